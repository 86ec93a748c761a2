"""The attention of one layer, with its four projections compressed: a decode or a short chunk step from hidden states to hidden states.

Six launches, or seven where long sequences are split: rows to E4M3 (``ecfa_quant``), the three products of q, k and v with their weights decoded on
the way (``ecf8_gemm_fp8_grouped``), rotation and append to the paged cache (``ecfa_append``), attention over it (``ecfa_attend``), rows to
E4M3 again and the output product (``ecf8_gemm_fp8_scaled``).  Nothing is allocated after construction and nothing looks at a
tensor's values on the host, so a step can be captured in a graph while the serving loop rewrites the batch's tensors in place.
"""
import torch

from . import ecf8, ecfa


class CompressedAttention:
    """weights: {"q", "k", "v", "o"}: (header, blob on the device, fp32 scale per 128 x 128 weights) each, as ``ecf8_encode(w, lane_syms=64,
    tile_rows=16)`` makes them, of shapes (heads * head_dim, hidden), (kv_heads * head_dim, hidden) twice and (hidden, heads * head_dim).
    cache, batch: ``ecfa.Cache`` and ``ecfa.Batch``, of up to 64 new tokens; rope: ``ecfa.Rope`` or None.  options: scale, window, softcap,
    slopes, prefix as ``ecfa_attend`` takes them.  What a step would refuse is refused here."""

    def __init__(self, weights, heads, cache, batch, rope=None, **options):
        n, dim, kv, dev = batch.n_tokens, cache.head_dim, cache.kv_heads, cache.device
        hidden = weights["o"][0].rows
        want = {"q": (heads * dim, hidden), "k": (kv * dim, hidden), "v": (kv * dim, hidden), "o": (hidden, heads * dim)}
        if not 1 <= n <= 64 or any((weights[w][0].rows, weights[w][0].cols) != shape for w, shape in want.items()):
            raise ecf8.Ecf8Error("CompressedAttention", ecf8.E_ARG)
        if any(t is None or t.get_device() != cache.on for w in want for t in weights[w][1:]):
            raise ecf8.Ecf8Error("CompressedAttention", ecf8.E_ARG)
        ecfa.check_layer("CompressedAttention", cache, batch, heads, rope, **options)
        self.cache, self.batch, self.rope, self.options, self.out_weight = cache, batch, rope, options, weights["o"]
        empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        self.x8, self.x_scale = empty((n, hidden), torch.uint8), empty((n, hidden // 128), torch.float32)
        self.group = ecf8.GemmGroup([{"hdr": weights[w][0], "blob": weights[w][1], "x": self.x8, "w_scale": weights[w][2], "x_scale": self.x_scale}
                                     for w in "qkv"])
        self.q, self.k, self.v = (y.view(n, -1, dim) for y in self.group.y)
        self.turned, self.seen = empty((n, heads, dim), torch.bfloat16), empty((n, heads, dim), torch.bfloat16)
        self.seen8, self.seen_scale = empty((n, heads * dim), torch.uint8), empty((n, heads * dim // 128), torch.float32)
        self.y = empty((n, hidden), torch.float32)
        self.workspace = ecfa.attend_workspace(cache, batch, heads)
        # the output product as a group of one, whose preparation refuses what the product would: nothing else is done with it
        ecf8.GemmGroup([{"hdr": weights["o"][0], "blob": weights["o"][1], "x": self.seen8, "w_scale": weights["o"][2], "x_scale": self.seen_scale, "y": self.y}])

    def __call__(self, x, stream=None):
        """x (n_tokens, hidden), BF16 or fp32 -> (n_tokens, hidden) fp32, in a buffer that the next call writes again."""
        ecfa.ecfa_quant(x, 128, self.x8, self.x_scale, stream)
        ecf8.ecf8_gemm_fp8_grouped(self.group, stream)
        ecfa.ecfa_append(self.cache, self.batch, self.k, self.v, self.q, self.turned, self.rope, stream)
        ecfa.ecfa_attend(self.cache, self.batch, self.turned, out=self.seen, workspace=self.workspace, stream=stream, **self.options)
        ecfa.ecfa_quant(self.seen.view(self.seen8.shape), 128, self.seen8, self.seen_scale, stream)
        hdr, blob, scale = self.out_weight
        return ecf8.ecf8_gemm_fp8_scaled(hdr, blob, self.seen8, scale, self.seen_scale, self.y, stream)
