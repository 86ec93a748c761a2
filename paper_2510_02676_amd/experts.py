"""The experts of one layer with their weights compressed: any number of tokens, from hidden states and a router's logits to hidden states.

Seven launches, or eight or nine where many tokens are sorted: rows to E4M3 (``ecfa_quant``), all experts' weights are decoded into a buffer
(``ecf8_decode_batched``), the tokens to their experts (``ecfm_route``), gate and up of every expert with its tokens (``ecfm_gemm_experts``), silu(gate) * up
to E4M3 (``ecfm_gate``), down (``ecfm_gemm_experts``), and what came back to the tokens (``ecfm_combine``).  Nothing is allocated after
construction and nothing looks at a tensor's values on the host, so a step can be captured in a graph.
"""
import torch

from . import ecf8, ecfa, ecfm


class CompressedExperts:
    """experts: a list of {"gate", "up", "down"}: (header, blob on the device, fp32 scale per 128 x 128 weights) each, as ``ecf8_encode(w)`` makes them, of
    shapes (inner, hidden) twice and (hidden, inner), both multiples of 128.  tokens: of a step; top: experts of a token; options as ``ecfm_route``
    takes them.  room: the buffers that the weights are decoded into, (experts, 2 * inner, hidden) and (experts, hidden, inner) uint8, which layers
    that run one after the other on a stream share (``layer.room``).  What a step would refuse is refused here."""

    def __init__(self, experts, tokens, top, room=None, **options):
        if not experts:
            raise ecf8.Ecf8Error("CompressedExperts", ecf8.E_ARG)
        inner, hidden = experts[0]["gate"][0].rows, experts[0]["gate"][0].cols
        dev = experts[0]["gate"][1].device
        want = {"gate": (inner, hidden), "up": (inner, hidden), "down": (hidden, inner)}
        bad = inner % 128 or hidden % 128 or max(inner, hidden) > 1 << 20 or dev.type == "cpu"      # (2^20: what quant, gate and combine take)
        for e in experts:
            for name, (rows, cols) in want.items():
                hdr, blob, scale = e[name]
                bad = (bad or (hdr.rows, hdr.cols) != (rows, cols) or blob.device != dev or scale.device != dev
                       or scale.dtype != torch.float32 or scale.shape != (rows // 128, cols // 128)
                       # (the decode reads as far as the header says)
                       or blob.dtype != torch.uint8 or not blob.is_contiguous() or blob.numel() < hdr.total_size)
        if bad:
            raise ecf8.Ecf8Error("CompressedExperts", ecf8.E_ARG)
        n, pairs = len(experts), tokens * top
        empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        shapes = (n, 2 * inner, hidden), (n, hidden, inner)
        if room is None:
            room = tuple(empty(s, torch.uint8) for s in shapes)
        if any(r.shape != s or r.dtype != torch.uint8 or r.device != dev or not r.is_contiguous() for r, s in zip(room, shapes)):
            raise ecf8.Ecf8Error("CompressedExperts", ecf8.E_ARG)
        self.room, self.top, self.options = room, top, options
        parts = [(e["gate"], room[0][i, :inner]) for i, e in enumerate(experts)] + [(e["up"], room[0][i, inner:]) for i, e in enumerate(experts)]
        parts += [(e["down"], room[1][i]) for i, e in enumerate(experts)]
        self.decode = ecf8.Batch([w[0] for w, _ in parts], [w[1] for w, _ in parts], [out for _, out in parts])
        self.gate_up = ecfm.Weights(room[0], torch.stack([torch.cat((e["gate"][2], e["up"][2])) for e in experts]))
        self.down = ecfm.Weights(room[1], torch.stack([e["down"][2] for e in experts]))
        self.routes = ecfm.Routes(tokens, top, n, dev)
        self.x8, self.x_scale = empty((tokens, hidden), torch.uint8), empty((tokens, hidden // 128), torch.float32)
        self.mid = empty((pairs, 2 * inner), torch.bfloat16)
        self.h8, self.h_scale = empty((pairs, inner), torch.uint8), empty((pairs, inner // 128), torch.float32)
        self.back, self.y = empty((pairs, hidden), torch.bfloat16), empty((tokens, hidden), torch.bfloat16)
        ecfm.ecfm_route(empty((0, n), torch.float32), top, routes=None, stream=None, **options)      # refuses what a step's would, and chooses nothing

    def __call__(self, x, logits, add=None, stream=None):
        """x (tokens, hidden), BF16 or fp32, logits (tokens, experts), add (tokens, hidden) or None, as of a shared expert -> (tokens, hidden) BF16, in a
        buffer that the next call writes again."""
        inner = self.h8.shape[1]
        ecfa.ecfa_quant(x, 128, self.x8, self.x_scale, stream)     # (in front of the decode: this call refuses other devices and streams)
        ecf8.ecf8_decode_batched(self.decode, stream)
        r = ecfm.ecfm_route(logits, self.top, routes=self.routes, stream=stream, **self.options)
        ecfm.ecfm_gemm_experts(self.gate_up, r.starts, self.x8, self.x_scale, rows=r.rows, y=self.mid, stream=stream)
        ecfm.ecfm_gate(self.mid[:, :inner], self.mid[:, inner:], 128, self.h8, self.h_scale, stream)
        ecfm.ecfm_gemm_experts(self.down, r.starts, self.h8, self.h_scale, y=self.back, stream=stream)
        return ecfm.ecfm_combine(self.back, r.place, r.weights, add=add, out=self.y, stream=stream)
