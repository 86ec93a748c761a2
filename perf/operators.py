"""What stands between the compressed projections of a transformer layer, as cases to be timed and compared.

A program that serves a model with its weights compressed has q, k and v from the fused products, as fp32 rows.  It then

  append  turns q and k by their positions and writes k and v into a paged cache (BF16, or E4M3 with a scale per head)
  attend  lets the new tokens, one or many of each sequence, attend to the keys of their sequence in that cache
  quant   rounds the rows that come out to E4M3 with a scale per row or per 128 columns: X of the next product

Caches, page tables and lengths are what a serving loop has after some time: pages in no order, sequences of unlike lengths.
The layer sizes are those of the 8B-class LLM (32 heads of 128 over 8 of keys and values, 4096 and 14336 columns) and of the
14B-class diffusion transformer (40 heads of 128) that the package's benchmark uses; others are small or odd ones.

The plain forms are elementary operations of torch in 32 bits.  A rotation's angle is an integer: the position times the
frequency in 2^-64 of a turn, modulo one turn.
"""
import math
import random

import torch

own = False                          # set from outside: run the package's kernels, not the plain forms
DEV = "cuda:0"
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -100               # of a row that holds nothing but zeros, the largest magnitude is taken to be this


def listed():
    return [
        # the next token of one conversation: launch and start-up are all of it
        _append("append_1_token", 1, 1, 1, 5000, src="f32", page=16),
        # a decode step of 64 sequences whose cache is held in E4M3
        _append("append_64_tokens_e4m3", 64, 1, 1, 6000, src="f32", cache="e4m3", page=64),
        # prompts: three sequences of up to 3000 new tokens, interleaved pairs, half of each head turned, pages split by head
        _append("append_chunks_interleaved", 3, 700, 3001, 9000, src="bf16", cache="bf16", page=32, rot=64, interleaved=True, order="head"),
        # the next token of one conversation of ordinary length
        _attend("attend_1_token_4k", 1, 1, 1, 4096, 4096),
        # a full decode step: 64 sequences from one token to 8 thousand, E4M3
        _attend("attend_64_seqs_e4m3", 64, 1, 1, 1, 8192, cache="e4m3", page=64),
        # the next token over a long document; page by page all over the pool
        _attend("attend_1_token_128k", 1, 1, 1, 131072, 131072),
        # a prompt that is taken in chunks: the fourth of them
        _attend("attend_chunk_2048_of_8k", 1, 2048, 2048, 8192, 8192, page=64),
        # chunks and single tokens in one step: scores capped, a sliding window, small heads, E4M3
        _attend("attend_mixed_capped_e4m3", 13, 1, 517, 1, 4100, cache="e4m3", heads=16, kv_heads=4, dim=64, window=1000, cap=30.0, order="head"),
        # a diffusion block: every token sees every token; an odd number of them
        _attend("attend_all_4680", 1, 4680, 4680, 4680, 4680, heads=40, kv_heads=40, causal=False, page=128),
        # a picture or a system prompt that is seen from both sides, then text; a bias by distance; heads of 96
        _attend("attend_prefix_distance", 3, 40, 900, 900, 1300, heads=12, kv_heads=12, dim=96, prefix=300, slopes=True),
        # X of the output projection of 16 sequences
        _quant("quant_16x4096", 16, 4096),
        # X of the down projection of a prompt, a scale for each 128 columns
        _quant("quant_4096x14336_groups", 4096, 14336, src="f32", groups=True),
    ]


def _append(name, seqs, min_q, max_q, max_kv, src="bf16", cache="bf16", heads=32, kv_heads=8, dim=128, page=16, rot=None, interleaved=False, order="token"):
    return {"name": name, "op": "append", "seqs": seqs, "min_q": min_q, "max_q": max_q, "min_kv": max_q, "max_kv": max_kv, "src": src, "cache": cache,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "rot": dim if rot is None else rot, "interleaved": interleaved, "order": order}


def _attend(name, seqs, min_q, max_q, min_kv, max_kv, cache="bf16", heads=32, kv_heads=8, dim=128, page=16, causal=True, window=0, cap=0.0, prefix=0,
            slopes=False, order="token"):
    return {"name": name, "op": "attend", "seqs": seqs, "min_q": min_q, "max_q": max_q, "min_kv": min_kv, "max_kv": max_kv, "cache": cache, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "causal": causal, "window": window, "cap": cap, "prefix": prefix, "slopes": slopes, "order": order}


def _quant(name, rows, cols, src="bf16", groups=False):
    return {"name": name, "op": "quant", "rows": rows, "cols": cols, "src": src, "groups": groups}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "token", "token", "chunk", "chunk", "chunk", "quant"])
    if kind == "quant":
        groups = rng.random() < 0.5
        return _unnamed(_quant("", _log(rng, 1, 4096), 128 * _log(rng, 2, 112) if groups else 16 * _log(rng, 4, 900), rng.choice(["f32", "bf16"]), groups))
    kv_heads, share = rng.choice([(8, 4), (8, 4), (8, 8), (1, 8), (4, 2), (16, 1), (40, 1), (5, 3), (2, 16)])
    common = {"heads": kv_heads * share, "kv_heads": kv_heads, "dim": rng.choice([128, 128, 128, 64, 64, 96, 256, 80]), "cache": rng.choice(["bf16", "bf16", "e4m3"]),
              "page": rng.choice([16, 16, 64, 128, 32, 1, 256]), "order": rng.choice(["token", "head"])}
    wide = kv_heads * common["dim"]
    if kind == "append":
        seqs = _log(rng, 1, 64)
        max_q = 1 if rng.random() < 0.4 else _log(rng, 2, 8192 // seqs)
        rot = rng.choice([common["dim"], common["dim"], 16 * rng.randint(1, common["dim"] // 16)])
        return _unnamed(_append("", seqs, 1, max_q, max_q + _log(rng, 1, 8000), rng.choice(["f32", "bf16"]), rot=rot, interleaved=rng.random() < 0.5, **common))
    window = rng.choice([0, 0, 0, _log(rng, 16, 3000)])
    extra = {"cap": rng.choice([0.0, 0.0, 0.0, 30.0]), "slopes": rng.random() < 0.2}
    if kind == "token":
        seqs = _log(rng, 1, 128)
        most = min(131072, int(4e8 / (seqs * wide)), int(4e8 / (seqs * common["heads"])))    # the padded copies of the plain form have to stay small
        max_kv = _log(rng, 2, most)
        return _unnamed(_attend("", seqs, 1, 1, rng.choice([1, max_kv, max(1, max_kv // 3)]), max_kv, window=window, **extra, **common))
    seqs = _log(rng, 1, 16)
    max_q = _log(rng, 2, min(4096, int(math.sqrt(7e8 / (seqs * common["heads"])))))
    max_kv = max_q + int(_log(rng, 1, max(2, min(16384, int(1e9 / (seqs * common["heads"] * max_q)), int(4e8 / (seqs * wide))) - max_q)))
    causal = rng.random() < 0.8
    prefix = _log(rng, 1, max_kv) if causal and not window and rng.random() < 0.3 else 0
    return _unnamed(_attend("", seqs, rng.choice([1, max_q, max(1, max_q // 4)]), max_q, max_q, max_kv, causal=causal, window=window if causal else 0, prefix=prefix,
                            **extra, **common))


def _unnamed(case):
    return {k: v for k, v in case.items() if k != "name"}


def _lengths(case):
    """(new tokens, tokens in the cache with them) of each sequence: the first has the most of both, the others anything between."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    q, kv = [case["max_q"]], [case["max_kv"]]
    for _ in range(case["seqs"] - 1):
        q.append(_log(rng, case["min_q"], case["max_q"]))
        kv.append(max(q[-1], _log(rng, case["min_kv"], case["max_kv"])))
    return q, kv


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pool(case, pages, gen, scale):
    """A pool of pages with what earlier tokens have left in it: (pages, page, kv_heads, dim), in one of two orders in memory."""
    shape = (pages, case["page"], case["kv_heads"], case["dim"])
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    if scale is not None:
        x = (x.float() / scale[:, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    if case["order"] == "head":
        x = x.view(torch.uint8 if scale is not None else x.dtype).transpose(1, 2).contiguous().transpose(1, 2)
        x = x.view(torch.float8_e4m3fn) if scale is not None else x
    return x


def _paged(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 11)
    q, kv = _lengths(case)
    width = -(-max(kv) // case["page"])
    need = [-(-n // case["page"]) for n in kv]
    spare = 3                                    # pages that belong to nobody
    order = torch.randperm(sum(need) + spare, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((case["seqs"], width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    start = [0]
    for n in q:
        start.append(start[-1] + n)
    st = {"case": case, "gen": gen, "table": table, "kv_len": _i32(kv), "q_start": _i32(start), "tokens": start[-1], "max_q": max(q), "max_kv": max(kv),
          "k_scale": None, "v_scale": None}
    if case["cache"] == "e4m3":                  # as calibrated: the largest keys and values of a head fill most of the format's range
        st["k_scale"] = torch.rand(case["kv_heads"], generator=gen, device=DEV) * 0.01 + 0.01
        st["v_scale"] = torch.rand(case["kv_heads"], generator=gen, device=DEV) * 0.01 + 0.01
    st["k"], st["v"] = (_pool(case, sum(need) + spare, gen, st[n]) for n in ("k_scale", "v_scale"))
    return st


def _rows(st, heads, dtype):
    return torch.randn((st["tokens"], heads, st["case"]["dim"]), generator=st["gen"], device=DEV).to(dtype)


def _handles(st):
    """What a program makes once and keeps: the cache, the step's batch, the rotation."""
    from paper_2510_02676_amd import ecfa
    case = st["case"]
    single = case["max_q"] == 1
    st["cache"] = ecfa.Cache(st["k"], st["v"], st["k_scale"], st["v_scale"])
    st["batch"] = ecfa.Batch(st["table"], st["kv_len"], None if single else st["q_start"], n_tokens=st["tokens"], max_q=st["max_q"], max_kv=st["max_kv"])
    if case["op"] == "append":
        st["rope"] = ecfa.Rope(st["freq"], interleaved=case["interleaved"])
    else:
        st["work"] = ecfa.attend_workspace(st["cache"], st["batch"], case["heads"])


def prepare(case, seed):
    if case["op"] == "quant":
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed * 7919 + 5)
        x = torch.randn((case["rows"], case["cols"]), generator=gen, device=DEV)
        x *= torch.exp(torch.randn((case["rows"], 1), generator=gen, device=DEV))            # rows of unlike size
        x = x.to(torch.float32 if case["src"] == "f32" else torch.bfloat16)
        groups = case["cols"] // 128 if case["groups"] else 0
        st = {"case": case, "x": x, "q": torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=DEV),
              "scale": torch.empty((case["rows"], groups) if groups else (case["rows"],), dtype=torch.float32, device=DEV)}
        if own:
            from paper_2510_02676_amd import ecfa  # noqa: F401  (loads the library, once)
        return st
    st = _paged(case, seed)
    if case["op"] == "append":
        dtype = torch.float32 if case["src"] == "f32" else torch.bfloat16
        st["new_q"], st["new_k"], st["new_v"] = _rows(st, case["heads"], dtype), _rows(st, case["kv_heads"], dtype), _rows(st, case["kv_heads"], dtype)
        st["q_out"] = torch.empty(st["new_q"].shape, dtype=torch.bfloat16, device=DEV)
        st["freq"] = torch.tensor([int(500000.0 ** (-2.0 * j / case["rot"]) / (2 * math.pi) * 2.0 ** 64) for j in range(case["rot"] // 2)], dtype=torch.int64, device=DEV)
    else:
        # some heads look at a few keys, others at all of them
        temper = torch.rand((case["heads"], 1), generator=st["gen"], device=DEV) * 2 + 0.5
        st["q"] = (_rows(st, case["heads"], torch.float32) * temper).to(torch.bfloat16)
        st["out"] = torch.empty(st["q"].shape, dtype=torch.bfloat16, device=DEV)
        st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["heads"] + 1, device=DEV) / case["heads"]) if case["slopes"] else None
        st["prefix"] = torch.clamp(st["kv_len"], max=case["prefix"]) if case["prefix"] else None
    if own:
        _handles(st)
    return st


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2510_02676_amd import ecfa
        if op == "quant":
            return ecfa.ecfa_quant(state["x"], 128 if state["case"]["groups"] else 0, state["q"], state["scale"])
        if op == "append":
            q = ecfa.ecfa_append(state["cache"], state["batch"], state["new_k"], state["new_v"], state["new_q"], state["q_out"], state["rope"])
            return q, state["k"], state["v"]
        case = state["case"]
        return ecfa.ecfa_attend(state["cache"], state["batch"], state["q"], causal=case["causal"], window=case["window"], softcap=case["cap"],
                                slopes=state["slopes"], prefix=state["prefix"], out=state["out"], workspace=state["work"])
    return {"quant": _plain_quant, "append": _plain_append, "attend": _plain_attend}[op](state)


def _plain_quant(st):
    x = st["x"].float()
    if st["case"]["groups"]:
        x = x.view(x.shape[0], -1, 128)
    most = x.abs().amax(dim=-1).clamp(min=SMALLEST)
    q = (x * (E4M3_MAX / most)[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(st["x"].shape), most / E4M3_MAX


def _turned(x, place, freq, interleaved, dtype):
    """x (tokens, heads, dim) turned by its places, in `dtype`."""
    half = freq.numel()
    phase = place[:, None] * freq[None, :]                       # 64-bit integers wrap around: whole turns fall away
    angle = (phase >> 32).to(dtype) * (2.0 * math.pi / 2.0 ** 32)
    c, s = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
    x = x.to(dtype)
    rot, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if interleaved else (rot[..., :half], rot[..., half:])
    a, b = a * c - b * s, b * c + a * s
    rot = torch.stack((a, b), dim=-1).flatten(-2) if interleaved else torch.cat((a, b), dim=-1)
    return torch.cat((rot, rest), dim=-1)


def _token_places(st):
    """(sequence, place in the cache) of each new token."""
    t = torch.arange(st["tokens"], device=DEV)
    start = st["q_start"].long()
    seq = torch.searchsorted(start, t, right=True) - 1
    return seq, st["kv_len"].long()[seq] - start[seq + 1] + t


def _plain_append(st):
    case = st["case"]
    seq, place = _token_places(st)
    page = st["table"].long()[seq, place // case["page"]]
    at = place % case["page"]
    q = _turned(st["new_q"], place, st["freq"], case["interleaved"], torch.float32).to(torch.bfloat16)
    k = _turned(st["new_k"], place, st["freq"], case["interleaved"], torch.float32)
    v = st["new_v"].float()
    if case["cache"] == "e4m3":
        k = (k / st["k_scale"][:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        v = (v / st["v_scale"][:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        st["k"].view(torch.uint8)[page, at] = k
        st["v"].view(torch.uint8)[page, at] = v
    else:
        st["k"][page, at] = k.to(torch.bfloat16)
        st["v"][page, at] = v.to(torch.bfloat16)
    return q, st["k"], st["v"]


def _sequences(st, pool, scale):
    """The cache of every sequence in one piece, (seqs, kv_heads, max_kv, dim), in 32 bits."""
    x = pool.view(torch.uint8) if scale is not None else pool
    x = x[st["table"].clamp(min=0).long()]                       # (seqs, pages, page, kv_heads, dim)
    x = x.flatten(1, 2)[:, :st["max_kv"]].transpose(1, 2).contiguous()
    return x.float() if scale is None else x.view(torch.float8_e4m3fn).float() * scale[:, None, None]


def _visible(st):
    """(seqs, max_q, max_kv): which keys a token sees; and the tokens' places."""
    case = st["case"]
    kv, start = st["kv_len"].long(), st["q_start"].long()
    place = (kv - start[1:] + start[:-1])[:, None] + torch.arange(st["max_q"], device=DEV)
    key = torch.arange(st["max_kv"], device=DEV)
    seen = (key < kv[:, None])[:, None, :]
    if case["causal"]:
        past = key <= place[:, :, None]
        if st["prefix"] is not None:
            past = past | (key < st["prefix"][:, None, None])
        seen = seen & past
    if case["window"]:
        seen = seen & (key > place[:, :, None] - case["window"])
    return seen.expand(-1, st["max_q"], -1), place


def _plain_attend(st):
    case = st["case"]
    seqs, heads, kv_heads, dim = case["seqs"], case["heads"], case["kv_heads"], case["dim"]
    share = heads // kv_heads
    seq, _ = _token_places(st)
    row = torch.arange(st["tokens"], device=DEV) - st["q_start"].long()[seq]
    q = torch.zeros((seqs, st["max_q"], heads, dim), device=DEV)
    q[seq, row] = st["q"].float()
    q = q.view(seqs, st["max_q"], kv_heads, share, dim).permute(0, 2, 3, 1, 4).reshape(seqs, kv_heads, share * st["max_q"], dim)
    k, v = _sequences(st, st["k"], st["k_scale"]), _sequences(st, st["v"], st["v_scale"])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * dim ** -0.5
    x = x.view(seqs, kv_heads, share, st["max_q"], st["max_kv"])
    seen, place = _visible(st)
    if case["cap"]:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    if st["slopes"] is not None:
        far = (place[:, :, None] - torch.arange(st["max_kv"], device=DEV)).abs().float()
        x = x - st["slopes"].view(kv_heads, share, 1, 1) * far[:, None, None]
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    most = x.amax(dim=-1, keepdim=True)
    x = torch.exp(x - torch.where(most == -math.inf, torch.zeros_like(most), most))
    total = x.sum(dim=-1, keepdim=True)
    y = torch.matmul(x.view(seqs, kv_heads, -1, st["max_kv"]), v).view(seqs, kv_heads, share, st["max_q"], dim)
    y = torch.where(total > 0, y / total, torch.zeros_like(y))
    y = y.permute(0, 3, 1, 2, 4).reshape(seqs, st["max_q"], heads, dim)[seq, row]
    return y.to(torch.bfloat16)


def work(case):
    if case["op"] == "quant":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (5 if case["src"] == "f32" else 3) + 4 * (n // 128 if case["groups"] else case["rows"]), "flops": 0}
    q, kv = _lengths(case)
    e = 1 if case["cache"] == "e4m3" else 2
    wide, narrow = case["heads"] * case["dim"], case["kv_heads"] * case["dim"]
    if case["op"] == "append":
        src = 4 if case["src"] == "f32" else 2
        return {"bytes": sum(q) * ((wide + 2 * narrow) * src + 2 * wide + 2 * narrow * e), "flops": 0}
    keys = pairs = 0
    for n, m in zip(q, kv):
        low = max(0, m - n + 1 - case["window"]) if case["window"] else 0
        keys += m - low
        if not case["causal"]:
            pairs += n * m
            continue
        for p in range(m - n, m):
            pairs += max(p + 1, min(case["prefix"], m)) - (max(0, p + 1 - case["window"]) if case["window"] else 0)
    return {"bytes": keys * 2 * narrow * e + sum(q) * wide * 4, "flops": 4.0 * pairs * wide}


def exact(case, seed):
    """The same from the definitions, in 64 bits, a sequence and a head of keys at a time."""
    st = prepare(case, seed)
    if case["op"] == "quant":
        x = st["x"].double()
        parts = x.view(x.shape[0], -1, 128) if case["groups"] else x
        most = parts.abs().max(dim=-1).values.clamp(min=SMALLEST)
        return (parts * (E4M3_MAX / most).unsqueeze(-1)).view(x.shape), most / E4M3_MAX
    page = case["page"]
    q_start, kv_len, table = st["q_start"].tolist(), st["kv_len"].tolist(), st["table"].long()
    if case["op"] == "append":
        return _exact_append(st, q_start, kv_len, table, page)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    share = case["heads"] // case["kv_heads"]
    for s in range(case["seqs"]):
        a, b, n = q_start[s], q_start[s + 1], kv_len[s]
        key = torch.arange(n, device=DEV)
        places = torch.arange(n - (b - a), n, device=DEV)
        slot = table[s, key // page]
        prefix = int(st["prefix"][s]) if st["prefix"] is not None else 0
        for g in range(case["kv_heads"]):
            k, v = (st[x].view(torch.uint8)[slot, key % page, g].view(torch.float8_e4m3fn).double() * st[x + "_scale"][g].double()
                    if st["k_scale"] is not None else st[x][slot, key % page, g].double() for x in ("k", "v"))
            for first in range(0, b - a, 1024):
                place = places[first:first + 1024, None]
                rows = slice(a + first, min(b, a + first + 1024))
                hide = torch.zeros((place.numel(), n), dtype=torch.bool, device=DEV)
                if case["causal"]:
                    hide |= (key > place) & (key >= prefix)
                if case["window"]:
                    hide |= key <= place - case["window"]
                for h in range(g * share, (g + 1) * share):
                    x = st["q"][rows, h].double() @ k.T / math.sqrt(case["dim"])
                    if case["cap"]:
                        x = case["cap"] * torch.tanh(x / case["cap"])
                    if case["slopes"]:
                        x -= st["slopes"][h].double() * (place - key).abs()
                    w = torch.softmax(x.masked_fill(hide, -math.inf), dim=-1)
                    out[rows, h] = torch.nan_to_num(w) @ v
    return out


def _exact_append(st, q_start, kv_len, table, page):
    case = st["case"]
    place = torch.cat([torch.arange(n - (b - a), n, device=DEV) for a, b, n in zip(q_start, q_start[1:], kv_len)])
    slot = torch.cat([table[s, torch.arange(n - (b - a), n, device=DEV) // page] for s, (a, b, n) in enumerate(zip(q_start, q_start[1:], kv_len))])
    half = case["rot"] // 2
    wraps = place.unsqueeze(1) * st["freq"].unsqueeze(0)
    turn = torch.polar(torch.ones(wraps.shape, dtype=torch.float64, device=DEV), wraps.double() * (math.pi / 2.0 ** 63))[:, None]

    def turned(x):
        x = x.double().clone()
        if case["interleaved"]:
            x[..., :2 * half] = torch.view_as_real(torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:2], half, 2)) * turn).flatten(-2)
        else:
            z = torch.complex(x[..., :half], x[..., half:2 * half]) * turn
            x[..., :half], x[..., half:2 * half] = z.real, z.imag
        return x

    pools = []
    for pool, new, scale in ((st["k"], turned(st["new_k"]), st["k_scale"]), (st["v"], st["new_v"].double(), st["v_scale"])):
        pool = pool.double()
        pool[slot, place % page] = new if scale is None else (new / scale.double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
        pools.append(pool)
    return turned(st["new_q"]), pools[0], pools[1]
