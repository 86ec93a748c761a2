"""The attention calls from their definitions, in 64 bits on the CPU, a token and a head at a time.  Shares nothing with the package."""
import math

import numpy as np
import torch


def e4m3_values():
    """The 256 numbers of E4M3, from its definition."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = math.nan if e == 15 and m == 7 else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out[b] = -x if b & 128 else x
    return out


E4M3 = e4m3_values()


def values(pool, scale=None):
    """A pool (pages, page, heads, dim) as 64-bit numbers: BF16, or E4M3 bytes times the scale of their head."""
    if pool.dtype == torch.bfloat16:
        return pool.cpu().double().numpy()
    x = E4M3[pool.cpu().view(torch.uint8).numpy()]
    return x if scale is None else x * scale.cpu().double().numpy()[:, None]


def tokens(q_start, kv_len, table, page, pages):
    """For each new token: (sequence, place, [slot of each key of its sequence, or None for a hole])."""
    out = []
    for s in range(len(kv_len)):
        n = q_start[s + 1] - q_start[s]
        slots = []
        for j in range(max(0, kv_len[s])):
            p = table[s][j // page] if j // page < len(table[s]) else -1
            slots.append((p, j % page) if 0 <= p < pages else None)
        for i in range(n):
            out.append((s, max(0, kv_len[s]) - n + i, slots))
    return out


def attend(q, k, v, toks, scale, causal=True, window=0, cap=0.0, slopes=None, prefix=None):
    """(out, sum of weight * |v|): what the result is, and what its error is measured by.  q (tokens, heads, dim); k, v: values()."""
    q = q.cpu().double().numpy()
    share = q.shape[1] // k.shape[2]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for t, (s, place, slots) in enumerate(toks):
        keys = [j for j, sl in enumerate(slots) if sl is not None and (not causal or j <= place or (prefix is not None and j < prefix[s]))
                and (not window or j > place - window)]
        if not keys:
            continue
        pg, at = np.array([slots[j][0] for j in keys]), np.array([slots[j][1] for j in keys])
        for h in range(q.shape[1]):
            kk, vv = k[pg, at, h // share], v[pg, at, h // share]
            with np.errstate(invalid="ignore", over="ignore"):
                x = scale * (kk @ q[t, h])
                if cap:
                    x = cap * np.tanh(x / cap)
                if slopes is not None:
                    x = x - float(slopes[h]) * np.abs(place - np.array(keys))
                w = np.exp(x - np.max(x))
                w /= w.sum()
                out[t, h] = w @ vv
                size[t, h] = w @ np.abs(vv)
    return out, size


def attend_bound(out, size):
    """Weights are rounded to BF16 (eight significant bits: 2^-8 of each at most, in the sum and in what it is divided by), the result too;
    2^-12 for fp32 scores and sums."""
    return (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * np.abs(out) + 1e-30


def turned(x, pos, freq, rot, interleaved, scale=1.0):
    """x (tokens, heads, dim) in 64 bits, its first `rot` elements turned; freq: integers, 2^-64 of a turn."""
    x = x.astype(np.float64).copy()
    for t in range(x.shape[0]):
        for j in range(rot // 2):
            phase = int(pos[t]) * int(freq[j]) % 2 ** 64
            ang = (phase if phase < 2 ** 63 else phase - 2 ** 64) / 2.0 ** 64 * 2 * math.pi
            c, s = scale * math.cos(ang), scale * math.sin(ang)
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
            x[t, :, a], x[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
    return x


def near_bf16(got, want, size):
    """Within half a step of BF16 (eight significant bits: 2^-8 of the number) and 2^-20 of the largest term for fp32 sines and products."""
    return np.abs(got - want) <= 2.0 ** -8 * np.abs(want) * 1.001 + 2.0 ** -20 * size + 1e-38


def near_e4m3(got, want, size):
    """`want` before rounding, limited to 448: half a step (2^-4 of the number, 2^-10 below 2^-6) and 2^-20 of the largest term."""
    want = np.clip(want, -448, 448)
    return np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) * 1.001 + 2.0 ** -20 * size
