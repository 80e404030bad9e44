"""Plain 64-bit forms of rotary positions, of the paged cache and of the attention over it, for the tests: loops over sequences, one
statement per definition."""
from __future__ import annotations

import math

import torch

PAGE = 64


def turned(x, pos, freq, layout, magnitude=1.0, back=False):
    """x [T, heads, d] in float64, pairs as complex numbers."""
    r, y = 2 * len(freq), x.double().clone()
    angle = pos.double()[:, None] * freq.double()[None, :] * (-1 if back else 1)
    z = (torch.complex(angle.cos(), angle.sin()) * magnitude)[:, None, :]
    i = torch.arange(r // 2, device=x.device)
    a, b = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    w = torch.complex(y[..., a], y[..., b]) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y


def frequencies(rot_dim, base=10000.0, device="cuda"):
    return base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)


def scale_for(top):
    """smallest power of two with top <= 448 * scale, its exponent in [-100, 119]"""
    if top == 0:
        return 2.0 ** -100
    e = math.ceil(math.log2(top / 448.0))
    while 448.0 * 2.0 ** (e - 1) >= top:
        e -= 1
    while 448.0 * 2.0 ** e < top:
        e += 1
    return 2.0 ** min(max(e, -100), 119)


def to_codes(x):
    """values in units of the scale -> e4m3 (nearest even, saturating, NaN for what is not finite)"""
    y = x.clamp(-448, 448).float().to(torch.float8_e4m3fn)
    bits = torch.where(torch.isfinite(x), y.view(torch.uint8), torch.tensor(0x7f, dtype=torch.uint8, device=x.device))
    return bits.view(torch.float8_e4m3fn)


def pages_for(lens, spare=3, seed=0, device="cuda"):
    """(page table [batch, blocks] with the pages in random order and -1 behind a sequence's last, number of pages)"""
    counts = [(n + PAGE - 1) // PAGE for n in lens]
    total = sum(counts) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lens), max(max(counts), 1)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table.to(device), total


def append(k, v, scales, new_k, new_v, table, news, prevs):
    """The pages after an append, in place; k, v [pages, hkv, 64, d], new_k / new_v [hkv, T, d] float64 (already turned);
    scales: (k_scale, v_scale) or None"""
    for cache, new, scale in ((k, new_k, scales and scales[0]), (v, new_v, scales and scales[1])):
        t0 = 0
        for b, (n, p) in enumerate(zip(news, prevs)):
            t = p
            while t < p + n:
                m, page, at = min(PAGE - t % PAGE, p + n - t), int(table[b, t // PAGE]), t % PAGE
                rows = new[:, t0 + t - p:t0 + t - p + m]
                if 0 <= page < cache.shape[0]:
                    for h in range(cache.shape[1]):
                        if scale is None:
                            cache[page, h, at:at + m] = rows[h].to(cache.dtype)
                            continue
                        mag = rows[h].abs()
                        s = scale_for(float(mag[torch.isfinite(mag)].max()) if torch.isfinite(mag).any() else 0.0)
                        if at:
                            was = float(scale[page, h])
                            s = max(s, was)
                            bits = cache.view(torch.uint8)
                            old = cache[page, h, :at].double()
                            bits[page, h, :at] = to_codes(old * (was / s)).view(torch.uint8)
                        cache.view(torch.uint8)[page, h, at:at + m] = to_codes(rows[h] / s).view(torch.uint8)
                        scale[page, h] = s
                t += m
            t0 += n


def rows_of(cache, scale, table, b, n, h):
    """(rows [n, d] in float64, which of them are there)"""
    out = torch.zeros((n, cache.shape[3]), dtype=torch.float64, device=cache.device)
    there = torch.zeros(n, dtype=torch.bool, device=cache.device)
    for j in range((n + PAGE - 1) // PAGE):
        page, m = int(table[b, j]), min(PAGE, n - j * PAGE)
        if 0 <= page < cache.shape[0]:
            x = cache[page, h, :m].double()
            out[j * PAGE:j * PAGE + m] = x if scale is None else x * scale[page, h].double()
            there[j * PAGE:j * PAGE + m] = True
    return out, there


def attention(q, k, v, scales, table, news, ctxs, softmax_scale, blocks=None, dense_below=0):
    """(out [T, hq, d], lse [T, hq], sum of weights times |v| [T, hq, d]) in float64: one softmax per token and head, over the keys that it sees"""
    T, hq, d = q.shape
    mass = torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
    hkv = k.shape[1]
    G = hq // hkv
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=q.device)
    t0 = 0
    for b, (n, L) in enumerate(zip(news, ctxs)):
        for h in range(hkv):
            if n == 0:
                continue
            K, there = rows_of(k, scales and scales[0], table, b, L, h)
            V, _ = rows_of(v, scales and scales[1], table, b, L, h)
            for i in range(n):
                pos = L - n + i
                see = there[:pos + 1].clone()
                if blocks is not None and L >= dense_below:
                    has = torch.zeros(pos + 1, dtype=torch.bool, device=q.device)
                    for j in blocks[t0 + i, h].tolist():
                        if 0 <= j <= pos // PAGE:
                            has[j * PAGE:(j + 1) * PAGE] = True
                    see &= has
                u = torch.nonzero(see)[:, 0]
                if len(u) == 0:
                    continue
                z = q[t0 + i, h * G:(h + 1) * G].double() @ K[u].T * softmax_scale
                p = torch.softmax(z, -1)
                out[t0 + i, h * G:(h + 1) * G] = p @ V[u]
                mass[t0 + i, h * G:(h + 1) * G] = p @ V[u].abs()
                lse[t0 + i, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
        t0 += n
    return out, lse, mass
