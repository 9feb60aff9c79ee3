"""Plain implementations in 64 bits, on the CPU, of the four-bit key/value cache and attention over it, from the definitions in include/apmm.h."""
import numpy as np
import torch


def quantise(x):
    """Rows x (any leading dimensions, a torch tensor of 16-bit floats): codes and scales as apmm_kv_write makes them, decided in exact arithmetic (64 bits hold every
    product of a 16-bit float's 11 significant bits and an integer up to 16)."""
    y = x.double()
    finite = torch.isfinite(y).all(-1)
    y = torch.where(finite[..., None], y, torch.zeros_like(y))
    s = (y.abs().amax(-1) / 15.0).to(x.dtype)     # 64 bits to the type: one rounding too many only for a quotient within 2^-53 of a tie, and max / 15 is none
    s64 = s.double()[..., None]
    # code c or more where x >= (2 c - 16) s: the lower border of a cell belongs to it
    codes = torch.zeros(y.shape, dtype=torch.uint8)
    for c in range(1, 16):
        codes += (y >= (2 * c - 16) * s64).to(torch.uint8)
    codes = torch.where(s64 > 0, codes, torch.full_like(codes, 8))
    s = torch.where(finite, s, torch.full_like(s, float("nan")))
    return codes, s


def value(codes, scales):
    """What codes and scales stand for, rounded once to the scales' type, no finite product beyond its largest number."""
    top = torch.finfo(scales.dtype).max
    y = (2.0 * codes.double() - 15.0) * scales.double()[..., None]
    return torch.where(torch.isnan(y), y, y.clamp(-top, top)).to(scales.dtype)


def layout(codes_k, codes_v):
    """Codes (pages, heads, page_size, D) -> the cache's bytes (pages, heads, 2, page_size * D / 2)."""
    pages, heads, ps, D = codes_k.shape
    k = codes_k.numpy()
    kb = np.zeros((pages, heads, ps, D // 2), dtype=np.uint8)
    vb = np.zeros((pages, heads, ps // 8, D // 4, 8, 2), dtype=np.uint8)
    v = codes_v.numpy()
    for c in range(D):
        kb[..., c // 2] |= (k[..., c] << (4 * (c % 2))).astype(np.uint8)
        for t in range(8):
            vb[:, :, :, c // 4, t, c % 4 // 2] |= (v[:, :, t::8, c] << (4 * (c % 2))).astype(np.uint8)
    return torch.from_numpy(np.stack([kb.reshape(pages, heads, -1), vb.reshape(pages, heads, -1)], 2))


def unlayout(codes, ps):
    """The cache's bytes -> codes of keys and of values (pages, heads, page_size, D)."""
    pages, heads, _, n = codes.shape
    D = 2 * n // ps
    raw = codes.cpu().numpy()
    kb, vb = raw[:, :, 0].reshape(pages, heads, ps, D // 2), raw[:, :, 1].reshape(pages, heads, ps // 8, D // 4, 8, 2)
    k, v = np.zeros((pages, heads, ps, D), dtype=np.uint8), np.zeros((pages, heads, ps, D), dtype=np.uint8)
    for c in range(D):
        k[..., c] = (kb[..., c // 2] >> (4 * (c % 2))) & 15
        for t in range(8):
            v[:, :, t::8, c] = (vb[:, :, :, c // 4, t, c % 4 // 2] >> (4 * (c % 2))) & 15
    return torch.from_numpy(k), torch.from_numpy(v)


def attention(q, codes, scales, table, lengths, starts, window, sinks, scale):
    """Results in 64 bits, and for each result how far a kernel with 32-bit sums and weights of 11 bits may be from it before its own rounding."""
    ps = scales.shape[3]
    ck, cv = unlayout(codes, ps)
    sk, sv = scales[:, :, 0].cpu().double(), scales[:, :, 1].cpu().double()
    k = (2.0 * ck.double() - 15.0) * sk[..., None]
    v = (2.0 * cv.double() - 15.0) * sv[..., None]
    q = q.cpu().double()
    T, Hq, D = q.shape
    H, pages, width = codes.shape[1], codes.shape[0], table.shape[1]
    out, near = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
    for b in range(len(lengths)):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            p = lengths[b] - n + i
            keys = [j for j in range(min(p + 1, lengths[b], width * ps)) if (not window or j > p - window or j < sinks) and 0 <= int(table[b, j // ps]) < pages]
            if not keys:
                continue
            j = torch.tensor(keys)
            page, at = table[b].long()[j // ps], j % ps
            kk, vv = k[page, :, at], v[page, :, at]  # keys, heads, D
            for h in range(Hq):
                g = h // (Hq // H)
                x = q[starts[b] + i, h]
                w = torch.softmax(scale * (kk[:, g] @ x), 0)
                out[starts[b] + i, h] = w @ vv[:, g]
                # the score: D products and as many sums of the codes' 0 to 15 times |q|, twice that with what is taken off, to 2^-24 each; the weight follows it and is
                # rounded to 2^-11; what is below 2^-24 of the range of 16 bits (2^9 for the largest scale) is lost
                d = (2 * D + 16) * 2.0 ** -24 * scale * 30.0 * float(x.abs().sum()) * sk[page, g, at]
                near[starts[b] + i, h] = ((w * (2.0 ** -11 + 2.0 * d.max() + 2.0 ** -20))[:, None] * (vv[:, g].abs() + sv[page, g, at][:, None] * 15.0 * 2.0 ** -10)).sum(0) + \
                    len(keys) * 2.0 ** -33 * 30.0 * float(sv[page, g, at].max())
    return out, near
