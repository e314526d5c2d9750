"""Plain forms, in 64 bits on the CPU, of the operators on packed patch tokens, and how far a
16-bit result may be from them.  Written from the formulas in include/l3_tokens.h, apart from the kernels.

Tolerances count roundings: `half(dtype)` is the most that one rounding to the type moves a value, relative
to it.  32-bit sums and the hardware's exp2, sin and cos are allowed SLACK = 2^-17 relative to the sum of the
absolute terms: 32-bit sums of n <= 1000 terms of random signs are good to some sqrt(n) 2^-24, the worst
n 2^-24 = 2^-14 does not occur in the tests' data; exp2 of a score that itself is off by 2^-22 of up to
about 16 is off by 2^-18; sines and cosines are off by at most 2^-18.
"""
import math

import numpy as np
import torch

SLACK = 2.0 ** -17
LEAST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}      # smallest subnormal


def half(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, bound, what):
    """Every element of got within bound of want; bound in addition to the rounding of the result itself."""
    got = got.detach().cpu()
    worst = half(got.dtype) * want.abs() + LEAST[got.dtype] if got.dtype in LEAST else 0.0
    off = (got.double() - want).abs()
    ok = off <= bound + worst
    assert bool(ok.all()), "%s: %d of %d elements, worst %g over (at %s: got %g, want %g)" % (
        what, int((~ok).sum()), ok.numel(), float((off - bound - worst).nan_to_num(1e30).max()),
        tuple((~ok).nonzero()[0].tolist()), float(got[tuple((~ok).nonzero()[0])]), float(want[tuple((~ok).nonzero()[0])]))


# ---- dropout ----------------------------------------------------------------------------------


def philox(blocks, high, key, rounds=7):
    """[len(blocks), 4] words (Python integers in an object array would be slow: uint64 arithmetic)."""
    low32 = np.uint64(0xFFFFFFFF)
    blocks = np.asarray(blocks, dtype=np.uint64)
    c = [blocks & low32, blocks >> np.uint64(32), np.full_like(blocks, high & 0xFFFFFFFF), np.full_like(blocks, high >> 32)]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low32]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1)


def kept(count, p, seed, offset):
    words = philox(np.arange((count + 7) // 8), offset & (2 ** 64 - 1), seed)
    bits = np.stack((words & np.uint64(0xFFFF), words >> np.uint64(16)), 2).reshape(-1)[:count]
    return torch.from_numpy((bits >= int(p * 65536 + 0.5)))


# ---- positions and norms ----------------------------------------------------------------------


def angles(turns, axes, positions):
    """[tokens, pairs] angles from the integer table: exact products, then 64 bits."""
    pairs = len(turns)
    positions = positions.cpu().reshape(-1, axes).tolist()
    out = torch.empty((len(positions), pairs), dtype=torch.float64)
    for t, where in enumerate(positions):
        for j in range(pairs):
            turn = (where[j * axes // pairs] * turns[j]) % 2 ** 64
            out[t, j] = 2 * math.pi * (turn / 2.0 ** 64)
    return out


def split(x, pairs, interleaved):
    return (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])


def turned(x, angle, pairs, interleaved, magnitude, back=False):
    """(result, sum of the absolute terms)"""
    a, b = split(x, pairs, interleaved)
    c, s = angle.cos()[:, None] * magnitude, angle.sin()[:, None] * magnitude * (-1 if back else 1)
    y, size = x.clone(), x.abs()
    ya, yb = split(y, pairs, interleaved)
    za, zb = split(size, pairs, interleaved)
    na, nb = a * c - b * s, a * s + b * c
    most = (a.abs() + b.abs()) * abs(magnitude)
    ya.copy_(na), yb.copy_(nb)
    za.copy_(most), zb.copy_(most)
    return y, size


def normed(x, weight, eps):
    return x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight


def norm_back(x, weight, eps, g):
    """Gradients of normed() for x and weight given g, and the sizes of their terms."""
    d = x.shape[-1]
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n, h = x * r, g * weight
    dot, size = (h * n).sum(-1, keepdim=True) / d, (h * n).abs().sum(-1, keepdim=True) / d
    return r * (h - n * dot), r * (h.abs() + n.abs() * size), (g * n).sum((0, 1)), (g * n).abs().sum((0, 1))


# ---- attention --------------------------------------------------------------------------------


def limits(n, m, mask, prefix):
    """Keys that each of n queries sees of m: those below."""
    own = torch.arange(n) + m - n + 1
    if mask == 0:
        return torch.full((n,), m)
    return torch.maximum(own.clamp(0, m), torch.tensor(min(max(prefix, 0), m) if mask == 2 else 0))


def scores(q, k, mask, prefix, scale, cap, slope):
    """One head of one image: scores (-inf where not seen) and the derivative by the scaled product."""
    n, m = q.shape[0], k.shape[0]
    s = q @ k.t() * scale
    steep = torch.ones_like(s)
    if cap:
        t = torch.tanh(s / cap)
        s, steep = cap * t, 1 - t * t
    if slope:
        s = s - slope * ((torch.arange(n) + m - n)[:, None] - torch.arange(m)).abs()
    return s.masked_fill(torch.arange(m) >= limits(n, m, mask, prefix)[:, None], -math.inf), steep


def weights(s):
    top = s.amax(-1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=s.dtype)
    w = (s - top.clamp(min=-1e300)).exp()
    total = w.sum(-1, keepdim=True)
    return w / total.clamp(min=1e-300), (top + total.log()).squeeze(-1)


def attention(q, k, v, q_first, kv_first, mask, prefix, scale, cap, slopes, dtype, grad=None):
    """Dictionary name -> (result, how far a kernel's may be) for out, lse and, with grad, q_grad, k_grad, v_grad.
    Tokens behind the last image: NaN in the result (not to be looked at)."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    group, u = q.shape[1] // k.shape[1], half(dtype)
    out, spread = torch.full_like(q, math.nan), torch.zeros_like(q)
    lse = torch.full((q.shape[1], q.shape[0]), math.nan, dtype=torch.float64)
    names = {}
    if grad is not None:
        grad = grad.detach().cpu().double()
        names = {"q_grad": (torch.full_like(q, math.nan), torch.zeros_like(q))}
        for name, t in (("k_grad", k), ("v_grad", v)):
            value = torch.full_like(t, math.nan)
            value[:kv_first[-1]] = 0
            names[name] = (value, torch.zeros_like(t))
    for i in range(len(q_first) - 1):
        a, b, c, d = q_first[i], q_first[i + 1], kv_first[i], kv_first[i + 1]
        for h in range(q.shape[1]):
            kv = h // group
            qh, kh, vh = q[a:b, h], k[c:d, kv], v[c:d, kv]
            s, steep = scores(qh, kh, mask, prefix[i] if prefix else 0, scale, cap, slopes[h] if slopes else 0.0)
            w, lse[h, a:b] = weights(s)
            # a narrowed weight is off by a rounding, or in fp16 by half its smallest step where weights (taken
            # against a reference point up to 2^8 below the largest) are tiny
            err = w * (u + 2 * SLACK) + (2.0 ** -25 if dtype == torch.float16 else 0.0) * (s > -math.inf)
            out[a:b, h], spread[a:b, h] = w @ vh, err @ vh.abs()
            if grad is None:
                continue
            g, o = grad[a:b, h], out[a:b, h]
            names["v_grad"][0][c:d, kv] += w.t() @ g
            names["v_grad"][1][c:d, kv] += err.t() @ g.abs()
            delta = (g * o).sum(-1, keepdim=True)
            # the kernel's delta comes from the narrowed results
            delta_err = (g.abs() * (u * o.abs() + spread[a:b, h])).sum(-1, keepdim=True) + SLACK * (g * o).abs().sum(-1, keepdim=True)
            dp = g @ vh.t()
            ds = w * (dp - delta) * steep
            ds_err = ds.abs() * (u + 2 * SLACK) + w * (delta_err + SLACK * (g.abs() @ vh.abs().t()) + 4 * SLACK * (dp - delta).abs())
            if dtype == torch.float16:
                ds_err = ds_err + 2.0 ** -25 * (s > -math.inf)
            names["q_grad"][0][a:b, h] = ds @ kh * scale
            names["q_grad"][1][a:b, h] = ds_err @ kh.abs() * scale
            names["k_grad"][0][c:d, kv] += ds.t() @ qh * scale
            names["k_grad"][1][c:d, kv] += ds_err.t() @ qh.abs() * scale
    names["out"], names["lse"] = (out, spread), (lse, 2.0 ** -16 + 2.0 ** -20 * lse.abs().nan_to_num(0, 0, 0))
    return names
