"""Plain 64-bit forms (numpy, CPU) of the 4-bit generation operators, and the error bounds their tests use."""
import numpy as np
import torch


def f64(t):
    return t.detach().to("cpu").to(torch.float64).numpy()


def bf16(a):
    """Rounds float64 values to bf16 the way the stored scale and mid are: through fp32."""
    return torch.from_numpy(np.asarray(a, np.float64)).to(torch.float32).to(torch.bfloat16).to(torch.float64).numpy()


def quantise(x, group):
    """(codes 0..15, scale, mid, values) of float64 x [..., n]; groups along the last axis."""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    hi, lo = g.max(-1), g.min(-1)
    scale = bf16((hi - lo) / 15.0)
    mid = bf16(0.5 * (hi + lo) + 0.5 * scale)
    s, m = scale[..., None], mid[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s > 0, np.clip(np.rint((g - m) / s) + 8, 0, 15), 8.0)
    return c.reshape(x.shape).astype(np.int64), scale, mid, (s * (c - 8) + m).reshape(x.shape)


def nibbles(codes):
    c = codes.detach().to("cpu").numpy()
    return np.stack([c & 15, c >> 4], -1).reshape(c.shape[:-1] + (-1,)).astype(np.int64)


def split_params(params):
    p = f64(params)
    return p[..., 0], p[..., 1]


def values(codes, params):
    """float64 values of packed codes [..., n / 2] in the order of the codes, with scale and mid per element."""
    c = nibbles(codes)
    s, m = split_params(params)
    rep = c.shape[-1] // s.shape[-1]
    s, m = np.repeat(s, rep, -1), np.repeat(m, rep, -1)
    return s * (c - 8) + m, s, m


def key_dims(d):
    """dim held at every storage position of a key row."""
    return np.array([32 * t + 8 * c + j for c in range(4) for t in range(d // 32) for j in range(8)])


def value_dims(d):
    return np.array([32 * t + 4 * g + j for g in range(8) for t in range(d // 32) for j in range(4)])


def cache_rows(codes, params, dims):
    """Rows of one head in the order of the dims: codes [rows, d / 2] -> (values, codes - 8, scale, mid), each [rows, d]."""
    stored = nibbles(codes)
    c = np.empty_like(stored)
    c[:, dims] = stored
    s, m = split_params(params)
    rep = c.shape[-1] // s.shape[-1]
    s, m = np.repeat(s, rep, -1), np.repeat(m, rep, -1)
    return s * (c - 8) + m, c - 8, s, m


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def gemv(x, w, dtype, norm=False, w2=None, residual=None, fp32_out=False, eps=1e-5):
    """y [n, out] in 64 bits and the bound on its error.

    The kernels hold sums in fp32.  A product of the matrix path is code * x, at most 15 |x| (codes are exact, x is exact in
    fp16 after a power of two down to 2^-30 of the token's largest element), and 8 times the sum of x is taken off per group, so
    all partial sums of an output stay below sum (23 scale + |mid|) |x|; A = sum (56 scale + |mid|) |x| is taken.  Roundings
    follow one another at most r = 8 (matrix steps of a group) + in / group (groups) + 24 (lanes, warps, epilogue) times,
    each off by at most 2^-23 of A (matrix units may truncate): r 2^-23 A.  For outputs in the storage type -8 sum x and
    sum x are held in two bf16 pieces, off by 2^-17: (8 scale + |mid|) 2^-17 sum |x| more, which the part of A between 23 and
    56 covers while |mid| <= 9 scale (r >= 33, and 33 * 33 scale 2^-23 >= 17 scale 2^-17); for fp32 outputs in three (2^-26).
    The CUDA-core form has in / 256 lane steps of eight terms each of size below A / steps, covered by the same bound with
    r' = 8 in / 256 < r.  The row norm is a sum of squares of positive terms in fp32: relative error below
    (in / 32 + 16) 2^-24 / 2 + 2^-22."""
    def one(w):
        v, s, m = values(w.codes, w.params)
        y = x @ v.T
        a = np.abs(x) @ (56 * s + np.abs(m)).T
        steps = 8 + w.in_features / w.group + 24
        return y, steps * 2.0 ** -23 * a
    k = x.shape[1]
    y, e = one(w)
    if norm:
        rs = 1 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
        re = (k / 32 + 16) * 2.0 ** -25 + 2.0 ** -22
        y, e = y * rs, (e + re * np.abs(y)) * rs
    if w2 is not None:
        u, eu = one(w2)
        if norm:
            u, eu = u * rs, (eu + re * np.abs(u)) * rs
        g, eg = y, e
        silu = g / (1 + np.exp(-g))
        # |silu'| <= 1.1; exp and the division of fp32: a few 2^-22
        y = silu * u
        e = (1.1 * eg + 2.0 ** -20 * np.abs(silu)) * (np.abs(u) + eu) + np.abs(silu) * eu
    if residual is not None:
        y = y + residual
        e = e + 2.0 ** -23 * (np.abs(y) + np.abs(residual))
    if not fp32_out:
        e = e * (1 + half_step(dtype)) + half_step(dtype) * np.abs(y)
    return y, e + 1e-30


def attention(q, k_codes, k_params, v_codes, v_params, length, dtype):
    """O [H, d] in 64 bits for one sequence (codes [Hkv, capacity, d / 2]) and the bound on its error.

    bf16: the weight p * scale of a row is rounded once, to fp16 (2^-11 relative; the bound takes bf16's 2^-8), before it meets
    the code, and the -8 multiplies the same rounded weight; p and mid are rounded to bf16 for the mid term (mid exactly
    representable or off by half a step): 2^-8 sum p scale |code| + 2 * 2^-8 sum p |mid|.  The fp32 sums leave 2^-23 per step
    of sum p scale 56 (codes up to 15 and 8 taken off), steps = rows / 16 / 8 + 40.
    Scores: the -8 and mid terms 8 scale |sum q| and |mid| |sum q| go through two bf16 pieces of the sum of q (2^-17 relative;
    the bound takes 2^-16 and 24), the rest through fp32 steps; an error of e in a score moves every weight by a factor within
    exp(+-2 e), which moves an output by at most 2.2 e sum p |v|.  fp32 storage: only the fp32 steps."""
    h, d = q.shape
    hkv = k_codes.shape[0]
    out, bound = np.zeros((h, d)), np.full((h, d), 1e-30)
    if length == 0:
        return out, bound
    low = dtype == torch.bfloat16
    half = half_step(dtype)
    for kv in range(hkv):
        k, kc, ks, km = cache_rows(k_codes[kv, :length], k_params[kv, :length], key_dims(d))
        v, vc, vs, vm = cache_rows(v_codes[kv, :length], v_params[kv, :length], value_dims(d))
        heads = slice(kv * (h // hkv), (kv + 1) * (h // hkv))
        qh = q[heads]
        s = qh @ k.T / np.sqrt(d)
        steps_s = d / 16 + 24
        es = steps_s * 2.0 ** -23 * (np.abs(qh) @ (56 * ks + np.abs(km)).T) / np.sqrt(d)
        if low:
            es = es + 2.0 ** -16 * (np.abs(qh) @ (24 * ks + np.abs(km)).T) / np.sqrt(d)
        # exp2 of fp32: the argument's rounding
        es = es + 2.0 ** -22 * (np.abs(s) + np.abs(s).max(1, keepdims=True) + 16)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        o = p @ v
        steps = length / 128 + 40
        e = steps * 2.0 ** -23 * (p @ (56 * vs + np.abs(vm)))
        if low:
            e = e + half * (p @ (vs * np.abs(vc))) + 2 * half * (p @ np.abs(vm))
        worst = np.minimum(es.max(1, keepdims=True), 0.05)
        e = e + 2.2 * worst * (p @ np.abs(v))
        out[heads] = o
        bound[heads] = e * (1 + half) + half * np.abs(o) + 1e-30
    return out, bound


def logits(x, rules, b, vocab):
    """fp32 steps of one row, token by token as the header defines them; (row, token)."""
    f = np.float32
    l = x.astype(np.float32).copy()
    r = {k: (v.detach().cpu().numpy() if v is not None else None) for k, v in rules.t.items()}
    if r["history"] is not None and any(r[n] is not None for n in ("repetition", "presence", "frequency")):
        i0, i1 = max(0, int(r["history_start"][b])), min(len(r["history"]), int(r["history_start"][b + 1]))
        g0 = int(r["generated_start"][b]) if r["generated_start"] is not None else i0
        count, seen = {}, set()
        for i in range(i0, i1):
            t = int(r["history"][i])
            if 0 <= t < vocab:
                seen.add(t)
                if i >= g0:
                    count[t] = count.get(t, 0) + 1
        rep = f(r["repetition"][b]) if r["repetition"] is not None else f(1)
        fre = f(r["frequency"][b]) if r["frequency"] is not None else f(0)
        pre = f(r["presence"][b]) if r["presence"] is not None else f(0)
        for t in seen:
            l[t] = l[t] / rep if l[t] > 0 else l[t] * rep
        for t, c in count.items():
            l[t] = f(f(l[t] - f(fre * f(c))) - pre)
    if r["bias_token"] is not None:
        i0, i1 = max(0, int(r["bias_start"][b])), min(len(r["bias_token"]), int(r["bias_start"][b + 1]))
        last = {}
        for i in range(i0, i1):
            t = int(r["bias_token"][i])
            if 0 <= t < vocab:
                last[t] = f(r["bias_value"][i])
        for t, v in last.items():
            l[t] = f(l[t] + v)
    if r["mask"] is not None:
        bits = ((r["mask"][b].astype(np.int64)[:, None] >> np.arange(32)) & 1).reshape(-1)[:vocab]
        l[bits == 0] = -np.inf
    c = np.where(np.isnan(l), -np.inf, l)
    return l, (-1 if c.max() == -np.inf else int(c.argmax()))
