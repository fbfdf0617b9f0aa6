"""Cases, plain forms and calls of the 4-bit generation operators: matrix-vector products with 4-bit weights, the
4-bit KV cache (append, and attention of single tokens over it) and the rules a generation puts on its logits.

A 4-bit group holds value = scale * (code - 8) + mid with code in 0..15 and bf16 scale and mid.
  weights    codes [out, in / 2] (element 2i in the low nibble of byte i), params [out, in / group, 2] = (scale, mid)
  KV cache   codes [n_seq, Hkv, capacity, d / 2], params [n_seq, Hkv, capacity, d / group, 2]; within a row of d codes,
             storage position ((c * d / 32) + t) * 8 + j of a key is dim 32 t + 8 c + j (c < 4, j < 8), and position
             ((g * d / 32) + t) * 4 + j of a value is dim 32 t + 4 g + j (g < 8, j < 4)
"""
import math

import torch

own = False

LLAMA = {"heads": 32, "kv_heads": 8, "dim": 128}
QWEN = {"heads": 28, "kv_heads": 4, "dim": 128}
TINY = {"heads": 4, "kv_heads": 2, "dim": 64}


def listed():
    return [
        # one decode token through the 8B output projection, the residual added: latency counts
        {"name": "gemv_1x4096x4096", "op": "gemv", "n": 1, "out": 4096, "in": 4096, "group": 128, "form": "residual", "dtype": "bf16"},
        # the next-token head over the full vocabulary
        {"name": "gemv_1x128256x4096", "op": "gemv", "n": 1, "out": 128256, "in": 4096, "group": 64, "form": "logits", "dtype": "bf16"},
        # eight sequences through the 8B gate and up projections with norm and SwiGLU
        {"name": "gemv_8x14336x4096_swiglu", "op": "gemv", "n": 8, "out": 14336, "in": 4096, "group": 128, "form": "swiglu", "dtype": "bf16"},
        # an odd number of sequences through the wide down projection, fine groups
        {"name": "gemv_21x3584x18944", "op": "gemv", "n": 21, "out": 3584, "in": 18944, "group": 32, "form": "residual", "dtype": "bf16"},
        # one decode step of a running batch: one new row per sequence
        {"name": "append_64x1", "op": "append", **LLAMA, "n_seq": 64, "rows": 1, "capacity": 8192, "group": 32, "dtype": "bf16"},
        # packed prompts of different lengths enter the cache after their prefill
        {"name": "append_8_prompts", "op": "append", **LLAMA, "n_seq": 8, "rows": 4099, "capacity": 16384, "group": 64, "dtype": "bf16"},
        # a short context: latency counts
        {"name": "attention_1x777", "op": "attention", **LLAMA, "n_seq": 1, "longest": 777, "capacity": 1024, "group": 32, "dtype": "bf16"},
        # one very long context
        {"name": "attention_1x131072", "op": "attention", **LLAMA, "n_seq": 1, "longest": 131072, "capacity": 131104, "group": 32, "dtype": "bf16"},
        # a ragged batch with an odd number of query heads per KV head and an empty sequence in it
        {"name": "attention_48_ragged", "op": "attention", **QWEN, "n_seq": 48, "longest": 16384, "capacity": 16384, "group": 64, "dtype": "bf16"},
        # fp32 storage, the small head size
        {"name": "attention_fp32_3x1000", "op": "attention", **TINY, "n_seq": 3, "longest": 1000, "capacity": 1024, "group": 32, "dtype": "fp32"},
        # one generation after a long prompt
        {"name": "logits_1x128256", "op": "logits", "n": 1, "vocab": 128256, "prompt": 32768, "generated": 256, "bias": 20, "grammar": True},
        # a running batch, odd vocabulary
        {"name": "logits_64x152063", "op": "logits", "n": 64, "vocab": 152063, "prompt": 4096, "generated": 1000, "bias": 300, "grammar": True},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gemv", "append", "attention", "logits"])
    if op == "gemv":
        group = rng.choice([32, 64, 128])
        n = _spread(rng, 1, 32)
        k = group * _spread(rng, max(1, 256 // group), 19456 // group)
        out = _spread(rng, 1, min(131072, 500_000_000 // k))
        form = rng.choice(["plain", "residual", "logits", "swiglu"])
        if form == "swiglu":
            out = max(1, out // 2)
        dtype = "bf16"
        if rng.random() < 0.15:
            dtype, out, n = "fp32", min(out, 8192), min(n, 8)
        return {"op": op, "n": n, "out": out, "in": k, "group": group, "form": form, "dtype": dtype}
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 3, 4, 7, 8, 16])
    dim = rng.choice([64, 128])
    group = rng.choice([g for g in (32, 64, 128) if g <= dim])
    if op == "append":
        n_seq = _spread(rng, 1, 256)
        rows = 1 if rng.random() < 0.3 else _spread(rng, 1, max(2, 32768 // n_seq))
        cap = -(-(2 * rows + rng.randrange(0, 1000) + 32) // 32) * 32
        return {"op": op, "heads": heads, "kv_heads": kv, "dim": dim, "n_seq": n_seq, "rows": rows, "capacity": cap, "group": group, "dtype": dtype}
    if op == "attention":
        n_seq = _spread(rng, 1, 128)
        longest = _spread(rng, 1, (16384 if dtype == "fp32" else 131072) // n_seq)
        cap = -(-(longest + rng.randrange(0, 200)) // 32) * 32
        return {"op": op, "heads": heads, "kv_heads": kv, "dim": dim, "n_seq": n_seq, "longest": longest, "capacity": cap, "group": group, "dtype": dtype}
    n = _spread(rng, 1, 64)
    return {"op": op, "n": n, "vocab": _spread(rng, 100, 160000), "prompt": _spread(rng, 1, 131072 // n), "generated": rng.randrange(0, 1200),
            "bias": rng.choice([0, 1, 20, 300]), "grammar": rng.random() < 0.6}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _bytes(shape, gen):
    """Random codes, two to a byte, more in the middle of the range than at its ends."""
    a = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=gen)
    b = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=gen)
    high = ((a >> 4) + (b >> 4)) >> 1
    low = ((a & 15) + (b & 15) + 1) >> 1
    return (high << 4) | low


def _params(shape, scale, gen):
    s = scale * (0.7 + 0.6 * torch.rand(shape, device="cuda", generator=gen))
    m = s * torch.randn(shape, device="cuda", generator=gen)
    return torch.stack([s, m], -1).to(torch.bfloat16)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case, gen):
    """Cache lengths of a ragged batch: one sequence of the longest length, and an empty one where there are several."""
    n, longest = case["n_seq"], case["longest"]
    f = torch.rand(n, device="cuda", generator=gen)
    lens = torch.clamp((longest * f ** 1.5).to(torch.int32), min=1)
    lens[0] = longest
    if n > 2:
        lens[n // 2] = 0
    return lens


def _context(heads, kv_heads, dim, dtype):
    from paper_2601_13155_b200 import binding, synth

    shape = synth.ModelShape(hidden=heads * dim, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=dim, ffn_dim=256, ltp_dlow=64, ltp_rank=16,
                             n_layers=1, vocab=64, dtype=dtype)
    return binding.Spts(shape, max_seq=64), shape


def prepare(case, seed):
    gen = _generator(seed)
    st = {"case": case}
    if case["op"] == "gemv":
        n, o, k, g = case["n"], case["out"], case["in"], case["group"]
        dt = _type(case)
        names = ["w", "w2"] if case["form"] == "swiglu" else ["w"]
        for name in names:
            st[name] = (_bytes((o, k // 2), gen), _params((o, k // g), 0.02 / 3, gen))
        st["x"] = torch.randn(n, k, device="cuda", generator=gen).to(dt)
        st["residual"] = torch.randn(n, o, device="cuda", generator=gen).to(dt) if case["form"] == "residual" else None
        if own:
            from paper_2601_13155_b200 import binding

            st["lib"], _ = _context(4, 2, 64, case["dtype"])
            for name in names:
                st[name] = binding.W4Weight(*st[name])
        return st
    if case["op"] == "logits":
        n, v = case["n"], case["vocab"]
        st["logits"] = 3.0 * torch.randn(n, v, device="cuda", generator=gen)
        lens = (case["prompt"] * (0.5 + 0.5 * torch.rand(n, device="cuda", generator=gen))).to(torch.int64)
        made = (case["generated"] * torch.rand(n, device="cuda", generator=gen)).to(torch.int64)
        lens[0], made[0] = case["prompt"], case["generated"]
        start = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
        start[1:] = torch.cumsum(lens + made, 0)
        total = int(start[-1])
        # tokens of a text: few of them often, many of them seldom
        st["history"] = (v * torch.rand(max(total, 1), device="cuda", generator=gen) ** 4).to(torch.int32).clamp_(max=v - 1)
        st["history_start"] = start.to(torch.int32)
        st["generated_start"] = (start[:-1] + lens).to(torch.int32)
        st["repetition"] = 1.0 + 0.3 * torch.rand(n, device="cuda", generator=gen)
        st["presence"] = torch.rand(n, device="cuda", generator=gen)
        st["frequency"] = 0.5 * torch.rand(n, device="cuda", generator=gen)
        b = case["bias"]
        st["bias_start"] = (torch.arange(n + 1, device="cuda") * b).to(torch.int32)
        st["bias_token"] = torch.randint(0, v, (max(n * b, 1),), dtype=torch.int32, device="cuda", generator=gen)
        st["bias_value"] = 4.0 * torch.randn(max(n * b, 1), device="cuda", generator=gen)
        st["mask"] = None
        if case["grammar"]:
            words = (v + 31) // 32
            m = torch.randint(-2 ** 31, 2 ** 31, (n, words), dtype=torch.int64, device="cuda", generator=gen)
            m &= torch.randint(-2 ** 31, 2 ** 31, (n, words), dtype=torch.int64, device="cuda", generator=gen)
            m = m.to(torch.int32)
            if n > 2:
                m[n // 2] = 0              # a state of the grammar that allows no token
            st["mask"] = m
        if own:
            from paper_2601_13155_b200 import binding

            st["lib"], _ = _context(4, 2, 64, "bf16")
            st["rules"] = binding.LogitsRules(
                history=st["history"], history_start=st["history_start"], generated_start=st["generated_start"], repetition=st["repetition"],
                presence=st["presence"], frequency=st["frequency"], bias_token=st["bias_token"] if b else None,
                bias_value=st["bias_value"] if b else None, bias_start=st["bias_start"] if b else None, mask=st["mask"])
        return st
    n, hkv, cap, d, g = case["n_seq"], case["kv_heads"], case["capacity"], case["dim"], case["group"]
    dt = _type(case)
    for name in ("k", "v"):
        st[name + "_codes"] = _bytes((n, hkv, cap, d // 2), gen)
        st[name + "_params"] = _params((n, hkv, cap, d // g), 0.35, gen)
    if case["op"] == "attention":
        st["len"] = _lengths(case, gen)
        behind = torch.arange(cap, device="cuda")[None, :] >= st["len"][:, None]
        for name in ("k_params", "v_params"):       # nothing has been written behind a sequence's end
            st[name].masked_fill_(behind[:, None, :, None, None], float("nan"))
        st["q"] = torch.randn(n, case["heads"], d, device="cuda", generator=gen).to(dt)
    else:
        rows = torch.ones(n, device="cuda", dtype=torch.int64)
        if case["rows"] > 1:
            # one prompt of the full length; of two others one is as much longer than half of it as the other is shorter
            half = case["rows"] // 2
            rows.fill_(half)
            rows[0] = case["rows"]
            pairs = (n - 1) // 2
            off = (half * torch.rand(pairs, device="cuda", generator=gen)).to(torch.int64)
            rows[1:1 + pairs] += off
            rows[1 + pairs:1 + 2 * pairs] -= off
        room = (cap - rows).clamp(min=0)
        at = (room * torch.rand(n, device="cuda", generator=gen)).to(torch.int64)
        if case["rows"] > 1:
            at.zero_()
        st["at"] = at.to(torch.int32)
        start = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
        start[1:] = torch.cumsum(rows, 0)
        st["row_start"] = start.to(torch.int32)
        total = int(start[-1])
        st["k"] = torch.randn(total, hkv, d, device="cuda", generator=gen).to(dt)
        st["v"] = torch.randn(total, hkv, d, device="cuda", generator=gen).to(dt)
        st["k_read"] = torch.empty_like(st["k"])
        st["v_read"] = torch.empty_like(st["v"])
        st["len"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    if own:
        from paper_2601_13155_b200 import binding

        st["lib"], shape = _context(case["heads"], hkv, d, case["dtype"])
        st["cache"] = binding.Kv4Cache(shape, n, cap, group=g, k_codes=st["k_codes"], v_codes=st["v_codes"], k_params=st["k_params"],
                                       v_params=st["v_params"], length=st["len"])
    return st


def run(state):
    return {"gemv": _gemv, "append": _append, "attention": _attention, "logits": _logits}[state["case"]["op"]](state)


def _nibbles(codes):
    return torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)


def _values(codes, params):
    """scale * (code - 8) + mid, in 32 bits, of codes [..., n] with params [..., n / group, 2]."""
    groups = params.shape[-2]
    c = codes.to(torch.float32).reshape(*codes.shape[:-1], groups, -1) - 8.0
    p = params.to(torch.float32)
    return (c * p[..., 0:1] + p[..., 1:2]).reshape(codes.shape)


def _gemv(st):
    form, x = st["case"]["form"], st["x"]
    if own:
        if form == "swiglu":
            return st["lib"].w4_gemv(st["w"], x, w2=st["w2"], norm=True)
        if form == "residual":
            return st["lib"].w4_gemv(st["w"], x, residual=st["residual"])
        if form == "logits":
            return st["lib"].w4_gemv(st["w"], x, norm=True, fp32_out=True)
        return st["lib"].w4_gemv(st["w"], x)
    x32 = x.to(torch.float32)
    y = x32 @ _values(_nibbles(st["w"][0]), st["w"][1]).T
    if form in ("swiglu", "logits"):
        rs = 1.0 / torch.sqrt((x32 * x32).mean(-1, keepdim=True) + 1e-5)
        y = y * rs
    if form == "swiglu":
        u = (x32 @ _values(_nibbles(st["w2"][0]), st["w2"][1]).T) * rs
        y = y / (1.0 + torch.exp(-y)) * u
    if form == "residual":
        y = st["residual"].to(torch.float32) + y
    return y if form == "logits" else y.to(x.dtype)


def _key_order(d):
    return torch.arange(d, device="cuda").reshape(d // 32, 4, 8).permute(1, 0, 2).reshape(d)        # dim at storage position


def _value_order(d):
    return torch.arange(d, device="cuda").reshape(d // 32, 8, 4).permute(1, 0, 2).reshape(d)


def _quantise(x, group):
    """Codes, params and the values they stand for.  The border between two codes is found in 64 bits."""
    d = x.shape[-1]
    x64 = x.to(torch.float64).reshape(*x.shape[:-1], d // group, group)
    hi, lo = x64.amax(-1, keepdim=True), x64.amin(-1, keepdim=True)
    s = ((hi - lo) / 15.0).to(torch.float32).to(torch.bfloat16)
    m = (0.5 * (hi + lo) + 0.5 * s.to(torch.float64)).to(torch.float32).to(torch.bfloat16)
    s64, m64 = s.to(torch.float64), m.to(torch.float64)
    c = torch.clamp(torch.round((x64 - m64) / torch.where(s64 > 0, s64, 1.0)) + 8.0, 0.0, 15.0)
    c = torch.where(s64 > 0, c, 8.0)
    read = (s64 * (c - 8.0) + m64).to(torch.float32)
    return c.reshape(x.shape).to(torch.uint8), torch.cat([s, m], -1), read.reshape(x.shape)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _append(st):
    case = st["case"]
    if own:
        st["lib"].kv4_append(st["cache"], st["k"], st["v"], at=st["at"], row_start=st["row_start"], K_out=st["k_read"], V_out=st["v_read"])
        return {"k_read": st["k_read"], "v_read": st["v_read"], "len": st["len"]}
    d, g, n = case["dim"], case["group"], case["n_seq"]
    start = st["row_start"].to(torch.int64)
    row = torch.arange(st["k"].shape[0], device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), row, right=True)
    slot = st["at"].to(torch.int64)[seq] + row - start[seq]
    for name, order in (("k", _key_order(d)), ("v", _value_order(d))):
        codes, params, read = _quantise(st[name], g)
        st[name + "_codes"][seq, :, slot] = _pack(codes[..., order])
        st[name + "_params"][seq, :, slot] = params
        st[name + "_read"].copy_(read)
    st["len"].copy_((st["at"].to(torch.int64) + start[1:] - start[:-1]).to(torch.int32))
    return {"k_read": st["k_read"], "v_read": st["v_read"], "len": st["len"]}


def _attention(st):
    case, q = st["case"], st["q"]
    if own:
        return st["lib"].kv4_attention(st["cache"], q)
    n, h, hkv, d, cap = case["n_seq"], case["heads"], case["kv_heads"], case["dim"], case["capacity"]
    out = torch.zeros(n, h * d, dtype=q.dtype, device="cuda")
    back_k, back_v = torch.argsort(_key_order(d)), torch.argsort(_value_order(d))
    places = torch.arange(cap, device="cuda")
    # as many sequences at a time as stay below some gigabytes of values
    step = max(1, min(n, (1 << 28) // (hkv * cap * d)))
    for b in range(0, n, step):
        s = slice(b, min(b + step, n))
        held = (places[None, :] < st["len"][s, None])[:, None, :]
        k = _values(_nibbles(st["k_codes"][s])[..., back_k], st["k_params"][s])
        v = _values(_nibbles(st["v_codes"][s])[..., back_v], st["v_params"][s])
        v = torch.where(held[..., None], v, 0.0)
        qf = q[s].to(torch.float32).reshape(-1, hkv, h // hkv, d)
        a = (qf @ k.transpose(-1, -2)) / math.sqrt(d)
        a = torch.where(held[:, :, None, :], a, float("-inf"))
        top = a.amax(-1, keepdim=True)
        p = torch.exp(a - torch.where(top == float("-inf"), 0.0, top))
        o = (p @ v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
        out[s] = o.reshape(-1, h * d).to(q.dtype)
    return out


def _logits(st):
    if own:
        out, token = st["lib"].process_logits(st["logits"], st["rules"])
        return {"logits": out, "token": token}
    case, x = st["case"], st["logits"]
    n, v = x.shape
    start, made = st["history_start"].to(torch.int64), st["generated_start"].to(torch.int64)
    total = int(case["prompt"]) + int(case["generated"])
    place = torch.arange(max(total, 1), device="cuda")[None, :]
    at = start[:-1, None] + place
    inside = at < start[1:, None]
    token = st["history"][at.clamp(max=st["history"].shape[0] - 1)].to(torch.int64)
    seen = torch.zeros(n, v, device="cuda").scatter_add_(1, token, inside.to(torch.float32))
    count = torch.zeros(n, v, device="cuda").scatter_add_(1, token, (inside & (at >= made[:, None])).to(torch.float32))
    r = st["repetition"][:, None]
    y = torch.where(seen > 0, torch.where(x > 0, x / r, x * r), x)
    y = y - st["frequency"][:, None] * count
    y = y - st["presence"][:, None] * (count > 0).to(torch.float32)
    b = case["bias"]
    if b:
        # of two entries for one token the later counts
        key = st["bias_token"][: n * b].to(torch.int64).reshape(n, b)
        last = torch.full((n, v), -1, dtype=torch.int64, device="cuda")
        last.scatter_reduce_(1, key, torch.arange(n * b, device="cuda").reshape(n, b), "amax")
        y = torch.where(last >= 0, y + st["bias_value"][last.clamp(min=0)], y)
    if st["mask"] is not None:
        bits = torch.arange(v, device="cuda")
        allowed = (st["mask"][:, bits >> 5] >> (bits & 31).to(torch.int32)) & 1
        y = torch.where(allowed > 0, y, float("-inf"))
    best = torch.argmax(y, -1).to(torch.int32)
    best = torch.where(y.amax(-1) == float("-inf"), -1, best)
    return {"logits": y, "token": best.to(torch.int32)}


def work(case):
    """Bytes and operations of one pass that no way of computing it can do without."""
    op = case["op"]
    if op == "gemv":
        n, o, k, g = case["n"], case["out"], case["in"], case["group"]
        e = 2 if case["dtype"] == "bf16" else 4
        m = 2 if case["form"] == "swiglu" else 1
        y = n * o * (4 if case["form"] == "logits" else 2 * e if case["form"] == "residual" else e)
        return {"bytes": m * o * (k // 2 + 4 * (k // g)) + n * k * e + y, "flops": 2.0 * m * n * o * k}
    if op == "logits":
        n, v = case["n"], case["vocab"]
        return {"bytes": n * (8 * v + (v // 8 if case["grammar"] else 0) + 8 * case["bias"]) + n * 4 * (0.75 * case["prompt"] + 0.5 * case["generated"]),
                "flops": 6.0 * n * v}
    hkv, d, g = case["kv_heads"], case["dim"], case["group"]
    e = 2 if case["dtype"] == "bf16" else 4
    row = 2 * hkv * (d // 2 + 4 * (d // g))
    if op == "append":
        rows = case["n_seq"] if case["rows"] == 1 else case["rows"] + case["rows"] // 2 * (case["n_seq"] - 1)
        return {"bytes": rows * (row + 4 * hkv * d * e), "flops": rows * 2 * hkv * d * 6.0}
    rows = case["longest"] * (1 + 0.4 * (case["n_seq"] - 1))
    return {"bytes": rows * row + 2 * case["n_seq"] * case["heads"] * d * e, "flops": 4.0 * rows * case["heads"] * d}


def _exact_values(codes, params, group):
    """The values in 64 bits, element by element from the two nibbles of every byte (natural order of positions)."""
    low, high = (codes % 16).to(torch.float64), torch.div(codes, 16, rounding_mode="floor").to(torch.float64)
    flat = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    flat[..., 0::2], flat[..., 1::2] = low, high
    return flat


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    op = case["op"]
    if op == "gemv":
        x = st["x"].to(torch.float64)
        k, g = case["in"], case["group"]

        def product(w):
            codes, params = w
            out = []
            for rows in range(0, case["out"], 8192):
                c = _exact_values(codes[rows:rows + 8192], None, g) - 8.0
                p = params[rows:rows + 8192].to(torch.float64)
                scale = p[..., 0].repeat_interleave(g, -1)
                mid = p[..., 1].repeat_interleave(g, -1)
                out.append(torch.matmul(x, (c * scale + mid).transpose(0, 1)))
            return torch.cat(out, 1)

        y = product(st["w"])
        norm = (x.pow(2).sum(1, keepdim=True) / k + 1e-5).rsqrt()
        if case["form"] == "logits":
            return y * norm
        if case["form"] == "swiglu":
            gate = y * norm
            return gate * torch.sigmoid(gate) * (product(st["w2"]) * norm)
        return y + st["residual"].to(torch.float64) if case["form"] == "residual" else y
    if op == "append":
        g = case["group"]
        got = {}
        for name in ("k", "v"):
            x = st[name].to(torch.float64).unflatten(-1, (-1, g))
            top, bottom = x.max(-1, keepdim=True).values, x.min(-1, keepdim=True).values
            scale = ((top - bottom) / 15).float().bfloat16().double()
            mid = ((top + bottom) / 2 + scale / 2).float().bfloat16().double()
            steps = torch.round((x - mid) / scale).nan_to_num(0.0).clamp(-8, 7)
            got[name + "_read"] = (mid + scale * steps).flatten(-2)
        got["len"] = (st["at"] + st["row_start"][1:] - st["row_start"][:-1]).to(torch.int32)
        return got
    if op == "attention":
        n, h, hkv, d, g = case["n_seq"], case["heads"], case["kv_heads"], case["dim"], case["group"]
        out = torch.zeros(n, h, d, dtype=torch.float64, device="cuda")
        for b, ln in enumerate(st["len"].tolist()):
            if ln == 0:
                continue
            for kv in range(hkv):
                rows = []
                for name, lanes, run_ in (("k", 4, 8), ("v", 8, 4)):
                    c = _exact_values(st[name + "_codes"][b, kv, :ln], None, g) - 8.0
                    c = c.reshape(ln, lanes, d // 32, run_).transpose(1, 2).reshape(ln, d)
                    p = st[name + "_params"][b, kv, :ln].to(torch.float64)
                    rows.append(c * p[..., 0].repeat_interleave(g, -1) + p[..., 1].repeat_interleave(g, -1))
                heads = slice(kv * (h // hkv), (kv + 1) * (h // hkv))
                a = torch.softmax(st["q"][b, heads].to(torch.float64) @ rows[0].T * d ** -0.5, -1)
                out[b, heads] = a @ rows[1]
        return out.reshape(n, h * d)
    x = st["logits"].to(torch.float64).clone()
    start, made = st["history_start"].tolist(), st["generated_start"].tolist()
    best = []
    for i in range(case["n"]):
        hist = st["history"][start[i]:start[i + 1]].long()
        count = torch.bincount(st["history"][made[i]:start[i + 1]].long(), minlength=case["vocab"]).double()
        seen = torch.unique(hist)
        r = st["repetition"][i].double()
        x[i, seen] = torch.where(x[i, seen] > 0, x[i, seen] / r, x[i, seen] * r)
        x[i] -= st["frequency"][i].double() * count + st["presence"][i].double() * (count > 0)
        entries = {}
        b0 = i * case["bias"]
        for t, value in zip(st["bias_token"][b0:b0 + case["bias"]].tolist(), st["bias_value"][b0:b0 + case["bias"]].tolist()):
            entries[t] = value
        if entries:
            x[i, list(entries)] += torch.tensor(list(entries.values()), dtype=torch.float64, device="cuda")
        if st["mask"] is not None:
            shifts = torch.arange(32, device="cuda", dtype=torch.int64)
            bits = ((st["mask"][i].long()[:, None] >> shifts) & 1).reshape(-1)[: case["vocab"]]
            x[i, bits == 0] = float("-inf")
        top = x[i].max()
        best.append(-1 if top == float("-inf") else int((x[i] == top).nonzero()[0]))
    return {"logits": x, "token": torch.tensor(best, dtype=torch.int32, device="cuda")}
