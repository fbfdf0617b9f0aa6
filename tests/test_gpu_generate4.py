"""Generation with 4-bit weights and caches: quantiser, matrix-vector products, cache append, attention over the cache and
the rules on logits, each against a plain 64-bit form."""
import ctypes as C
from dataclasses import replace

import numpy as np
import pytest
import torch

import generate4_ref as R
from paper_2601_13155_b200 import synth
from parity_utils import Guarded, dev, i32

pytestmark = pytest.mark.gpu

BF16 = replace(synth.LLAMA8B, hidden=256, n_q_heads=8, n_kv_heads=2, head_dim=128, ffn_dim=256, ltp_dlow=64, ltp_rank=16, n_layers=1,
               vocab=64)


def shape_of(heads=8, kv_heads=2, dim=128, dtype="bf16"):
    return replace(BF16, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=dim, dtype=dtype)


def context(shape=BF16, plain=False):
    from paper_2601_13155_b200 import binding
    lib = binding.Spts(shape, max_seq=64)
    if plain and shape.dtype == "bf16" and shape.head_dim == 128:
        lib.set_reference_kernels(True)
    return lib


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand_w4(out, k, group, seed, mids=True):
    from paper_2601_13155_b200 import binding
    g = gen(seed)
    codes = torch.randint(0, 256, (out, k // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = 0.01 * (0.2 + torch.rand(out, k // group, device="cuda", generator=g))
    m = s * torch.randn(out, k // group, device="cuda", generator=g) * (1.0 if mids else 0.0)
    return binding.W4Weight(codes, torch.stack([s, m], -1).to(torch.bfloat16))


def close(got, want, bound, what):
    got = R.f64(got)
    assert np.isfinite(got).all(), f"{what}: non-finite output"
    over = np.abs(got - want) / bound
    assert over.max() <= 1.0, f"{what}: error {np.abs(got - want).max():.3e}, {over.max():.3f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


# ---------------------------------------------------------------------------------------------- quantiser
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("out,k,group", [(1, 32, 32), (3, 96, 32), (5, 256, 128), (33, 192, 64), (257, 4096, 128)])
def test_quantised_weights_are_the_exact_ones(out, k, group, dtype):
    lib = context(shape_of(dtype=dtype))
    W = (torch.randn(out, k, device="cuda", generator=gen(out + k)) * 0.02).to(lib.dtype)
    if out > 2:
        W[0, :group] = 0.5                          # one value: scale 0
        W[1, :group] = torch.linspace(-8, 7, group, device="cuda").round().to(lib.dtype)    # every border a tie or a code
        W[2] *= 1e-20
    w = lib.w4_quantize(W, group)
    codes, scale, mid, _ = R.quantise(R.f64(W), group)
    s, m = R.split_params(w.params)
    assert np.array_equal(s, scale) and np.array_equal(m, mid)
    assert np.array_equal(R.nibbles(w.codes), codes)
    assert lib.device_status() == 0
    lib.close()


def test_quantiser_ties_go_to_even():
    """Halves of a step everywhere: the exact quotient decides, not an approximate one."""
    lib = context()
    x = torch.empty(8, 128)
    for r in range(8):
        x[r] = (torch.arange(128) % 31) * 0.5 * 2.0 ** -r           # range 15 steps of 2^-r, elements on halves of a step
    W = x.to(torch.bfloat16).cuda()
    w = lib.w4_quantize(W, 128)
    codes, scale, mid, _ = R.quantise(R.f64(W), 128)
    assert np.array_equal(R.nibbles(w.codes), codes)
    assert np.array_equal(R.split_params(w.params)[0], scale)
    lib.close()


def test_non_finite_weights_are_reported():
    lib = context()
    for bad in (float("nan"), float("inf"), -float("inf")):
        W = torch.randn(4, 128, device="cuda").to(torch.bfloat16)
        W[2, 40] = bad
        w = lib.w4_quantize(W, 32)
        assert lib.device_status() == 6 and lib.device_status() == 0
        s, m = R.split_params(w.params)
        assert s[2, 1] == 0 and np.isnan(m[2, 1])
        keep = np.ones((4, 4), bool)
        keep[2, 1] = False
        assert np.isfinite(m[keep]).all()
    lib.close()


# ---------------------------------------------------------------------------------------------- matrix-vector products
GEMV_CASES = [  # n, out, in, group
    (1, 1, 32, 32), (1, 7, 64, 64), (1, 16, 128, 128), (1, 17, 4096, 128), (1, 250, 1056, 32), (1, 4100, 768, 64),
    (2, 33, 192, 64), (8, 64, 4096, 128), (9, 65, 384, 128), (16, 48, 544, 32), (21, 129, 2048, 32), (32, 31, 1152, 64),
    (1, 3, 19456, 128), (5, 1030, 160, 32), (32, 300, 14336, 128),
]


@pytest.mark.parametrize("dtype,plain", [("bf16", False), ("bf16", True), ("fp32", False)])
@pytest.mark.parametrize("n,out,k,group", GEMV_CASES)
def test_gemv_forms(n, out, k, group, dtype, plain):
    lib = context(shape_of(dtype=dtype), plain)
    w, w2 = rand_w4(out, k, group, 7 * n + out), rand_w4(out, k, group, 11 * n + out, mids=False)
    x = torch.randn(n, k, device="cuda", generator=gen(n + k)).to(lib.dtype)
    r = torch.randn(n, out, device="cuda", generator=gen(n + 1)).to(lib.dtype)
    xr, rr = R.f64(x), R.f64(r)
    eps = lib.shape.rms_eps
    y, e = R.gemv(xr, w, lib.dtype)
    close(lib.w4_gemv(w, x), y, e, "plain")
    y, e = R.gemv(xr, w, lib.dtype, norm=True, fp32_out=True, eps=eps)
    close(lib.w4_gemv(w, x, norm=True, fp32_out=True), y, e, "logits")
    y, e = R.gemv(xr, w, lib.dtype, norm=True, w2=w2, eps=eps)
    close(lib.w4_gemv(w, x, w2=w2, norm=True), y, e, "swiglu")
    y, e = R.gemv(xr, w, lib.dtype, residual=rr)
    close(lib.w4_gemv(w, x, residual=r), y, e, "residual")
    got = lib.w4_gemv(w, x, residual=r, out=r)                       # in place
    assert got is r
    close(r, y, e, "residual in place")
    assert lib.device_status() == 0 and lib.check_guards() == 0
    lib.close()


def test_gemv_strided_rows_and_guarded_output():
    lib = context()
    w = rand_w4(50, 256, 64, 3)
    wide = torch.randn(3, 4 * 256 + 8, device="cuda", generator=gen(5)).to(torch.bfloat16)
    x = wide[:, 264:520]
    g = Guarded((3, 70), torch.bfloat16)
    g.t.fill_(7.0)
    lib.w4_gemv(w, x, out=g.t[:, :50])
    y, e = R.gemv(R.f64(x), w, torch.bfloat16)
    close(g.t[:, :50], y, e, "strided")
    assert g.intact() and bool((g.t[:, 50:] == 7.0).all())
    lib.close()


def test_gemv_non_finite_input_reaches_its_own_row_only():
    lib = context()
    w = rand_w4(40, 256, 64, 3)
    x = torch.randn(4, 256, device="cuda", generator=gen(5)).to(torch.bfloat16)
    clean = lib.w4_gemv(w, x)
    x[2, 100] = float("inf")
    y = lib.w4_gemv(w, x)
    assert not torch.isfinite(y[2]).any()
    keep = torch.tensor([0, 1, 3], device="cuda")
    assert torch.equal(y[keep], clean[keep])
    lib.close()


def test_gemv_refusals():
    from paper_2601_13155_b200 import binding
    lib = context()
    w, w2 = rand_w4(16, 256, 64, 1), rand_w4(16, 256, 128, 2)
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    r = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda")
    assert lib.w4_gemv(w, x[:0]).shape == (0, 16)
    for call in (lambda: lib.w4_gemv(w, torch.zeros(33, 256, dtype=torch.bfloat16, device="cuda")),
                 lambda: lib.w4_gemv(w, x, w2=w2), lambda: lib.w4_gemv(w, x, w2=w, residual=r),
                 lambda: lib.w4_gemv(w, x, residual=r, fp32_out=True),
                 lambda: lib.w4_gemv(w, torch.zeros(4, 260, dtype=torch.bfloat16, device="cuda")[:, 3:259])):
        with pytest.raises(binding.SptsError):
            call()
    for call in (lambda: lib.w4_gemv(w, x.float()), lambda: lib.w4_gemv(w, x[:, :128]), lambda: lib.w4_gemv(w, x.cpu()),
                 lambda: lib.w4_gemv(w, x, residual=r[:2]), lambda: lib.w4_gemv(w, x.t().contiguous().t()),
                 lambda: lib.w4_quantize(x[:, :100].contiguous(), 32), lambda: lib.w4_quantize(x, 16)):
        with pytest.raises(ValueError):
            call()
    c = binding.W4C(w.codes.data_ptr(), w.params.data_ptr(), 16, 256, 48)
    args = (C.c_void_p(x.data_ptr()), 256, 1, None, 0)
    assert lib.lib.spts_w4_gemv(lib.h, C.byref(c), None, *args, 0, C.c_void_p(r.data_ptr()), 16) == 2
    assert lib.lib.spts_w4_gemv(lib.h, C.byref(w.c), None, *args, 8, C.c_void_p(r.data_ptr()), 16) == 1
    assert lib.lib.spts_w4_gemv(lib.h, C.byref(w.c), None, *args, 0, None, 16) == 1
    lib.close()


# ---------------------------------------------------------------------------------------------- cache append
def fill_garbage(cache, seed):
    """Codes at random and NaN params: what memory nobody has written may hold."""
    g = gen(seed)
    for t in (cache.k_codes, cache.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, dtype=torch.uint8, device="cuda", generator=g))
    for t in (cache.k_params, cache.v_params):
        t.fill_(float("nan"))


def check_rows(cache, which, rows64, seq, slot, group, dim):
    """The slots (seq, slot) of the cache hold the exact quantisation of rows64 [len, Hkv, d]."""
    codes_t, params_t = (cache.k_codes, cache.k_params) if which == "k" else (cache.v_codes, cache.v_params)
    order = R.key_dims(dim) if which == "k" else R.value_dims(dim)
    codes, scale, mid, vals = R.quantise(rows64, group)
    s, m = R.split_params(params_t[seq, :, slot])
    assert np.array_equal(s, scale) and np.array_equal(m, mid)
    assert np.array_equal(R.nibbles(codes_t[seq, :, slot]), codes[..., order])
    return vals


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv_heads,dim,group", [(1, 64, 32), (2, 64, 64), (3, 128, 32), (8, 128, 64), (2, 128, 128)])
def test_append_packed_prompts_then_single_rows(kv_heads, dim, group, dtype):
    from paper_2601_13155_b200 import binding
    shape = shape_of(kv_heads * 2, kv_heads, dim, dtype)
    lib = context(shape)
    lens, pad = [5, 0, 33, 1, 70], 4
    total = sum(lens)
    cache = binding.Kv4Cache(shape, 5, 96, group=group, positions=True)
    fill_garbage(cache, 1)
    before = [t.clone() for t in (cache.k_codes, cache.v_codes)]
    K = (2.0 * torch.randn(total + pad, kv_heads, dim, device="cuda", generator=gen(2)) + 0.3).to(lib.dtype)
    V = torch.randn(total + pad, kv_heads, dim, device="cuda", generator=gen(3)).to(lib.dtype)
    pos = i32(np.arange(total + pad) * 3)
    start = i32(np.concatenate([[0], np.cumsum(lens)]))
    kr, vr = Guarded(K.shape, lib.dtype), Guarded(K.shape, lib.dtype)
    kr.t.fill_(9.0), vr.t.fill_(9.0)
    lib.kv4_append(cache, K, V, pos=pos, row_start=start, at=i32([0, 7, 2, 0, 20]), K_out=kr.t, V_out=vr.t)
    assert lib.device_status() == 0
    assert cache.length.tolist() == [5, 7, 35, 1, 90]
    written = np.zeros((5, 96), bool)
    at = [0, 7, 2, 0, 20]
    for b, n in enumerate(lens):
        seq = torch.full((n,), b, device="cuda")
        slot = torch.arange(at[b], at[b] + n, device="cuda")
        rows = slice(sum(lens[:b]), sum(lens[:b]) + n)
        written[b, at[b]:at[b] + n] = True
        if n == 0:
            continue
        assert cache.pos[b, at[b]:at[b] + n].tolist() == pos[rows].tolist()
        for which, src, read in (("k", K, kr), ("v", V, vr)):
            vals = check_rows(cache, which, R.f64(src[rows]), seq, slot, group, dim)
            want = torch.from_numpy(vals).to(torch.float32).to(lib.dtype)
            assert torch.equal(read.t[rows].cpu(), want)
    assert bool((kr.t[total:] == 9.0).all()) and bool((vr.t[total:] == 9.0).all()) and kr.intact() and vr.intact()
    keep = torch.from_numpy(~written).cuda()
    for t, old in zip((cache.k_codes, cache.v_codes), before):
        assert torch.equal(t.transpose(1, 2)[keep], old.transpose(1, 2)[keep])
    # single rows behind what is held, from strided views of one wider matrix
    wide = torch.randn(5, 3 * kv_heads * dim, device="cuda", generator=gen(4)).to(lib.dtype)
    k1, v1 = wide[:, kv_heads * dim:2 * kv_heads * dim], wide[:, 2 * kv_heads * dim:]
    lib.kv4_append(cache, k1, v1)
    assert cache.length.tolist() == [6, 8, 36, 2, 91]
    seq, slot = torch.arange(5, device="cuda"), (cache.length - 1).long()
    check_rows(cache, "k", R.f64(k1).reshape(5, kv_heads, dim), seq, slot, group, dim)
    check_rows(cache, "v", R.f64(v1).reshape(5, kv_heads, dim), seq, slot, group, dim)
    assert lib.device_status() == 0
    lib.close()


def test_append_without_room_and_with_bad_slots():
    from paper_2601_13155_b200 import binding
    lib = context()
    cache = binding.Kv4Cache(BF16, 3, 32, group=32)
    fill_garbage(cache, 1)
    before = cache.k_codes.clone()
    K = torch.randn(9, 2, 128, device="cuda", generator=gen(2)).to(torch.bfloat16)
    lib.kv4_append(cache, K, K, row_start=i32([0, 3, 6, 9]), at=i32([30, -2, 5]))
    assert lib.device_status() == 3 and lib.device_status() == 0
    assert cache.length.tolist() == [32, 1, 8]
    changed = (cache.k_codes != before).any(-1).any(1)
    want = torch.zeros(3, 32, dtype=torch.bool, device="cuda")
    want[0, 30:32] = True
    want[1, 0] = True
    want[2, 5:8] = True
    assert torch.equal(changed, want)
    cache.length.copy_(i32([32, 31, -5]))
    lib.kv4_append(cache, K[:3], K[:3])
    assert lib.device_status() == 3
    assert cache.length.tolist() == [32, 32, 0]
    lib.close()


def test_append_non_finite_rows_and_refusals():
    from paper_2601_13155_b200 import binding
    lib = context()
    cache = binding.Kv4Cache(BF16, 2, 40, group=64)
    assert cache.capacity == 64
    K = torch.randn(2, 2, 128, device="cuda").to(torch.bfloat16)
    V = K.clone()
    V[1, 1, 70] = float("nan")
    lib.kv4_append(cache, K, V)
    assert lib.device_status() == 6
    s, m = R.split_params(cache.v_params[1, 1, 0])
    assert s[1] == 0 and np.isnan(m[1]) and np.isfinite(m[0])
    for call in (lambda: lib.kv4_append(cache, K[:1], V[:1]),):
        with pytest.raises(binding.SptsError):
            call()
    other = binding.Kv4Cache(shape_of(kv_heads=4), 2, 32)
    for call in (lambda: lib.kv4_append(other, K, V), lambda: lib.kv4_append(cache, K.float(), V), lambda: lib.kv4_append(cache, K, V[:1]),
                 lambda: lib.kv4_append(cache, K, V, at=i32([0])), lambda: lib.kv4_append(cache, K, V, row_start=i32([0, 1])),
                 lambda: lib.kv4_attention(cache, K), lambda: binding.Kv4Cache(BF16, 2, 32, group=48),
                 lambda: binding.Kv4Cache(shape_of(dim=64), 2, 32, group=128)):
        with pytest.raises(ValueError):
            call()
    c = cache.c
    bad = binding.Kv4CacheC(c.k_codes, c.v_codes, c.k_params, c.v_params, None, c.len, 2, 40, 64)
    q, o = torch.zeros(2, 1024, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1024, dtype=torch.bfloat16, device="cuda")
    ptr = lambda t: C.c_void_p(t.data_ptr())
    assert lib.lib.spts_kv4_attention(lib.h, C.byref(bad), ptr(q), 1024, ptr(o), 1024) == 2
    bad = binding.Kv4CacheC(c.k_codes, c.v_codes, c.k_params, c.v_params, None, None, 2, 64, 64)
    assert lib.lib.spts_kv4_attention(lib.h, C.byref(bad), ptr(q), 1024, ptr(o), 1024) == 1
    assert lib.lib.spts_kv4_attention(lib.h, C.byref(c), ptr(q), 1000, ptr(o), 1024) == 1
    assert lib.lib.spts_kv4_attention(lib.h, C.byref(c), ptr(q), 1024, ptr(q), 1024) == 1
    lib.close()


# ---------------------------------------------------------------------------------------------- attention over the cache
def random_cache(shape, n_seq, capacity, group, lens, seed, k_scale=0.3):
    from paper_2601_13155_b200 import binding
    cache = binding.Kv4Cache(shape, n_seq, capacity, group=group)
    fill_garbage(cache, seed)
    g = gen(seed + 1)
    for t, base in ((cache.k_params, k_scale), (cache.v_params, 0.3)):
        s = base * (0.5 + torch.rand(t.shape[:-1], device="cuda", generator=g))
        m = s * torch.randn(t.shape[:-1], device="cuda", generator=g)
        held = torch.arange(cache.capacity, device="cuda")[None] < i32(lens)[:, None]
        p = torch.stack([s, m], -1).to(torch.bfloat16)
        t.copy_(torch.where(held[:, None, :, None, None], p, t))
    cache.length.copy_(i32(lens))
    return cache


def check_attention(lib, cache, q, out, lens):
    shape = lib.shape
    for b, n in enumerate(lens):
        want, bound = R.attention(R.f64(q[b]).reshape(shape.n_q_heads, shape.head_dim), cache.k_codes[b], cache.k_params[b],
                                  cache.v_codes[b], cache.v_params[b], min(max(n, 0), cache.capacity), lib.dtype)
        close(out[b].reshape(shape.n_q_heads, shape.head_dim), want, bound, f"sequence {b} of {n} rows")


ATTENTION_CASES = [  # heads, kv heads, dim, group, capacity, lens
    (2, 2, 64, 32, 32, [1]), (4, 2, 64, 64, 96, [0, 96, 33]), (8, 1, 64, 32, 320, [300]), (8, 2, 128, 32, 64, [2, 31, 32, 33, 0, 64]),
    (28, 4, 128, 64, 800, [777, 5, 400]), (8, 8, 128, 128, 544, [543, 128]), (16, 1, 128, 32, 1056, [1025]), (20, 1, 128, 64, 200, [199, 16]),
    (32, 8, 128, 32, 4128, [4099, 17, 0, 2048]), (40, 1, 64, 32, 96, [70]), (32, 8, 128, 128, 8192, [8192]), (9, 3, 128, 32, 64, [15, 16, 17]),
]


@pytest.mark.parametrize("dtype,plain", [("bf16", False), ("bf16", True), ("fp32", False)])
@pytest.mark.parametrize("heads,kv_heads,dim,group,capacity,lens", ATTENTION_CASES)
def test_attention_over_the_cache(heads, kv_heads, dim, group, capacity, lens, dtype, plain):
    shape = shape_of(heads, kv_heads, dim, dtype)
    lib = context(shape, plain)
    cache = random_cache(shape, len(lens), capacity, group, lens, seed=heads + dim)
    q = torch.randn(len(lens), heads, dim, device="cuda", generator=gen(5)).to(lib.dtype)
    out = Guarded((len(lens), heads * dim), lib.dtype)
    out.t.fill_(float("nan"))
    lib.kv4_attention(cache, q, O_out=out.t)
    check_attention(lib, cache, q, out.t, lens)
    assert out.intact() and lib.device_status() == 0 and lib.check_guards() == 0
    lib.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_when_the_largest_score_moves(dtype):
    """Scores that grow along the cache, and far outliers: the running maximum moves in every step or by hundreds."""
    shape = shape_of(8, 2, 128, dtype)
    lib = context(shape)
    lens = [700, 700, 64]
    cache = random_cache(shape, 3, 704, 32, lens, seed=3)
    ramp = torch.linspace(0, 1, 704, device="cuda")[None, None, :, None]
    p = cache.k_params[0:1].float()
    cache.k_params[0:1] = torch.stack([p[..., 0] * (0.2 + 4 * ramp), p[..., 1] * (0.2 + 4 * ramp)], -1).to(torch.bfloat16)
    for row in (0, 5, 130, 350, 699):
        cache.k_params[1, :, row] *= 30.0
    cache.k_params[2] *= 0.0                                        # all keys zero: equal weights
    q = (2.0 * torch.randn(3, 8, 128, device="cuda", generator=gen(5))).to(lib.dtype)
    out = lib.kv4_attention(cache, q)
    check_attention(lib, cache, q, out, lens)
    lib.close()


def test_attention_strided_rows_and_length_beyond_the_capacity():
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    cache = random_cache(shape, 3, 64, 64, [64, 10, 3], seed=9)
    wide = torch.randn(3, 2048, device="cuda", generator=gen(5)).to(torch.bfloat16)
    o = torch.full((3, 1500 * 2), 4.0, dtype=torch.bfloat16, device="cuda")
    cache.length.copy_(i32([1000, 10, -7]))
    lib.kv4_attention(cache, wide[:, 512:1536], O_out=o[:, 8:1032])
    check_attention(lib, cache, wide[:, 512:1536], o[:, 8:1032], [64, 10, 0])
    assert bool((o[:, :8] == 4.0).all()) and bool((o[:, 1032:] == 4.0).all())
    lib.close()


def test_attention_non_finite_rows_stay_with_their_head():
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    cache = random_cache(shape, 2, 128, 32, [100, 90], seed=9)
    q = torch.randn(2, 8, 128, device="cuda", generator=gen(5)).to(torch.bfloat16)
    clean = lib.kv4_attention(cache, q).reshape(2, 8, 128)
    cache.v_params[0, 1, 50, 2, 1] = float("nan")                   # dims 64..95 of KV head 1
    cache.k_params[1, 0, 7, 0, 1] = float("nan")                    # every score row of KV head 0
    out = lib.kv4_attention(cache, q).reshape(2, 8, 128)
    assert torch.isnan(out[0, 4:, 64:96]).all() and torch.isnan(out[1, :4]).all()
    assert torch.equal(out[0, :4], clean[0, :4]) and torch.equal(out[1, 4:], clean[1, 4:])
    assert torch.isfinite(out[0, 4:, :64]).all() and torch.isfinite(out[0, 4:, 96:]).all()
    lib.close()


def test_attention_many_sequences_and_repeatability():
    """1024 sequences of 0 to 70 rows; two runs give the same bits, and so does each sequence on its own."""
    from paper_2601_13155_b200 import binding
    shape = shape_of(8, 2, 64)
    lib = context(shape)
    rng = np.random.default_rng(3)
    lens = [int(v) for v in rng.integers(0, 71, 1024)]
    cache = random_cache(shape, 1024, 96, 32, lens, seed=1)
    q = torch.randn(1024, 8, 64, device="cuda", generator=gen(5)).to(torch.bfloat16)
    a, b = lib.kv4_attention(cache, q), lib.kv4_attention(cache, q)
    assert torch.equal(a, b)
    for s in (0, 1, 17, 500, 1023):
        check_attention(lib, cache_of(cache, s, shape), q[s:s + 1], a[s:s + 1], lens[s:s + 1])
    assert bool((a[[i for i, n in enumerate(lens) if n == 0]] == 0).all())
    with pytest.raises(binding.SptsError):
        big = binding.Kv4Cache(shape, 1025, 32, group=32)
        lib.kv4_attention(big, torch.zeros(1025, 8, 64, dtype=torch.bfloat16, device="cuda"))
    lib.close()


def cache_of(cache, s, shape):
    from paper_2601_13155_b200 import binding
    cut = lambda t: t[s:s + 1].contiguous()
    return binding.Kv4Cache(shape, 1, cache.capacity, group=cache.group, k_codes=cut(cache.k_codes), v_codes=cut(cache.v_codes),
                            k_params=cut(cache.k_params), v_params=cut(cache.v_params), length=cut(cache.length))


def test_attention_offsets_beyond_32_bits():
    """A cache of more than 4 GB per code buffer: the last sequences lie behind 2^32 bytes."""
    from paper_2601_13155_b200 import binding
    shape = shape_of(8, 8, 128)
    lib = context(shape)
    n, cap = 34, 262144
    cache = binding.Kv4Cache(shape, n, cap, group=128)
    assert cache.k_codes.numel() > 2 ** 32
    lens = [0] * n
    lens[0], lens[n - 1] = 40, 70
    cache.length.copy_(i32(lens))
    rows = torch.randn(110, 8, 128, device="cuda", generator=gen(5)).to(torch.bfloat16)
    start = np.zeros(n + 1, np.int32)
    start[1:n] = 40
    start[n] = 110
    at = np.zeros(n, np.int32)
    at[n - 1] = cap - 70
    lib.kv4_append(cache, rows, rows, row_start=i32(start), at=i32(at))
    check_rows(cache, "v", R.f64(rows[40:]), torch.full((70,), n - 1, device="cuda"), torch.arange(cap - 70, cap, device="cuda"), 128, 128)
    at[n - 1] = 0
    lib.kv4_append(cache, rows, rows, row_start=i32(start), at=i32(at))
    q = torch.randn(n, 8, 128, device="cuda", generator=gen(6)).to(torch.bfloat16)
    out = lib.kv4_attention(cache, q)
    for s in (0, n - 1):
        want, bound = R.attention(R.f64(q[s]), cache.k_codes[s, :, :96], cache.k_params[s, :, :96], cache.v_codes[s, :, :96],
                                  cache.v_params[s, :, :96], lens[s], torch.bfloat16)
        close(out[s].reshape(8, 128), want, bound, f"sequence {s}")
    assert bool((out[1:n - 1] == 0).all())
    lib.close()


# ---------------------------------------------------------------------------------------------- rules on logits
def random_rules(n, vocab, seed, history=True, bias=True, mask=True, gstart=True, longest=500):
    from paper_2601_13155_b200 import binding
    rng = np.random.default_rng(seed)
    kw = {}
    f = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()
    if history:
        lens = rng.integers(0, longest, n)
        start = np.concatenate([[0], np.cumsum(lens)])
        h = (vocab * rng.random(max(1, start[-1])) ** 3).astype(np.int32)
        h[::17] = -1                                                # padding
        h[5::31] = vocab                                            # outside
        kw.update(history=i32(h), history_start=i32(start), repetition=f(1 + rng.random(n)), presence=f(rng.random(n)),
                  frequency=f(rng.random(n) * 0.3))
        if gstart:
            kw["generated_start"] = i32(start[:-1] + lens // 2)
    if bias:
        nb = rng.integers(0, 40, n)
        start = np.concatenate([[0], np.cumsum(nb)])
        tok = rng.integers(-1, vocab + 1, max(1, start[-1])).astype(np.int32)
        tok[1::3] = tok[0]                                          # the same token again and again
        kw.update(bias_token=i32(tok), bias_value=f(rng.normal(size=len(tok)) * 3), bias_start=i32(start))
    if mask:
        m = rng.integers(-2 ** 31, 2 ** 31, (n, (vocab + 31) // 32 + 2)).astype(np.int32)
        if n > 1:
            m[n // 2] = 0
        kw["mask"] = i32(m)
    return binding.LogitsRules(**kw)


def check_logits(x, rules, out, token):
    n, vocab = x.shape
    xs = x.cpu().numpy()
    for b in range(n):
        want, tok = R.logits(xs[b], rules, b, vocab)
        if out is not None:
            assert np.array_equal(out[b].cpu().numpy(), want, equal_nan=True), f"row {b}"
        assert int(token[b]) == tok, f"row {b}: token {int(token[b])}, {tok} is right"


@pytest.mark.parametrize("n,vocab,kw", [
    (1, 1, {}), (1, 31, {}), (2, 33, {}), (3, 1000, {}), (5, 1003, dict(bias=False)), (4, 777, dict(history=False)), (3, 512, dict(mask=False)),
    (2, 5000, dict(gstart=False)), (7, 128256, {}), (1, 152064, dict(longest=40000)), (2, 400001, {}), (2, 64, dict(history=False, bias=False, mask=False)),
    (70, 4099, {}),
])
def test_logits_rules(n, vocab, kw):
    lib = context()
    rules = random_rules(n, vocab, seed=n + vocab, **kw)
    x = 3 * torch.randn(n, vocab, device="cuda", generator=gen(vocab))
    out, token = lib.process_logits(x, rules)
    check_logits(x, rules, out, token)
    only = lib.process_logits(x, rules, want_logits=False)
    assert only[0] is None and torch.equal(only[1], token)
    y = x.clone()
    same, token2 = lib.process_logits(y, rules, out=y)               # in place
    assert same is y and torch.equal(y, out) and torch.equal(token2, token)
    assert lib.check_guards() == 0
    lib.close()


def test_logits_special_values_and_strides():
    lib = context()
    vocab = 999
    wide = 3 * torch.randn(4, 1200, device="cuda", generator=gen(1))
    x = wide[:, 101:101 + vocab]
    x[0, 5] = float("nan")
    x[0, 600] = float("inf")
    x[1] = -float("inf")
    x[2] = 1.5                                                      # all equal: the lowest index wins
    x[3, 7] = -float("inf")
    rules = random_rules(4, vocab, seed=2, mask=False)
    g = Guarded((4, vocab + 3), torch.float32)
    g.t.fill_(8.0)
    out, token = lib.process_logits(x, rules, out=g.t[:, :vocab])
    check_logits(x, rules, out, token)
    assert int(token[1]) == -1 and g.intact() and bool((g.t[:, vocab:] == 8.0).all())
    from paper_2601_13155_b200 import binding
    out, token = lib.process_logits(x, binding.LogitsRules())
    assert torch.equal(out.nan_to_num(0.25), x.nan_to_num(0.25)) and int(token[2]) == 0 and int(token[0]) == 600
    lib.close()


def test_logits_refusals():
    from paper_2601_13155_b200 import binding
    lib = context()
    x = torch.zeros(3, 100, device="cuda")
    ones = torch.ones(3, device="cuda")
    assert lib.process_logits(x[:0], binding.LogitsRules())[0].shape == (0, 100)
    for call in (lambda: binding.LogitsRules(history=i32([1])), lambda: binding.LogitsRules(bias_token=i32([1])),
                 lambda: binding.LogitsRules(mask=i32([1])), lambda: binding.LogitsRules(repetition=ones.double()),
                 lambda: lib.process_logits(x, binding.LogitsRules(repetition=ones[:2].contiguous())),
                 lambda: lib.process_logits(x, binding.LogitsRules(mask=i32(np.zeros((3, 3))))),
                 lambda: lib.process_logits(x.half(), binding.LogitsRules()), lambda: lib.process_logits(x, binding.LogitsRules(), out=x[:2])):
        with pytest.raises(ValueError):
            call()
    r = binding.LogitsRules()
    assert lib.lib.spts_process_logits(lib.h, C.c_void_p(x.data_ptr()), 100, 3, 100, C.byref(r.c), None, 0, None) == 1
    assert lib.lib.spts_process_logits(lib.h, C.c_void_p(x.data_ptr()), 90, 3, 100, C.byref(r.c), C.c_void_p(x.data_ptr()), 90, None) == 1
    lib.close()


# ---------------------------------------------------------------------------------------------- streams and graphs
def test_other_stream_and_captured_replay():
    """A step captured once (append, attention, product, rules) follows the device-side lengths when it is replayed."""
    from paper_2601_13155_b200 import binding
    shape = shape_of(8, 2, 128)
    st = torch.cuda.Stream()
    lib = binding.Spts(shape, max_seq=64, stream=st)
    w = rand_w4(500, 1024, 128, 1)
    rules = random_rules(3, 500, seed=1)
    caches = [random_cache(shape, 3, 256, 32, [100, 0, 31], seed=4) for _ in range(2)]
    K = torch.randn(3, 2, 128, device="cuda", generator=gen(2)).to(torch.bfloat16)
    q = torch.randn(3, 8, 128, device="cuda", generator=gen(3)).to(torch.bfloat16)
    o = torch.empty(3, 1024, dtype=torch.bfloat16, device="cuda")
    lg, out = torch.empty(3, 500, device="cuda"), torch.empty(3, 500, device="cuda")
    tok = torch.empty(3, dtype=torch.int32, device="cuda")

    def step(cache):
        lib.kv4_append(cache, K, K)
        lib.kv4_attention(cache, q, O_out=o)
        lib.w4_gemv(w, o, norm=True, fp32_out=True, out=lg)
        lib.process_logits(lg, rules, out=out, token_out=tok)
    torch.cuda.synchronize()
    want = []
    with torch.cuda.stream(st):
        for i in range(4):
            step(caches[0])
            want.append([t.clone() for t in (o, lg, out, tok)])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step(caches[1])
    assert caches[1].length.tolist() == [100, 0, 31]
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        for got, w_ in zip((o, lg, out, tok), want[i]):
            assert torch.equal(got, w_)
    assert caches[1].length.tolist() == [104, 4, 35]
    assert lib.device_status() == 0
    del graph
    lib.close()
