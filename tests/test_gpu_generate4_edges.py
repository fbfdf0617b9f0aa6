"""The ends of the ranges of the 4-bit generation operators: values at the ends of their types, inputs that take several
launches, buffers beyond 4 GB, calls side by side, pointers of any alignment that a row may have."""
import ctypes as C

import numpy as np
import pytest
import torch

import generate4_ref as R
from parity_utils import Guarded, i32
from test_gpu_generate4 import (cache_of, check_attention, check_logits, check_rows, close, context, fill_garbage, gen, rand_w4,
                                random_cache, random_rules, shape_of)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- quantiser
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantiser_at_the_ends_of_the_types(dtype):
    """Subnormal and tiny groups, groups whose range or sum leaves fp32, one value near the largest, and the step between."""
    lib = context(shape_of(dtype=dtype))
    g = torch.randn(12, 128, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    top = float(torch.finfo(lib.dtype).max) * 0.98
    scales = [1e-45, 1e-41, 1e-39, 2e-38, 1e-37, 1e-33, 1e-30, 1e30, 1e36]
    rows = [g[i] * s for i, s in enumerate(scales)]
    rows += [torch.clamp(g[9] * 2e38, -top, top), torch.full((128,), top, dtype=torch.float64), g[11] * 1e30 + 1e36]
    W = torch.stack(rows).to(torch.float32).to(lib.dtype).cuda()
    for group in (32, 128):
        w = lib.w4_quantize(W, group)
        codes, scale, mid, _ = R.quantise(R.f64(W), group)
        s, m = R.split_params(w.params)
        assert np.array_equal(s, scale) and np.array_equal(m, mid)
        assert np.array_equal(R.nibbles(w.codes), codes)
    assert lib.device_status() == 0
    lib.close()


# ---------------------------------------------------------------------------------------------- matrix-vector products
@pytest.mark.parametrize("n,out,k,group", [(32, 40, 65536, 64), (9, 17, 131072, 128), (20, 65, 32800, 32), (25, 33, 40000, 32)])
def test_gemv_of_more_than_one_launch(n, out, k, group):
    lib = context()
    w, w2 = rand_w4(out, k, group, n), rand_w4(out, k, group, n + 1, mids=False)
    x = torch.randn(n, k, device="cuda", generator=gen(1)).to(lib.dtype)
    r = torch.randn(n, out, device="cuda", generator=gen(2)).to(lib.dtype)
    y, e = R.gemv(R.f64(x), w, lib.dtype, residual=R.f64(r))
    close(lib.w4_gemv(w, x, residual=r), y, e, "residual")
    y, e = R.gemv(R.f64(x), w, lib.dtype, norm=True, fp32_out=True, eps=lib.shape.rms_eps)
    close(lib.w4_gemv(w, x, norm=True, fp32_out=True), y, e, "logits")
    y, e = R.gemv(R.f64(x), w, lib.dtype, norm=True, w2=w2, eps=lib.shape.rms_eps)
    close(lib.w4_gemv(w, x, norm=True, w2=w2), y, e, "swiglu")
    lib.close()


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("n,out,k", [(1, 60, 512), (3, 2500, 4096), (20, 60, 512)])
def test_gemv_of_the_smallest_and_largest_tokens(n, out, k, plain):
    """Tokens of 2^107 and 2^-110 and one that holds both an element of 2^20 and elements of 2^-6, side by side."""
    lib = context(plain=plain)
    w = rand_w4(out, k, 64, 5)
    x = torch.randn(n, k, device="cuda", generator=gen(1))
    x[0] = x[0].clamp(-2, 2) * 2.0 ** 106
    if n > 1:
        x[1] *= 2.0 ** -110
        x[2] *= 2.0 ** -6
        x[2, 77] = 2.0 ** 20
    x = x.to(lib.dtype)
    y, e = R.gemv(R.f64(x), w, lib.dtype, fp32_out=True)
    got = lib.w4_gemv(w, x, fp32_out=True)
    close(got, y, e, "fp32")
    # 2^115: beyond what a power of two and the codes' unit could carry in one factor
    x[0] *= 2.0 ** 8
    if n > 1:
        x[1] = 0.0
    y, e = R.gemv(R.f64(x), w, lib.dtype, fp32_out=True)
    got = lib.w4_gemv(w, x, fp32_out=True)
    close(got, y, e, "2^115")
    assert n == 1 or not got[1].any()
    lib.close()


def test_gemv_codes_beyond_4_gb():
    from paper_2601_13155_b200 import binding
    lib = context()
    out, k, group = 131081, 65536, 128
    w = binding.W4Weight(torch.empty(out, k // 2, dtype=torch.uint8, device="cuda"), torch.empty(out, k // group, 2, dtype=torch.bfloat16, device="cuda"))
    assert w.codes.numel() > 2 ** 32
    w.codes.random_(0, 256, generator=gen(1))
    w.params.uniform_(-0.01, 0.02, generator=gen(2))
    x = torch.randn(2, k, device="cuda", generator=gen(3)).to(lib.dtype)
    rows = torch.tensor([0, 1, 65535, 131072, out - 2, out - 1])
    some = binding.W4Weight(w.codes[rows].contiguous(), w.params[rows].contiguous())
    y, e = R.gemv(R.f64(x), some, lib.dtype)
    first = lib.w4_gemv(w, x)
    close(first[:, rows], y, e, "rows")
    lib.set_reference_kernels(True)
    close(lib.w4_gemv(w, x)[:, rows], y, e, "rows, plain")
    lib.close()


def test_gemv_is_the_same_for_a_token_in_any_place():
    """A token's result depends neither on the tokens beside it nor on the call before."""
    lib = context()
    w = rand_w4(700, 2048, 128, 1)
    x = torch.randn(8, 2048, device="cuda", generator=gen(2)).to(lib.dtype)
    a = lib.w4_gemv(w, x)
    lib.w4_gemv(rand_w4(3000, 4096, 32, 2), torch.randn(30, 4096, device="cuda").to(lib.dtype))
    assert torch.equal(lib.w4_gemv(w, x), a)
    perm = torch.tensor([5, 0, 7, 2, 1, 6, 3, 4], device="cuda")
    assert torch.equal(lib.w4_gemv(w, x[perm].contiguous()), a[perm])
    lib.close()


# ---------------------------------------------------------------------------------------------- cache
@pytest.mark.parametrize("kv_heads,dim,group", [(5, 64, 32), (24, 128, 64), (9, 64, 64)])
def test_append_of_many_or_odd_heads_in_place(kv_heads, dim, group):
    from paper_2601_13155_b200 import binding
    shape = shape_of(kv_heads, kv_heads, dim)
    lib = context(shape)
    n = 700                                                         # enough rows that a warp takes several passes
    cache = binding.Kv4Cache(shape, 2, 704, group=group)
    fill_garbage(cache, 1)
    K = (3 * torch.randn(n, kv_heads, dim, device="cuda", generator=gen(2))).to(lib.dtype)
    V = torch.randn(n, kv_heads, dim, device="cuda", generator=gen(3)).to(lib.dtype)
    k64, v64 = R.f64(K), R.f64(V)
    lib.kv4_append(cache, K, V, row_start=i32([0, 1, n]), at=i32([703, 4]), K_out=K, V_out=V)      # the values take K's and V's place
    for which, src, got in (("k", k64, K), ("v", v64, V)):
        for b, rows, slot in ((0, slice(0, 1), torch.tensor([703])), (1, slice(1, n), torch.arange(4, n + 3))):
            vals = check_rows(cache, which, src[rows], torch.full((len(slot),), b, device="cuda"), slot.cuda(), group, dim)
            assert torch.equal(got[rows].cpu(), torch.from_numpy(vals).to(torch.float32).to(lib.dtype))
    assert cache.length.tolist() == [704, n + 3] and lib.device_status() == 0
    lib.close()


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("k_scale,v_scale", [(1e-30, 1e-30), (0.3, 0.0), (0.0, 1e-36), (0.3, 1e30)])
def test_attention_over_the_smallest_and_largest_values(k_scale, v_scale, plain):
    shape = shape_of(24, 2, 128)
    lib = context(shape, plain)
    lens = [400, 1, 0, 2100]
    cache = random_cache(shape, 4, 2112, 32, lens, seed=6, k_scale=k_scale)
    cache.v_params.copy_((cache.v_params.float() / 0.3 * v_scale).to(torch.bfloat16))
    q = torch.randn(4, 24, 128, device="cuda", generator=gen(5)).to(lib.dtype)
    out = lib.kv4_attention(cache, q)
    for b, n in enumerate(lens):
        want, bound = R.attention(R.f64(q[b]), cache.k_codes[b], cache.k_params[b], cache.v_codes[b], cache.v_params[b], n, lib.dtype)
        close(out[b].reshape(24, 128), want, bound + 2.0 ** -133, f"sequence {b}")          # 2^-133: the smallest bf16 number
    lib.close()


def test_attention_long_rows_of_shared_heads_cut_between_blocks():
    """16 and 20 query heads to a KV head, whose rows no block holds alone; each sequence on its own gives the same bits only
    where its cuts are the same, so both are held against the plain form."""
    for heads, kv in ((32, 2), (20, 1)):
        shape = shape_of(heads, kv, 128)
        lib = context(shape)
        lens = [9000, 3, 12345]
        cache = random_cache(shape, 3, 12352, 64, lens, seed=2)
        q = torch.randn(3, heads, 128, device="cuda", generator=gen(5)).to(lib.dtype)
        out = lib.kv4_attention(cache, q)
        check_attention(lib, cache, q, out, lens)
        one = lib.kv4_attention(cache_of(cache, 2, shape), q[2:3])
        check_attention(lib, cache_of(cache, 2, shape), q[2:3], one, lens[2:])
        assert torch.equal(out, lib.kv4_attention(cache, q))
        lib.close()


@pytest.mark.parametrize("heads,kv_heads,dim,group,lens", [
    (16, 1, 128, 32, "short"), (20, 1, 128, 64, "mixed"), (10, 1, 128, 128, "short"), (8, 1, 128, 32, "mixed"), (6, 2, 128, 64, "mixed"),
    (4, 2, 128, 128, "short"), (16, 1, 64, 32, "mixed"), (12, 1, 64, 64, "short"), (5, 1, 64, 64, "mixed"), (2, 2, 64, 32, "equal"),
])
def test_attention_of_more_units_than_blocks(heads, kv_heads, dim, group, lens):
    """340 sequences: of 0 to 40 rows, of which most units lie in one block; with a few of thousands, which are cut; and equal ones."""
    shape = shape_of(heads, kv_heads, dim)
    lib = context(shape)
    rng = np.random.default_rng(heads)
    n = [int(v) for v in rng.integers(0, 41, 340)]
    if lens == "mixed":
        for b, rows in ((0, 3000), (7, 1), (100, 2500), (101, 2111), (339, 1777)):
            n[b] = rows
    if lens == "equal":
        n = [33] * 340
    cache = random_cache(shape, 340, max(n), group, n, seed=1)
    q = torch.randn(340, heads, dim, device="cuda", generator=gen(5)).to(lib.dtype)
    out = Guarded((340, heads * dim), lib.dtype)
    out.t.fill_(float("nan"))
    lib.kv4_attention(cache, q, O_out=out.t)
    for b in [0, 1, 2, 7, 50, 99, 100, 101, 102, 200, 338, 339]:
        check_attention(lib, cache_of(cache, b, shape), q[b:b + 1], out.t[b:b + 1], n[b:b + 1])
    assert bool(torch.isfinite(out.t).all()) and bool((out.t[[b for b in range(340) if n[b] == 0]] == 0).all())
    assert torch.equal(lib.kv4_attention(cache, q), out.t)
    assert out.intact() and lib.check_guards() == 0
    lib.close()


@pytest.mark.parametrize("heads,kv_heads,dim", [(32, 8, 128), (8, 1, 64), (28, 4, 128)])
@pytest.mark.parametrize("lens", [[1], [31, 32, 33], [257, 0, 0, 1], [0, 0, 4000], [900, 900, 900], [5000, 1, 1, 1, 1, 1, 1, 1, 2000], [63] * 18, [1, 0, 2]])
def test_attention_pieces_of_every_kind(heads, kv_heads, dim, lens):
    """Cuts at units' borders, inside a unit's fixed cost, one step before the end, and units of one step."""
    shape = shape_of(heads, kv_heads, dim)
    lib = context(shape)
    cache = random_cache(shape, len(lens), max(lens), 32, lens, seed=len(lens))
    q = torch.randn(len(lens), heads, dim, device="cuda", generator=gen(5)).to(lib.dtype)
    out = lib.kv4_attention(cache, q)
    check_attention(lib, cache, q, out, lens)
    assert torch.equal(out, lib.kv4_attention(cache, q))
    lib.close()


# ---------------------------------------------------------------------------------------------- rules on logits
@pytest.mark.parametrize("n,vocab", [(2100, 53), (1025, 1000)])
def test_logits_of_many_rows(n, vocab):
    lib = context()
    rules = random_rules(n, vocab, seed=n, longest=30)
    x = 3 * torch.randn(n, vocab, device="cuda", generator=gen(vocab))
    out, token = lib.process_logits(x, rules)
    check_logits(x, rules, out, token)
    lib.close()


@pytest.mark.parametrize("n", [2, 12])
def test_logits_with_long_bias_lists_and_wide_vocabularies(n):
    """More than 65534 bias entries, many for one token, and slices of more tokens than the tables hold at a time."""
    from paper_2601_13155_b200 import binding
    lib = context()
    vocab = 700_001
    rules = random_rules(n, vocab, seed=4, bias=False, mask=False, longest=3000)
    rng = np.random.default_rng(1)
    m = 90_000
    tok = rng.integers(0, vocab, m).astype(np.int32)
    tok[::3] = vocab - 1
    start = np.linspace(0, m, n + 1).astype(np.int32)
    kw = {k: v for k, v in rules.t.items() if v is not None}
    kw.update(bias_token=i32(tok), bias_value=torch.from_numpy(rng.normal(size=m).astype(np.float32)).cuda(), bias_start=i32(start))
    rules = binding.LogitsRules(**kw)
    x = 3 * torch.randn(n, vocab, device="cuda", generator=gen(3))
    out, token = lib.process_logits(x, rules)
    check_logits(x, rules, out, token)
    lib.close()


def test_logits_lists_and_rows_of_any_alignment_and_starts_outside_the_lists():
    from paper_2601_13155_b200 import binding
    lib = context()
    n, vocab = 5, 2003
    base = random_rules(n, vocab, seed=9)
    kw = {}
    for name, t in base.t.items():
        if t is None:
            continue
        wide = torch.zeros(t.numel() + 1, dtype=t.dtype, device="cuda")
        wide[1:] = t.reshape(-1)
        kw[name] = wide[1:].reshape(t.shape)                         # 4 bytes off a 16-byte boundary
    nh, nb = len(kw["history"]), len(kw["bias_token"])
    for name, m in (("history_start", nh), ("bias_start", nb)):
        kw[name][0] = -7                                            # begins before the list, ends behind it
        kw[name][n] = m + 1000
    rules = binding.LogitsRules(**kw)
    x = (3 * torch.randn(n, vocab + 6, device="cuda", generator=gen(3)))[:, 1:vocab + 1]
    store = Guarded((n, vocab + 3), torch.float32)
    out, token = lib.process_logits(x, rules, out=store.t[:, 2:vocab + 2])
    check_logits(x, rules, out, token)
    assert store.intact()
    kw["history_start"][:] = 2 ** 31 - 1                            # all behind the list: no history
    kw["bias_start"][:] = 2 ** 31 - 2
    out, token = lib.process_logits(x, binding.LogitsRules(**kw))
    only = binding.LogitsRules(mask=kw["mask"])
    want, want_token = lib.process_logits(x, only)
    assert torch.equal(out, want) and torch.equal(token, want_token)
    lib.close()


# ---------------------------------------------------------------------------------------------- refusals, calls side by side
def test_misaligned_pointers_and_sizes_out_of_range_are_refused():
    from paper_2601_13155_b200 import binding
    lib = context()
    w = rand_w4(16, 256, 64, 1)
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(4, 64, device="cuda")
    at = lambda t, b: C.c_void_p(t.data_ptr() + b)
    call = lib.lib.spts_w4_gemv
    assert call(lib.h, C.byref(w.c), None, at(x, 0), 256, 1, None, 0, 0, at(y, 1), 16) == 1
    assert call(lib.h, C.byref(w.c), None, at(x, 0), 256, 1, at(y, 1), 16, 0, at(y, 64), 16) == 1
    assert call(lib.h, C.byref(w.c), None, at(x, 0), 256, 1, None, 0, 2, at(f, 2), 16) == 1
    big = binding.W4C(w.codes.data_ptr(), w.params.data_ptr(), 2 ** 30 + 1, 256, 64)
    assert call(lib.h, C.byref(big), None, at(x, 0), 256, 1, None, 0, 0, at(y, 0), 16) == 2
    assert lib.lib.spts_w4_quantize(lib.h, at(x, 0), 1, 131072 + 64, 64, at(y, 0), at(y, 0)) == 2
    r = binding.LogitsRules().c
    logits = lib.lib.spts_process_logits
    assert logits(lib.h, at(f, 0), 64, 1, 2 ** 30 + 1, C.byref(r), at(f, 0), 64, None) == 2
    assert logits(lib.h, at(f, 0), 64, 1, 64, C.byref(r), at(f, 0), 64, at(f, 2)) == 1
    h = i32(np.zeros(8))
    bad = binding.LogitsRules(history=h[:4], history_start=h[4:6], presence=f[0, :1]).c
    bad.history = h.data_ptr() + 1
    assert logits(lib.h, at(f, 0), 64, 1, 64, C.byref(bad), at(f, 0), 64, None) == 1
    cache = binding.Kv4Cache(shape_of(), 1, 32, group=64)
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    assert lib.lib.spts_kv4_append(lib.h, C.byref(cache.c), at(k, 0), 256, at(k, 0), 256, None, None, at(h, 2), 1, None, None) == 1
    lib.close()


def test_two_contexts_at_once_on_their_own_streams():
    """Interleaved calls of two contexts whose kernels overlap give what each gives alone."""
    from paper_2601_13155_b200 import binding
    shape = shape_of(8, 2, 128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    libs = [binding.Spts(shape, max_seq=64, stream=s) for s in streams]
    ws = [rand_w4(3000, 8192, 128, 1), rand_w4(900, 16384, 64, 2)]
    xs = [torch.randn(12, w.in_features, device="cuda", generator=gen(3 + i)).to(torch.bfloat16) for i, w in enumerate(ws)]
    lens = [[700, 3, 5000], [64, 0, 4097]]
    caches = [random_cache(shape, 3, 5024, 32, l, seed=4 + i) for i, l in enumerate(lens)]
    q = torch.randn(3, 8, 128, device="cuda", generator=gen(8)).to(torch.bfloat16)
    rules = [random_rules(3, 20000, seed=i) for i in range(2)]
    lg = torch.randn(3, 20000, device="cuda", generator=gen(9))

    def run(i):
        with torch.cuda.stream(streams[i]):
            y = libs[i].w4_gemv(ws[i], xs[i])
            o = libs[i].kv4_attention(caches[i], q)
            l, t = libs[i].process_logits(lg, rules[i])
            return y, o, l, t
    torch.cuda.synchronize()
    alone = []
    for i in range(2):
        alone.append(run(i))
        torch.cuda.synchronize()
    for _ in range(20):
        got = [run(0), run(1)]
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(got[i], alone[i]):
                assert torch.equal(a, b)
    for lib in libs:
        lib.close()
