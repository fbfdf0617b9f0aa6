"""What a caller of the 4-bit generation operators may do beside the plain calls: options, refused arguments, streams of their
own, scales of either sign, caches of a skipping prefill; and bounds that see a lost rounding piece."""
import ctypes as C
import os
import subprocess
import sys
from dataclasses import replace

import numpy as np
import pytest
import torch

import generate4_ref as R
from paper_2601_13155_b200 import synth
from parity_utils import host, i32, rel_rms_err, up
from test_gpu_decode4 import WIDE, build, reference_layer
from test_gpu_generate4 import check_attention, close, context, fill_garbage, gen, rand_w4, random_cache, shape_of

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- options
def test_plain_kernels_of_heads_of_64_dims():
    """SPTS_REFERENCE_KERNELS reaches the 4-bit calls of a bf16 context whose shape has no tensor-core prefill: one launch for 16
    tokens (the matrix route lays x out in a launch of its own), and the plain kernels' fp32 arithmetic, which is that of an fp32
    context on the same values: its results rounded once are the same bits."""
    from paper_2601_13155_b200 import binding
    shape = shape_of(8, 2, 64)
    lib, full = context(shape), context(replace(shape, dtype="fp32"))
    w = rand_w4(70, 512, 64, 1)
    x = torch.randn(16, 512, device="cuda", generator=gen(2)).to(torch.bfloat16)
    lens = [300, 0, 45]
    cache = random_cache(shape, 3, 320, 32, lens, seed=3)
    q = torch.randn(3, 8, 64, device="cuda", generator=gen(4)).to(torch.bfloat16)

    def launches(call):
        before = lib.launch_count()
        call()
        return lib.launch_count() - before
    with pytest.raises(binding.SptsError):                           # nothing to take back
        lib.set_reference_kernels(False)
    assert launches(lambda: lib.w4_gemv(w, x)) > 1
    matrix = lib.kv4_attention(cache, q)
    lib.set_reference_kernels(True)
    assert launches(lambda: lib.w4_gemv(w, x)) == 1
    assert torch.equal(lib.w4_gemv(w, x, fp32_out=True), full.w4_gemv(w, x.float(), fp32_out=True))
    assert torch.equal(lib.kv4_attention(cache, q), full.kv4_attention(cache, q.float()).to(torch.bfloat16))
    lib.set_reference_kernels(False)
    assert launches(lambda: lib.w4_gemv(w, x)) > 1
    assert torch.equal(lib.kv4_attention(cache, q), matrix)
    full.set_reference_kernels(True)
    with pytest.raises(binding.SptsError):                           # fp32 has no other kernels
        full.set_reference_kernels(False)
    lib.close()
    full.close()


@pytest.mark.parametrize("heads,kv_heads,group,lens", [(2, 2, 32, [1]), (4, 2, 64, [0, 96, 33]), (8, 1, 32, [300]), (40, 1, 32, [70]), (6, 2, 64, [1500, 1, 64])])
def test_plain_attention_of_heads_of_64_dims_in_bf16(heads, kv_heads, group, lens):
    shape = shape_of(heads, kv_heads, 64)
    lib = context(shape)
    lib.set_reference_kernels(True)
    cache = random_cache(shape, len(lens), max(lens), group, lens, seed=heads)
    q = torch.randn(len(lens), heads, 64, device="cuda", generator=gen(5)).to(lib.dtype)
    check_attention(lib, cache, q, lib.kv4_attention(cache, q), lens)
    assert lib.device_status() == 0 and lib.check_guards() == 0
    lib.close()


@pytest.mark.parametrize("n,out,k,group", [(1, 7, 64, 64), (5, 1030, 160, 32), (21, 129, 2048, 32)])
def test_plain_products_beside_heads_of_64_dims_in_bf16(n, out, k, group):
    lib = context(shape_of(8, 2, 64))
    lib.set_reference_kernels(True)
    w = rand_w4(out, k, group, n)
    x = torch.randn(n, k, device="cuda", generator=gen(n + k)).to(lib.dtype)
    y, e = R.gemv(R.f64(x), w, lib.dtype, norm=True, eps=lib.shape.rms_eps)
    close(lib.w4_gemv(w, x, norm=True), y, e, "norm")
    lib.close()


# ---------------------------------------------------------------------------------------------- a step that is refused
def test_a_step_with_refused_rules_leaves_the_caches():
    """Rules that spts_process_logits refuses are refused by the step before anything is launched: lengths, codes and logits stay."""
    from paper_2601_13155_b200 import binding
    lens = [4, 5]
    lib, shape, model, q, lm, embed, caches = build(WIDE, 128, 64, lens, seed=2)
    pos, token = i32([4, 5]), i32([1, 2])
    logits = torch.full((2, shape.vocab), 3.0, device="cuda")
    good = binding.LogitsRules(history=i32([1, 2, 3]), history_start=i32([0, 1, 3]), presence=torch.ones(2, device="cuda"),
                               bias_token=i32([1]), bias_value=torch.ones(1, device="cuda"), bias_start=i32([0, 1, 1]),
                               mask=torch.full((2, 32), -1, dtype=torch.int32, device="cuda"))

    def with_(**kw):
        c = binding.LogitsRulesC.from_buffer_copy(good.c)
        for k, v in kw.items():
            setattr(c, k, v)
        return c
    bad = [with_(history=good.c.history + 1), with_(mask=good.c.mask + 2), with_(history_start=None), with_(bias_value=None),
           with_(bias_start=None), with_(ld_mask=31), with_(n_history=-1), with_(n_bias=2 ** 29 + 1), with_(presence=good.c.presence + 1)]
    before = [(c.length.clone(), c.k_codes.clone(), c.v_params.clone()) for c in caches.layers]
    ptr = lambda t: C.c_void_p(t.data_ptr())

    def step(rules, logits_out, token_out):
        return lib.lib.spts_decode_step4(lib.h, C.byref(model.c), caches.c, None, ptr(token), ptr(pos), C.byref(rules), None,
                                         logits_out, token_out)
    launched = lib.launch_count()
    for c in bad:
        assert step(c, ptr(logits), None) == 1
    assert step(good.c, None, None) == 1                             # rules and nothing that they apply to
    assert lib.launch_count() == launched
    for (length, codes, params), c in zip(before, caches.layers):
        assert torch.equal(c.length, length) and torch.equal(c.k_codes, codes) and torch.equal(c.v_params, params)
    assert bool((logits == 3.0).all())
    assert step(good.c, ptr(logits), ptr(token)) == 0
    assert lib.device_status() == 0 and caches.layers[0].length.tolist() == [5, 6]
    lib.close()


# ---------------------------------------------------------------------------------------------- streams
def test_a_layer_quantised_on_a_stream_of_its_own():
    """The stacked q / k / v matrix is made inside the call: the context's stream waits for it, whatever torch's stream still does."""
    from paper_2601_13155_b200 import binding
    tensors = {k: up(v, "bf16") for k, v in synth.layer_weights(WIDE, 9).items()}
    lib = binding.Spts(WIDE, max_seq=64)
    want = lib.quantize_layer4(tensors, 64)
    lib.close()
    lib = binding.Spts(WIDE, max_seq=64, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    for _ in range(3):
        late = {k: torch.zeros_like(v) for k, v in tensors.items()}
        torch.cuda._sleep(100_000_000)                              # the matrices arrive some 50 ms from now
        for k, v in tensors.items():
            late[k].copy_(v)
        got = lib.quantize_layer4(late, 64)
        for name, w in want.items():
            assert torch.equal(got[name].codes, w.codes) and torch.equal(got[name].params, w.params), name
    lib.close()


def test_products_of_several_launches_replayed():
    """Layout, product and join are dependents of one another: captured, the same bits as called, call after call over one workspace."""
    from paper_2601_13155_b200 import binding
    st = torch.cuda.Stream()
    lib = binding.Spts(shape_of(), max_seq=64, stream=st)
    cases = [(12, 3000, 8192, 128), (32, 300, 14336, 32), (5, 1030, 4096, 64), (20, 65, 40000, 32)]
    ws = [rand_w4(out, k, g, i) for i, (_, out, k, g) in enumerate(cases)]
    xs = [torch.randn(n, k, device="cuda", generator=gen(i)).to(torch.bfloat16) for i, (n, _, k, _) in enumerate(cases)]
    w2 = rand_w4(1030, 4096, 64, 9)

    def run():
        return [lib.w4_gemv(w, x, norm=i % 2 == 0, w2=w2 if i == 2 else None) for i, (w, x) in enumerate(zip(ws, xs))]
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        want = run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        got = run()
    for _ in range(5):
        for y in got:
            y.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert lib.device_status() == 0 and lib.check_guards() == 0
    del g
    lib.close()


FIRST_CAPTURED = """
import sys, torch
sys.path[:0] = [{root!r}, {root!r} + "/tests"]
import test_gpu_decode4 as T
from paper_2601_13155_b200 import binding
from parity_utils import i32
lib, shape, model, q, lm, embed, caches = T.build(T.WIDE, 128, 64, [9, 30], seed=11)
lib.close()
st = torch.cuda.Stream()
lib = binding.Spts(shape, max_seq=64, stream=st)
pos, token = i32([9, 30]), i32([3, 4])
logits = torch.empty(2, shape.vocab, device="cuda")
rules = binding.LogitsRules(bias_token=i32([5]), bias_value=torch.ones(1, device="cuda"), bias_start=i32([0, 1, 1]))
torch.cuda.synchronize()
step = lambda: lib.decode_step4(model, caches, pos, token_in=token, rules=rules, logits_out=logits, token_out=token)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=st):
    step()
g.replay()
torch.cuda.synchronize()
assert lib.device_status() == 0 and caches.layers[0].length.tolist() == [10, 31]
first = logits.clone()
for c in caches.layers:
    c.length.copy_(i32([9, 30]))
token.copy_(i32([3, 4]))
torch.cuda.synchronize()
step()
torch.cuda.synchronize()
assert torch.equal(first, logits)
del g
print("same")
"""


def test_a_step_whose_first_call_is_captured():
    """In a process of its own, where no kernel of the step has been loaded before."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CAPTURED.format(root=root)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("same"), r.stderr[-2000:]


# ---------------------------------------------------------------------------------------------- scales of either sign
@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,group", [(8, 2, 128, 32), (24, 2, 128, 128), (4, 2, 64, 32)])
@pytest.mark.parametrize("sign", ["negative", "mixed"])
def test_attention_with_negative_scales(heads, kv_heads, dim, group, sign, plain):
    """A group may hold its values with a negative scale (a cache made elsewhere).  Bound: R.attention's, whose terms are absolute
    values of scale times code; it takes the scales' absolute values with the codes mirrored, which are the same values:
    s (c - 8) + m = |s| (8 - c) + m, where 8 - c may be 8, one more than its formula's |code| of at most 8."""
    shape = shape_of(heads, kv_heads, dim)
    lib = context(shape)
    if plain:
        lib.set_reference_kernels(True)
    lens = [700, 3, 0, 64]
    cache = random_cache(shape, 4, 704, group, lens, seed=7)
    for t in (cache.k_params, cache.v_params):
        flip = -1.0 if sign == "negative" else torch.where(torch.rand(t.shape[:-1], device="cuda", generator=gen(8)) < 0.5, -1.0, 1.0)
        t[..., 0] = t[..., 0] * flip
    large = 2.0 ** 17 if sign == "negative" else torch.where(cache.v_params[..., 0] < 0, 2.0 ** 17, 1.0)
    cache.v_params[..., 0] = cache.v_params[..., 0] * large
    q = torch.randn(4, heads, dim, device="cuda", generator=gen(5)).to(lib.dtype)
    out = lib.kv4_attention(cache, q).reshape(4, heads, dim)
    for b, n in enumerate(lens):
        if n == 0:
            assert not out[b].any()
            continue
        want, bound = signed_attention(R.f64(q[b]), cache, b, n)
        close(out[b], want, bound, f"sequence {b}")
    lib.close()


def signed_attention(q, cache, b, length):
    """R.attention's result and bound (bf16) with the absolute values of the scales in the bound."""
    h, d = q.shape
    hkv = cache.k_codes.shape[1]
    out, bound = np.zeros((h, d)), np.zeros((h, d))
    half = R.half_step(torch.bfloat16)
    for kv in range(hkv):
        k, _, ks, km = R.cache_rows(cache.k_codes[b, kv, :length], cache.k_params[b, kv, :length], R.key_dims(d))
        v, vc, vs, vm = R.cache_rows(cache.v_codes[b, kv, :length], cache.v_params[b, kv, :length], R.value_dims(d))
        ks, vs = np.abs(ks), np.abs(vs)
        g = slice(kv * (h // hkv), (kv + 1) * (h // hkv))
        s = q[g] @ k.T / np.sqrt(d)
        es = (d / 16 + 24) * 2.0 ** -23 * (np.abs(q[g]) @ (56 * ks + np.abs(km)).T) / np.sqrt(d)
        es = es + 2.0 ** -16 * (np.abs(q[g]) @ (24 * ks + np.abs(km)).T) / np.sqrt(d)
        es = es + 2.0 ** -22 * (np.abs(s) + np.abs(s).max(1, keepdims=True) + 16)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        e = (length / 128 + 40) * 2.0 ** -23 * (p @ (56 * vs + np.abs(vm)))
        e = e + half * (p @ (vs * np.abs(vc))) + 2 * half * (p @ np.abs(vm))
        e = e + 2.2 * np.minimum(es.max(1, keepdims=True), 0.05) * (p @ np.abs(v))
        out[g] = p @ v
        bound[g] = e * (1 + half) + half * np.abs(out[g]) + 1e-30
    return out, bound


# ---------------------------------------------------------------------------------------------- bounds that see a lost piece
@pytest.mark.parametrize("dim,group,heads", [(128, 32, 8), (128, 128, 32), (64, 64, 8)])
@pytest.mark.parametrize("weight", [1.0 + 2.0 ** -8 * 0.97, 1.0 + 2.0 ** -8 * 1.03, 2.0 + 2.0 ** -7 * 0.97])
def test_attention_of_a_constant_under_weights_that_bf16_cannot_hold(dim, group, heads, weight):
    """Values that are one constant come back as it: the softmax's weights sum to one, whatever they are.  The scores of the first
    rows are lower than those of the rest by the logarithm of `weight`, which lies next to the middle between two bf16 numbers, so
    weights rounded to bf16 on one side of the division only would move the output by up to 2^-8.
    Bound: the weights of the mids are held to 2^-17 relative, the sums of a unit's 1280 rows in fp32 (2^-23 a step, 50 steps), the
    division and the exponentials cancel: 2^-17 + 2^-17; and half a step of the output."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    shape = shape_of(heads, 2, dim)
    lib = context(shape)
    n, rows, first = sms, 1280, 128                                  # as many units as resident blocks; four warps' first steps
    from paper_2601_13155_b200 import binding
    cache = binding.Kv4Cache(shape, n, rows, group=group)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(0x88)                                                # code 8 stands for the mid
    cache.k_params.zero_()
    cache.k_params[:, :, first:, :, 1] = float(np.log(weight) / np.sqrt(dim))       # q = 1: score = sqrt(d) mid
    const = 61.0
    cache.v_params[..., 0] = 2.0 ** -6
    cache.v_params[..., 1] = const
    cache.length.fill_(rows)
    q = torch.ones(n, heads, dim, dtype=torch.bfloat16, device="cuda")
    out = lib.kv4_attention(cache, q)
    # 61 lies between 32 and 64: half a step is 2^-3
    assert float((out.double() - const).abs().max()) <= 2.0 ** -3 * 0.999
    assert bool((out == const).all())                                # 61 is a bf16 number, and 2^-16 * 61 is less than half a step
    lib.close()


@pytest.mark.parametrize("n,out,k,group", [(1, 1000, 4096, 64), (8, 500, 4096, 128), (20, 300, 8192, 32)])
def test_fp32_outputs_hold_fp32_sums(n, out, k, group):
    """The root mean square of the error, where the element by element bound is too wide to see a lost piece of the groups' sums.

    With s the scale, x ~ N(0, 1) and g groups of m elements, an output's RMS is 4.6 sqrt(g m) s.  A group's sum of x, about sqrt(m),
    in two bf16 pieces instead of three would be off by 2^-17 * 0.436 of a number in [1, 2) (the second piece rounds what is left,
    uniform below 2^-8, to eight bits), 2.3e-6 of the sum: 8 s sqrt(m) 2.3e-6 sqrt(g), 4.0e-6 of the RMS.
    In three pieces what is left are fp32 steps, of matrix units that may truncate (2^-24 of the partial sum on average): m / 16
    steps of a group, whose partial sums are about 8.8 sqrt(m) s and of either sign: m / 16 2^-24 8.8 sqrt(m) sqrt(g) s, 9e-7 of the
    RMS for m = 128; and here at most 18 steps of a warp's outputs: 18 * 2^-24 = 1.1e-6 if all erred to one side at the output's
    full size, of which they have half on average.  The root of the squares' sum is below 1.1e-6; 2e-6 lies between it and 4.0e-6."""
    lib = context()
    w = rand_w4(out, k, group, 21, mids=False)
    x = torch.randn(n, k, device="cuda", generator=gen(4)).to(lib.dtype)
    want = R.f64(x) @ R.values(w.codes, w.params)[0].T
    err = R.f64(lib.w4_gemv(w, x, fp32_out=True)) - want
    assert np.sqrt((err ** 2).mean()) <= 2e-6 * np.sqrt((want ** 2).mean())
    lib.close()


@pytest.mark.parametrize("n,out", [(8, 60000), (12, 40000)])
def test_bf16_outputs_are_those_of_fp32_sums(n, out):
    """How many outputs round to another bf16 number than the exact ones do.  An output that is off by e rounds differently with the
    probability |e| / ulp; of outputs of a normal distribution of RMS 1 above a quarter, the mean of 1 / ulp is 2^7 * 1.44 * 1.45 =
    267.  With the errors of the test above (in three pieces below 1.1e-6 in the root mean square, in two 4.0e-6; the mean size is
    0.8 of it) that are at most 2.3e-4 of the outputs, or 8.5e-4; 5e-4 lies between."""
    lib = context()
    k, group = 1024, 64
    w = rand_w4(out, k, group, 21, mids=False)
    x = torch.randn(n, k, device="cuda", generator=gen(4)).to(lib.dtype)
    c = torch.stack([w.codes & 15, w.codes >> 4], -1).reshape(out, k).double() - 8
    want = x.double() @ (c * w.params[..., 0].double().repeat_interleave(group, -1)).T
    got = lib.w4_gemv(w, x)
    seen = want.abs() > 0.25 * want.square().mean().sqrt()
    assert float((got != want.to(torch.bfloat16))[seen].double().mean()) <= 5e-4
    lib.close()


# ---------------------------------------------------------------------------------------------- from the prefill to the 4-bit step
@pytest.mark.parametrize("shape", [replace(WIDE, n_layers=3, vocab=1024), replace(synth.TINY, hidden=256, ffn_dim=672, n_layers=3)], ids=["bf16", "fp32"])
def test_from_a_skipping_prefill_to_generation(shape):
    """A prompt goes through the skipping prefill, whose caches differ in length and positions from layer to layer; they enter the
    4-bit caches layer by layer, and two tokens are generated.  Each step against the plain 64-bit layers on what the 4-bit caches
    and weights stand for, within the bounds of the other decode tests."""
    from paper_2601_13155_b200 import binding, schedule
    seed, N, L = 31, 300, shape.n_layers
    lib = binding.Spts(shape, max_seq=N)
    arrays = [synth.layer_weights(shape, seed, l) for l in range(L)]
    hw = synth.head_weights(shape, seed)
    embed = up(hw["embed"], shape.dtype)
    model = binding.Model([binding.LayerWeights(a, shape.dtype) for a in arrays], up(hw["lm_head"], shape.dtype), embed)
    ids = np.random.default_rng(seed).integers(0, shape.vocab, N)
    X = embed[torch.from_numpy(ids).cuda()].clone()
    plan = [(N, N, 200), (120, 90, 0), (77, 64, 0)]
    cache = binding.KvCache(shape, L, [p[0] for p in plan])
    pos, orig = i32(np.arange(N)), i32(np.arange(N))
    token = torch.empty(1, dtype=torch.int32, device="cuda")
    lib.prefill(model, plan, X, pos, orig, torch.empty_like(X), torch.empty_like(pos), torch.empty_like(orig), cache, token_out=token)
    lens = [cache.length(l) for l in range(L)]
    assert lens == [300, 120, 77]

    caches = binding.Kv4Caches(shape, L, 1, max(lens) + 8, group=32)
    for l in range(L):
        k, v, at = cache.k[l][:lens[l]], cache.v[l][:lens[l]], i32([0])
        lib.kv4_append(caches.layers[l], k, v, pos=cache.pos[l][:lens[l]], row_start=i32([0, lens[l]]), at=at)
        assert caches.layers[l].length.tolist() == [lens[l]]
        assert torch.equal(caches.layers[l].pos[0, :lens[l]], cache.pos[l][:lens[l]])
        held = R.cache_rows(caches.layers[l].k_codes[0, 0, :lens[l]], caches.layers[l].k_params[0, 0, :lens[l]], R.key_dims(shape.head_dim))[0]
        assert np.array_equal(held, R.quantise(R.f64(k[:, 0]), 32)[3])
    q = [lib.quantize_layer4({n: up(a[n], shape.dtype) for n in a}, 32) for a in arrays]
    lm = lib.w4_quantize(up(hw["lm_head"], shape.dtype), 32)
    model4 = binding.Model4(q, lm, embed)
    x_out, logits = torch.empty(1, shape.hidden, dtype=lib.dtype, device="cuda"), torch.empty(1, shape.vocab, device="cuda")
    tol = 4e-2 if shape.dtype == "bf16" else 2e-4
    for step in range(2):
        before, at = int(token), i32([N + step])
        assert 0 <= before < shape.vocab
        lib.decode_step4(model4, caches, at, token_in=token, x_out=x_out, logits_out=logits, token_out=token)
        assert lib.device_status() == 0 and lib.check_guards() == 0
        x = host(embed[before])
        for l in range(L):
            x = reference_layer(x, N + step, q[l], shape, caches.layers[l], 0, lens[l] + step + 1, shape.dtype)
        assert rel_rms_err(host(x_out[0]), x) <= tol * L
        assert int(token) == int(np.argmax(host(logits[0])))
        assert [c.length.tolist() for c in caches.layers] == [[n + step + 1] for n in lens]
    lib.close()


# ---------------------------------------------------------------------------------------------- quantiser
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_stored_numbers_are_rounded_by_way_of_fp32(dtype):
    """Scale and mid are 64-bit numbers rounded to fp32 and from there to bf16.  A largest element far below half a step of
    the sum shows it: (-248 + tiny + 16.5) / 2 rounds to -115.75 in fp32, a tie that goes to -116, where one rounding gives -115.5."""
    lib = context(shape_of(dtype=dtype))
    x = torch.full((4, 32), -100.0)
    x[:, 3] = -248.0
    x[:, 9] = torch.tensor([2.0 ** -20, 2.0 ** -30, 0.0, 2.0 ** -10])
    W = x.to(lib.dtype).cuda()
    w = lib.w4_quantize(W, 32)
    codes, scale, mid, _ = R.quantise(R.f64(W), 32)
    s, m = R.split_params(w.params)
    assert np.array_equal(s, scale) and np.array_equal(m, mid) and np.array_equal(R.nibbles(w.codes), codes)
    assert m[:, 0].tolist() == [-116.0, -116.0, -116.0, -115.5]
    lib.close()


# ---------------------------------------------------------------------------------------------- cache append
@pytest.mark.parametrize("start,want,code", [
    ([0, 3, 12], [3, 15], 8),            # the last sequence claims four rows more than there are
    ([0, 9, 9], [8, 10], 8),
    ([0, 20, 30], [8, 10], 8),           # a sequence that begins behind the last row
    ([0, 3, 8], [3, 15], 0),
    ([2, 3, 5], [1, 12], 0),             # rows before the first and behind the last sequence are nobody's
    ([5, 3, 8], [0, 15], 8),             # starts that descend
    ([-2, 3, 8], [3, 15], 8),            # rows before the first row
])
def test_append_counts_the_rows_that_there_are(start, want, code):
    from paper_2601_13155_b200 import binding
    lib = context()
    cache = binding.Kv4Cache(shape_of(), 2, 32, group=64)
    fill_garbage(cache, 1)
    before = cache.k_codes.clone()
    K = torch.randn(8, 2, 128, device="cuda", generator=gen(2)).to(torch.bfloat16)
    lib.kv4_append(cache, K, K, row_start=i32(start), at=i32([0, 10]))
    assert lib.device_status() == code
    assert cache.length.tolist() == want
    changed = (cache.k_codes != before).any(-1).any(1)
    held = torch.zeros(2, 32, dtype=torch.bool, device="cuda")
    held[0, :want[0]] = True
    held[1, 10:want[1]] = True
    assert torch.equal(changed, held)                                # every row that the length counts was written, and no other
    lib.close()


def test_append_refuses_values_that_take_the_other_matrix_s_place():
    """K_out may be K and V_out V where their rows are packed; anything else would be read and written in no order."""
    from paper_2601_13155_b200 import binding
    lib = context()
    cache = binding.Kv4Cache(shape_of(), 3, 32, group=64)
    wide = torch.randn(3, 2 * 256, device="cuda", generator=gen(2)).to(torch.bfloat16)
    K, V = torch.randn(3, 2, 128, device="cuda").to(torch.bfloat16), torch.randn(3, 2, 128, device="cuda").to(torch.bfloat16)
    ptr = lambda t: C.c_void_p(t.data_ptr())
    call = lambda k, ldk, v, ldv, kr, vr: lib.lib.spts_kv4_append(lib.h, C.byref(cache.c), ptr(k), ldk, ptr(v), ldv, None, None, None, 3, kr, vr)
    assert call(K, 256, V, 256, ptr(V), None) == 1
    assert call(K, 256, V, 256, None, ptr(K)) == 1
    assert call(wide, 512, V, 256, ptr(wide), None) == 1
    assert call(K, 256, wide, 512, None, ptr(wide)) == 1
    assert cache.length.tolist() == [0, 0, 0]
    assert call(K, 256, V, 256, ptr(K), ptr(V)) == 0
    assert cache.length.tolist() == [1, 1, 1] and lib.device_status() == 0
    lib.close()
