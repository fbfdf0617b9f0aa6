"""Decode steps with 4-bit weights and caches: the calls together, against the plain 64-bit layer on the values that the 4-bit
forms stand for, against the same calls one by one, and replayed from a captured graph."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import generate4_ref as R
from oracle import spts_oracle as O
from paper_2601_13155_b200 import synth
from parity_utils import dev, host, i32, rel_rms_err, up

pytestmark = pytest.mark.gpu

WIDE = replace(synth.LLAMA8B, hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=128, ffn_dim=1024, ltp_dlow=64, ltp_rank=16, n_layers=2,
               vocab=1003)
ODD = replace(synth.TINY, hidden=256, n_q_heads=6, n_kv_heads=2, head_dim=64, ffn_dim=672, n_layers=2, vocab=515)


def build(shape, group, cache_group, lens, seed, dtype=None):
    from paper_2601_13155_b200 import binding
    shape = replace(shape, dtype=dtype or shape.dtype)
    lib = binding.Spts(shape, max_seq=64)
    arrays = [synth.layer_weights(shape, seed, l) for l in range(shape.n_layers)]
    tensors = [{k: up(v, shape.dtype) for k, v in a.items()} for a in arrays]
    q = [lib.quantize_layer4(t, group) for t in tensors]
    head = synth.head_weights(shape, seed)
    lm, embed = lib.w4_quantize(up(head["lm_head"], shape.dtype), group), up(head["embed"], shape.dtype)
    model = binding.Model4(q, lm, embed)
    caches = binding.Kv4Caches(shape, shape.n_layers, len(lens), max(lens) + 40, group=cache_group)
    rng = np.random.default_rng(seed)
    start = i32(np.concatenate([[0], np.cumsum(lens)]))
    total = int(sum(lens))
    for cache in caches.layers:                                   # what a prompt left behind
        k, v = (torch.from_numpy(rng.normal(size=(total, shape.n_kv_heads, shape.head_dim)).astype(np.float32)).to(dev()).to(lib.dtype) for _ in range(2))
        lib.kv4_append(cache, k, v, pos=i32(np.arange(total)), row_start=start, at=i32(np.zeros(len(lens))))
    return lib, shape, model, q, lm, embed, caches


def reference_layer(x, pos, w, shape, cache, b, ln, mode):
    """One token through one layer in 64 bits; the cache's rows and the quantised new row are read back from the device."""
    rnd = O.rounding(mode)
    H, Hkv, d = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    vals = {n: R.values(w[n].codes, w[n].params)[0] for n in w}
    ones = np.ones(len(x))
    a = O.rmsnorm(x[None], ones, shape.rms_eps)
    qkv = (a @ vals["wqkv"].T)[0]
    q = rnd(O.rope(qkv[:H * d].reshape(1, H, d), [pos], shape.rope_theta))[0]
    k = O.rope(qkv[H * d:(H + Hkv) * d].reshape(1, Hkv, d), [pos], shape.rope_theta)[0]
    v = qkv[(H + Hkv) * d:].reshape(Hkv, d)
    att = np.zeros((H, d))
    for kv in range(Hkv):
        K = R.cache_rows(cache.k_codes[b, kv, :ln], cache.k_params[b, kv, :ln], R.key_dims(d))[0]
        V = R.cache_rows(cache.v_codes[b, kv, :ln], cache.v_params[b, kv, :ln], R.value_dims(d))[0]
        # the row that the step appended stands for its k and v within half a step of its groups (and the rounding to storage)
        for held, new, prm in ((K[-1], k[kv], cache.k_params), (V[-1], v[kv], cache.v_params)):
            s, m = R.split_params(prm[b, kv, ln - 1])
            s, m = np.repeat(s, d // len(s)), np.repeat(m, d // len(m))
            assert (np.abs(held - new) <= 0.54 * s + 2.0 ** -7 * (np.abs(m) + 8 * s) + 2e-2 * np.abs(new).max()).all()
        g = slice(kv * (H // Hkv), (kv + 1) * (H // Hkv))
        z = q[g] @ K.T / np.sqrt(d)
        e = np.exp(z - z.max(1, keepdims=True))
        att[g] = (e / e.sum(1, keepdims=True)) @ V
    x = rnd(x + vals["wo"] @ rnd(att.reshape(-1)))
    hm = O.rmsnorm(x[None], ones, shape.rms_eps)[0]
    return rnd(x + vals["w_down"] @ rnd(O.silu(vals["w_gate"] @ hm) * (vals["w_up"] @ hm)))


@pytest.mark.parametrize("shape,dtype,group,cache_group,lens", [
    (WIDE, "bf16", 128, 32, [33]), (WIDE, "bf16", 64, 128, [5, 0, 70, 12]), (WIDE, "fp32", 32, 64, [40, 3]),
    (ODD, "bf16", 32, 32, [17, 1, 64]), (ODD, "fp32", 32, 64, [9]), (WIDE, "bf16", 128, 64, [3] * 11),
])
def test_step_against_the_plain_layers(shape, dtype, group, cache_group, lens):
    """Two steps; hidden state and logits within the bounds of the other decode tests (twice the layer bound of the storage
    type, per layer: 4e-2 of the RMS in bf16, 2e-4 in fp32), the token that of the step's own logits."""
    lib, shape, model, q, lm, embed, caches = build(shape, group, cache_group, lens, seed=77, dtype=dtype)
    n, D = len(lens), shape.hidden
    tol = 4e-2 if dtype == "bf16" else 2e-4
    x_out = torch.empty(n, D, dtype=lib.dtype, device=dev())
    logits, token = torch.empty(n, shape.vocab, device=dev()), i32(np.arange(n) * 7 + 1)
    for step in range(2):
        before = token.tolist()
        pos = i32([100 + 3 * b + step for b in range(n)])
        lib.decode_step4(model, caches, pos, token_in=token, x_out=x_out, logits_out=logits, token_out=token)
        assert lib.device_status() == 0 and lib.check_guards() == 0
        assert caches.layers[-1].length.tolist() == [v + step + 1 for v in lens]
        lm_vals = R.values(lm.codes, lm.params)[0]
        for b in range(n):
            x = host(embed[before[b]])
            ln = lens[b] + step + 1
            for l in range(shape.n_layers):
                x = reference_layer(x, int(pos[b]), q[l], shape, caches.layers[l], b, ln, dtype)
                assert int(caches.layers[l].pos[b, ln - 1]) == int(pos[b])
            assert rel_rms_err(host(x_out[b]), x) <= tol * shape.n_layers
            want = lm_vals @ O.rmsnorm(x[None], np.ones(D), shape.rms_eps)[0]
            assert rel_rms_err(host(logits[b]), want) <= tol * shape.n_layers
            assert int(token[b]) == int(np.argmax(host(logits[b])))
    lib.close()


def test_step_equals_its_calls_one_by_one():
    lens = [20, 0, 7]
    lib, shape, model, q, lm, embed, caches = build(WIDE, 128, 32, lens, seed=5)
    _, _, _, _, _, _, other = build(WIDE, 128, 32, lens, seed=5)
    H, Hkv, d = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    from paper_2601_13155_b200 import binding
    hist = i32([1, 2, 3, 3, 9, 9, 9, 500])
    rules = binding.LogitsRules(history=hist, history_start=i32([0, 3, 5, 8]), repetition=torch.full((3,), 1.3, device=dev()),
                                frequency=torch.full((3,), 0.2, device=dev()), mask=torch.full((3, 32), -1431655766, dtype=torch.int32, device=dev()))
    x_in = torch.randn(3, shape.hidden, device=dev(), generator=torch.Generator(device="cuda").manual_seed(1)).to(lib.dtype)
    pos = i32([50, 60, 70])
    x_out, logits = torch.empty_like(x_in), torch.empty(3, shape.vocab, device=dev())
    token = torch.empty(3, dtype=torch.int32, device=dev())
    lib.decode_step4(model, caches, pos, x_in=x_in, rules=rules, x_out=x_out, logits_out=logits, token_out=token)
    x = x_in.clone()
    for l in range(shape.n_layers):
        y = lib.w4_gemv(q[l]["wqkv"], x, norm=True, fp32_out=True)
        # the rotation in 32 bits, with the cosines and sines of 64 bits
        i = torch.arange(d // 2, dtype=torch.float64, device=dev())
        ang = pos.double()[:, None] * torch.exp2(-(2 * i) / d * np.log2(np.float64(np.float32(shape.rope_theta))))
        c, s = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
        heads = y.reshape(3, H + 2 * Hkv, d)
        a, b = heads[:, :H + Hkv, :d // 2], heads[:, :H + Hkv, d // 2:]
        rot = torch.cat([a * c - b * s, b * c + a * s], -1).to(lib.dtype)
        v = heads[:, H + Hkv:].to(lib.dtype)
        lib.kv4_append(other.layers[l], rot[:, H:].contiguous(), v.contiguous(), pos=pos)
        att = lib.kv4_attention(other.layers[l], rot[:, :H].contiguous())
        x = lib.w4_gemv(q[l]["wo"], att, residual=x)
        hm = lib.w4_gemv(q[l]["w_gate"], x, w2=q[l]["w_up"], norm=True)
        x = lib.w4_gemv(q[l]["w_down"], hm, residual=x)
    # the rotation's two products may be fused into one rounding: a stored bit here and there, no more than a bf16 step of the state
    assert rel_rms_err(host(x_out), host(x)) <= 2e-2
    lg, tok = lib.process_logits(lib.w4_gemv(lm, x_out, norm=True, fp32_out=True), rules)
    assert torch.equal(lg, logits) and torch.equal(tok, token)
    assert other.layers[0].length.tolist() == [21, 1, 8] == caches.layers[0].length.tolist()
    lib.close()


def test_generation_replayed_from_one_graph():
    """Eight tokens: stepped one by one, and one captured step (with the positions' increment) replayed."""
    from paper_2601_13155_b200 import binding
    runs = []
    for mode in ("steps", "graph"):
        st = torch.cuda.Stream()
        lib, shape, model, q, lm, embed, caches = build(WIDE, 128, 64, [9, 30], seed=11)
        lib.close()
        lib = binding.Spts(shape, max_seq=64, stream=st)
        pos, token = i32([9, 30]), i32([3, 4])
        logits = torch.empty(2, shape.vocab, device=dev())
        one = torch.ones(2, dtype=torch.int32, device=dev())
        got = []
        torch.cuda.synchronize()

        def step():
            lib.decode_step4(model, caches, pos, token_in=token, logits_out=logits, token_out=token)
            pos.add_(one)
        if mode == "steps":
            with torch.cuda.stream(st):
                for _ in range(8):
                    step()
                    got.append((token.clone(), logits.clone()))
            torch.cuda.synchronize()
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                step()
            for _ in range(8):
                g.replay()
                torch.cuda.synchronize()
                got.append((token.clone(), logits.clone()))
            del g
        assert caches.layers[1].length.tolist() == [17, 38] and lib.device_status() == 0
        runs.append(got)
        lib.close()
    for (ta, la), (tb, lb) in zip(*runs):
        assert torch.equal(ta, tb) and torch.equal(la, lb)


def test_step_refusals():
    from paper_2601_13155_b200 import binding
    lib, shape, model, q, lm, embed, caches = build(WIDE, 128, 64, [4, 5], seed=2)
    pos, token = i32([4, 5]), i32([1, 2])
    logits = torch.empty(2, shape.vocab, device=dev())
    for kw in (dict(token_in=None), dict(token_in=token, token_out=token)):
        with pytest.raises(binding.SptsError):
            lib.decode_step4(model, caches, pos, **kw)
    with pytest.raises(ValueError):
        lib.decode_step4(model, caches, pos[:1], token_in=token)
    with pytest.raises(ValueError):
        lib.decode_step4(binding.Model4(q[:1], lm, embed), caches, pos, token_in=token)
    bad = [dict(q[0]), dict(q[1])]
    bad[1]["wo"] = q[1]["w_gate"]
    with pytest.raises(binding.SptsError):
        lib.decode_step4(binding.Model4(bad, lm, embed), caches, pos, token_in=token)
    many = binding.Kv4Caches(shape, 2, 33, 32)
    with pytest.raises(binding.SptsError):
        lib.decode_step4(model, many, i32(np.zeros(33)), token_in=i32(np.zeros(33)))
    # a token outside the vocabulary (a dead end of the rules gives -1) is reported, not read
    lib.decode_step4(model, caches, pos, token_in=i32([-1, shape.vocab]), logits_out=logits)
    assert lib.device_status() == 8
    assert torch.isfinite(logits).all()
    # caches without room: reported, lengths stay at the capacity
    for cache in caches.layers:
        cache.length.fill_(cache.capacity)
    lib.decode_step4(model, caches, pos, token_in=token, logits_out=logits)
    assert lib.device_status() == 3 and caches.layers[0].length.tolist() == [caches.layers[0].capacity] * 2
    lib.close()
