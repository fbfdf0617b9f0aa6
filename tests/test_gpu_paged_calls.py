"""The paged cache beside the framework's other paths: what a skipping prefill leaves enters a pool that all layers share, attention agrees
with the reduced attention of the prefill, a next turn attends to it, and the logits of the head are scored."""
import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2601_13155_b200 import binding, synth
from test_gpu_paged import near

pytestmark = pytest.mark.gpu

SMALL = synth.ModelShape(hidden=512, n_q_heads=4, n_kv_heads=2, head_dim=128, ffn_dim=512, ltp_dlow=64, ltp_rank=16, n_layers=3, vocab=1003,
                         dtype="bf16")


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("shape", [SMALL, synth.TINY], ids=["bf16", "fp32"])
def test_from_a_skipping_prefill_to_a_next_turn(shape):
    seed, N, L = 7, 300, shape.n_layers
    lib = binding.Spts(shape, max_seq=N)
    arrays = [synth.layer_weights(shape, seed, l) for l in range(L)]
    hw = synth.head_weights(shape, seed)
    embed, lm_head = binding.to_device(hw["embed"], shape.dtype), binding.to_device(hw["lm_head"], shape.dtype)
    model = binding.Model([binding.LayerWeights(a, shape.dtype) for a in arrays], lm_head, embed)
    ids = np.random.default_rng(seed).integers(0, shape.vocab, N)
    X = embed[torch.from_numpy(ids).cuda()].clone()
    plan = ([(N, N, 200), (120, 90, 0), (77, 64, 0)] + [(70, 60, 0)] * L)[:L]
    cache = binding.KvCache(shape, L, [p[0] for p in plan])
    pos, orig = i32(np.arange(N)), i32(np.arange(N))
    _, in_alt = lib.prefill(model, plan, X, pos, orig, X_alt := torch.empty_like(X), torch.empty_like(pos), torch.empty_like(orig), cache)
    lens = [cache.length(l) for l in range(L)]
    assert lens == [p[0] for p in plan]
    # one pool for all layers: every layer has a table of its own
    page, hkv, d, h = 16, shape.n_kv_heads, shape.head_dim, shape.n_q_heads
    need = [-(-(n + 40) // page) for n in lens]
    order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(seed)).to(torch.int32).to("cuda")
    pool = binding.PagedKv(shape, order[None], page_size=page, n_pages=sum(need), positions=True, weights=True)
    layers = []
    for l in range(L):
        table = order[sum(need[:l]):sum(need[:l + 1])][None].contiguous()
        layers.append(binding.PagedKv(shape, table, page_size=page, k=pool.k, v=pool.v, pos=pool.pos, weight=pool.weight))
        lib.paged_append(layers[l], cache.k[l][:lens[l]], cache.v[l][:lens[l]], pos=cache.pos[l][:lens[l]], row_start=i32([0, lens[l]]))
    assert lib.device_status() == 0
    g = torch.Generator().manual_seed(seed)

    def rows_of(c, n):
        j = torch.arange(n, device="cuda")
        slot = c.table[0].long()[j // page] * page + j % page
        return c.k.view(-1, hkv, d)[slot], c.v.view(-1, hkv, d)[slot], c.pos.view(-1)[slot], c.weight.view(-1)[slot]
    for l in range(L):
        n = lens[l]
        k, v, at, _ = rows_of(layers[l], n)
        assert torch.equal(k, cache.k[l][:n]) and torch.equal(v, cache.v[l][:n]) and torch.equal(at, cache.pos[l][:n])
        # all rows as one chunk: the causal attention among them, as the prefill computes it
        q = torch.randn(n, h, d, generator=g).to(lib.dtype).to("cuda")
        o, e, _, _ = R.attention(q, k, v, 0, lib.dtype)
        near(lib.reduced_attention(q, k.contiguous(), v.contiguous()).view(n, h, d), o, e)
        out, lse = lib.paged_attention(layers[l], q, row_start=i32([0, n]), want_lse=True)
        near(out.view(n, h, d), o, e)
        # its last queries judge the rows, a third of them stays, and the next turn attends to those
        lib.paged_weights(layers[l], q[-16:], lse[-16:].contiguous(), row_start=i32([0, 16]), decay=0.0)
        before = rows_of(layers[l], n)
        lib.paged_evict(layers[l], i32([n // 3]), n_sink=4, n_recent=8)
        kept = R.evict(*before, n // 3, 4, 8)
        new = [torch.randn(25, hkv, d, generator=g).to(lib.dtype).to("cuda") for _ in range(2)]
        lib.paged_append(layers[l], new[0], new[1], pos=i32(np.arange(N, N + 25)), row_start=i32([0, 25]))
        q = torch.randn(25, h, d, generator=g).to(lib.dtype).to("cuda")
        out = lib.paged_attention(layers[l], q, row_start=i32([0, 25]))
        assert lib.device_status() == 0 and lib.check_guards() == 0
        o, e, _, _ = R.attention(q, torch.cat([kept[0], new[0]]), torch.cat([kept[1], new[1]]), n // 3, lib.dtype)
        near(out.view(25, h, d), o, e)
    # the layers share the pool and leave each other's rows alone
    for l in range(L):
        assert int(layers[l].length[0]) == lens[l] // 3 + 25
        assert int(rows_of(layers[l], int(layers[l].length[0]))[2].max()) == N + 24
    # the head's logits: its token has rank 0, a given one the place that sorting gives it
    logits, token = torch.empty(shape.vocab, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    last = (X_alt if in_alt else X)[plan[-1][0] - 1].contiguous()
    lib.first_token(last, lm_head, logits_out=logits, token_out=token)
    scored = lib.token_logprobs(logits[None].expand(2, -1).contiguous(), torch.cat([token, i32([5])]), n_top=3)
    lp, rank, ent, top, tok, e, ee = R.logprobs(logits, 5, 3)
    assert scored["rank"].tolist() == [0, rank] and scored["top_token"][0].tolist() == tok and int(token) == tok[0]
    assert abs(float(scored["logprob"][1]) - lp) <= e + 2.0 ** -23 * abs(lp) and abs(float(scored["entropy"][0]) - ent) <= ee + 2.0 ** -23 * abs(ent)
    lib.close()


def test_an_option_selects_the_plain_kernels_and_takes_them_back():
    """SPTS_REFERENCE_KERNELS reaches these calls of a bf16 context: fp32 weights of the softmax, not rounded before they meet V."""
    lib = binding.Spts(SMALL, max_seq=64)
    pages = R.Pages(SMALL, [200], 32, seed=1)
    q, start = R.queries(SMALL, [9], seed=1)
    first = lib.paged_attention(pages.c, q, row_start=start)
    lib.set_reference_kernels(True)
    plain = lib.paged_attention(pages.c, q, row_start=start)
    lib.set_reference_kernels(False)
    again = lib.paged_attention(pages.c, q, row_start=start)
    assert torch.equal(first, again) and not torch.equal(first, plain)
    k, v = pages.held(0)[:2]
    o, e, _, _ = R.attention(q, k, v, 191, torch.bfloat16)
    near(first.view(9, 4, 128), o, e)
    near(plain.view(9, 4, 128), o, e)
    lib.close()
