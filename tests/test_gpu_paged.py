"""Serving over a paged cache on the GPU against plain 64-bit forms: append, chunk attention, gathered weights, eviction."""
import pytest
import torch

import paged_ref as R
from paper_2601_13155_b200 import binding, synth

pytestmark = pytest.mark.gpu


def shape_of(heads, kv, dim, dtype="bf16"):
    return synth.ModelShape(hidden=heads * dim, n_q_heads=heads, n_kv_heads=kv, head_dim=dim, ffn_dim=256, ltp_dlow=64, ltp_rank=16, n_layers=1,
                            vocab=64, dtype=dtype)


_contexts = {}


def context(shape, plain=False):
    key = (shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.dtype, plain)
    if key not in _contexts:
        lib = binding.Spts(shape, max_seq=64)
        if plain:
            lib.set_reference_kernels(True)
        _contexts[key] = lib
    return _contexts[key]


@pytest.fixture(autouse=True, scope="module")
def _close():
    yield
    for lib in _contexts.values():
        assert lib.check_guards() == 0
        lib.close()
    _contexts.clear()


def done(lib, status=0):
    assert lib.device_status() == status
    assert lib.check_guards() == 0


def near(got, want, bound, what=""):
    got, want, bound = got.double(), want.double(), bound.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    assert bool((off <= bound).all()), f"{what}: worst {float((off / bound).max()):.3g} of the bound"


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim,kv", [(128, 8), (64, 1), (64, 3), (128, 1)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_append_rows_of_ragged_sequences(dtype, dim, kv, page):
    shape = shape_of(kv, kv, dim, dtype)
    lib = context(shape)
    lens, new = [0, 5, page, 3 * page - 1, 17], [3, 0, 2 * page + 1, 1, page - 1]
    pages = R.Pages(shape, lens, page, seed=dim + kv, room=2 * page + 8)
    before = [pages.held(b) for b in range(5)]
    total = sum(new)
    wide_k = torch.randn(total + 2, kv * dim + 16, device="cuda").to(lib.dtype)
    wide_v = torch.randn(total + 2, kv * dim + 32, device="cuda").to(lib.dtype)
    K, V = wide_k[:, 8:8 + kv * dim], wide_v[:, 16:16 + kv * dim]
    pos = torch.randint(0, 1 << 30, (total + 2,), dtype=torch.int32, device="cuda")
    start = torch.tensor([sum(new[:i]) for i in range(6)], dtype=torch.int32, device="cuda")
    untouched = pages.c.k.clone()
    lib.paged_append(pages.c, K, V, pos=pos, row_start=start)
    done(lib)
    written = torch.zeros(untouched.shape[:2], dtype=torch.bool)
    for b in range(5):
        k, v, p, w = pages.held(b)
        r = slice(int(start[b]), int(start[b + 1]))
        assert k.shape[0] == lens[b] + new[b]
        for got, old, add in ((k, before[b][0], K[r].reshape(-1, kv, dim)), (v, before[b][1], V[r].reshape(-1, kv, dim)), (p, before[b][2], pos[r])):
            assert torch.equal(got, torch.cat([old, add]))
        assert torch.equal(w, torch.cat([before[b][3], torch.zeros(new[b], device="cuda")]))
        written.view(-1)[pages.slots(b, torch.arange(lens[b], lens[b] + new[b]))] = True
    same = (pages.c.k == untouched) | (torch.isnan(pages.c.k) & torch.isnan(untouched))
    assert bool(same[~written.to("cuda")].all())


def test_append_single_rows_at_given_places():
    shape = shape_of(4, 2, 64)
    lib = context(shape)
    pages = R.Pages(shape, [40, 1, 0, 33], 16, room=20)
    K, V = torch.randn(4, 2, 64, device="cuda").bfloat16(), torch.randn(4, 2, 64, device="cuda").bfloat16()
    at = torch.tensor([30, 1, 0, 33], dtype=torch.int32, device="cuda")        # the first sequence goes back ten rows
    lib.paged_append(pages.c, K, V, at=at)
    done(lib)
    assert pages.c.length.tolist() == [31, 2, 1, 34]
    for b in range(4):
        assert torch.equal(pages.held(b)[0][-1], K[b]) and torch.equal(pages.held(b)[1][-1], V[b])
        assert float(pages.held(b)[3][-1]) == 0.0
    # places given by the lengths themselves are the rows behind
    lib.paged_append(pages.c, K, V, at=pages.c.length)
    done(lib)
    assert pages.c.length.tolist() == [32, 3, 2, 35]


def test_append_beyond_the_table_and_with_bad_entries_is_reported():
    shape = shape_of(4, 2, 64)
    lib = context(shape)
    pages = R.Pages(shape, [30, 4], 16)
    K, V = torch.randn(12, 2, 64, device="cuda").bfloat16(), torch.randn(12, 2, 64, device="cuda").bfloat16()
    start = torch.tensor([0, 6, 12], dtype=torch.int32, device="cuda")
    kept = pages.held(0)[0]
    lib.paged_append(pages.c, K, V, row_start=start)
    done(lib, 3)                                    # two rows of room, SPTS_ERR_WORKSPACE
    assert pages.c.length.tolist() == [32, 10]
    assert torch.equal(pages.held(0)[0], torch.cat([kept, K[:2]])) and torch.equal(pages.held(1)[0][4:], K[6:])
    # an entry that names no page, one beyond the pages
    for beyond in (False, True):
        pages = R.Pages(shape, [16, 4], 16, room=16)
        pages.c.table[0, 1] = pages.c.n_pages if beyond else -1
        before = pages.c.k.clone()
        lib.paged_append(pages.c, K[:2], V[:2])
        done(lib, 8)                                # SPTS_ERR_INDEX
        assert pages.c.length.tolist() == [17, 5]
        changed = (pages.c.k != before) & ~(torch.isnan(pages.c.k) & torch.isnan(before))
        assert int(changed.flatten(2).any(-1).sum()) == 1


@pytest.mark.parametrize("start,lens", [([0, 9, 6], [9, 0]), ([0, 3, 100], [3, 3]), ([-4, 2, 6], [2, 4])])
def test_starts_that_break_the_rule_are_reported_and_stay_in_bounds(start, lens):
    shape = shape_of(4, 2, 64)
    lib = context(shape)
    pages = R.Pages(shape, [0, 0], 16, room=40)
    K, V = torch.randn(6, 2, 64, device="cuda").bfloat16(), torch.randn(6, 2, 64, device="cuda").bfloat16()
    lib.paged_append(pages.c, K, V, row_start=torch.tensor(start, dtype=torch.int32, device="cuda"))
    done(lib, 8)
    assert all(a <= 6 for a in pages.c.length.tolist())
    q = torch.randn(6, 4, 64, device="cuda").bfloat16()
    o, lse = lib.paged_attention(pages.c, q, row_start=torch.tensor(start, dtype=torch.int32, device="cuda"), want_lse=True)
    done(lib, 8)


# ------------------------------------------------------------------------------------------------ attention
def check_attention(shape, lens, rows, page, plain=False, seed=0, scale=1.0, pad=0, weights=True):
    lib = context(shape, plain)
    pages = R.Pages(shape, lens, page, seed=seed)
    q, start = R.queries(shape, rows, seed=seed, scale=scale, pad=pad)
    single = all(r == 1 for r in rows) and pad == 0
    h, d = shape.n_q_heads, shape.head_dim
    out = torch.full((q.shape[0], h * d), 7.0, dtype=lib.dtype, device="cuda")
    lse = torch.full((q.shape[0], h), 7.0, device="cuda")
    lib.paged_attention(pages.c, q, row_start=None if single else start, O_out=out, lse_out=lse)
    done(lib)
    for b, m in enumerate(rows):
        if m == 0:
            continue
        k, v = pages.held(b)[:2]
        r = slice(int(start[b]), int(start[b]) + m)
        o, e, l, el = R.attention(q[r], k, v, lens[b] - m, lib.dtype)
        near(out[r].view(m, h, d), o, e, f"O of sequence {b}")
        near(lse[r], l, el, f"lse of sequence {b}")
    assert bool((out[sum(rows):] == 7.0).all()) and bool((lse[sum(rows):] == 7.0).all())
    if weights:
        before = [pages.held(b)[3].clone() for b in range(len(lens))]
        whole = pages.c.weight.clone()
        lib.paged_weights(pages.c, q, lse, row_start=None if single else start, decay=0.5)
        done(lib)
        touched = torch.zeros_like(whole, dtype=torch.bool)
        for b, m in enumerate(rows):
            r = slice(int(start[b]), int(start[b]) + m)
            w, e = R.weights(q[r], pages.held(b)[0], lse[r], lens[b] - m)
            near(pages.held(b)[3], 0.5 * before[b].double() + w, e + 2.0 ** -23 * (before[b].double() + w), f"weights of sequence {b}")
            touched.view(-1)[pages.slots(b, torch.arange(lens[b])).to("cuda")] = True
        assert bool(torch.isnan(pages.c.weight[~touched]).all())
    return lib, pages, q, start, out, lse


KINDS = [("bf16", False), ("bf16", True), ("fp32", False)]


@pytest.mark.parametrize("dtype,plain", KINDS)
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (4, 4, 64), (7, 1, 128), (6, 2, 64), (32, 2, 128)])
@pytest.mark.parametrize("page", [16, 32, 128, 256])
def test_attention_of_ragged_chunks(dtype, plain, heads, kv, dim, page):
    """Lengths on both sides of tiles and pages, one query, one more than a tile of queries, a sequence without queries, one without rows."""
    lens = [1, 0, 127, 128, 129, 300, 513, 40]
    rows = [1, 2, 5, 128, 33, 0, 290, 40]
    check_attention(shape_of(heads, kv, dim, dtype), lens, rows, page, plain, seed=heads + page, pad=3)


@pytest.mark.parametrize("dtype,plain", KINDS)
@pytest.mark.parametrize("heads,kv,dim", [(32, 8, 128), (28, 4, 128), (4, 2, 64), (16, 1, 64)])
def test_attention_of_single_tokens(dtype, plain, heads, kv, dim):
    lens = [777, 1, 0, 4099, 128, 64, 2]
    check_attention(shape_of(heads, kv, dim, dtype), lens, [1] * 7, 64, plain, seed=dim)


@pytest.mark.parametrize("dtype,plain", KINDS)
def test_more_queries_than_rows(dtype, plain):
    """The first queries of a chunk that is longer than the cache see nothing: zeros and -inf."""
    shape = shape_of(8, 2, 128, dtype)
    lib, pages, q, start, out, lse = check_attention(shape, [3, 0, 200], [70, 9, 500], 16, plain, seed=5)
    for b, (held, m) in enumerate(zip([3, 0, 200], [70, 9, 500])):
        r = slice(int(start[b]), int(start[b]) + m - held)
        assert bool((out[r] == 0).all()) and bool((lse[r] == float("-inf")).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores(dtype):
    """Scores in the hundreds: one weight takes all, and the running maximum moves far and often."""
    check_attention(shape_of(8, 2, 128, dtype), [700, 260], [9, 260], 32, seed=9, scale=30.0)


@pytest.mark.parametrize("dtype,plain", KINDS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -3e38])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_is_not_seen_does_not_matter(dtype, plain, value, dim):
    """Rows that later queries alone see hold NaN, infinities or the lowest values: earlier queries are what they are without them."""
    shape = shape_of(8, 2, dim, dtype)
    lib = context(shape, plain)
    lens, rows = [150, 400], [60, 300]
    pages = R.Pages(shape, lens, 16, seed=2)
    q, start = R.queries(shape, rows, seed=2)
    clean, lse0 = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
    for b, cut in enumerate((120, 333)):
        j = pages.slots(b, torch.arange(cut, lens[b])).to("cuda")
        for t in (pages.c.k, pages.c.v):
            t.view(-1, 2, dim)[j] = value
    out, lse1 = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
    done(lib)
    for b, cut in enumerate((120, 333)):
        m = cut - (lens[b] - rows[b])
        r = slice(int(start[b]), int(start[b]) + m)
        o, e, l, el = R.attention(q[r], pages.held(b)[0][:cut], pages.held(b)[1][:cut], lens[b] - rows[b], lib.dtype)
        near(out[r].view(m, 8, dim), o, e, f"O of sequence {b}")
        near(lse1[r], l, el, "lse")
        later = out[int(start[b]) + m:int(start[b + 1])]
        if value != value:
            assert bool(torch.isnan(later).all())
    assert bool(torch.isfinite(clean).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [1, 40])
def test_values_that_are_not_finite_reach_the_queries_that_see_them(value, rows):
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    pages = R.Pages(shape, [3000], 64, seed=4)
    q, start = R.queries(shape, [rows], seed=4)
    pages.c.v.view(-1, 2, 128)[int(pages.slots(0, torch.tensor(1234))), 1, 5] = value
    out = lib.paged_attention(pages.c, q, row_start=start).view(rows, 8, 128)
    done(lib)
    hit = torch.zeros(rows, 8, 128, dtype=torch.bool)
    hit[:, 4:, 5] = True
    assert bool((~torch.isfinite(out.cpu()) == hit).all())
    assert bool((out.cpu()[hit] == value).all()) if value == value else bool(torch.isnan(out.cpu()[hit]).all())


@pytest.mark.parametrize("dtype,plain", KINDS)
def test_strided_queries_and_outputs(dtype, plain):
    shape = shape_of(8, 2, 128, dtype)
    lib = context(shape, plain)
    lens, rows = [200, 31], [50, 31]
    pages = R.Pages(shape, lens, 32, seed=3)
    q, start = R.queries(shape, rows, seed=3)
    want, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
    wide = torch.randn(81, 8 * 128 + 24, device="cuda").to(lib.dtype)
    wide[:, 16:16 + 1024] = q.view(81, -1)
    out = torch.full((81, 8 * 128 + 40), 5.0, device="cuda", dtype=lib.dtype)
    lib.paged_attention(pages.c, wide[:, 16:16 + 1024], row_start=start, O_out=out[:, 8:8 + 1024])
    done(lib)
    assert torch.equal(out[:, 8:1032], want) and bool((out[:, :8] == 5).all()) and bool((out[:, 1032:] == 5).all())
    w0 = pages.c.weight.clone()
    lib.paged_weights(pages.c, q, lse, row_start=start, decay=0.0)
    w1 = pages.c.weight.clone()
    pages.c.weight.copy_(w0)
    lib.paged_weights(pages.c, wide[:, 16:16 + 1024], lse, row_start=start, decay=0.0)
    done(lib)
    assert torch.equal(pages.c.weight.nan_to_num(-1.0), w1.nan_to_num(-1.0))


@pytest.mark.parametrize("plain", [False, True])
def test_entries_that_name_no_page_read_as_zeros(plain):
    shape = shape_of(8, 2, 128)
    lib = context(shape, plain)
    for bad in (-1, -2 ** 31, 10 ** 6, 2 ** 31 - 1):
        pages = R.Pages(shape, [200], 32, seed=6)
        q, start = R.queries(shape, [20], seed=6)
        k, v = pages.held(0)[0].clone(), pages.held(0)[1].clone()
        pages.c.table[0, 3] = bad
        k[96:128], v[96:128] = 0, 0
        out = lib.paged_attention(pages.c, q, row_start=start)
        done(lib, 8)
        o, e, _, _ = R.attention(q, k, v, 180, lib.dtype)
        near(out.view(20, 8, 128), o, e)


def test_sequences_that_share_pages():
    """Two sequences with the same first pages, as after a common prompt."""
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    pages = R.Pages(shape, [256, 100], 64, seed=8, room=64)
    pages.c.table[1, :4] = pages.c.table[0, :4]
    pages.c.length[1] = 250
    q, start = R.queries(shape, [3, 7], seed=8)
    out = lib.paged_attention(pages.c, q, row_start=start)
    done(lib)
    k, v = pages.held(0)[:2]
    o, e, _, _ = R.attention(q[3:], k[:250], v[:250], 243, lib.dtype)
    near(out[3:].view(7, 8, 128), o, e)


def test_one_sequence_after_another_and_all_at_once_agree():
    """What a sequence gets does not depend on its batch, within the bound of either."""
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    lens, rows = [700, 90, 2000, 1], [30, 90, 1, 1]
    pages = R.Pages(shape, lens, 16, seed=12)
    q, start = R.queries(shape, rows, seed=12)
    out = lib.paged_attention(pages.c, q, row_start=start)
    for b in range(4):
        one = binding.PagedKv(shape, pages.c.table[b:b + 1].contiguous(), page_size=16, k=pages.c.k, v=pages.c.v, length=pages.c.length[b:b + 1].contiguous())
        r = slice(int(start[b]), int(start[b + 1]))
        alone = lib.paged_attention(one, q[r], row_start=torch.tensor([0, rows[b]], dtype=torch.int32, device="cuda"))
        k, v = pages.held(b)[:2]
        o, e, _, _ = R.attention(q[r], k, v, lens[b] - rows[b], lib.dtype)
        near(alone.view(-1, 8, 128), o, e)
        near(out[r].view(-1, 8, 128), o, e)
    done(lib)


# ------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("dtype,plain", KINDS)
def test_weights_forget_or_add_up(dtype, plain):
    shape = shape_of(8, 2, 64, dtype)
    lib = context(shape, plain)
    lens, rows = [300, 0, 77], [1, 1, 1]
    pages = R.Pages(shape, lens, 64, seed=7)
    q, _ = R.queries(shape, rows, seed=7)
    _, lse = lib.paged_attention(pages.c, q, want_lse=True)
    pages.c.weight.fill_(float("nan"))
    lib.paged_weights(pages.c, q, lse, decay=0.0)
    done(lib)
    for b in (0, 2):
        w, e = R.weights(q[b:b + 1], pages.held(b)[0], lse[b:b + 1], lens[b] - 1)
        near(pages.held(b)[3], w, e)
        # the weights of one query and head add up to one
        assert abs(float(pages.held(b)[3].double().sum()) - 1) < float(e.sum()) + 1e-5
    once = [pages.held(b)[3].clone() for b in range(3)]
    lib.paged_weights(pages.c, q, lse, decay=1.0)
    done(lib)
    for b in range(3):
        near(pages.held(b)[3], 2 * once[b].double(), 2.0 ** -22 * once[b].double() + 1e-30)


def test_weights_of_a_window_of_the_last_queries():
    """The last 20 queries of a prompt of 500 alone: their lse is what the whole prompt's attention gave them."""
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    pages = R.Pages(shape, [500], 16, seed=17)
    q, start = R.queries(shape, [500], seed=17)
    _, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
    lib.paged_weights(pages.c, q[480:], lse[480:].contiguous(), row_start=torch.tensor([0, 20], dtype=torch.int32, device="cuda"), decay=0.0)
    done(lib)
    w, e = R.weights(q[480:], pages.held(0)[0], lse[480:], 480)
    near(pages.held(0)[3], w, e)


def test_weights_without_queries_only_fade():
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    pages = R.Pages(shape, [70, 3], 16, seed=1)
    before = [pages.held(b)[3].clone() for b in range(2)]
    q = torch.empty(0, 8, 128, dtype=torch.bfloat16, device="cuda")
    lib.paged_weights(pages.c, q, torch.empty(0, 8, device="cuda"), row_start=torch.zeros(3, dtype=torch.int32, device="cuda"), decay=0.25)
    done(lib)
    for b in range(2):
        assert torch.equal(pages.held(b)[3], 0.25 * before[b])


# ------------------------------------------------------------------------------------------------ eviction
def check_evict(pages, lib, keep, n_sink, n_recent, status=0):
    before = [pages.held(b) for b in range(pages.n)]
    lens = pages.c.length.tolist()
    pools = [t.clone() for t in (pages.c.k, pages.c.v, pages.c.pos, pages.c.weight)]
    lib.paged_evict(pages.c, torch.tensor(keep, dtype=torch.int32, device="cuda"), n_sink=n_sink, n_recent=n_recent)
    done(lib, status)
    kept = torch.zeros(pools[3].numel(), dtype=torch.bool)
    for b in range(pages.n):
        want = R.evict(*before[b], keep[b], n_sink, n_recent)
        got = pages.held(b)
        assert int(pages.c.length[b]) == len(want[3])
        for x, y in zip(got, want):
            assert torch.equal(x.nan_to_num(-5.0), y.nan_to_num(-5.0)), f"sequence {b}"
        kept[pages.slots(b, torch.arange(len(want[3])))] = True
    kept = kept.view(pools[3].shape).to("cuda")
    for old, new in zip(pools, (pages.c.k, pages.c.v, pages.c.pos, pages.c.weight)):       # all other places are as they were
        assert torch.equal(old[~kept].nan_to_num(-5.0), new[~kept].nan_to_num(-5.0))
    return lens


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n_sink,n_recent", [(0, 0), (4, 0), (0, 9), (30, 100), (10 ** 6, 0)])
def test_evict_ragged_sequences(dtype, page, n_sink, n_recent):
    shape = shape_of(4, 2, 64, dtype)
    lens = [0, 1, 300, 300, 300, 511, 512, 513, 70, 2000]
    keep = [0, 0, 299, 1, 0, 256, 255, 257, -1, 1000]
    check_evict(R.Pages(shape, lens, page, seed=page + n_sink), context(shape), keep, n_sink, n_recent)


@pytest.mark.parametrize("held,keep", [(5000, 4999), (9000, 100), (9000, 8000), (40000, 20000)])
def test_evict_sequences_shared_by_several_blocks(held, keep):
    shape = shape_of(2, 1, 64)
    check_evict(R.Pages(shape, [held, 37, held - 1111], 64, seed=held + keep), context(shape), [keep, 40, keep // 3], 2, 33)


def test_evict_a_sequence_beyond_shared_memory():
    shape = shape_of(1, 1, 64)
    check_evict(R.Pages(shape, [200000], 256, seed=3), context(shape), [70000], 2, 33)


def test_evict_goes_by_capacity_beyond_shared_memory_and_by_rows_held():
    """A long table with short sequences: the same rows as with a short one."""
    shape = shape_of(2, 1, 64)
    pages = R.Pages(shape, [700, 90], 16, seed=4)
    wide = torch.full((2, 20000), -1, dtype=torch.int32, device="cuda")
    wide[:, : pages.c.max_pages] = pages.c.table
    pages.c = binding.PagedKv(shape, wide, page_size=16, k=pages.c.k, v=pages.c.v, pos=pages.c.pos, weight=pages.c.weight, length=pages.c.length)
    check_evict(pages, context(shape), [300, 60], 1, 5)


@pytest.mark.parametrize("kind", ["equal", "zeros", "few values", "nan", "infinite", "descending", "ascending"])
@pytest.mark.parametrize("held", [600, 6000])
def test_evict_ties_and_values_that_are_not_finite(kind, held):
    shape = shape_of(2, 1, 64)
    pages = R.Pages(shape, [held, 50], 32, seed=11)
    slots = pages.slots(0, torch.arange(held)).to("cuda")
    g = torch.Generator().manual_seed(5)
    w = {"equal": torch.full((held,), 0.25), "zeros": torch.where(torch.arange(held) % 2 == 0, 0.0, -0.0),
         "few values": torch.randint(0, 4, (held,), generator=g).float(), "nan": torch.rand(held, generator=g),
         "infinite": torch.rand(held, generator=g), "descending": torch.arange(held, 0, -1).float(), "ascending": torch.arange(held).float()}[kind]
    if kind == "nan":
        w[::3] = float("nan")
    if kind == "infinite":
        w[::5], w[1::5] = float("inf"), float("-inf")
    pages.c.weight.view(-1)[slots] = w.to("cuda")
    keep = held // 3 + 400 if kind == "nan" else held // 3
    check_evict(pages, context(shape), [keep, 20], 0, 0, status=6 if kind == "nan" and held > keep else 0)
    if kind == "nan":
        # (of 6000 rows the NaN ones are gone by now)
        check_evict(pages, context(shape), [held // 3 + 150, 20], 0, 0, status=6 if held == 600 else 0)


def test_evict_again_and_with_nothing_to_do():
    shape = shape_of(2, 1, 64)
    lib = context(shape)
    pages = R.Pages(shape, [900, 300], 64, seed=13)
    check_evict(pages, lib, [500, 300], 4, 10)
    check_evict(pages, lib, [500, 500], 4, 10)
    check_evict(pages, lib, [123, 7], 4, 10)


def test_evict_reports_entries_that_name_no_page():
    shape = shape_of(2, 1, 64)
    lib = context(shape)
    pages = R.Pages(shape, [160], 16, seed=14)
    pages.c.table[0, 4] = -1
    lib.paged_evict(pages.c, torch.tensor([100], dtype=torch.int32, device="cuda"))
    done(lib, 8)
    assert pages.c.length.tolist() == [100]


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,plain", KINDS)
def test_a_conversation_over_a_paged_cache_at_its_budget(dtype, plain):
    """Prompt, gathered weights, eviction, next turn, single tokens with an eviction every few, each step against the plain form."""
    shape = shape_of(8, 2, 128, dtype)
    lib = context(shape, plain)
    pages = R.Pages(shape, [0, 0], 16, seed=21, room=700)
    g = torch.Generator().manual_seed(3)
    budget = torch.tensor([96, 128], dtype=torch.int32, device="cuda")
    at = [0, 0]
    for step, rows in enumerate([[300, 150], [40, 7], [1, 1], [1, 0], [1, 1], [5, 3]]):
        n = sum(rows)
        new = [torch.randn(n, 2, 128, generator=g).to(lib.dtype).to("cuda") for _ in range(2)]
        q, start = R.queries(shape, rows, seed=step)
        pos = torch.cat([torch.arange(a, a + r) for a, r in zip(at, rows)]).to(torch.int32).to("cuda")
        at = [a + r for a, r in zip(at, rows)]
        lib.paged_append(pages.c, new[0], new[1], pos=pos, row_start=start)
        out, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
        done(lib)
        want = []
        for b in range(2):
            r, held = slice(int(start[b]), int(start[b + 1])), int(pages.c.length[b])
            k, v, p, w = pages.held(b)
            assert torch.equal(k[held - rows[b]:], new[0][r]) and torch.equal(p[held - rows[b]:], pos[r])
            if rows[b]:
                o, e, l, el = R.attention(q[r], k, v, held - rows[b], lib.dtype)
                near(out[r].view(-1, 8, 128), o, e)
                near(lse[r], l, el)
            want.append((w, R.weights(q[r], k, lse[r], held - rows[b])))
        lib.paged_weights(pages.c, q, lse, row_start=start, decay=0.9)
        done(lib)
        for b in range(2):
            old, (w, e) = want[b]
            near(pages.held(b)[3], 0.9 * old.double() + w, e + 2.0 ** -22 * (old.double() + w))
        if step != 3:
            before = [pages.held(b) for b in range(2)]
            lib.paged_evict(pages.c, budget, n_sink=4, n_recent=16)
            done(lib)
            for b in range(2):
                for x, y in zip(pages.held(b), R.evict(*before[b], int(budget[b]), 4, 16)):
                    assert torch.equal(x, y)


def test_a_captured_step_is_replayed():
    """Append, attention, weights and eviction of single tokens in one graph: lengths, weights and pages move on with every replay."""
    shape = shape_of(8, 2, 128)
    stream = torch.cuda.Stream()
    lib = binding.Spts(shape, max_seq=64, stream=stream)
    lens = [60, 33, 64]
    eager, graph = R.Pages(shape, lens, 16, seed=30, room=8), R.Pages(shape, lens, 16, seed=30, room=8)
    K, V = torch.zeros(3, 2, 128, device="cuda").bfloat16(), torch.zeros(3, 2, 128, device="cuda").bfloat16()
    q, pos = torch.zeros(3, 8, 128, device="cuda").bfloat16(), torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(3, 1024, device="cuda").bfloat16(), torch.zeros(3, 8, device="cuda")
    budget = torch.tensor([62, 40, 64], dtype=torch.int32, device="cuda")

    def step(c):
        lib.paged_append(c, K, V, pos=pos)
        lib.paged_attention(c, q, O_out=out, lse_out=lse)
        lib.paged_weights(c, q, lse, decay=0.9)
        lib.paged_evict(c, budget, n_sink=2, n_recent=4)

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        cuda_graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cuda_graph, stream=stream):
            step(graph.c)
    torch.cuda.synchronize()
    assert graph.c.length.tolist() == lens
    for i in range(9):
        g = torch.Generator().manual_seed(i)
        with torch.cuda.stream(stream):
            for t in (K, V, q):
                t.copy_(torch.randn(t.shape, generator=g).bfloat16())
            pos.fill_(1000 + i)
            step(eager.c)
            want = out.clone(), lse.clone()
            out.zero_(), lse.zero_()
            cuda_graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert torch.equal(eager.c.length, graph.c.length)
        for b in range(3):
            for x, y in zip(eager.held(b), graph.held(b)):
                assert torch.equal(x, y)
    assert graph.c.length.tolist() == [62, 40, 64]
    assert lib.device_status() == 0
    del cuda_graph
    lib.close()


# ------------------------------------------------------------------------------------------------ refusals
def test_calls_that_cannot_be_made_are_refused_before_anything_is_launched():
    import ctypes as C
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    pages = R.Pages(shape, [20, 3], 16, room=8)
    L, h, c = lib.lib, lib.h, pages.c.c
    q = torch.randn(2, 8 * 128, device="cuda").bfloat16()
    kv = torch.randn(2, 2 * 128, device="cuda").bfloat16()
    out, lse, ints = torch.zeros_like(q), torch.zeros(2, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    Q, K, O, E, I = q.data_ptr(), kv.data_ptr(), out.data_ptr(), lse.data_ptr(), ints.data_ptr()
    state = [t.clone() for t in (pages.c.k, pages.c.length, pages.c.weight)]
    launched = lib.launch_count()

    def with_(**kw):
        d = binding.PagedKvC()
        C.memmove(C.byref(d), C.byref(pages.c.c), C.sizeof(d))
        for name, value in kw.items():
            setattr(d, name, value)
        return C.byref(d)
    broken = [(with_(page_size=48), 2), (with_(page_size=0), 2), (with_(n_seq=1025), 2), (with_(n_seq=-1), 2), (with_(max_pages=0), 2),
              (with_(max_pages=(1 << 25) // 16 + 1), 2), (with_(n_pages=0), 2), (with_(n_pages=1 << 27), 2), (with_(k=None), 1), (with_(v=None), 1),
              (with_(table=None), 1), (with_(len=None), 1), (with_(k=pages.c.k.data_ptr() + 8), 1), (with_(v=pages.c.k.data_ptr()), 1),
              (with_(table=pages.c.table.data_ptr() + 2), 1), (with_(pos=pages.c.pos.data_ptr() + 1), 1), (None, 1)]
    for cache, code in broken:
        assert L.spts_paged_append(h, cache, K, 256, K + 16, 256, None, None, None, 2) == code
        assert L.spts_paged_attention(h, cache, Q, 1024, None, 2, O, 1024, None) == code
        assert L.spts_paged_weights(h, cache, Q, 1024, None, 2, E, 1.0) == code
        assert L.spts_paged_evict(h, cache, I, 0, 0) == code
    c = C.byref(c)
    for args in [(None, 256, K, 256, None, None, None, 2), (K, 256, None, 256, None, None, None, 2), (K + 2, 256, K, 256, None, None, None, 2),
                 (K, 255, K, 256, None, None, None, 2), (K, 260, K, 256, None, None, None, 2), (K, 256, K, 256, I + 1, None, None, 2),
                 (K, 256, K, 256, None, I + 2, None, 2), (K, 256, K, 256, None, None, I + 3, 2), (K, 256, K, 256, None, None, None, 3),
                 (K, 256, K, 256, None, None, None, -1), (pages.c.k.data_ptr(), 256, K, 256, None, None, None, 2)]:
        assert L.spts_paged_append(h, c, *args) == 1, args
    for args in [(None, 1024, None, 2, O, 1024, None), (Q, 1024, None, 2, None, 1024, None), (Q, 1024, None, 2, Q, 1024, None),
                 (Q + 8, 1024, None, 2, O, 1024, None), (Q, 1023, None, 2, O, 1024, None), (Q, 1024, None, 2, O, 1028, None),
                 (Q, 1024, None, 1, O, 1024, None), (Q, 1024, I, -2, O, 1024, None), (Q, 1024, None, 2, O, 1024, E + 2)]:
        assert L.spts_paged_attention(h, c, *args) == 1, args
    for args in [(None, 1024, None, 2, E, 1.0), (Q, 1024, None, 2, None, 1.0), (Q, 1024, None, 2, E, -0.5), (Q, 1024, None, 2, E, float("nan")),
                 (Q, 1024, None, 2, E, float("inf")), (Q, 1020, None, 2, E, 1.0), (Q, 1024, None, 3, E, 1.0)]:
        assert L.spts_paged_weights(h, c, *args) == 1, args
    assert L.spts_paged_weights(h, with_(weight=None), Q, 1024, None, 2, E, 1.0) == 1
    for cache, keep, sink, recent in [(c, None, 0, 0), (c, I, -1, 0), (c, I, 0, -1), (c, I + 2, 0, 0), (with_(weight=None), I, 0, 0), (with_(pos=None), I, 1, 0)]:
        assert L.spts_paged_evict(h, cache, keep, sink, recent) == 1
    x = torch.randn(2, 64, device="cuda").data_ptr()
    for args, code in [((None, 64, 2, 64, I, 0, E, None, None, None, None), 1), ((x, 63, 2, 64, I, 0, E, None, None, None, None), 1),
                       ((x, 64, 2, 0, I, 0, E, None, None, None, None), 2), ((x, 64, -1, 64, I, 0, E, None, None, None, None), 1),
                       ((x, 64, 2, 64, None, 0, E, None, None, None, None), 1), ((x, 64, 2, 64, I, 0, None, None, None, None, None), 1),
                       ((x, 64, 2, 64, I, 33, E, None, None, None, None), 1), ((x, 64, 2, 64, None, 0, None, None, None, E, I), 1),
                       ((x + 2, 64, 2, 64, I, 0, E, None, None, None, None), 1), ((x, 64, 2, 64, None, 0, None, I, None, None, None), 1)]:
        assert L.spts_token_logprobs(h, *args) == code, args
    # nothing to do is no error
    assert L.spts_paged_attention(h, with_(n_seq=0), None, 0, None, 0, None, 0, None) == 0
    assert L.spts_paged_append(h, with_(n_seq=0), None, 0, None, 0, None, I, None, 0) == 0
    assert L.spts_paged_attention(h, c, None, 0, I, 0, None, 0, None) == 0
    assert L.spts_token_logprobs(h, None, 0, 0, 64, None, 0, None, None, None, None, None) == 0
    assert lib.launch_count() == launched
    done(lib)
    for old, new in zip(state, (pages.c.k, pages.c.length, pages.c.weight)):
        assert torch.equal(old.nan_to_num(-1.0), new.nan_to_num(-1.0))
