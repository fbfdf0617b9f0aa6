"""Calls around a paged cache at the ends of what they allow: kernels that run for seconds, lengths out of range, weights that are not
numbers in rows that stay whatever they are, a context that goes on after a wait that gave up."""
import pytest
import torch

import paged_ref as R
from paper_2601_13155_b200 import binding
from test_gpu_paged import check_attention, check_evict, context, near, shape_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _close():
    yield
    import test_gpu_paged
    for lib in test_gpu_paged._contexts.values():
        assert lib.check_guards() == 0
        lib.close()
    test_gpu_paged._contexts.clear()


def test_an_attention_of_several_seconds_is_no_wait_that_gave_up():
    """4,194,247 fresh tokens of one head, 8.8e12 pairs: the block whose rows behind the last one are to be cleared comes at the very end of the
    last CTA's piece, which takes longer than the two seconds that a wait within the kernel may last without a sign of life."""
    shape = shape_of(1, 1, 128)
    lib = context(shape)
    page, n_pages = 256, 16384
    n = n_pages * page - 57
    g = torch.Generator(device="cuda").manual_seed(9)
    held = [torch.randn(n_pages * page, 1, 128, device="cuda", generator=g, dtype=torch.bfloat16) for _ in range(2)]
    held[1][..., 0] = 1.0                            # a column whose result is known for every query
    for t in held:
        t[n:] = float("nan")
    q = torch.randn(n, 128, device="cuda", generator=g, dtype=torch.bfloat16)
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(9)).to(torch.int32)[None].to("cuda")
    k, v = (torch.empty(n_pages, page, 1, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for pool, rows in ((k, held[0]), (v, held[1])):
        pool[table[0].long()] = rows.view(n_pages, page, 1, 128)
    c = binding.PagedKv(shape, table, page_size=page, k=k, v=v, length=torch.tensor([n], dtype=torch.int32, device="cuda"))
    out = torch.full((n, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    lse = torch.full((n, 1), float("nan"), device="cuda")
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    lib.paged_attention(c, q, row_start=start, O_out=out, lse_out=lse)
    end.record()
    assert lib.device_status() == 0
    assert begin.elapsed_time(end) > 2000
    # a weight's rounding and the result's, half a step each, and two sums over the rows in (rows / 8 + 80) steps of 2^-23
    rows = torch.arange(1, n + 1, device="cuda", dtype=torch.float64)
    assert bool(((out[:, 0].double() - 1).abs() <= 2.01 * 2.0 ** -8 + 2.01 * (rows / 8 + 80) * 2.0 ** -23).all())
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    for first in (0, 1000, 70000):
        m = 40
        o, e, l, el = R.attention(q[first:first + m].view(m, 1, 128), held[0][:first + m], held[1][:first + m], first, torch.bfloat16)
        near(out[first:first + m].view(m, 1, 128), o, e)
        near(lse[first:first + m], l, el)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("by", ["nothing", "lengths", "places"])
def test_append_behind_lengths_out_of_range(dtype, by):
    """A length below zero counts as none, so the rows begin at place 0; one beyond the table leaves no room.  A place that is given is taken as
    it is: rows before place 0 are reported and not written."""
    shape = shape_of(4, 2, 64, dtype)
    lib = context(shape)
    for lens, new in (([-5, 3, -2 ** 31], [8, 2, 1]), ([-5, 3, -1], [3, 0, 0]), ([2 ** 31 - 1, 3, 33], [2, 1, 1])):
        pages = R.Pages(shape, [0, 3, 0], 16, seed=2, room=29)             # tables of 32 rows
        kept = pages.held(1)[0].clone()
        pages.c.length.copy_(torch.tensor(lens, dtype=torch.int32))
        start = torch.tensor([0, new[0], new[0] + new[1], sum(new)], dtype=torch.int32, device="cuda")
        K, V = (torch.randn(sum(new), 2, 64, device="cuda").to(lib.dtype) for _ in range(2))
        at = {"nothing": None, "lengths": pages.c.length, "places": pages.c.length.clone()}[by]
        lib.paged_append(pages.c, K, V, row_start=start, at=at)
        begin = [held if by == "places" else min(max(held, 0), 32) for held in lens]
        lost = any(a < 0 or a + m > 32 for a, m in zip(begin, new) if m)
        assert lib.device_status() == (3 if lost else 0)                   # SPTS_ERR_WORKSPACE
        assert pages.c.length.tolist() == [min(max(a + m, 0), 32) for a, m in zip(begin, new)]
        for b in (0, 1, 2):
            for i in range(new[b]):
                if 0 <= begin[b] + i < 32:
                    slot = int(pages.slots(b, torch.tensor(begin[b] + i)))
                    assert torch.equal(pages.c.k.view(-1, 2, 64)[slot], K[int(start[b]) + i])
                    assert torch.equal(pages.c.v.view(-1, 2, 64)[slot], V[int(start[b]) + i])
        assert torch.equal(pages.c.k.view(-1, 2, 64)[pages.slots(1, torch.arange(3)).to("cuda")], kept)
        assert lib.check_guards() == 0


@pytest.mark.parametrize("capacity", [640, 9600, 200704])
@pytest.mark.parametrize("n_sink,n_recent", [(9, 0), (0, 9), (9, 9)])
def test_weights_that_are_no_numbers_in_rows_that_stay_before_all_others(capacity, n_sink, n_recent):
    """Reported whatever room the table has (one block, a cluster, keys beyond shared memory), and the same rows stay."""
    shape = shape_of(2, 1, 64)
    lib = context(shape)
    for bad, status in ((0, 6 if n_sink else 0), (599, 6 if n_recent else 0), (None, 0)):      # SPTS_ERR_NONFINITE
        pages = R.Pages(shape, [600, 50], 64, seed=capacity + n_sink)
        wide = torch.full((2, capacity // 64), -1, dtype=torch.int32, device="cuda")
        wide[:, : pages.c.max_pages] = pages.c.table
        pages.c = binding.PagedKv(shape, wide, page_size=64, k=pages.c.k, v=pages.c.v, pos=pages.c.pos, weight=pages.c.weight, length=pages.c.length)
        if bad is not None and status:
            pages.c.weight.view(-1)[int(pages.slots(0, torch.tensor(bad)))] = float("nan")
        check_evict(pages, lib, [300, 50], n_sink, n_recent, status=status)


def test_calls_after_a_wait_that_gave_up():
    """A CTA that gives up leaves what others have counted: reading the status puts that in order for everything that is joined by the one that
    comes last, single tokens and chunks over long caches, weights, appends, evictions and long rows of logits."""
    shape = shape_of(8, 2, 128)
    lib = binding.Spts(shape, max_seq=64)
    want = None
    for gave_up in (False, True, False):
        if gave_up:
            lib.selftest_wait_timeout(1000)
            assert lib.device_status() == 5                                # SPTS_ERR_TIMEOUT
        got = []
        for rows in (1, 90):
            pages = R.Pages(shape, [9000, 700], 64, seed=rows, room=100)
            q, start = R.queries(shape, [rows, rows], seed=rows)
            K, V = (torch.randn(2 * rows, 2, 128, generator=torch.Generator().manual_seed(rows)).to(torch.bfloat16).to("cuda") for _ in range(2))
            lib.paged_append(pages.c, K, V, row_start=start)
            out, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
            lib.paged_weights(pages.c, q, lse, row_start=start, decay=0.0)
            lib.paged_evict(pages.c, torch.tensor([4000, 690], dtype=torch.int32, device="cuda"))
            got += [out, lse, pages.c.weight.nan_to_num(-1.0), pages.c.length, pages.c.k.nan_to_num(-1.0)]
        x = torch.randn(2, 128256, generator=torch.Generator().manual_seed(3)).to("cuda")
        got += list(lib.token_logprobs(x, torch.tensor([5, 128000], dtype=torch.int32, device="cuda"), n_top=6).values())
        assert lib.device_status() == 0 and lib.check_guards() == 0
        want = want or got
        assert got[3].tolist() == [4000, 690]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    lib.close()


def test_joined_results_never_hold_another_calls_shares():
    """Two calls in turn, many times over: a share that was read before it was written would be the other call's."""
    shape = shape_of(8, 2, 128)
    lib = context(shape)
    made = []
    for seed in (1, 2):
        pages = R.Pages(shape, [30000, 9000, 700], 64, seed=seed, room=64)
        q, start = R.queries(shape, [1, 1, 1], seed=seed)
        x = torch.randn(3, 128256, generator=torch.Generator().manual_seed(seed)).to("cuda")
        K, V = (torch.randn(3, 2, 128, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to("cuda") for _ in range(2))
        made.append((pages, q, x, K, V, pages.c.length.clone(), []))
    for _ in range(60):
        for pages, q, x, K, V, lens, seen in made:
            lib.paged_append(pages.c, K, V, at=lens)
            out, lse = lib.paged_attention(pages.c, q, want_lse=True)
            lib.paged_weights(pages.c, q, lse, decay=0.0)
            got = [out, lse, pages.c.weight.nan_to_num(-1.0), pages.c.length.clone()]
            got += list(lib.token_logprobs(x, torch.arange(3, dtype=torch.int32, device="cuda"), n_top=4).values())
            seen.append(got)
    assert lib.device_status() == 0
    for pages, q, x, K, V, lens, seen in made:
        assert seen[0][3].tolist() == [30001, 9001, 701]
        for got in seen[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got, seen[0]))
        for b, held in enumerate([30001, 9001, 701]):
            k, v = pages.held(b)[:2]
            o, e, l, el = R.attention(q[b:b + 1], k, v, held - 1, torch.bfloat16)
            near(seen[0][0][b:b + 1].view(1, 8, 128), o, e)
            near(seen[0][1][b:b + 1], l, el)


@pytest.mark.parametrize("dtype,plain", [("bf16", False), ("bf16", True), ("fp32", False)])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (4, 4, 128), (14, 2, 64), (32, 4, 128)])
@pytest.mark.parametrize("chunk,others", [(512, 63), (300, 40), (33, 200)])
def test_one_long_chunk_beside_many_single_tokens(dtype, plain, heads, kv, dim, chunk, others):
    """What goes by the batch's average chunk (tiles of one or two, who joins, boxes of queries, rows or tiles) holds for those far from it."""
    lens = [9000] + [1 + 37 * i % 900 for i in range(others)]
    rows = [chunk] + [1] * others
    check_attention(shape_of(heads, kv, dim, dtype), lens, rows, 64, plain, seed=chunk + heads)
    check_attention(shape_of(heads, kv, dim, dtype), lens[::-1], rows[::-1], 16, plain, seed=others)


@pytest.mark.parametrize("n_sink,n_recent", [(0, 0), (4, 64)])
def test_evict_more_rows_than_have_their_numbers_in_shared_memory(n_sink, n_recent):
    """Beyond 1,048,576 rows; a sequence beside it that gives up a few."""
    shape = shape_of(1, 1, 64)
    check_evict(R.Pages(shape, [1100003, 5000], 256, seed=3), context(shape), [400001, 4990], n_sink, n_recent)
