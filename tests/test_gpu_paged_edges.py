"""Edges of the calls around a paged cache: groups of very many heads, many sequences, long caches, pools beyond 32-bit offsets, other
streams, two contexts at a time, equal bits from equal calls."""
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


@pytest.mark.parametrize("heads,kv", [(128, 1), (144, 1), (65, 1), (50, 2)])
def test_groups_of_many_heads(heads, kv):
    """A tile of one token, of none whole (the plain kernels), and groups that leave rows of a tile unused."""
    check_attention(shape_of(heads, kv, 64), [200, 3, 130], [5, 3, 1], 32, seed=heads)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_as_many_sequences_as_there_may_be(dtype):
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 90, (1024,), generator=g).tolist()
    rows = [min(r, held) if held else r for r, held in zip(torch.randint(0, 4, (1024,), generator=g).tolist(), lens)]
    shape = shape_of(4, 2, 64, dtype)
    lib, pages, *_ = check_attention(shape, lens, rows, 16, seed=2)
    for b in range(1024):                        # (the weights of all sequences were checked above)
        assert not bool(torch.isnan(pages.held(b)[3]).any())
    check_evict(pages, lib, [max(0, held - 30) for held in lens], 2, 5)


def test_more_sequences_than_fit_the_workspace_at_once():
    """700 tables of 65536 rows: their rows have more bits than the workspace has room for, so the eviction goes round by round."""
    shape = shape_of(2, 1, 64)
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 70, (700,), generator=g).tolist()
    pages = R.Pages(shape, lens, 16, seed=3)
    wide = torch.full((700, 4096), -1, dtype=torch.int32, device="cuda")
    wide[:, : pages.c.max_pages] = pages.c.table
    pages.c = binding.PagedKv(shape, wide, page_size=16, k=pages.c.k, v=pages.c.v, pos=pages.c.pos, weight=pages.c.weight, length=pages.c.length)
    from test_gpu_paged import context
    check_evict(pages, context(shape), [max(0, held - 20) for held in lens], 0, 3)


@pytest.mark.parametrize("rows", [1, 5, 70, 300])
def test_long_caches(rows):
    """131,072 rows: many CTAs share each unit."""
    check_attention(shape_of(4, 1, 128), [131072], [rows], 256, seed=rows)


@pytest.mark.parametrize("rows", [1, 3, 20, 100, 600])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (7, 1, 64)])
def test_units_shared_by_several_blocks(rows, heads, kv, dim):
    check_attention(shape_of(heads, kv, dim), [9000, 0, 777], [rows, 2, min(rows, 40)], 64, seed=rows + heads)


def test_equal_calls_give_equal_bits():
    shape = shape_of(8, 2, 128)
    from test_gpu_paged import context
    lib = context(shape)
    pages = R.Pages(shape, [9000, 300, 40, 0], 16, seed=5)
    q, start = R.queries(shape, [70, 300, 1, 2], seed=5)
    first = None
    for _ in range(4):
        out, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
        lib.paged_weights(pages.c, q, lse, row_start=start, decay=0.0)
        got = [out, lse, pages.c.weight.nan_to_num(-1.0).clone()]
        if first is None:
            first = got
        assert all(torch.equal(x, y) for x, y in zip(got, first))


def test_pools_beyond_32_bit_offsets():
    """More than 2^31 elements of K and of V; the sequences lie in the last pages."""
    shape = shape_of(16, 8, 128)
    from test_gpu_paged import context
    lib = context(shape)
    page, n_pages = 256, 8400                     # 2,150,400 rows of 1024 elements: 2.2e9
    k, v = (torch.zeros(n_pages, page, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3], [n_pages - 2, n_pages - 4, 1]], dtype=torch.int32, device="cuda")
    c = binding.PagedKv(shape, table, page_size=page, k=k, v=v, positions=True, weights=True)
    lens, held = [700, 300], []
    g = torch.Generator().manual_seed(6)
    K, V = (torch.randn(1000, 8, 128, generator=g).bfloat16().to("cuda") for _ in range(2))
    start = torch.tensor([0, 700, 1000], dtype=torch.int32, device="cuda")
    lib.paged_append(c, K, V, pos=torch.arange(1000, dtype=torch.int32, device="cuda"), row_start=start)
    q, qs = R.queries(shape, [30, 1], seed=6)
    out, lse = lib.paged_attention(c, q, row_start=qs, want_lse=True)
    lib.paged_weights(c, q, lse, row_start=qs, decay=0.0)
    assert lib.device_status() == 0
    for b, (first, m) in enumerate([(0, 30), (700, 1)]):
        r, rows = slice(int(qs[b]), int(qs[b]) + m), slice(first, first + lens[b])
        o, e, l, el = R.attention(q[r], K[rows], V[rows], lens[b] - m, torch.bfloat16)
        near(out[r].view(m, 16, 128), o, e)
        near(lse[r], l, el)
        w, ew = R.weights(q[r], K[rows], lse[r], lens[b] - m)
        j = torch.arange(lens[b], device="cuda")
        slot = table[b].long()[j // page] * page + j % page
        near(c.weight.view(-1)[slot], w, ew)
        held.append((k.view(-1, 8, 128)[slot], v.view(-1, 8, 128)[slot], c.pos.view(-1)[slot], c.weight.view(-1)[slot]))
        assert torch.equal(held[b][0], K[rows]) and torch.equal(held[b][1], V[rows])
    keep = torch.tensor([300, 20], dtype=torch.int32, device="cuda")
    lib.paged_evict(c, keep, n_sink=2, n_recent=30)
    assert lib.device_status() == 0
    for b in range(2):
        j = torch.arange(int(keep[b]), device="cuda")
        slot = table[b].long()[j // page] * page + j % page
        for got, want in zip((k.view(-1, 8, 128)[slot], v.view(-1, 8, 128)[slot], c.pos.view(-1)[slot], c.weight.view(-1)[slot]),
                             R.evict(*held[b], int(keep[b]), 2, 30)):
            assert torch.equal(got, want)


def test_values_not_seen_at_the_end_of_very_long_caches():
    """160 sequences share 524,288 rows, the last of which, not finite, only the last of their 16 queries see: what the others get takes longer
    to compute again than a wait within the kernel may last without a sign of life."""
    shape = shape_of(8, 1, 128)
    from test_gpu_paged import context
    lib = context(shape)
    n_seq, n, held, page = 160, 16, 524288, 256
    g = torch.Generator().manual_seed(7)
    k, v = (torch.randn(held // page, page, 1, 128, generator=g).bfloat16().to("cuda") for _ in range(2))
    k.view(held, 128)[-1] = float("inf")
    v.view(held, 128)[-1] = float("nan")
    table = torch.arange(held // page, dtype=torch.int32, device="cuda").repeat(n_seq, 1)
    length = torch.full((n_seq,), held, dtype=torch.int32, device="cuda")
    c = binding.PagedKv(shape, table, page_size=page, k=k, v=v, length=length)
    q, start = R.queries(shape, [n] * n_seq, seed=7)
    out, lse = lib.paged_attention(c, q, row_start=start, want_lse=True)
    assert lib.device_status() == 0
    for b in (0, 77, 159):
        r = slice(n * b, n * b + n - 1)
        o, e, l, el = R.attention(q[r], k.view(held, 1, 128)[:held - 1], v.view(held, 1, 128)[:held - 1], held - n, torch.bfloat16)
        near(out[r].view(n - 1, 8, 128), o, e)
        near(lse[r], l, el)
    out = out.view(n_seq, n, 8, 128)
    assert bool(torch.isfinite(out[:, :-1]).all()) and bool(torch.isnan(out[:, -1]).all())


def test_two_contexts_on_two_streams():
    """Each has its workspace: calls that run at the same time do not meet."""
    shape = shape_of(8, 2, 128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    made = []
    for i, st in enumerate(streams):
        with torch.cuda.stream(st):
            lib = binding.Spts(shape, max_seq=64, stream=st)
            pages = R.Pages(shape, [9000 - 700 * i, 500], 32, seed=40 + i)
            q, start = R.queries(shape, [60, 9], seed=40 + i)
        made.append((lib, pages, q, start))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, (lib, pages, q, start) in enumerate(made):
            with torch.cuda.stream(streams[i]):
                out, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
                lib.paged_weights(pages.c, q, lse, row_start=start, decay=0.0)
                outs[i].append((out, lse, pages.c.weight.clone()))
    torch.cuda.synchronize()
    for i, (lib, pages, q, start) in enumerate(made):
        assert lib.device_status() == 0 and lib.check_guards() == 0
        for out, lse, w in outs[i]:
            assert torch.equal(out, outs[i][0][0]) and torch.equal(w.nan_to_num(-1), outs[i][0][2].nan_to_num(-1))
        for b, (held, m) in enumerate([(9000 - 700 * i, 60), (500, 9)]):
            r = slice(int(start[b]), int(start[b]) + m)
            o, e, _, _ = R.attention(q[r], pages.held(b)[0], pages.held(b)[1], held - m, torch.bfloat16)
            near(outs[i][0][0][r].view(m, 8, 128), o, e)
        lib.close()


def test_lengths_out_of_range_are_held_in_it():
    """A length beyond the table counts as the table's rows, one below zero as none."""
    shape = shape_of(8, 2, 128)
    from test_gpu_paged import context
    for plain in (False, True):
        lib = context(shape, plain)
        pages = R.Pages(shape, [64, 64], 32, seed=50)
        pages.c.length.copy_(torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32))
        q, start = R.queries(shape, [3, 2], seed=50)
        out, lse = lib.paged_attention(pages.c, q, row_start=start, want_lse=True)
        lib.paged_weights(pages.c, q, lse, row_start=start, decay=0.0)
        assert lib.device_status() == 0
        k, v = pages.rows[0][0].to("cuda"), pages.rows[0][1].to("cuda")
        o, e, _, _ = R.attention(q[:3], k, v, 61, lib.dtype)
        near(out[:3].view(3, 8, 128), o, e)
        assert bool((out[3:] == 0).all()) and bool((lse[3:] == float("-inf")).all())
        lib.paged_evict(pages.c, torch.tensor([40, 1], dtype=torch.int32, device="cuda"))
        assert lib.device_status() == 0 and pages.c.length.tolist() == [40, -5]


def test_evictions_budget_of_nothing_and_everything():
    shape = shape_of(2, 1, 64)
    from test_gpu_paged import context
    check_evict(R.Pages(shape, [5000, 4097, 1], 64, seed=60), context(shape), [0, 4096, 1], 0, 0)


@pytest.mark.parametrize("n_sink,n_recent", [(0, 0), (4, 64)])
@pytest.mark.parametrize("longest", [700, 9000, 200000])
def test_evictions_of_the_few_rows_that_a_step_brought(longest, n_sink, n_recent):
    """Up to 32 rows go, or just more: of sequences of one block, of a cluster of blocks and beyond shared memory."""
    shape = shape_of(2, 1, 64)
    lens = [longest, longest - 1, longest - 300, 400, 400, 33, 32, 1, 260]
    gone = [1, 32, 33, 31, 32, 33, 32, 1, 7]
    check_evict(R.Pages(shape, lens, 64, seed=longest), context(shape), [held - x for held, x in zip(lens, gone)], n_sink, n_recent)
