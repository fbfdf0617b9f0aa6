"""Log probabilities, ranks, entropy and alternatives of rows of logits against 64 bits."""
import math

import pytest
import torch

import paged_ref as R
from paper_2601_13155_b200 import binding, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    x = binding.Spts(synth.ModelShape(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=256, ltp_dlow=64, ltp_rank=16, n_layers=1, vocab=64,
                                      dtype="bf16"), max_seq=64)
    yield x
    x.close()


def check(lib, x, targets, n_top, rows=None):
    out = lib.token_logprobs(x, targets, n_top=n_top)
    assert lib.device_status() == 0 and lib.check_guards() == 0
    t = targets.tolist() if targets is not None else [None] * x.shape[0]

    def same(got, want, bound):
        if want != want:
            return got != got
        return got == want or abs(got - want) <= bound + 2.0 ** -23 * abs(want)
    for i in (range(x.shape[0]) if rows is None else rows):
        lp, rank, ent, top, tok, e, ee = R.logprobs(x[i], t[i], n_top)
        if t[i] is not None:
            assert same(float(out["logprob"][i]), lp, e), (i, float(out["logprob"][i]), lp, e)
            assert int(out["rank"][i]) == rank, (i, int(out["rank"][i]), rank)
        assert same(float(out["entropy"][i]), ent, ee), (i, float(out["entropy"][i]), ent, ee)
        if n_top:
            assert out["top_token"][i].tolist() == tok, i
            for a, b in zip(out["top_logprob"][i].tolist(), top):
                assert same(a, b, e), (i, a, b, e)
    return out


@pytest.mark.parametrize("vocab", [1, 2, 3, 31, 100, 2047, 2048, 4097, 8191, 33000])
@pytest.mark.parametrize("n_top", [0, 1, 5, 32])
def test_rows_of_all_lengths(lib, vocab, n_top):
    g = torch.Generator().manual_seed(vocab + n_top)
    x = (3 * torch.randn(3, vocab, generator=g)).to("cuda")
    check(lib, x, torch.randint(0, vocab, (3,), generator=g).to(torch.int32).to("cuda"), n_top)


@pytest.mark.parametrize("n", [1, 7, 40, 700])
def test_few_and_many_rows(lib, n):
    g = torch.Generator().manual_seed(n)
    x = (3 * torch.randn(n, 20001, generator=g)).to("cuda")
    rows = range(n) if n <= 7 else range(0, n, n // 7)
    check(lib, x, torch.randint(0, 20001, (n,), generator=g).to(torch.int32).to("cuda"), 20, rows=rows)


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("ld", [5003, 5004, 5006])
def test_rows_at_any_place(lib, shift, ld):
    g = torch.Generator().manual_seed(shift + ld)
    flat = (3 * torch.randn(4 * ld + 8, generator=g)).to("cuda")
    flat[:shift] = 99.0
    x = flat[shift:shift + 4 * ld].view(4, ld)[:, :5001]
    flat[shift + 5001::ld] = 99.0                   # between the rows
    check(lib, x, torch.tensor([0, 5000, 77, 4096], dtype=torch.int32, device="cuda"), 7)


@pytest.mark.parametrize("vocab", [300, 9000, 70000])
@pytest.mark.parametrize("n_top", [5, 32])
@pytest.mark.parametrize("kind", ["equal", "two values", "ascending", "descending", "masked", "one left", "empty", "late", "low", "tied at the cut"])
def test_hard_rows(lib, vocab, n_top, kind):
    """Ties beyond any list, orders that make every token the best so far, masks that leave few tokens, one or none."""
    x = torch.zeros(2, vocab)
    v = torch.arange(vocab).float()
    if kind == "two values":
        x[:, 1::2] = 1.0
    elif kind == "ascending":
        x[:] = v / vocab * 9
    elif kind == "descending":
        x[:] = -v / vocab * 9
    elif kind in ("masked", "one left", "empty"):
        x[:] = torch.randn(vocab, generator=torch.Generator().manual_seed(1))
        left = {"masked": 17, "one left": 1, "empty": 0}[kind]
        keep = torch.randperm(vocab, generator=torch.Generator().manual_seed(2))[:left]
        hide = torch.ones(vocab, dtype=torch.bool)
        hide[keep] = False
        x[:, hide] = float("-inf")
    elif kind == "late":
        x[:] = -3e38
        x[:, vocab - 40:] = v[:40] * 0.1
    elif kind == "low":
        x[:] = torch.finfo(torch.float32).min
    elif kind == "tied at the cut":
        x[:] = torch.randn(vocab, generator=torch.Generator().manual_seed(3)).clamp(max=1.5)
        x[:, 200:203] = 2.0
    x = x.to("cuda")
    check(lib, x, torch.tensor([vocab - 1, vocab // 2], dtype=torch.int32, device="cuda"), n_top)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("vocab", [500, 50000])
def test_rows_that_are_not_finite(lib, value, vocab):
    x = torch.randn(4, vocab, generator=torch.Generator().manual_seed(4)).to("cuda")
    x[1, vocab // 3], x[2, vocab - 1], x[2, 3] = value, value, float("-inf")
    check(lib, x, torch.tensor([5, 6, vocab - 1, -1], dtype=torch.int32, device="cuda"), 6)


def test_padding_and_missing_targets(lib):
    x = torch.randn(5, 3001, device="cuda")
    check(lib, x, torch.tensor([-1, 3001, 2 ** 31 - 1, -2 ** 31, 3000], dtype=torch.int32, device="cuda"), 3)
    check(lib, x, None, 3)
    out = lib.token_logprobs(x, torch.zeros(5, dtype=torch.int32, device="cuda"), entropy=False)
    assert set(out) == {"logprob", "rank"}
    # a target at -inf, with others there before and behind it
    x[:, 100:2000] = float("-inf")
    check(lib, x, torch.tensor([100, 1999, 1000, 99, 2000], dtype=torch.int32, device="cuda"), 3)


def test_ranks_at_minus_infinity_across_slices(lib):
    """A long row shared by many blocks, the target at -inf among others."""
    x = torch.randn(1, 128256, generator=torch.Generator().manual_seed(6)).to("cuda")
    x[:, ::3] = float("-inf")
    for t in (0, 60000, 128253):
        check(lib, x, torch.tensor([t], dtype=torch.int32, device="cuda"), 2)


def test_log_probabilities_of_a_decode_steps_logits(lib):
    """The greedy token of spts_process_logits has rank 0, and exp of all alternatives' log probabilities stays below one."""
    x = (3 * torch.randn(9, 32003, generator=torch.Generator().manual_seed(8))).to("cuda")
    mask = torch.randint(-2 ** 31, 2 ** 31, (9, 1001), generator=torch.Generator().manual_seed(9)).to(torch.int32).to("cuda")
    logits, token = lib.process_logits(x, binding.LogitsRules(mask=mask))
    out = check(lib, logits, token, 20)
    assert out["rank"].tolist() == [0] * 9 and torch.equal(out["top_token"][:, 0], token)
    assert torch.equal(out["top_logprob"][:, 0], out["logprob"])
    assert bool((out["top_logprob"].double().exp().sum(-1) < 1).all())


def test_many_rows_of_a_short_vocabulary(lib):
    """More rows than the workspace has counters for."""
    x = torch.randn(3000, 65, generator=torch.Generator().manual_seed(10)).to("cuda")
    check(lib, x, (torch.arange(3000) % 65).to(torch.int32).to("cuda"), 4, rows=range(0, 3000, 97))


def test_a_captured_call_is_replayed():
    stream = torch.cuda.Stream()
    own = binding.Spts(synth.ModelShape(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=256, ltp_dlow=64, ltp_rank=16, n_layers=1, vocab=64,
                                        dtype="bf16"), max_seq=64, stream=stream)
    x, t = torch.zeros(2, 40001, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = own.token_logprobs(x, t, n_top=4)
    for i in range(4):
        g = torch.Generator().manual_seed(i)
        with torch.cuda.stream(stream):
            x.copy_(torch.randn(2, 40001, generator=g))
            t.copy_(torch.randint(0, 40001, (2,), generator=g).to(torch.int32))
            graph.replay()
        torch.cuda.synchronize()
        for r in range(2):
            lp, rank, ent, top, tok, e, ee = R.logprobs(x[r], int(t[r]), 4)
            assert abs(float(out["logprob"][r]) - lp) <= e + 2.0 ** -23 * abs(lp) and int(out["rank"][r]) == rank
            assert out["top_token"][r].tolist() == tok and abs(float(out["entropy"][r]) - ent) <= ee + 2.0 ** -23 * abs(ent)
    assert not math.isnan(float(out["logprob"][0]))
    del graph
    own.close()
