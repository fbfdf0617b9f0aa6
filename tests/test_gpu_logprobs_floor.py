"""The floor below which none of the best alternatives lies: found once from the warps' largest tokens and once from those of stretches of
512, each in words of shared memory of its own."""
import pytest
import torch

from paper_2601_13155_b200 import binding, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [17000, 40000, 152063])
@pytest.mark.parametrize("n", [5, 600])
@pytest.mark.parametrize("where", ["anywhere", "one warp", "one stretch", "the first tokens"])
def test_alternatives_whichever_floor_is_the_higher(vocab, n, where):
    """Rows whose largest tokens lie in one warp's places (its floor is far above the others'), in one stretch or everywhere."""
    lib = binding.Spts(synth.ModelShape(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=256, ltp_dlow=64, ltp_rank=16, n_layers=1, vocab=64,
                                        dtype="bf16"), max_seq=64)
    g = torch.Generator(device="cuda").manual_seed(vocab + n)
    x = torch.randn(n, vocab, device="cuda", generator=g)
    token = torch.arange(vocab, device="cuda")
    lift = {"anywhere": token < 0, "one warp": token % 1024 < 128, "one stretch": (token >= 8192) & (token < 8704), "the first tokens": token < 40}[where]
    x += 10.0 * lift
    value, index = torch.sort(x, dim=-1, descending=True, stable=True)
    lse = torch.logsumexp(x.double(), -1, keepdim=True)
    for n_top in (1, 20, 32):
        for _ in range(3):
            out = lib.token_logprobs(x, n_top=n_top)
            assert torch.equal(out["top_token"], index[:, :n_top].to(torch.int32))
            # a term of the sum is off by 2 (2^-21 + 2^-23 |l - m|) of itself, |l - m| < 24 here, the sum of positive terms by
            # (vocab / 512 + 60) 2^-24, the logarithm, the last differences and the result by 2^-22 of what they meet
            want = value[:, :n_top].double() - lse
            bound = 2 * (2.0 ** -21 + 24 * 2.0 ** -23) + (vocab / 512 + 60) * 2.0 ** -24 + 2.0 ** -22 * (1 + want.abs() + 24)
            assert bool(((out["top_logprob"].double() - want).abs() <= bound).all())
    assert lib.device_status() == 0 and lib.check_guards() == 0
    lib.close()


@pytest.mark.parametrize("n", [2, 700])
def test_stretches_of_several_pieces(n):
    """The longest rows: a stretch whose largest token is noted is several pieces' 512 where a row is not shared."""
    vocab = 1 << 20
    lib = binding.Spts(synth.ModelShape(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=256, ltp_dlow=64, ltp_rank=16, n_layers=1, vocab=64,
                                        dtype="bf16"), max_seq=64)
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, vocab, device="cuda", generator=g)
    target = torch.randint(0, vocab, (n,), device="cuda", generator=g, dtype=torch.int32)
    out = lib.token_logprobs(x, target, n_top=32)
    assert lib.device_status() == 0 and lib.check_guards() == 0
    for i in range(0, n, max(1, n // 7)):
        value, index = torch.sort(x[i], descending=True, stable=True)
        assert torch.equal(out["top_token"][i], index[:32].to(torch.int32))
        xt = x[i, int(target[i])]
        assert int(out["rank"][i]) == int((x[i] > xt).sum() + ((x[i] == xt) & (torch.arange(vocab, device="cuda") < int(target[i]))).sum())
        want = xt.double() - torch.logsumexp(x[i].double(), -1)
        bound = 2 * (2.0 ** -21 + 16 * 2.0 ** -23) + (vocab / 512 + 60) * 2.0 ** -24 + 2.0 ** -22 * (1 + want.abs() + 16)
        assert abs(float(out["logprob"][i]) - float(want)) <= float(bound)
    lib.close()
