"""Plain 64-bit forms of the operators around a paged cache, and the error bounds their tests use."""
import torch


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Pages:
    """A cache whose pages lie in a random order, with something else in all places that no sequence holds."""

    def __init__(self, shape, lens, page, seed=0, spare=3, room=0, junk=float("nan"), sink=None):
        from paper_2601_13155_b200 import binding
        g = torch.Generator().manual_seed(seed)
        n, hkv, d = len(lens), shape.n_kv_heads, shape.head_dim
        dt = binding.torch_dtype(shape.dtype)
        most = max(1, -(-(max(lens) + room) // page))
        need = [-(-(held + room) // page) for held in lens]
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        table = torch.full((n, most), -7, dtype=torch.int32)
        at = 0
        for b in range(n):
            table[b, : need[b]] = torch.tensor(order[at:at + need[b]], dtype=torch.int32)
            at += need[b]
        self.lens, self.page, self.n, self.shape = list(lens), page, n, shape
        k = torch.full((n_pages, page, hkv, d), junk, dtype=torch.float32)
        v, pos = k.clone(), torch.full((n_pages, page), -99, dtype=torch.int32)
        weight = torch.full((n_pages, page), junk)
        self.rows = []
        for b, held in enumerate(lens):
            kk, vv = torch.randn(held, hkv, d, generator=g), torch.randn(held, hkv, d, generator=g)
            pp = torch.cumsum(torch.randint(1, 4, (held,), generator=g), 0).to(torch.int32)
            ww = torch.rand(held, generator=g)
            self.rows.append((kk.to(dt), vv.to(dt), pp, ww))
            j = torch.arange(held)
            slot = table[b].long()[j // page] * page + j % page
            for t, x in ((k.view(-1, hkv, d), kk), (v.view(-1, hkv, d), vv), (pos.view(-1), pp), (weight.view(-1), ww)):
                t[slot] = x
        self.table = table
        dev = "cuda:0"
        self.c = binding.PagedKv(shape, table.to(dev), page_size=page, k=k.to(dt).to(dev), v=v.to(dt).to(dev), pos=pos.to(dev),
                                 weight=weight.to(dev), length=torch.tensor(lens, dtype=torch.int32, device=dev))

    def slots(self, b, j):
        return self.table[b].long()[j // self.page] * self.page + j % self.page

    def held(self, b):
        """(K, V, pos, weight) of the rows that sequence b holds now."""
        j = torch.arange(int(self.c.length[b]))
        s = self.slots(b, j).to(self.c.k.device)
        hkv, d = self.c.heads
        return (self.c.k.view(-1, hkv, d)[s], self.c.v.view(-1, hkv, d)[s], self.c.pos.view(-1)[s], self.c.weight.view(-1)[s])


def queries(shape, rows, seed=0, scale=1.0, pad=0):
    """Packed queries of sequences with rows[b] of them, and their starts."""
    from paper_2601_13155_b200 import binding
    g = torch.Generator().manual_seed(1000 + seed)
    q = scale * torch.randn(sum(rows) + pad, shape.n_q_heads, shape.head_dim, generator=g)
    start = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32, device="cuda:0")
    return q.to(binding.torch_dtype(shape.dtype)).to("cuda:0"), start


def attention(q, k, v, off, dtype):
    """(O [m, H, d], its bound, lse [m, H], its bound) of m queries, query i seeing rows j <= off + i of k, v [rows, Hkv, d].

    Scores: d products, exact in 64 bits, added in fp32 in at most d / 4 + 8 steps, each off by at most 2^-23 of the partial sums (matrix
    units may truncate), which stay below sum |q| |k|; the scale, the maximum and the exponential's argument cost 2^-22 of the numbers they
    meet (|s|, the largest |s| and 16 for the lazy maximum).  An error of e in a score moves every weight by a factor within exp(+-2 e): an
    output by at most 2.2 e sum p |v|.  Sums over the rows: (rows / 8 + 80) steps of 2^-23 sum p |v|.  bf16 storage: a weight is rounded
    once, half_step sum p |v|.  One rounding at the end.  lse: the largest error of a score, the sum's rounding, 2^-22 of itself."""
    m, h, d = q.shape
    rows, hkv = k.shape[:2]
    if rows == 0:
        z = torch.zeros(m, h, d, dtype=torch.float64, device=q.device)
        return z, z + 1e-30, z[..., 0] - float("inf"), z[..., 0]
    q, k, v = q.double(), k.double(), v.double()
    kk, vv = k.repeat_interleave(h // hkv, 1), v.repeat_interleave(h // hkv, 1)
    seen = torch.arange(rows, device=q.device)[None, :] <= off + torch.arange(m, device=q.device)[:, None]
    zero = torch.zeros((), dtype=torch.float64, device=q.device)
    # what is not seen does not count, whatever it holds
    ever = seen.any(0)
    kk, vv = torch.where(ever[:, None, None], kk, zero), torch.where(ever[:, None, None], vv, zero)
    s = torch.einsum("mhd,rhd->hmr", q, kk) / d ** 0.5
    es = (d / 4 + 8) * 2.0 ** -23 * torch.einsum("mhd,rhd->hmr", q.abs(), kk.abs()) / d ** 0.5
    s, es = torch.where(seen, s, float("-inf")), torch.where(seen, es, zero)
    size = torch.where(seen, s.abs(), zero)
    es = es + 2.0 ** -22 * (size + size.amax(-1, keepdim=True) + 16)
    empty = ~seen.any(1)
    lse = torch.logsumexp(s, -1)
    p = torch.where(empty[:, None], zero, torch.exp(s - torch.where(empty, zero, lse)[..., None]))
    safe = torch.where(seen[None, :, :, None] & (p[..., None] >= 0), vv.permute(1, 0, 2)[:, None], zero) if not torch.isfinite(vv).all() else None
    if safe is None:
        o, a = p @ vv.permute(1, 0, 2), p @ vv.abs().permute(1, 0, 2)
    else:
        o, a = (p[..., None] * safe).sum(2), (p[..., None] * safe.abs()).sum(2)
    half = half_step(dtype)
    worst = es.amax(-1, keepdim=True)
    e = ((rows / 8 + 80) * 2.0 ** -23 + 2.2 * worst) * a
    if dtype == torch.bfloat16:
        e = e + half * a
    e = e * (1 + half) + half * o.abs() + 1e-30
    el = worst[..., 0] + (rows / 8 + 80) * 2.0 ** -23 + 2.0 ** -22 * torch.where(empty, zero, lse).abs()
    return o.permute(1, 0, 2), e.permute(1, 0, 2), lse.T, el.T


def weights(q, k, lse, off):
    """(sum of the weights that the rows of k get from the queries, over H; its bound).  lse is taken as given; a score's error e moves a
    weight by a factor within exp(+-1.1 e), and the sum of m * H positive terms is off by at most m H 2^-24 of it."""
    m, h, d = q.shape
    rows, hkv = k.shape[:2]
    if m == 0 or rows == 0:
        z = torch.zeros(rows, dtype=torch.float64, device=k.device)
        return z, z
    q, k, lse = q.double(), k.double(), lse.double()
    kk = k.repeat_interleave(h // hkv, 1)
    s = torch.einsum("mhd,rhd->hmr", q, kk) / d ** 0.5
    es = (d / 4 + 8) * 2.0 ** -23 * torch.einsum("mhd,rhd->hmr", q.abs(), kk.abs()) / d ** 0.5
    es = es + 2.0 ** -22 * (s.abs() + lse.T[..., None].abs() + 16)
    seen = torch.arange(rows, device=q.device)[None, :] <= off + torch.arange(m, device=q.device)[:, None]
    zero = torch.zeros((), dtype=torch.float64, device=q.device)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(lse), zero, lse).T[..., None]), zero)
    w = p.sum((0, 1)) / h
    e = (1.1 * torch.where(seen, es, zero) * p).sum((0, 1)) / h + (m * h + 40) * 2.0 ** -24 * w
    return w, e + 1e-30


def evict(k, v, pos, weight, keep, n_sink, n_recent):
    """The rows of one sequence after its eviction, row by row as the header defines it."""
    held = len(weight)
    if keep < 0 or held <= keep:
        return k, v, pos, weight
    p, w = pos.tolist(), weight.tolist()
    newest = max(p)
    first = [(x < n_sink) or (n_recent > 0 and x > newest - n_recent) for x in p]
    rank = sorted(range(held), key=lambda j: (not first[j], 0.0 if first[j] else float("inf") if w[j] != w[j] else -w[j],
                                              (w[j] != w[j]) and not first[j], j))
    stay = set(rank[:keep])
    holes = [j for j in range(keep) if j not in stay]
    movers = [j for j in range(keep, held) if j in stay]
    assert len(holes) == len(movers)
    src = list(range(keep))
    for a, b in zip(holes, movers):
        src[a] = b
    src = torch.tensor(src, dtype=torch.long, device=k.device)
    return k[src], v[src], pos[src], weight[src]


def logprobs(x, target, n_top):
    """One row in 64 bits: (logprob, rank, entropy, top logprobs, top tokens, bound of the log probabilities, bound of the entropy).

    A term e^(l - m) is off by 2^-21 + 2^-23 |l - m| of itself (the difference, its product with log2 e, the exponential; twice where the
    maximum moved), sums of positive terms by (vocab / 512 + 60) 2^-24 of them, and the last differences by 2^-22 of what they meet."""
    x = x.double().cpu()
    v = x.shape[0]
    live = x > float("-inf")
    bad = bool((~(x < float("inf"))).any())
    clean = torch.where(torch.isnan(x), torch.tensor(float("-inf"), dtype=torch.float64), x)
    order = sorted((j for j in range(v) if clean[j] > float("-inf")), key=lambda j: (-float(clean[j]), j))[:n_top]
    tokens = order + [-1] * (n_top - len(order))
    nan, inf = float("nan"), float("inf")
    if target is None or not 0 <= target < v:
        lp, rank = 0.0, -1
    else:
        xt = float(x[target])
        rank = int((x > xt).sum() + ((x == xt) & (torch.arange(v) < target)).sum())
        lp = None
    if bad:
        return (nan if lp is None else lp), rank, nan, [nan] * n_top, tokens, 0.0, 0.0
    if not live.any():
        return (-inf if lp is None else lp), rank, 0.0, [-inf] * n_top, tokens, 0.0, 0.0
    # differences from the maximum throughout: of logits near the end of the range even 64 bits do not hold m + log A
    m = x.max()
    d = torch.where(live, x - m, torch.zeros((), dtype=torch.float64))
    log_a = torch.log(torch.where(live, torch.exp(d), torch.zeros((), dtype=torch.float64)).sum())
    p = torch.where(live, torch.exp(d - log_a), torch.zeros((), dtype=torch.float64))
    steps = (v / 512 + 60) * 2.0 ** -24
    rel = 2 * (p * (2.0 ** -21 + 2.0 ** -23 * d.abs())).sum() + steps
    mean = (p * d.abs()).sum()
    entropy = float(log_a + mean)
    e_entropy = float(rel + 2 * (p * d.abs() * (2.0 ** -20 + 2.0 ** -22 * d.abs())).sum() + (steps + rel) * mean + 2.0 ** -22 * (mean + log_a.abs() + 1))
    top = [float((x[j] - m) - log_a) if j >= 0 else -inf for j in tokens]
    if lp is None:
        lp = float((x[target] - m) - log_a)
    return lp, rank, entropy, top, tokens, float(rel + 2.0 ** -23 * log_a.abs()) + 2.0 ** -22, e_entropy
