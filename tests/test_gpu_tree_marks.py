"""No token is lost and none counted twice: with queries of zeros all weights are equal, with the identity for a basis an output is the mean of one component, and
every token has a single one in its last component.  Outputs times the number of tokens are then counts of tokens, by rank; one token more or less shows
as a whole number.  (Counts stay below 2^7, so that 16-bit outputs, off by half a step, still round to them.)"""
import pytest
import torch

from .test_gpu_tree import B, DT, Batch, run  # noqa: F401  (B: fixture)

pytestmark = pytest.mark.gpu


def spread_ranks(n, d, most):
    """Ranks 1 .. d in turn, no more than `most` tokens each: so many are short, the rest have the full rank and a mark in no component."""
    r = torch.arange(n) % d + 1
    return r, torch.arange(n) // d < most


@pytest.mark.parametrize("ctx,nodes,hq,hkv,dt,out_dt", [
    ([20000], [4], 16, 8, "f16", "f32"),                     # many splits
    ([20000], [1], 8, 8, "bf16", "f32"),
    ([20000], [24], 8, 4, "bf16", "bf16"),
    ([9000, 700, 1, 0, 4100], [9, 64, 3, 2, 17], 16, 4, "f16", "f16"),
    ([1250] * 90, [16, 15] * 45, 16, 2, "bf16", "f32"),      # one split, ten tiles behind one another
    ([500, 513, 130, 16, 17, 15] * 6, [3, 13, 1, 2, 8, 5] * 6, 32, 8, "f16", "f32"),      # joint tiles, boxes of one token
    ([140001], [3], 2, 1, "f16", "f32"),                     # more V tiles than the plan has threads
    ([139993], [2], 1, 1, "bf16", "bf16"),
    ([70000] * 8, [64] * 8, 8, 1, "f16", "f16"),             # more than 128 tiles in a CTA: accumulators emptied for 16-bit outputs
    ([70000] * 8, [64] * 8, 8, 1, "bf16", "bf16"),
])
def test_every_token_counts_once(B, ctx, nodes, hq, hkv, dt, out_dt):  # noqa: F811
    d, n = hkv * 128, len(ctx)
    b = Batch(601, [1] * n, nodes, hq=hq, hkv=hkv, dt=DT[dt], out_dt=DT[out_dt], max_tokens=max(ctx) + 8)
    b.uk = b.uv = torch.eye(d).to(DT[dt])
    b.q = torch.zeros_like(b.q)
    b.ctx = ctx
    b.positions = [c + bin(m).count("1") - 1 for c, ms in zip(ctx, b.masks) for m in ms]
    g = torch.Generator()
    g.manual_seed(9)
    ranks, values, cached = [], [], []
    for c in ctx:
        r, marked = spread_ranks(c, d, 100)
        at = torch.randperm(c, generator=g)
        r, marked = r[at], marked[at]
        x = torch.zeros(c, d, dtype=DT[dt])
        x[torch.arange(c)[marked], r[marked] - 1] = 1.0
        ranks.append(r)
        values.append(x)
        cached.append(x.double().sum(0) if c else torch.zeros(d, dtype=torch.float64))
    r = torch.cat(ranks)
    b.ranks = torch.stack([r.flip(0), r], 1)                 # K ranks of their own
    b.xv = torch.cat(values)
    b.xk = torch.ones(len(r), d).to(DT[dt])
    b.levels = torch.randint(1, d + 1, (sum(nodes), 2), generator=g)
    b.nv = torch.zeros(sum(nodes), d, dtype=DT[dt])
    b.nv[torch.arange(sum(nodes)), b.levels[:, 1] - 1] = 1.0
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    out = out.double().cpu()
    for i, ms in enumerate(b.masks):
        for j, m in enumerate(ms):
            seen = [k for k in range(nodes[i]) if m >> k & 1]
            want = cached[i] + b.nv[[b.offsets[i] + k for k in seen]].double().sum(0)
            got = out[b.offsets[i] + j].view(hkv, hq // hkv, 128) * (ctx[i] + len(seen))
            want = want.view(hkv, 1, 128).expand_as(got)
            if out_dt == "f32":
                assert (got - want).abs().max() <= 128 * 2.0 ** -18          # 2^-18 of a count: two sums that lose 1e-6 each at most, and the division
            assert torch.equal(got.round(), want), (i, j)
    B.twkv_cache_destroy(h)
