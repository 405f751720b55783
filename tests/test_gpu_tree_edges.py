"""Tree attention at its edges: states that are not finite, queries at the ends of the f16 range, softmax scales of either sign and zero."""
import types

import pytest
import torch

from .test_gpu_tree import B, REL, Batch, close, run  # noqa: F401  (B: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_key_that_is_not_finite_reaches_all_heads_of_those_who_see_it(B, dt, bad):  # noqa: F811
    """Every component of a state is part of all heads' keys.  Of an infinite pair (a, b) rotation makes a cos - b sin and b cos + a sin, one of which is the
    difference of two infinities whatever the signs: a NaN in every pair, and so in every score.  Behind the node's rank it is no part of the state."""
    b = Batch(501, [60, 200], [10, 40], dt=dt)
    b.levels[:] = 700
    want, top = b.want()
    nodes = {0: (3,), 1: (5, 21)}                     # by request
    for i, js in nodes.items():
        for j in js:
            b.nk[b.offsets[i] + j, 699 if j == 5 else 2] = bad
    b.nk[b.offsets[1] + 7, 700] = bad
    sees = torch.tensor([any(m >> j & 1 for j in nodes[i]) for i in range(2) for m in b.masks[i]])
    assert sees.sum() >= 3 and (~sees).sum() >= 10
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    out = out.cpu()
    assert torch.isnan(out[sees]).all()
    close(out[~sees], want[~sees], top, torch.float32)
    B.twkv_cache_destroy(h)


def scaled(B, scale):  # noqa: F811
    """The binding with a softmax scale in every configuration it makes."""
    names = {k: getattr(B, k) for k in dir(B) if not k.startswith("__")}
    names["make_config"] = lambda **kw: B.make_config(sm_scale=scale, **kw)
    return types.SimpleNamespace(**names)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("scale", [-0.05, -128 ** -0.5, 0.0, 0.001, 0.25])
def test_scales(B, dt, scale):  # noqa: F811
    """Two empty caches and nodes that see nothing among the requests; masks stay masks whatever the scale's sign.  Score errors go with the scale: REL is for
    128^-0.5."""
    b = Batch(502, [0, 300, 64, 0], [5, 9, 30, 1], dt=dt)
    b.masks[0][2] = 0
    b.masks[1][4] = 0                                 # sees cached tokens only
    b.masks[3][0] = 0                                 # sees nothing at all
    want, top = b.want(scale=scale)
    h = b.cache(scaled(B, scale))
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    assert (out.double().cpu() - want).abs().max() <= REL * max(1.0, abs(scale) * 128 ** 0.5) * top
    assert (out[2] == 0).all() and (out[b.offsets[3]] == 0).all()
    B.twkv_cache_destroy(h)


def test_bf16_queries_at_the_ends_of_the_f16_range(B):  # noqa: F811
    """Below 2^-14 a query keeps 2^-25: with 128 components and keys of less than 8 an error of 128 x 8 x 2^-25 x 128^-0.5 < 3e-6 in a score.  Beyond 65504 it is
    clamped and reported; the other rows are right."""
    b = Batch(503, [150, 40], [6, 7], dt=torch.bfloat16)
    b.q = (b.q.float() * 2.0 ** -20).bfloat16()
    want, top = b.want()
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(out, want, top, torch.float32)
    b.q[8, 3, 17] = 70000.0
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_ERR_DEVICE_CHECK
    rows = [r for r in range(13) if r != 8]
    close(out[rows], want[rows], top, torch.float32)
    B.twkv_cache_destroy(h)


def test_after_eviction_and_growth_behind_it(B):  # noqa: F811
    """A third of one sequence stays, nothing of the other, and both grow by tokens of other ranks before the call."""
    b = Batch(504, [200, 77], [6, 10], max_tokens=400, max_seqs=8)      # (room: evicted tiles are not used again)
    h = b.cache(B)
    keep = [set(range(0, 200, 3)), set()]
    for s, k in zip(b.seqs, keep):
        B.twkv_evict(h, 0, s, torch.tensor(sorted(k), dtype=torch.int32, device="cuda"))
    more = Batch(505, [90, 140], [6, 10])
    pos = [range(200, 290), range(77, 217)]
    B.twkv_compress(h, 0, more.xk.cuda(), more.xv.cuda(), torch.tensor([s for s, p in zip(b.seqs, pos) for _ in p], dtype=torch.int32).cuda(),
                    torch.tensor([x for p in pos for x in p], dtype=torch.int32).cuda(), None, more.ranks.to(torch.int16).cuda(), B.TWKV_GATE_FORCED)
    # both together, as one batch of longer contexts
    both = Batch(504, [290, 217], [6, 10])
    for name in ("xk", "xv", "ranks"):
        x, y = getattr(b, name), getattr(more, name)
        setattr(both, name, torch.cat([x[:200], y[:90], x[200:], y[90:]]))
    for name in ("uk", "uv", "nk", "nv", "levels", "q", "parents", "masks", "offsets", "seqs"):
        setattr(both, name, getattr(b, name))
    both.positions = [c + bin(m).count("1") - 1 for c, ms in zip(both.ctx, both.masks) for m in ms]
    want, top = both.want([keep[0] | set(pos[0]), set(pos[1])])
    out, _ = run(B, h, both)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(out, want, top, torch.float32)
    assert B.twkv_cache_check(h) == (B.TWKV_OK, 0)
    B.twkv_cache_destroy(h)
