"""Speculative decoding over the compressed cache against plain forms in 64 bits: twkv_slot_map, twkv_tree_map, twkv_tree_attn,
twkv_tree_accept, alone and as a step that uses them together.

Tolerance of the attention, against the definition in 64 bits on the same 16-bit inputs.  A rotated key is carried to 2^-21 of its size (two
f16 parts) and accumulated in fp32 over at most 64 products, each cut to 2^-23: relative 64 * 2^-23 + 2^-21 < 8.2e-6.  A score is
off by that times scale * |q| |k| <= 128^-0.5 * sqrt(128) * 1.5 * sqrt(128) * 1.5 = 26 (norms with half as much again), i.e. 2.1e-4, a weight relative to
the others by twice that, and an output by at most that times the largest value: 4.3e-4 max|v|.  The sums of values (fp32, weights in two parts
of the type, 2^-16 for bf16) stay below 2^-15 max|v| = 3.1e-5.  Together below 5e-4 max|v|, besides half a step of the output type.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BASE = 500000.0
REL = 5e-4


@pytest.fixture(scope="module")
def B():
    from paper_2603_04411_b200 import build
    build.build()
    from paper_2603_04411_b200 import binding
    return binding


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def random_parents(g, n):
    return [-1] + [int(torch.randint(0, j, (1,), generator=g)) for j in range(1, n)]


def masks_of(parents):
    out = []
    for j, p in enumerate(parents):
        out.append((1 << j) | (out[p] if p >= 0 else 0))
    return out


def as_i64(masks):
    return torch.tensor([m - (1 << 64) if m >= 1 << 63 else m for m in masks], dtype=torch.int64)


def states(g, n, d, dt, scale=1.0):
    size = (1.0 + torch.arange(d) / (d / 16)).rsqrt()
    size *= math.sqrt(d) / size.norm()
    return (torch.randn(n, d, generator=g) * size * scale).to(dt)


class Batch:
    """Sequences with cached tokens, trees behind them, and the definition in 64 bits."""

    def __init__(self, seed, ctx, nodes, *, hq=32, hkv=8, dt=torch.float16, out_dt=torch.float32, seqs=None, max_seqs=None, ranks="any", n_layers=1, layer=0,
                 base_pos=None, max_tokens=None):
        g = gen(seed)
        self.ctx, self.nodes, self.hq, self.hkv, self.dt, self.out_dt, self.layer = ctx, nodes, hq, hkv, dt, out_dt, layer
        self.n_req, self.d, self.rep = len(ctx), hkv * 128, hq // hkv
        self.max_seqs = max_seqs or self.n_req
        self.n_layers = n_layers
        self.seqs = seqs if seqs is not None else torch.randperm(self.max_seqs, generator=g)[:self.n_req].tolist()
        self.base_pos = base_pos or [0] * self.n_req
        d = self.d
        self.uk, self.uv = (torch.linalg.qr(torch.randn(d, d, generator=g))[0].to(dt).contiguous() for _ in range(2))
        n_tok, n = sum(ctx), sum(nodes)
        self.xk, self.xv = states(g, n_tok, d, dt), states(g, n_tok, d, dt)
        self.nk, self.nv = states(g, n, d, dt), states(g, n, d, dt)

        def draw(m):
            if ranks == "any":
                return torch.randint(1, d + 1, (m, 2), generator=g)
            if ranks == "small":
                return torch.randint(1, d // 4 + 1, (m, 2), generator=g)
            return torch.full((m, 2), int(ranks))
        self.ranks, self.levels = draw(n_tok), draw(n)
        self.q = torch.randn(n, hq, 128, generator=g).to(dt)
        self.parents = [random_parents(g, k) if k else [] for k in nodes]
        self.masks = [masks_of(p) for p in self.parents]
        self.offsets = [0] + np.cumsum(nodes).tolist()
        self.positions = [b + c + bin(m).count("1") - 1 for b, c, ms in zip(self.base_pos, ctx, self.masks) for m in ms]
        self.max_tokens = max_tokens or max(1, max(ctx) + 8)

    def token_rows(self):
        seq, pos = [], []
        for s, c, b in zip(self.seqs, self.ctx, self.base_pos):
            seq += [s] * c
            pos += range(b, b + c)
        return torch.tensor(seq, dtype=torch.int32), torch.tensor(pos, dtype=torch.int32)

    def cache(self, B, shuffle=True):
        cfg = B.make_config(n_layers=self.n_layers, n_q_heads=self.hq, n_kv_heads=self.hkv, dtype=self.dt, out_dtype=self.out_dt, max_seqs=self.max_seqs,
                            max_tokens_per_seq=self.max_tokens, rope_base=BASE)
        payload = int(((self.ranks + 63) // 64 * 128).sum()) + (1 << 22)
        self.pool = torch.empty(B.twkv_cache_required_bytes(cfg, payload), dtype=torch.uint8, device="cuda")
        h = B.twkv_cache_create(cfg, self.pool)
        self.dev_u = self.uk.cuda(), self.uv.cuda()
        B.twkv_cache_set_layer_params(h, self.layer, *self.dev_u)
        seq, pos = self.token_rows()
        n = len(seq)
        if n:
            at = torch.randperm(n, generator=gen(7)) if shuffle else torch.arange(n)
            B.twkv_compress(h, self.layer, self.xk[at].cuda(), self.xv[at].cuda(), seq[at].cuda(), pos[at].cuda(), None,
                            self.ranks[at].to(torch.int16).cuda(), B.TWKV_GATE_FORCED)
        assert B.twkv_cache_status(h) == B.TWKV_OK
        return h

    def args(self):
        dev = lambda x, dt: torch.tensor(x, dtype=dt).cuda()  # noqa: E731
        return dict(q=self.q.cuda(), K=self.nk.cuda(), V=self.nv.cuda(), levels=self.levels.to(torch.int16).cuda(), req_seqs=dev(self.seqs, torch.int32),
                    offsets=dev(self.offsets, torch.int32), positions=dev(self.positions, torch.int32),
                    masks=as_i64([m for ms in self.masks for m in ms]).cuda())

    def rotate(self, x, pos):
        a = torch.tensor(pos, dtype=torch.float64)[:, None] * BASE ** (-torch.arange(64, dtype=torch.float64) / 64)
        c, s = a.cos()[:, None], a.sin()[:, None]
        return torch.cat([x[..., :64] * c - x[..., 64:] * s, x[..., 64:] * c + x[..., :64] * s], -1)

    def rebuilt(self, x, ranks, u):
        keep = torch.arange(self.d)[None] < ranks[:, None]
        return (torch.where(keep, x.double(), 0.0) @ u.double()).view(-1, self.hkv, 128)

    def want(self, keep=None, scale=128 ** -0.5):
        """Outputs in 64 bits and the largest value; keep: per request, the positions in the cache that count."""
        out, top = torch.zeros(sum(self.nodes), self.hq, 128, dtype=torch.float64), 0.0
        t0 = 0
        for i, (c, n) in enumerate(zip(self.ctx, self.nodes)):
            rows = slice(self.offsets[i], self.offsets[i + 1])
            tok = slice(t0, t0 + c)
            t0 += c
            if n == 0:
                continue
            pos = list(range(self.base_pos[i], self.base_pos[i] + c))
            k = self.rotate(self.rebuilt(self.xk[tok], self.ranks[tok, 0], self.uk), pos)
            v = self.rebuilt(self.xv[tok], self.ranks[tok, 1], self.uv)
            if keep is not None:
                sel = [j for j, p in enumerate(pos) if p in keep[i]]
                k, v = k[sel], v[sel]
            k2 = self.rotate(self.rebuilt(self.nk[rows], self.levels[rows, 0], self.uk), self.positions[rows])
            v2 = self.rebuilt(self.nv[rows], self.levels[rows, 1], self.uv)
            for j, m in enumerate(self.masks[i]):
                at = [t for t in range(n) if m >> t & 1]
                kk, vv = torch.cat([k, k2[at]]), torch.cat([v, v2[at]])
                if len(kk) == 0:
                    continue
                top = max(top, float(vv.abs().max()))
                qq = self.q[rows][j].double().view(self.hkv, self.rep, 128)
                p = torch.softmax(torch.einsum("hrd,nhd->hrn", qq, kk) * scale, -1)
                out[rows.start + j] = torch.einsum("hrn,nhd->hrd", p, vv).reshape(self.hq, 128)
        return out, top


def run(B, h, b, args=None, ws_bytes=None, n_rows=None, max_nodes=None, stream=None, out=None):
    args = args or b.args()
    most = max_nodes or max(1, max(b.nodes))
    ws = torch.empty(ws_bytes or B.twkv_tree_required_bytes(h, b.n_req, most), dtype=torch.uint8, device="cuda")
    out = torch.full((args["q"].shape[0], b.hq, 128), 7.0, dtype=b.out_dt, device="cuda") if out is None else out
    B.twkv_tree_attn(h, b.layer, args["q"], args["K"], args["V"], args["levels"], args["req_seqs"], args["offsets"], args["positions"], args["masks"], out, ws,
                     max_nodes=most, stream=stream)
    return out, ws


def close(got, want, top, dt):
    got = got.double().cpu()
    tol = REL * top + torch.finfo(dt).eps / 2 * want.abs() + (0 if dt == torch.float32 else torch.finfo(dt).tiny)
    worst = ((got - want).abs() - tol).max()
    assert worst <= 0, float((got - want).abs().max())


CASES = [
    # contexts, nodes, heads, type, output type, ranks
    ([1], [1], 1, 1, "f16", "f32", "any"),
    ([0, 5, 0], [1, 64, 3], 8, 8, "f16", "f32", "any"),
    ([127, 128, 129, 700], [5, 1, 13, 7], 32, 8, "f16", "f16", "any"),
    ([300, 31], [64, 33], 32, 8, "bf16", "bf16", "any"),
    ([513, 1000], [9, 2], 64, 8, "bf16", "f32", "small"),
    ([200, 40, 77], [11, 17, 3], 12, 6, "f16", "f32", "any"),
    ([260], [3], 5, 5, "bf16", "f32", "any"),
    ([150, 90], [63, 12], 8, 1, "f16", "f32", "any"),
    ([128, 384], [16, 16], 32, 8, "f16", "f32", 1024),
    ([2000], [8], 16, 4, "f16", "bf16", 64),
    ([33] * 40, [4] * 40, 8, 4, "f16", "f32", "small"),
    ([20, 1500], [2, 31], 24, 3, "bf16", "f16", "any"),
    ([300, 0, 140], [20, 64, 33], 32, 8, "f16", "f32", 1024),         # wide classes with many query rows
    ([131, 40], [9, 5], 7, 7, "bf16", "f32", "any"),
    ([131], [3], 56, 7, "f16", "f32", "any"),
    ([700], [50], 40, 5, "bf16", "f32", "any"),
]
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("case", range(len(CASES)))
def test_tree_attention(B, case):
    ctx, nodes, hq, hkv, dt, out_dt, ranks = CASES[case]
    b = Batch(100 + case, ctx, nodes, hq=hq, hkv=hkv, dt=DT[dt], out_dt=DT[out_dt], ranks=ranks, max_seqs=len(ctx) + case % 3)
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = b.want()
    close(out, want, top, DT[out_dt])
    # the room for nodes is only a bound
    out2, _ = run(B, h, b, max_nodes=64)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(out2, want, top, DT[out_dt])
    code, bad = B.twkv_cache_check(h)
    assert code == B.TWKV_OK and bad == 0
    B.twkv_cache_destroy(h)


def test_one_layer_of_several_and_far_positions(B):
    b = Batch(3, [90, 400], [6, 21], n_layers=3, layer=1, base_pos=[100000, 500000], dt=torch.bfloat16)
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = b.want()
    close(out, want, top, torch.float32)
    B.twkv_cache_destroy(h)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_many_tiles_behind_one_another(B, dt):
    """More requests than there are SMs for splits: a CTA takes ten tiles, empties its accumulators on the way, and finds larger and larger scores
    (queries eight times as large, keys growing along the positions: score error 8 x that of the derivation above)."""
    b = Batch(15, [1250] * 90, [16, 15] * 45, hq=16, hkv=2, dt=dt, ranks=200)
    b.q = (b.q.float() * 8).to(dt)
    ramp = torch.linspace(0.05, 1.0, 1250).repeat(90)[:, None]
    b.xk = (b.xk.float() * ramp).to(dt)
    h = b.cache(B, shuffle=False)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = b.want()
    assert (out.double().cpu() - want).abs().max() <= 8 * REL * top
    again, _ = run(B, h, b)
    assert torch.equal(out, again)
    B.twkv_cache_destroy(h)


@pytest.mark.parametrize("dt,out_dt,nodes", [(torch.float16, torch.float32, 4), (torch.bfloat16, torch.float32, 1), (torch.bfloat16, torch.bfloat16, 24)])
def test_many_splits(B, dt, out_dt, nodes):
    b = Batch(16, [20000], [nodes], hq=4, hkv=2, dt=dt, out_dt=out_dt, ranks="any")
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = b.want()
    close(out, want, top, out_dt)
    B.twkv_cache_destroy(h)


def test_more_requests_than_a_cta_has_threads(B):
    n = 1500
    b = Batch(18, [j % 5 for j in range(n)], [1 + (j % 7 == 0) for j in range(n)], hq=2, hkv=1, ranks="any", max_seqs=4096)
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = b.want()
    close(out, want, top, torch.float32)
    # the last names the sequence of the first
    args = b.args()
    args["req_seqs"][-1] = args["req_seqs"][0]
    out, _ = run(B, h, b, args)
    assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG
    close(out[:b.offsets[-2]], want[:b.offsets[-2]], top, torch.float32)
    assert (out[b.offsets[-2]:] == 0).all()
    B.twkv_cache_destroy(h)


def test_fp32_outputs_are_as_good_as_fp32_sums(B):
    """Relative error of the whole output.  fp32 sums of n terms, each step rounded, wander by sqrt(n) 2^-24 / sqrt(3): a key's 256 products 5.5e-7, doubled by
    queries, scores and weights, and 1300 weighted values 1.2e-6; 4e-6 is twice their sum."""
    for dt in (torch.float16, torch.bfloat16):
        b = Batch(17, [1300] * 3, [12] * 3, hq=8, hkv=2, dt=dt, ranks="any")
        h = b.cache(B)
        out, _ = run(B, h, b)
        want, _ = b.want()
        assert float((out.double().cpu() - want).norm() / want.norm()) <= 4e-6
        B.twkv_cache_destroy(h)


@pytest.mark.parametrize("scale", [2.0 ** -7, 2.0 ** 9])
def test_small_and_large_values(B, scale):
    """Powers of two in the values change nothing in the relative error (the bound is the one above): mean components far below the fp16 range's normal numbers
    and near its end alike."""
    for dt in (torch.float16, torch.bfloat16):
        b = Batch(19, [1300, 60], [12, 7], hq=8, hkv=2, dt=dt, ranks="any")
        b.xv, b.nv = (b.xv.float() * scale).to(dt), (b.nv.float() * scale).to(dt)
        h = b.cache(B)
        out, _ = run(B, h, b)
        assert B.twkv_cache_status(h) == B.TWKV_OK
        want, _ = b.want()
        for i in range(2):
            rows = slice(b.offsets[i], b.offsets[i + 1])
            assert float((out[rows].double().cpu() - want[rows]).norm() / want[rows].norm()) <= 4e-6
        B.twkv_cache_destroy(h)


def test_negative_scale_and_scores_far_apart(B):
    # queries fifty times as large: the softmax is decided by one token (score error 50 x that of the derivation above)
    b = Batch(5, [300, 64], [9, 30])
    b.q = (b.q.float() * 50).half()
    h = b.cache(B)
    out, _ = run(B, h, b)
    want, top = b.want()
    got = out.double().cpu()
    assert (got - want).abs().max() <= 50 * REL * top
    B.twkv_cache_destroy(h)


def test_masks_of_any_form(B):
    # cross links, nodes that do not see themselves, nodes that see nothing: with an empty cache zeros
    b = Batch(11, [0, 50, 0], [7, 12, 64])
    g = gen(12)
    for i, n in enumerate(b.nodes):
        b.masks[i] = [int(torch.randint(0, 1 << 62, (1,), generator=g)) & ((1 << n) - 1) for _ in range(n)]
    b.masks[0][3] = 0
    b.masks[1][5] = 0
    b.masks[2][63] = (1 << 64) - 1
    want, top = b.want()
    # bits behind the tree's nodes say nothing
    b.masks[0][3] = 1 << 40
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(out, want, top, torch.float32)
    assert out[3].abs().max() == 0
    B.twkv_cache_destroy(h)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_what_is_not_a_number_stays_with_those_who_see_it(B, dt):
    b = Batch(21, [60, 200], [10, 40], dt=dt)
    b.levels[:] = 700
    b.nk[4, 3] = float("nan")
    b.nv[7, 100] = float("inf")
    b.nv[8, 900] = float("nan")                      # behind its rank: not part of the state
    b.nk[15, 699] = float("-inf")
    b.nv[30, 0] = float("nan")
    sees = torch.zeros(50, dtype=torch.bool)
    for i in range(2):
        for j, m in enumerate(b.masks[i]):
            for node in (4, 7, 15, 30):
                k = node - b.offsets[i]
                if 0 <= k < b.nodes[i] and m >> k & 1:
                    sees[b.offsets[i] + j] = True
    h = b.cache(B)
    out, _ = run(B, h, b)
    out = out.cpu()
    assert not torch.isfinite(out[sees]).any(-1).all()
    clean = Batch(21, [60, 200], [10, 40], dt=dt)
    clean.levels[:] = 700
    want, top = clean.want()
    close(out[~sees], want[~sees], top, torch.float32)
    assert sees.sum() >= 4 and (~sees).sum() > 10
    for node in (7, 30):                             # a value: every output of those who see it
        i = int(node >= 10)
        for j, m in enumerate(b.masks[i]):
            if m >> (node - b.offsets[i]) & 1:
                assert not torch.isfinite(out[b.offsets[i] + j]).any()
    B.twkv_cache_destroy(h)


def test_rows_behind_the_last_request_and_bytes_behind_the_workspace(B):
    b = Batch(31, [70, 10], [5, 9])
    h = b.cache(B)
    args = b.args()
    for k in ("q", "K", "V", "levels", "positions", "masks"):
        args[k] = torch.cat([args[k], args[k][:4]])
    need = B.twkv_tree_required_bytes(h, 2, 9)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    out = torch.full((18, 32, 128), 7.0, device="cuda")
    B.twkv_tree_attn(h, 0, args["q"], args["K"], args["V"], args["levels"], args["req_seqs"], args["offsets"], args["positions"], args["masks"], out,
                     ws[:need], max_nodes=9)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = b.want()
    close(out[:14], want, top, torch.float32)
    assert (out[14:] == 7).all() and (ws[need:] == 0x5a).all()
    B.twkv_cache_destroy(h)


def test_less_workspace_means_more_passes(B):
    b = Batch(41, [40, 300, 0, 129, 64, 5, 250], [3, 9, 1, 0, 7, 9, 2], max_seqs=9)
    h = b.cache(B)
    want, top = b.want()
    one, all_ = B.twkv_tree_required_bytes(h, 1, 9), B.twkv_tree_required_bytes(h, 7, 9)
    assert 0 < one < all_
    assert [B.twkv_tree_required_bytes(h, n, 9) for n in range(1, 10)] == sorted(B.twkv_tree_required_bytes(h, n, 9) for n in range(1, 10))
    for room in (one, B.twkv_tree_required_bytes(h, 3, 9), all_, 3 * all_):
        out, _ = run(B, h, b, ws_bytes=room)
        assert B.twkv_cache_status(h) == B.TWKV_OK
        close(out, want, top, torch.float32)
    with pytest.raises(B.TwkvError) as e:
        run(B, h, b, ws_bytes=one - 256)
    assert e.value.code == B.TWKV_ERR_CAPACITY
    # a sequence that an earlier pass has served is refused in a later one as well
    args = b.args()
    args["req_seqs"][6] = args["req_seqs"][1]
    out, _ = run(B, h, b, args, ws_bytes=one)
    assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG
    assert (out[b.offsets[6]:] == 0).all()
    close(out[:b.offsets[6]], want[:b.offsets[6]], top, torch.float32)
    B.twkv_cache_destroy(h)


def test_requests_that_are_refused_leave_the_others_alone(B):
    b = Batch(51, [90, 30, 60], [4, 6, 5], max_seqs=4)
    h = b.cache(B)
    want, top = b.want()
    spoil = {
        "unknown sequence": lambda a: a["req_seqs"].__setitem__(1, 4),
        "negative sequence": lambda a: a["req_seqs"].__setitem__(1, -1),
        "listed before": lambda a: a["req_seqs"].__setitem__(1, int(a["req_seqs"][0])),
        "rank zero": lambda a: a["levels"].__setitem__((6, 0), 0),
        "rank too large": lambda a: a["levels"].__setitem__((9, 1), 1025),
        "negative position": lambda a: a["positions"].__setitem__(5, -1),
        "position too large": lambda a: a["positions"].__setitem__(5, 524288),
    }
    for name, f in spoil.items():
        args = b.args()
        f(args)
        out, _ = run(B, h, b, args)
        assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG, name
        rows = torch.tensor([r for r in range(15) if not 4 <= r < 10])
        close(out[rows.cuda()], want[rows], top, torch.float32)
        assert (out[4:10] == 0).all(), name
    # offsets that name no rows: nothing of that request is written
    for bad in ([0, 4, 3, 8], [0, 4, 11, 15], [0, 4, 99, 103]):
        args = b.args()
        args["offsets"] = torch.tensor(bad, dtype=torch.int32).cuda()
        out, _ = run(B, h, b, args, max_nodes=6)
        assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG, bad
        close(out[:4], want[:4], top, torch.float32)
    # and the call after is whole again
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(out, want, top, torch.float32)
    B.twkv_cache_destroy(h)


def test_host_refusals(B):
    b = Batch(61, [20], [4])
    h = b.cache(B)
    a = b.args()
    out = torch.full((4, 32, 128), 7.0, device="cuda")
    ws = torch.empty(B.twkv_tree_required_bytes(h, 1, 4), dtype=torch.uint8, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    good = [h, 0, p(a["q"]), p(a["K"]), p(a["V"]), p(a["levels"]), p(a["req_seqs"]), p(a["offsets"]), p(a["positions"]), p(a["masks"]), 1, 4, 4, p(out), p(ws),
            ws.numel(), torch.cuda.current_stream().cuda_stream]
    launches = B.twkv_launch_count()
    for at, bad in [(1, -1), (1, 1), (2, None), (3, None), (4, None), (5, None), (6, None), (7, None), (8, None), (9, None), (10, -1), (10, 2), (11, -1),
                    (12, 0), (12, 65), (13, None), (14, None), (2, p(a["q"]) + 2), (3, p(a["K"]) + 8), (4, p(a["V"]) + 8), (5, p(a["levels"]) + 2),
                    (9, p(a["masks"]) + 4), (13, p(out) + 4), (14, p(ws) + 16)]:
        args = list(good)
        args[at] = bad
        assert B.lib.twkv_tree_attn(*args) == B.TWKV_ERR_INVALID_ARG, (at, bad)
    args = list(good)
    args[15] = ws.numel() - 1
    assert B.lib.twkv_tree_attn(*args) == B.TWKV_ERR_CAPACITY
    for at in (10, 11):
        args = list(good)
        args[at] = 0
        assert B.lib.twkv_tree_attn(*args) == B.TWKV_OK
    assert B.twkv_launch_count() == launches and (out == 7).all()
    assert [B.twkv_tree_required_bytes(h, *x) for x in ((0, 4), (2, 4), (1, 0), (1, 65), (-1, 4))] == [0] * 5
    # a layer without parameters
    b2 = Batch(62, [20], [4], n_layers=2)
    h2 = b2.cache(B)
    args = list(good)
    args[0], args[1] = h2, 1
    assert B.lib.twkv_tree_attn(*args) == B.TWKV_ERR_INVALID_ARG
    o32 = torch.zeros(8, dtype=torch.int32, device="cuda")
    m = torch.zeros(8, dtype=torch.int64, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    for args in ([h, 1, p(o32), p(o32), None, 1, 4, p(o32), p(o32), p(o32), s], [h, 0, None, p(o32), None, 1, 4, p(o32), p(o32), p(o32), s],
                 [h, 0, p(o32), p(o32), None, 2, 4, p(o32), p(o32), p(o32), s], [h, 0, p(o32), p(o32), None, 1, -1, p(o32), p(o32), p(o32), s],
                 [h, 0, p(o32), p(o32), None, 1, 4, None, p(o32), p(o32), s], [h, 0, p(o32), p(o32), None, 1, 4, p(o32), None, p(o32), s]):
        assert B.lib.twkv_slot_map(*args) == B.TWKV_ERR_INVALID_ARG
    for args in ([h, p(o32), p(o32), 1, 4, 65, p(o32), p(m), s], [h, p(o32), p(o32), 1, 4, 0, p(o32), p(m), s], [h, None, p(o32), 1, 4, 8, p(o32), p(m), s],
                 [h, p(o32), p(o32), 1, 4, 8, p(o32), p(m) + 4, s], [h, p(o32), p(o32), 2, 4, 8, p(o32), p(m), s]):
        assert B.lib.twkv_tree_map(*args) == B.TWKV_ERR_INVALID_ARG
    for args in ([h, p(o32), p(o32), p(o32), p(o32), 1, 4, 65, p(o32), p(o32), p(o32), s], [h, p(o32), p(o32), None, p(o32), 1, 4, 8, p(o32), p(o32), p(o32), s],
                 [h, p(o32), p(o32), p(o32), p(o32), 1, 4, 8, None, p(o32), p(o32), s]):
        assert B.lib.twkv_tree_accept(*args) == B.TWKV_ERR_INVALID_ARG
    B.twkv_cache_destroy(h)
    B.twkv_cache_destroy(h2)


def test_after_eviction_and_growth(B):
    b = Batch(71, [200, 77], [6, 10], max_tokens=400)
    h = b.cache(B)
    keep = [set(range(0, 200, 3)), set()]
    for s, k in zip(b.seqs, keep):
        B.twkv_evict(h, 0, s, torch.tensor(sorted(k), dtype=torch.int32, device="cuda"))
    want, top = b.want(keep)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(out, want, top, torch.float32)
    B.twkv_cache_destroy(h)


def test_one_node_is_a_decode_step(B):
    """A root alone sees what a decode query sees once its token is stored."""
    b = Batch(81, [150, 31, 400], [1, 1, 1], dt=torch.bfloat16, max_tokens=500)
    h = b.cache(B)
    a = b.args()
    out, _ = run(B, h, b, a)
    B.twkv_compress(h, 0, a["K"], a["V"], a["req_seqs"], a["positions"], None, a["levels"], B.TWKV_GATE_FORCED)
    step = torch.empty_like(out)
    B.twkv_decode_attn(h, 0, a["q"], a["req_seqs"], step)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    _, top = b.want()
    assert (out - step).abs().max() <= 2 * REL * top
    B.twkv_cache_destroy(h)


def test_captured_and_replayed(B):
    """A captured call follows the device's lengths, masks and cache; two caches' graphs share nothing but a workspace, in turn."""
    b = Batch(91, [100, 40], [8, 5], max_tokens=600)
    h = b.cache(B)
    args = b.args()
    ws = torch.empty(B.twkv_tree_required_bytes(h, 2, 8), dtype=torch.uint8, device="cuda")
    out = torch.empty(13, 32, 128, device="cuda")
    call = lambda: B.twkv_tree_attn(h, 0, args["q"], args["K"], args["V"], args["levels"], args["req_seqs"], args["offsets"], args["positions"],  # noqa: E731
                                    args["masks"], out, ws, max_nodes=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.current_stream().wait_stream(side)
    graph.replay()
    want, top = b.want()
    close(out, want, top, torch.float32)
    # other trees and more tokens than at the capture
    c = Batch(92, [500, 3], [2, 8], max_tokens=600, seqs=b.seqs)
    c.uk, c.uv = b.uk, b.uv
    B.twkv_cache_reset(h)
    seq, pos = c.token_rows()
    B.twkv_compress(h, 0, c.xk.cuda(), c.xv.cuda(), seq.cuda(), pos.cuda(), None, c.ranks.to(torch.int16).cuda(), B.TWKV_GATE_FORCED)
    for k, t in c.args().items():
        args[k][:len(t)].copy_(t)
    graph.replay()
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, top = c.want()
    close(out[:10], want, top, torch.float32)
    graph.replay()
    close(out[:10], want, top, torch.float32)
    B.twkv_cache_destroy(h)


def test_same_bits_every_time(B):
    b = Batch(93, [700, 90, 1100], [9, 16, 4], dt=torch.bfloat16)
    h = b.cache(B)
    first, _ = run(B, h, b)
    for _ in range(4):
        again, _ = run(B, h, b)
        assert torch.equal(first, again)
    B.twkv_cache_destroy(h)


def test_another_stream(B):
    b = Batch(95, [300], [12])
    h = b.cache(B)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    args = b.args()
    torch.cuda.synchronize()
    out = torch.empty(12, 32, 128, device="cuda")
    out, ws = run(B, h, b, args, stream=s, out=out)
    s.synchronize()
    want, top = b.want()
    close(out, want, top, torch.float32)
    B.twkv_cache_destroy(h)


# ------------------------------------------------------------------------------------------ maps
def map_cache(B, max_seqs=64, tokens=None):
    cfg = B.make_config(n_layers=2, n_q_heads=1, n_kv_heads=1, max_seqs=max_seqs, max_tokens_per_seq=256)
    pool = torch.empty(B.twkv_cache_required_bytes(cfg, 1 << 20), dtype=torch.uint8, device="cuda")
    h = B.twkv_cache_create(cfg, pool)
    return h, pool


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("n_req,most", [(1, 1), (1, 0), (3, 5), (64, 1), (64, 300), (1000, 40), (4096, 3), (2500, 129)])
def test_slot_map(B, n_req, most):
    h, pool = map_cache(B, max_seqs=max(64, n_req))
    g = gen(n_req + most)
    lens = torch.randint(0, most + 1, (n_req,), generator=g)
    if n_req == 1:
        lens[0] = most
    seqs = torch.randperm(max(64, n_req), generator=g)[:n_req]
    starts = torch.randint(0, 500000, (n_req,), generator=g)
    n = int(lens.sum())
    off, sid, pos = i32([-5] * (n_req + 1)), i32([-5] * (n + 3)), i32([-5] * (n + 3))
    B.twkv_slot_map(h, 1, i32(seqs.tolist()), i32(lens.tolist()), off, sid, pos, starts=i32(starts.tolist()))
    assert B.twkv_cache_status(h) == B.TWKV_OK
    assert off.tolist() == [0] + lens.cumsum(0).tolist()
    assert sid.tolist() == torch.repeat_interleave(seqs, lens).tolist() + [-5] * 3
    want = [int(s) + j for s, k in zip(starts, lens) for j in range(int(k))]
    assert pos.tolist() == want + [-5] * 3
    B.twkv_cache_destroy(h)


def test_slot_map_from_the_cache_and_without_requests(B):
    h, pool = map_cache(B)
    x = torch.randn(30, 128, device="cuda").half()
    B.twkv_compress(h, 1, x, x, i32([3] * 20 + [9] * 10), i32(list(range(20)) + list(range(10))), None, torch.full((30, 2), 5, dtype=torch.int16, device="cuda"),
                    B.TWKV_GATE_FORCED)
    off, sid, pos = i32([0] * 4), i32([0] * 6), i32([0] * 6)
    B.twkv_slot_map(h, 1, i32([9, 7, 3]), i32([2, 1, 3]), off, sid, pos)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    assert off.tolist() == [0, 2, 3, 6] and sid.tolist() == [9, 9, 7, 3, 3, 3] and pos.tolist() == [10, 11, 0, 20, 21, 22]
    B.twkv_slot_map(h, 0, i32([9, 7, 3]), i32([2, 1, 3]), off, sid, pos)          # the other layer holds nothing
    assert pos.tolist() == [0, 1, 0, 0, 1, 2]
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    off = i32([4])
    B.twkv_slot_map(h, 0, empty, empty, off, empty, empty)
    assert off.tolist() == [0]
    B.twkv_cache_destroy(h)


def test_slot_map_refusals(B):
    h, pool = map_cache(B)
    for seqs, lens, starts, code in [([0, 64], [1, 1], [0, 0], "i"), ([0, -1], [1, 1], [0, 0], "i"), ([0, 1], [1, -1], [0, 0], "i"), ([0, 1], [1, 1], [0, -1], "i"),
                                     ([0, 1], [1, 2], [0, 524287], "i"), ([5, 5], [1, 1], None, "i"), ([0, 1], [4, 5], [0, 0], "c"),
                                     ([0, 1], [2 ** 31 - 1, 2 ** 31 - 1], [0, 0], "i"), ([0, 1], [500000, 500000], [0, 0], "c")]:
        off, sid, pos = i32([9] * 3), i32([9] * 8), i32([9] * 8)
        B.twkv_slot_map(h, 0, i32(seqs), i32(lens), off, sid, pos, starts=None if starts is None else i32(starts))
        assert B.twkv_cache_status(h) == (B.TWKV_ERR_INVALID_ARG if code == "i" else B.TWKV_ERR_CAPACITY), (seqs, lens)
        assert off.tolist() == [0] * 3 and sid.tolist() == [9] * 8 and pos.tolist() == [9] * 8
    # two pieces of one sequence, with starts of their own
    off, sid, pos = i32([9] * 3), i32([9] * 8), i32([9] * 8)
    B.twkv_slot_map(h, 0, i32([5, 5]), i32([2, 1]), off, sid, pos, starts=i32([0, 2]))
    assert B.twkv_cache_status(h) == B.TWKV_OK and pos.tolist() == [0, 1, 2] + [9] * 5 and sid.tolist() == [5] * 3 + [9] * 5
    B.twkv_cache_destroy(h)


@pytest.mark.parametrize("nodes", [[1], [64], [0, 3, 0, 64, 1], [33, 32, 31] * 20])
def test_tree_map(B, nodes):
    h, pool = map_cache(B)
    g = gen(len(nodes))
    parents = [random_parents(g, n) if n else [] for n in nodes]
    if len(nodes) == 1 and nodes[0] == 64:
        parents = [list(range(-1, 63))]                                            # a chain
    offsets = [0] + np.cumsum(nodes).tolist()
    starts = torch.randint(0, 9999, (len(nodes),), generator=g).tolist()
    rows = [s + j for s, n in zip(starts, nodes) for j in range(n)]
    want = [m for p in parents for m in masks_of(p)]
    pos, masks = i32(rows + [-7]), torch.full((len(rows) + 1,), -7, dtype=torch.int64, device="cuda")
    for _ in range(2):                                                              # again on its own result: the same
        B.twkv_tree_map(h, i32(offsets), i32([p for ps in parents for p in ps] + [0]), pos, masks)
        assert B.twkv_cache_status(h) == B.TWKV_OK
        assert masks[:-1].tolist() == as_i64(want).tolist() and int(masks[-1]) == -7 and int(pos[-1]) == -7
        first = [s for s, n in zip(starts, nodes) for _ in range(n)]
        assert pos[:-1].tolist() == [f + bin(m).count("1") - 1 for f, m in zip(first, want)]
    B.twkv_cache_destroy(h)


def test_tree_map_roots_and_refusals(B):
    h, pool = map_cache(B)
    pos, masks = i32([10, 0, 0, 0]), torch.zeros(4, dtype=torch.int64, device="cuda")
    B.twkv_tree_map(h, i32([0, 4]), i32([-1, -1, 1, 0]), pos, masks)                # two roots
    assert B.twkv_cache_status(h) == B.TWKV_OK and masks.tolist() == [1, 2, 6, 9] and pos.tolist() == [10, 10, 11, 11]
    for bad in ([0, 0, 1, 2], [-1, 1, 0, 0], [-1, 0, 3, 0], [-2, 0, 0, 0], [-1, 0, 0, 9]):
        pos, masks = i32([10, 1, 2, 3, 50, 51]), torch.full((6,), 5, dtype=torch.int64, device="cuda")
        B.twkv_tree_map(h, i32([0, 4, 6]), i32(bad + [-1, 0]), pos, masks)
        assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG, bad
        assert masks.tolist() == [0] * 4 + [1, 3] and pos.tolist() == [10, 1, 2, 3, 50, 51]
    for off in ([0, 3, 2], [-1, 2, 4], [0, 2, 7], [0, 5, 6]):
        pos, masks = i32([10, 1, 2, 3, 4, 5]), torch.full((6,), 5, dtype=torch.int64, device="cuda")
        B.twkv_tree_map(h, i32(off), i32([-1, 0] * 3), pos, masks, max_nodes=4)
        assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG, off
    B.twkv_cache_destroy(h)


def plain_accept(parents, draft, target):
    if not parents:
        return [], -1
    cur, path = 0, [0]
    while True:
        kids = [j for j in range(cur + 1, len(parents)) if parents[j] == cur and draft[j] == target[cur]]
        if not kids:
            return path, target[cur]
        cur = kids[0]
        path.append(cur)


@pytest.mark.parametrize("nodes,words", [([1], 1), ([64], 1), ([64], 2), ([0, 5, 0, 64, 1], 2), ([33, 8, 63] * 21, 2), ([7, 0, 64, 31] * 300, 3)])
def test_tree_accept(B, nodes, words):
    h, pool = map_cache(B, max_seqs=max(64, len(nodes)))
    g = gen(words * 100 + len(nodes))
    parents = [random_parents(g, n) if n else [] for n in nodes]
    n = sum(nodes)
    offsets = [0] + np.cumsum(nodes).tolist()
    for chain in (False, True):
        if chain:
            parents = [list(range(-1, k - 1)) for k in nodes]
        draft, target = torch.randint(0, words, (2, n), generator=g).tolist()       # few words: many agree, and children tie
        acc, rows, nxt = i32([-9] * len(nodes)), i32([-9] * n), i32([-9] * len(nodes))
        B.twkv_tree_accept(h, i32(offsets), i32([p for ps in parents for p in ps]), i32(draft), i32(target), acc, rows, nxt)
        assert B.twkv_cache_status(h) == B.TWKV_OK
        want = [plain_accept(p, draft[o:o + len(p)], target[o:o + len(p)]) for p, o in zip(parents, offsets)]
        kept = [o + j for (path, _), o in zip(want, offsets) for j in path]
        assert acc.tolist() == [len(p) for p, _ in want] and nxt.tolist() == [t for _, t in want]
        assert rows.tolist() == kept + [-9] * (n - len(kept))
    B.twkv_cache_destroy(h)


def test_tree_accept_takes_broken_trees(B):
    # parents that are no earlier nodes are never walked to; offsets out of range keep nothing
    h, pool = map_cache(B)
    acc, rows, nxt = i32([5, 5]), i32([5] * 5), i32([5, 5])
    B.twkv_tree_accept(h, i32([0, 3, 5]), i32([0, 0, 2, 1, 0]), i32([4, 4, 4, 4, 4]), i32([4] * 5), acc, rows, nxt)
    assert B.twkv_cache_status(h) == B.TWKV_OK and acc.tolist() == [2, 2] and rows.tolist() == [0, 1, 3, 4, 5] and nxt.tolist() == [4, 4]
    B.twkv_tree_accept(h, i32([0, 3, 9]), i32([-1, 0, 1, -1, 0]), i32([4] * 5), i32([4] * 5), acc, rows, nxt)
    assert B.twkv_cache_status(h) == B.TWKV_ERR_INVALID_ARG and acc.tolist() == [3, 0] and nxt.tolist() == [4, -1]
    B.twkv_cache_destroy(h)


# ------------------------------------------------------------------------------------------ together
def test_a_step_of_speculative_decoding(B):
    """Slots, map, attention, verification, storing the kept rows; then a decode step sees exactly the kept path."""
    b = Batch(201, [130, 40, 7], [9, 24, 5], max_tokens=300, max_seqs=5)
    h = b.cache(B)
    a = b.args()
    n = sum(b.nodes)
    off, sid, pos = i32([0] * 4), i32([0] * n), i32([0] * n)
    B.twkv_slot_map(h, 0, a["req_seqs"], i32(b.nodes), off, sid, pos)
    masks = torch.zeros(n, dtype=torch.int64, device="cuda")
    parents = i32([p for ps in b.parents for p in ps])
    B.twkv_tree_map(h, off, parents, pos, masks, max_nodes=24)
    assert torch.equal(pos, a["positions"]) and torch.equal(masks, a["masks"]) and torch.equal(off, a["offsets"])
    a["positions"], a["masks"], a["offsets"] = pos, masks, off
    out, _ = run(B, h, b, a)
    want, top = b.want()
    close(out, want, top, torch.float32)
    # the chosen tokens follow one path of every tree
    draft = torch.arange(100, 100 + n, dtype=torch.int32)
    target = torch.full((n,), -3, dtype=torch.int32)
    paths = []
    for i in range(3):
        leaf = b.nodes[i] - 1
        path = [j for j in range(b.nodes[i]) if b.masks[i][leaf] >> j & 1]
        paths.append(path)
        for u, w in zip(path, path[1:]):
            target[b.offsets[i] + u] = draft[b.offsets[i] + w]
        target[b.offsets[i] + leaf] = 77 + i
    acc, rows, nxt = i32([0] * 3), i32([0] * n), i32([0] * 3)
    B.twkv_tree_accept(h, off, parents, draft.cuda(), target.cuda(), acc, rows, nxt, max_nodes=24)
    assert acc.tolist() == [len(p) for p in paths] and nxt.tolist() == [77, 78, 79]
    kept = int(acc.sum())
    rows = rows[:kept]
    assert rows.tolist() == [b.offsets[i] + j for i in range(3) for j in paths[i]]
    off2, sid2, pos2 = i32([0] * 4), i32([0] * kept), i32([0] * kept)
    B.twkv_slot_map(h, 0, a["req_seqs"], acc, off2, sid2, pos2)
    assert torch.equal(pos2, pos[rows.long()]) and torch.equal(sid2, sid[rows.long()])
    at = rows.long()
    B.twkv_compress(h, 0, a["K"][at], a["V"][at], sid2, pos2, None, a["levels"][at].contiguous(), B.TWKV_GATE_FORCED)
    leaves = torch.tensor([b.offsets[i + 1] - 1 for i in range(3)], device="cuda")
    step = torch.empty(3, 32, 128, device="cuda")
    B.twkv_decode_attn(h, 0, a["q"][leaves].contiguous(), a["req_seqs"], step)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    close(step, want[leaves.cpu()], top, torch.float32)
    assert B.twkv_cache_check(h) == (B.TWKV_OK, 0)
    B.twkv_cache_destroy(h)
