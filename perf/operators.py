"""Speculative decoding over the compressed cache, as cases that can be timed and compared.

Operators (a serving step calls them in this order):
  slots    request lengths -> first row of every request, sequence id and position of every row
  map      parents of drafted trees -> positions and ancestor masks of the nodes
  tree     attention of the drafted nodes over their sequence's cached tokens and their own ancestors
  accept   drafted and chosen tokens -> the path every request keeps, and its next token

`own` false computes them in elementary torch operations; true calls the library.
"""
import math

import torch

own = False

HEAD_DIM = 128
ROPE_BASE = 500000.0
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
LEVELS = (1.0, 0.5, 0.25, 0.125)              # of d_kv
VOCAB = 128256


def listed():
    return [
        # a decode batch: one new token per request, the map every step starts with
        dict(name="slots_64x1", op="slots", reqs=64, most=1),
        # prompts of many lengths admitted together, some requests without new tokens
        dict(name="slots_256x1024", op="slots", reqs=256, most=1024),
        # one small tree
        dict(name="map_1x8", op="map", reqs=1, most=8, shape="tree", ragged=False),
        # a full batch of the largest trees
        dict(name="map_64x64", op="map", reqs=64, most=64, shape="tree", ragged=True),
        # smallest call: one short sequence, one query head per KV head
        dict(name="tree_1x1024_8", op="tree", reqs=1, ctx=1024, ragged=False, most=8, shape="tree", hq=8, hkv=8, dtype="f16", out="f16", ranks="uniform"),
        # a small batch with chains of four drafted tokens behind the current one
        dict(name="chain_4x4096_5", op="tree", reqs=4, ctx=4096, ragged=True, most=5, shape="chain", hq=32, hkv=8, dtype="bf16", out="bf16", ranks="spread"),
        # short ragged sequences, ragged trees of odd sizes, any rank
        dict(name="tree_37x700_13_ragged", op="tree", reqs=37, ctx=700, ragged=True, most=13, shape="tree", hq=16, hkv=4, dtype="bf16", out="f32", ranks="any"),
        # high-batch serving: 64 sequences of 8192 tokens, small trees
        dict(name="tree_64x8192_8", op="tree", reqs=64, ctx=8192, ragged=False, most=8, shape="tree", hq=32, hkv=8, dtype="f16", out="f16", ranks="skewed"),
        # the benchmark's cache: 16 sequences of 32768 tokens, trees of 16 nodes
        dict(name="tree_16x32768_16", op="tree", reqs=16, ctx=32768, ragged=False, most=16, shape="tree", hq=32, hkv=8, dtype="f16", out="f16", ranks="spread"),
        # one long context with 64 query heads and the largest tree
        dict(name="tree_1x131072_64", op="tree", reqs=1, ctx=131072, ragged=False, most=64, shape="tree", hq=64, hkv=8, dtype="bf16", out="bf16", ranks="sink_recent"),
        # verification of one small tree, and of a full batch
        dict(name="accept_1x8", op="accept", reqs=1, most=8, shape="tree", ragged=False),
        dict(name="accept_64x64", op="accept", reqs=64, most=64, shape="tree", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "tree", "slots", "map", "accept"])
    if op == "slots":
        reqs = _log_int(rng, 1, 256)
        return dict(op=op, reqs=reqs, most=_log_int(rng, 1, 1024))
    shape, ragged = rng.choice(["tree", "tree", "chain"]), rng.random() < 0.6
    if op != "tree":
        return dict(op=op, reqs=_log_int(rng, 1, 64), most=_log_int(rng, 1, 64), shape=shape, ragged=ragged)
    hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (8, 8), (16, 4), (8, 1), (12, 6)])
    reqs = _log_int(rng, 1, 64)
    ctx = _log_int(rng, 1, min(131072, 524288 // reqs))
    most = _log_int(rng, 1, 64)
    while most > 1 and reqs * ctx * most * hq > 131072 * 64 * 64:
        most -= 1
    return dict(op=op, reqs=reqs, ctx=ctx, ragged=ragged, most=most, shape=shape, hq=hq, hkv=hkv, dtype=rng.choice(["f16", "bf16"]),
                out=rng.choice(["f16", "bf16", "f32"]), ranks=rng.choice(["uniform", "skewed", "sink_recent", "spread", "any"]))


# ------------------------------------------------------------------------------------------ inputs
def _contexts(case):
    """Cached tokens per sequence: ctx each, or (ragged) spread between none and all of it."""
    n, t = case["reqs"], case["ctx"]
    return [t - (i * 7919 + 13) % (t + 1) if case["ragged"] else t for i in range(n)]


def _counts(case):
    """New rows per request: any number up to the most (slots), the most each, or (ragged) one to the most."""
    n, t = case["reqs"], case["most"]
    if case["op"] == "slots":
        return [1] * n if t == 1 else [(i * 7919 + 29) % (t + 1) for i in range(n)]
    return [t - (i * 31 + 7) % t if case["ragged"] else t for i in range(n)]


def _generator(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _ranks(g, n, d, mix):
    """[n, 2] ranks of K and V."""
    if mix == "any":                                             # every rank, K and V apart
        return torch.randint(1, d + 1, (n, 2), generator=g, device="cuda")
    if mix == "spread":                                          # around a quarter of d, K and V apart
        z = torch.randn(n, 2, generator=g, device="cuda")
        return (0.22 * d * torch.exp(0.5 * z)).round().clamp_(1, d).long()
    p = {"uniform": (0.25, 0.25, 0.25, 0.25), "skewed": (0.10, 0.20, 0.40, 0.30), "sink_recent": (0.05, 0.0, 0.475, 0.475)}[mix]
    at = torch.searchsorted(torch.tensor(p, device="cuda").cumsum(0), torch.rand(n, generator=g, device="cuda")).clamp_(max=3)
    return (torch.tensor(LEVELS, device="cuda")[at] * d).long().clamp_(min=1)[:, None].expand(n, 2).contiguous()


def _mean_rank(mix, d):
    if mix == "any":
        return (d + 1) / 2
    if mix == "spread":
        return 0.22 * d * math.exp(0.125)
    p = {"uniform": (0.25, 0.25, 0.25, 0.25), "skewed": (0.10, 0.20, 0.40, 0.30), "sink_recent": (0.05, 0.0, 0.475, 0.475)}[mix]
    return d * sum(a * b for a, b in zip(p, LEVELS))


def _states(g, n, d, dt, ranks):
    """[n, d] spectral states, energy falling along the components; behind a token's rank zeros (ranks None: everything)."""
    x = torch.empty(n, d, dtype=dt, device="cuda")
    size = (1.0 + torch.arange(d, device="cuda") / (d / 16)).rsqrt()
    size *= math.sqrt(d) / size.norm()
    for lo in range(0, n, 65536):
        hi = min(n, lo + 65536)
        part = torch.randn(hi - lo, d, generator=g, device="cuda") * size
        if ranks is not None:
            part.masked_fill_(torch.arange(d, device="cuda")[None] >= ranks[lo:hi, None], 0.0)
        x[lo:hi] = part.to(dt)
    return x


def _trees(case, g):
    """Rows of every request's tree: request of a row, its number inside the request, parents (-1: the root)."""
    counts = torch.tensor(_counts(case), device="cuda")
    offsets = torch.zeros(len(counts) + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    n = sum(_counts(case))
    req = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts, output_size=n)
    local = torch.arange(n, device="cuda") - offsets[req].long()
    if case["shape"] == "chain":
        parents = local - 1
    else:                                                        # a later node hangs below any earlier one
        parents = torch.minimum((torch.rand(n, generator=g, device="cuda") * local).long(), local - 1)
    return n, offsets, req, local, parents.int()


def _inputs(case, seed):
    """Everything the operator is given, without the library."""
    g = _generator(case, seed)
    n_req = case["reqs"]
    s = dict(case=case)
    if case["op"] == "slots":
        s["n"] = max(1, sum(_counts(case)))
        s["lens"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda")[torch.randperm(n_req, generator=g, device="cuda")].contiguous()
        s["req_seqs"] = torch.randperm(n_req, generator=g, device="cuda").int()
        s["starts"] = torch.randint(0, 8192, (n_req,), generator=g, device="cuda").int()
        return s
    s["n"], s["offsets"], req, local, s["parents"] = _trees(case, g)
    if case["op"] == "map":
        s["starts"] = torch.randint(0, 8192, (n_req,), generator=g, device="cuda").int()
        s["rows"] = s["starts"][req] + local.int()               # positions as the slot map leaves them
        return s
    if case["op"] == "accept":
        s["draft"] = torch.randint(0, VOCAB, (s["n"],), generator=g, device="cuda").int()
        # the chosen token is the first child's draft in seven cases of ten
        first = torch.full((s["n"],), s["n"], device="cuda")
        has = s["parents"] >= 0
        up = (s["offsets"][req] + s["parents"])[has].long()
        first.scatter_reduce_(0, up, torch.arange(s["n"], device="cuda")[has], "amin")
        agree = (torch.rand(s["n"], generator=g, device="cuda") < 0.7) & (first < s["n"])
        other = torch.randint(0, VOCAB, (s["n"],), generator=g, device="cuda").int()
        s["target"] = torch.where(agree, s["draft"][first.clamp(max=s["n"] - 1)], other)
        return s
    d, dt, n = case["hkv"] * HEAD_DIM, DTYPES[case["dtype"]], s["n"]
    ctx = _contexts(case)
    s["ctx"] = ctx
    s["uk"], s["uv"] = (torch.linalg.qr(torch.randn(d, d, generator=g, device="cuda"))[0].to(dt).contiguous() for _ in range(2))
    s["ranks"] = _ranks(g, sum(ctx), d, case["ranks"])
    s["xk"] = _states(g, sum(ctx), d, dt, s["ranks"][:, 0])       # what the cache holds
    s["xv"] = _states(g, sum(ctx), d, dt, s["ranks"][:, 1])
    s["levels"] = _ranks(g, n, d, case["ranks"])
    s["nk"], s["nv"] = _states(g, n, d, dt, None), _states(g, n, d, dt, None)
    s["q"] = torch.randn(n, case["hq"], HEAD_DIM, generator=g, device="cuda").to(dt)
    # depth of a node, and its ancestors and itself as the bits of a word
    depth, masks, up = torch.zeros_like(local), torch.ones_like(local) << local, s["parents"].long()
    for _ in range(case["most"]):
        there = up >= 0
        depth += there
        masks |= torch.where(there, torch.ones_like(up) << up.clamp(min=0), torch.zeros_like(up))
        up = torch.where(there, s["parents"].long()[(s["offsets"][req] + up.clamp(min=0)).long()], up)
    s["masks"] = masks
    s["positions"] = (torch.tensor(ctx, device="cuda")[req] + depth).int()
    s["req_seqs"] = torch.randperm(n_req, generator=g, device="cuda").int()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, n_req = case["op"], case["reqs"]
    new = lambda *shape, dt=torch.int32: torch.full(shape, -1, dtype=dt, device="cuda")  # noqa: E731
    if op == "slots":
        s["out"] = (new(n_req + 1), new(s["n"]), new(s["n"]))
    elif op == "map":
        s["out"] = (s.pop("rows"), new(s["n"], dt=torch.int64))
    elif op == "accept":
        s["out"] = (new(n_req), new(s["n"]), new(n_req))
    else:
        s["out"] = torch.zeros(s["n"], case["hq"], HEAD_DIM, dtype=DTYPES[case["out"]], device="cuda")
    if not own:
        return s
    from paper_2603_04411_b200 import binding as B
    tree = op == "tree"
    ctx = s["ctx"] if tree else [0]
    d = case["hkv"] * HEAD_DIM if tree else HEAD_DIM
    cfg = B.make_config(n_layers=1, n_q_heads=case["hq"] if tree else 1, n_kv_heads=d // HEAD_DIM, dtype=DTYPES[case["dtype"]] if tree else torch.float16,
                        out_dtype=DTYPES[case["out"]] if tree else torch.float16, max_seqs=n_req, max_tokens_per_seq=max(1, max(ctx)), rope_base=ROPE_BASE)
    payload = int((((s["ranks"] + 63) // 64) * 128).sum()) if tree else 0
    s["pool"] = torch.empty(B.twkv_cache_required_bytes(cfg, payload), dtype=torch.uint8, device="cuda")
    s["cache"] = B.twkv_cache_create(cfg, s["pool"])
    if tree:
        B.twkv_cache_set_layer_params(s["cache"], 0, s["uk"], s["uv"])
        n_tok = sum(ctx)
        if n_tok:
            lens = torch.tensor(ctx, device="cuda")
            req = torch.repeat_interleave(torch.arange(n_req, device="cuda"), lens, output_size=n_tok)
            pos = torch.arange(n_tok, device="cuda") - (lens.cumsum(0) - lens)[req]
            B.twkv_compress(s["cache"], 0, s["xk"], s["xv"], s["req_seqs"][req].contiguous(), pos.int(), None, s["ranks"].to(torch.int16).contiguous(),
                            B.TWKV_GATE_FORCED)
        s["levels"] = s["levels"].to(torch.int16).contiguous()
        s["ws"] = torch.empty(B.twkv_tree_required_bytes(s["cache"], n_req, case["most"]), dtype=torch.uint8, device="cuda")
        if B.twkv_cache_status(s["cache"]) != B.TWKV_OK:
            raise RuntimeError("the cache of the case could not be filled")
        for k in ("xk", "xv", "ranks"):
            s.pop(k)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_slots(s):
    offsets, seq_ids, positions = s["out"]
    ends = s["lens"].cumsum(0)
    offsets[0] = 0
    offsets[1:] = ends
    at = torch.arange(s["n"], device="cuda")
    req = (at[:, None] >= ends[None]).sum(1)
    there, req = req < len(ends), req.clamp(max=len(ends) - 1)
    seq_ids.copy_(torch.where(there, s["req_seqs"][req], seq_ids))
    positions.copy_(torch.where(there, s["starts"][req] + (at - offsets[req]).int(), positions))
    return offsets, seq_ids, positions


def _row_requests(s):
    at = torch.arange(s["n"], device="cuda")
    return (at[:, None] >= s["offsets"][None, 1:]).sum(1)


def _plain_map(s):
    positions, masks = s["out"]
    req = _row_requests(s)
    first = s["offsets"][req].long()
    up = torch.arange(s["n"], device="cuda") - first
    bits = torch.zeros_like(up)
    depth = torch.full_like(up, -1)
    for _ in range(s["case"]["most"]):
        there = up >= 0
        depth += there
        bits |= torch.where(there, torch.ones_like(up) << up.clamp(min=0), torch.zeros_like(up))
        up = torch.where(there, s["parents"].long()[first + up.clamp(min=0)], up)
    masks.copy_(bits)
    positions.copy_(positions[first] + depth.int())
    return positions, masks


def _plain_accept(s):
    n_accepted, rows, next_tokens = s["out"]
    n_req, most, n = s["case"]["reqs"], s["case"]["most"], s["n"]
    first, last = s["offsets"][:-1].long(), s["offsets"][1:].long()
    at = first[:, None] + torch.arange(most, device="cuda")[None]                 # [request, node] -> row
    there, at = at < last[:, None], at.clamp(max=n - 1)
    parents = torch.where(there, s["parents"][at], -2)
    draft = s["draft"][at]
    cur, live = torch.zeros(n_req, dtype=torch.long, device="cuda"), last > first
    count, path = torch.zeros_like(cur), torch.zeros(n_req, most, dtype=torch.long, device="cuda")
    want = torch.full_like(next_tokens, -1)
    for step in range(most):
        path[:, step] = cur
        count += live
        want = torch.where(live, s["target"][(first + cur).clamp(max=n - 1)], want)
        hit = (parents == cur[:, None]) & (draft == want[:, None])
        live = live & hit.any(1)
        cur = torch.where(live, hit.int().argmax(1), cur)
    n_accepted.copy_(count)
    next_tokens.copy_(want)
    ends = count.cumsum(0)
    k = torch.arange(n, device="cuda")
    req = (k[:, None] >= ends[None]).sum(1)
    kept, req = req < n_req, req.clamp(max=n_req - 1)
    step = (k - (ends - count)[req]).clamp(min=0, max=most - 1)
    rows.copy_(torch.where(kept, (first[req] + path[req, step]).int(), rows))
    return n_accepted, rows, next_tokens


def _plain_tree(s):
    case = s["case"]
    hq, hkv, most = case["hq"], case["hkv"], case["most"]
    rep, d = hq // hkv, hkv * HEAD_DIM
    uk, uv = s["uk"].float(), s["uv"].float()
    freq = ROPE_BASE ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    comp = torch.arange(d, device="cuda")
    lo_tok = lo = 0
    for n_tok, n in zip(s["ctx"], _counts(case)):
        rows = slice(lo, lo + n)
        keep = comp[None, None] < s["levels"][rows].T[:, :, None]
        xk = torch.cat([s["xk"][lo_tok:lo_tok + n_tok].float(), torch.where(keep[0], s["nk"][rows].float(), 0.0)])
        xv = torch.cat([s["xv"][lo_tok:lo_tok + n_tok].float(), torch.where(keep[1], s["nv"][rows].float(), 0.0)])
        pos = torch.cat([torch.arange(n_tok, device="cuda"), s["positions"][rows]])
        angle = pos[:, None].double() * freq
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        k = (xk @ uk).view(-1, hkv, HEAD_DIM)
        k = torch.cat([k[..., :64] * cos - k[..., 64:] * sin, k[..., 64:] * cos + k[..., :64] * sin], -1)
        v = (xv @ uv).view(-1, hkv, HEAD_DIM)
        q = s["q"][rows].float().view(n, hkv, rep, HEAD_DIM).permute(1, 0, 2, 3).reshape(hkv, n * rep, HEAD_DIM)
        sc = (q @ k.permute(1, 2, 0)).view(hkv, n, rep, -1) * HEAD_DIM ** -0.5
        sees = (s["masks"][rows][:, None] >> torch.arange(n, device="cuda")[None]) & 1 == 1
        sc[..., n_tok:].masked_fill_(~sees[None, :, None], float("-inf"))
        sc = torch.exp(sc - sc.amax(-1, keepdim=True))
        p = (sc / sc.sum(-1, keepdim=True)).view(hkv, n * rep, -1)
        o = (p @ v.permute(1, 0, 2)).view(hkv, n, rep, HEAD_DIM).permute(1, 0, 2, 3).reshape(n, hq, HEAD_DIM)
        s["out"][rows] = o.to(s["out"].dtype)
        lo_tok, lo = lo_tok + n_tok, lo + n
    return s["out"]


def run(s):
    case = s["case"]
    if not own:
        return {"slots": _plain_slots, "map": _plain_map, "tree": _plain_tree, "accept": _plain_accept}[case["op"]](s)
    from paper_2603_04411_b200 import binding as B
    if case["op"] == "slots":
        B.twkv_slot_map(s["cache"], 0, s["req_seqs"], s["lens"], *s["out"], starts=s["starts"])
    elif case["op"] == "map":
        B.twkv_tree_map(s["cache"], s["offsets"], s["parents"], *s["out"], max_nodes=case["most"])
    elif case["op"] == "accept":
        B.twkv_tree_accept(s["cache"], s["offsets"], s["parents"], s["draft"], s["target"], *s["out"], max_nodes=case["most"])
    else:
        B.twkv_tree_attn(s["cache"], 0, s["q"], s["nk"], s["nv"], s["levels"], s["req_seqs"], s["offsets"], s["positions"], s["masks"], s["out"], s["ws"],
                         max_nodes=case["most"])
    return s["out"]


def work(case):
    n_req, n = case["reqs"], sum(_counts(case))
    if case["op"] == "slots":
        return {"bytes": 16 * n_req + 4 + 8 * n, "flops": 2 * n}
    if case["op"] == "map":
        return {"bytes": 4 * n_req + 4 + 20 * n, "flops": 4 * n}
    if case["op"] == "accept":
        return {"bytes": 12 * n_req + 4 + 16 * n, "flops": 2 * n}
    hq, d = case["hq"], case["hkv"] * HEAD_DIM
    r = _mean_rank(case["ranks"], d)
    tokens = sum(_contexts(case)) + n
    pairs = sum(c * t for c, t in zip(_contexts(case), _counts(case))) * hq           # (cached token, query row)
    out_size = torch.finfo(DTYPES[case["out"]]).bits // 8
    nbytes = 4 * r * tokens + n * hq * HEAD_DIM * (2 + out_size) + 4 * d * d + 24 * n
    # values are rebuilt, or summed in the basis and projected once, whichever is less
    values = min(2 * r * d * tokens + 2 * HEAD_DIM * pairs, 2 * r * pairs + 2 * HEAD_DIM * d * n * hq)
    return {"bytes": int(nbytes), "flops": int(2 * r * d * tokens + 2 * HEAD_DIM * pairs + values)}


# ------------------------------------------------------------------------------------------ by definition, in 64 bits
def exact(case, seed):
    """Outputs of the attention from its definition in 64 bits, a node at a time; the maps are whole numbers."""
    if case["op"] != "tree":
        return None
    s = _inputs(case, seed)
    hq, hkv = case["hq"], case["hkv"]
    rep, d = hq // hkv, hkv * HEAD_DIM
    counts = _counts(case)
    out = torch.zeros(s["n"], hq, HEAD_DIM, dtype=torch.float64, device="cuda")
    uk, uv = s["uk"].double(), s["uv"].double()
    turn = torch.arange(64, dtype=torch.float64, device="cuda").mul(-math.log(ROPE_BASE) / 64).exp()

    def rotated(x, pos):                                         # [tokens, hkv, 64] complex keys
        k = (x @ uk).view(-1, hkv, 2, 64)
        a = pos.double()[:, None] * turn
        return torch.complex(k[:, :, 0], k[:, :, 1]) * torch.polar(torch.ones_like(a), a)[:, None]

    parents = s["parents"].tolist()
    lo_tok = lo = 0
    for n_tok, n in zip(s["ctx"], counts):
        lv = s["levels"][lo:lo + n]
        xk, xv = s["nk"][lo:lo + n].double(), s["nv"][lo:lo + n].double()
        for j, (rk, rv) in enumerate(lv.tolist()):
            xk[j, rk:] = 0.0
            xv[j, rv:] = 0.0
        node_k = rotated(xk, s["positions"][lo:lo + n])
        kc = rotated(s["xk"][lo_tok:lo_tok + n_tok].double(), torch.arange(n_tok, device="cuda"))
        vc = s["xv"][lo_tok:lo_tok + n_tok].double()
        for j in range(n):
            path, at = [], j
            while at >= 0:
                path.append(at)
                at = parents[lo + at]
            q = s["q"][lo + j].double().view(hkv, rep, 2, 64)
            qc = torch.complex(q[:, :, 0], q[:, :, 1])
            keys = torch.cat([kc, node_k[path]])
            sc = torch.einsum("hri,nhi->hrn", torch.view_as_real(qc).flatten(-2), torch.view_as_real(keys).flatten(-2)) / math.sqrt(HEAD_DIM)
            w = torch.softmax(sc, -1).view(hq, -1)
            mixed = w[:, :n_tok] @ vc + w[:, n_tok:] @ xv[path]   # [hq, d] in the basis
            out[lo + j] = torch.einsum("hrc,chd->hrd", mixed.view(hkv, rep, d), uv.view(d, hkv, HEAD_DIM)).reshape(hq, HEAD_DIM)
        lo_tok, lo = lo_tok + n_tok, lo + n
    return out
