"""What the binding of the tree operators refuses before it calls the library: index arrays of another width than the library reads."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2603_04411_b200 import build
    build.build()
    from paper_2603_04411_b200 import binding
    return binding


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


CALLS = {
    "twkv_slot_map": (dict(req_seqs=2, req_lens=2, offsets=3, seq_ids=4, positions=4, starts=2), {}),
    "twkv_tree_map": (dict(offsets=3, parents=4, positions=4), dict(masks=torch.zeros(4, dtype=torch.int64))),
    "twkv_tree_accept": (dict(offsets=3, parents=4, draft=4, target=4, n_accepted=2, rows=4, next_tokens=2), {}),
    "twkv_tree_attn": (dict(req_seqs=2, offsets=3, positions=4),
                       dict(q=torch.zeros(4, 1, 128).half(), K=torch.zeros(4, 128).half(), V=torch.zeros(4, 128).half(),
                            levels=torch.ones(4, 2, dtype=torch.int16), masks=torch.zeros(4, dtype=torch.int64), out=torch.zeros(4, 1, 128),
                            workspace=torch.zeros(256, dtype=torch.uint8))),
}


def call(B, name, args):
    f = getattr(B, name)
    return f(None, 0, **args) if name in ("twkv_slot_map", "twkv_tree_attn") else f(None, **args)


@pytest.mark.parametrize("name", CALLS)
def test_index_arrays_are_int32(B, name):
    ids, others = CALLS[name]
    for at in ids:
        for dt in (torch.int64, torch.int16, torch.float32):
            args = {k: i32(n) for k, n in ids.items()} | others
            args[at] = args[at].to(dt)
            with pytest.raises(TypeError, match=f"{name}.*{at}.*int32"):
                call(B, name, args)


def test_states_and_masks_have_their_widths(B):
    ids, others = CALLS["twkv_tree_attn"]
    for at, dt in [("q", torch.float32), ("K", torch.float32), ("V", torch.float32), ("levels", torch.int32), ("masks", torch.int32), ("masks", torch.float64)]:
        args = {k: i32(n) for k, n in ids.items()} | others
        args[at] = args[at].to(dt)
        with pytest.raises(TypeError, match=f"twkv_tree_attn.*{at}"):
            call(B, "twkv_tree_attn", args)
    args = {k: i32(n) for k, n in CALLS["twkv_tree_map"][0].items()} | dict(masks=i32(4))
    with pytest.raises(TypeError, match="twkv_tree_map.*masks"):
        call(B, "twkv_tree_map", args)
    args = {k: i32(n) for k, n in CALLS["twkv_slot_map"][0].items()}
    args["starts"] = i32(1)
    with pytest.raises(AssertionError):
        call(B, "twkv_slot_map", args)
