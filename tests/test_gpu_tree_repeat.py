"""The same call gives the same bits: tree attention again on the same cache, and on a cache made anew from the same tokens."""
import pytest
import torch

from .test_gpu_tree import B, Batch, DT, run  # noqa: F401  (B: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ctx,nodes,hq,hkv,dt,out_dt", [
    # up to 18 splits to choose from, and tiles beyond the first range of panels in every warp that sums up the work of a range
    ([4096, 3000, 1777, 4000], [5, 4, 3, 5], 32, 8, "bf16", "bf16"),
    ([4096, 3000, 1777, 4000], [5, 4, 3, 5], 32, 8, "bf16", "f32"),
    ([9000], [4], 8, 8, "f16", "f32"),
    ([700, 90, 350, 512, 33, 699], [13, 2, 7, 1, 13, 9], 16, 4, "f16", "f16"),
])
def test_same_bits_on_the_same_and_on_a_new_cache(B, ctx, nodes, hq, hkv, dt, out_dt):  # noqa: F811
    first = None
    for _ in range(3):
        b = Batch(301, ctx, nodes, hq=hq, hkv=hkv, dt=DT[dt], out_dt=DT[out_dt], ranks="any")
        h = b.cache(B)
        args = b.args()
        for _ in range(12):
            out, _ = run(B, h, b, args)
            first = out.clone() if first is None else first
            assert torch.equal(out, first)
        assert B.twkv_cache_status(h) == B.TWKV_OK
        B.twkv_cache_destroy(h)
