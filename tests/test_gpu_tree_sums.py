"""What the tensor core's sums lose, and what the kernels give back for it: fp32 outputs of tree attention whose sums lose much, little and nothing.

An instruction cuts the fp32 sum by nothing at least and one unit in the last place at most, and the kernels give back what is expected between the two.
Outputs are then off by at most what is given back, in either direction, if all of an instruction's cuts are the extreme: 1.75e-8 for each instruction that has
long products in the sums of values, 2.15e-8 in the last product, where fp32 outputs have two sums, each of half of the instructions.  `bias` is the part of
the error that lies along the outputs: a rounding of single values to nearest (2^-24) has next to none of it over a hundred thousand of them.
"""
import pytest
import torch

from .test_gpu_tree import B, Batch, run  # noqa: F401  (B: fixture)

pytestmark = pytest.mark.gpu


def error_and_bias(got, want):
    got = got.double().cpu()
    return float((got - want).norm() / want.norm()), float(((got - want) * want).sum() / (want * want).sum())


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rank", [64, 256])
def test_components_behind_the_ranks_lose_nothing(B, dt, rank):  # noqa: F811
    """1024 components, few of them stored, and so many nodes that one CTA multiplies all of a row's: an instruction whose components are zeros cuts nothing.
    A request's 60 tokens and 16 nodes are five boxes, ten long instructions (1.8e-7); rank 256 has 16 steps of the last product, of up to three instructions,
    in two sums (24, 5.2e-7): below 7e-7.  (With all 64 steps counted, 1.4e-6 and 2.1e-6 too large.)"""
    b = Batch(401, [60] * 48, [16] * 48, hq=32, hkv=8, dt=dt, ranks=rank)
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, _ = b.want()
    _, bias = error_and_bias(out, want)
    assert abs(bias) <= 7e-7
    B.twkv_cache_destroy(h)
