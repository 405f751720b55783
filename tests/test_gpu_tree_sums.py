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


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_equal_weights_lose_nothing_in_the_sums_of_values(B, dt):  # noqa: F811
    """Queries of zeros: all weights are one power of two, products are no longer than the values and their sums of 1250 tokens (2^11 of 2^11 steps, fp16) all but
    exact.  What is left is the last product: 16 steps, at most three instructions each, in two sums: 24 x 2.15e-8 = 5.2e-7, and three roundings to nearest."""
    b = Batch(402, [1250] * 40, [16] * 40, hq=16, hkv=2, dt=dt, ranks=200)
    b.q = torch.zeros_like(b.q)
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, _ = b.want()
    err, bias = error_and_bias(out, want)
    assert abs(bias) <= 5.2e-7 and err <= 5.2e-7 + 3 * 2.0 ** -24
    B.twkv_cache_destroy(h)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_a_softmax_that_one_token_decides_loses_nothing(B, dt):  # noqa: F811
    """One token of 1250 has a key, and every query lies along it: the others' weights are below e^-50.  Outputs are that token's value; its sixteen tokens
    may count (twice 1.75e-8), and the last product as above."""
    n, at = 40, 777
    b = Batch(403, [1250] * n, [4] * n, hq=4, hkv=2, dt=dt, ranks=200)
    b.nk = torch.zeros_like(b.nk)
    keys = torch.zeros_like(b.xk)
    for i in range(n):
        keys[i * 1250 + at] = b.xk[i * 1250 + at]
        k = b.rotate(b.rebuilt(keys[i * 1250 + at][None], torch.tensor([200]), b.uk), [at])[0]              # [KV heads, 128]
        q = k * (60 / 128 ** -0.5 / (k * k).sum(-1, keepdim=True))                                          # scores of 60
        for j in range(4):
            b.q[b.offsets[i] + j] = q.repeat_interleave(2, 0).to(dt)
    b.xk = keys
    h = b.cache(B, shuffle=False)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, _ = b.want()
    err, bias = error_and_bias(out, want)
    assert abs(bias) <= 5.6e-7 and err <= 5.6e-7 + 3 * 2.0 ** -24
    B.twkv_cache_destroy(h)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ctx,nodes,hq,hkv,rank", [
    ([700] * 37, [13] * 37, 16, 4, "any"),
    ([1024] * 24, [8] * 24, 32, 8, 256),                      # full tiles, so that accumulators are emptied on the way
    ([4096] * 2, [5] * 2, 4, 2, 256),
    ([20000], [4], 4, 2, "any"),
])
def test_errors_are_those_of_fp32_sums(B, dt, ctx, nodes, hq, hkv, rank):  # noqa: F811
    """Relative error of the whole output, with the bound of test_fp32_outputs_are_as_good_as_fp32_sums: fp32 sums of n terms, each step rounded, wander by
    sqrt(n) 2^-24 / sqrt(3).  Twice what keys (d products, doubled by queries, scores and weights) and values (all tokens) come to."""
    b = Batch(404, ctx, nodes, hq=hq, hkv=hkv, dt=dt, ranks=rank)
    h = b.cache(B)
    out, _ = run(B, h, b)
    assert B.twkv_cache_status(h) == B.TWKV_OK
    want, _ = b.want()
    err, _ = error_and_bias(out, want)
    assert err <= 2 * (2 * b.d ** 0.5 + (max(ctx) + max(nodes)) ** 0.5) * 2.0 ** -24 / 3 ** 0.5
    B.twkv_cache_destroy(h)
