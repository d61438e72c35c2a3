"""How far the e4m3 product is off on the average, for every family of its kernels.

The bounds of test_gpu_ops.py hold for the worst sums there can be, and are therefore wide: for random rows they lie a hundred
times above what include/spec_ops.h states.  Here the error is averaged over a matrix of results and set against the
root of the sum of the squared terms of each result (rss), its size where the terms are independent and of either sign.

  sums   n = 128 + 3 + blocks roundings, each of at most 2^-23 of a partial sum, which stays below rss in the mean square;
         taken as independent they come to sqrt(n) 2^-23 rss.
  bf16   The e4m3 matrix instruction drops from each of eight neighbouring products what lies below 2^-13 of the power of two
         P of the largest: the other seven lose a remainder spread over 0 .. 2^-13 P, of the sign of the product, so 7 / 3
         (2^-13 P)^2 in the mean square.  P^2 is at most the group's sum of squares; over all groups sqrt(7 / 3) 2^-13 rss.
         The rounding to bf16 is taken out: a sum off by e crosses a border between two results a step apart with
         probability |e| / step, so the mean distance from the rounded exact result is the mean of |e|."""
import math

import numpy as np
import pytest
import torch

import ops_reference as ref
import paper_2504_00030_amd as pk
import test_gpu_ops as ops

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _exact(q, xs, w, ws):
    """(y, rss) in 64 bits on the GPU: plain products of blocks."""
    q, w = (torch.from_numpy(a).cuda() for a in (q, w))
    xs, ws = (torch.from_numpy(a).cuda().double() for a in (xs, ws))
    y = torch.zeros((q.shape[0], w.shape[0]), dtype=torch.float64, device="cuda")
    squares = torch.zeros_like(y)
    for b in range(xs.shape[0]):
        s = slice(b * ref.BLOCK, (b + 1) * ref.BLOCK)
        sc = xs[b][:, None] * ws[:, b].repeat_interleave(ref.BLOCK)[None, : w.shape[0]]
        wt = w[:, s].t().contiguous()
        y += (q[:, s] @ wt) * sc
        squares += (q[:, s] ** 2 @ wt ** 2) * sc ** 2
    return y, squares.sqrt()


# rows x columns x K: the stream with one and several tiles of rows, small tiles whole and in shares of K, large tiles
CASES = [(1, 8200, 4096, F32), (16, 2100, 8192, F32), (40, 4096, 4096, F32), (137, 4096, 11008, F32), (300, 6144, 2064, F32),
         (900, 8100, 2064, F32),
         (16, 8200, 4096, BF16), (40, 4096, 4096, BF16), (137, 4096, 11008, BF16), (192, 8192, 2048, BF16), (500, 6144, 2064, BF16),
         (1030, 12300, 2064, BF16)]


@pytest.mark.parametrize("R,N,K,y_dtype", CASES)
def test_mean_error_of_the_product(R, N, K, y_dtype):
    rng = np.random.default_rng(R + N + K)
    w, ws = ops._weights(rng, N, K)
    q, xs = ref.quantise(ops._activations(rng, R, K, F32).numpy())
    y = torch.zeros((R, N), dtype=y_dtype, device="cuda")
    work = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    pk.k_gemm_f8(ops._f8(w), torch.from_numpy(ws).cuda(), ops._f8(q), y, x_scale=torch.from_numpy(xs).cuda(), workspace=work,
                 stream=ops._stream())
    want, rss = _exact(q, xs, w, ws)
    off = (y.double() - want.to(y_dtype).double()).abs().mean().item() / rss.mean().item()
    bound = math.sqrt(128 + 3 + ref.blocks(K)) * 2.0 ** -23 + (math.sqrt(7 / 3) * 2.0 ** -13 if y_dtype == BF16 else 0.0)
    print(f"{R} x {N} x {K} {y_dtype}: {off:.2e}, bound {bound:.2e}")
    assert off <= bound
