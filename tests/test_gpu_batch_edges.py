"""Operators of include/spec_batch.h at the edges of what the header allows; tolerances as in test_gpu_batch.py unless stated."""
import numpy as np
import pytest
import torch

import paper_2504_00030_amd as pk
from test_gpu_batch import BF16, F32, Attn, _int, _stream

pytestmark = pytest.mark.gpu


# ---- attention: a prefix alone -------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [40, 128, 256])
@pytest.mark.parametrize("rows", [[3], [1, 0, 19], [40], [70], [1] * 140])  # 16, 32, 64, 128 and 256 columns a workgroup in bf16
def test_attention_of_a_prefix_alone(rows, hd, dtype):
    """Tables without pages: nothing to go through, a single part, several."""
    for prefix in (0, 100, 1000):
        a = Attn(hd + prefix, rows, [0] * len(rows), prefix, 2, 2, hd, 16, dtype, spare=0, extra_rows=1)
        assert a.table.shape[1] == 0
        got = a.check()
        assert (got[-1] == 3.0).all() and (prefix > 0 or not got[:-1].any())


def test_attention_of_a_prefix_alone_in_more_than_2_to_the_20_workgroups():
    """A grid beyond 2^20 workgroups ends in whole rows of them: those past the last one leave every row and what lies behind the
    workspace alone."""
    R, nq, hd, prefix, page = 524800, 32, 8, 64, 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn((R, nq, hd), generator=gen, device="cuda")
    k, v = (torch.randn((2, nq, page, hd), generator=gen, device="cuda") for _ in range(2))
    out = torch.full_like(q, 3.0)
    n = pk.k_attn_shared_workspace(R, 1, nq, nq, hd, F32, prefix, 0)
    assert R * nq // 16 > 1 << 20 and n > 0
    hold = torch.full((n + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    pk.k_attn_shared(q, k, v, _int([0, R]), torch.zeros((1, 0), dtype=torch.int32, device="cuda"), _int([0]), out, hold[:n], prefix_table=_int([1]),
                     prefix_len=prefix, stream=_stream())
    torch.cuda.synchronize()
    assert (hold[n:] == 0xff).all()
    kk, vv = k[1].double(), v[1].double()
    for r in range(0, R, 32768):
        x = q[r: r + 32768].double().transpose(0, 1).contiguous()
        s = torch.matmul(x, kk.transpose(1, 2).contiguous()) * hd ** -0.5
        size = torch.matmul(x.abs(), kk.abs().transpose(1, 2).contiguous()).amax(dim=2, keepdim=True) * hd ** -0.5
        w = torch.softmax(s, dim=2)
        want, mag = torch.matmul(w, vv), torch.matmul(w, vv.abs())
        rel = 2 * ((hd + 4) * size + 1) * 2.0 ** -23 + (4 * prefix + 16) * 2.0 ** -23
        err = (out[r: r + 32768].double().transpose(0, 1) - want).abs()
        assert (err <= rel * mag + 2.0 ** -24 * want.abs()).all(), f"rows from {r}: off by {err.max():.3g}"
