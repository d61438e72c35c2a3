"""Forms of the calls of include/spec_ops.h that the size lists of test_gpu_ops.py do not come to."""
import numpy as np
import pytest
import torch

import ops_reference as ref
import paper_2504_00030_amd as pk
import test_gpu_ops as ops

pytestmark = pytest.mark.gpu

F8, F32, BF16 = ops.F8, ops.F32, ops.BF16


@pytest.mark.parametrize("y_dtype", [F32, BF16])
@pytest.mark.parametrize("K", [384, 400, 512, 656, 1040])
def test_product_in_tiles_of_128_by_128(K, y_dtype):
    """512 tiles, which fp32 results take in two stages and bf16 results in three, over three to nine blocks of k: rounds of the
    loop over the stages, and every number of steps that can be left behind it."""
    ops.test_product_launch_shapes(900, 8100, K, y_dtype)


@pytest.mark.parametrize("y_dtype", [F32, BF16])
@pytest.mark.parametrize("x_kind", [F32, BF16])
@pytest.mark.parametrize("R,N,K", [(8, 2048, 2048), (8, 5000, 2000), (24, 5000, 2000), (40, 5000, 1024), (113, 3100, 672)])
def test_product_of_wide_rows_in_both_result_types(R, N, K, x_kind, y_dtype):
    """One and two groups of columns by one to four tiles of rows that the product quantises itself."""
    ops._gemm_case(np.random.default_rng(R + N), R, N, K, x_kind, y_dtype, ldy_extra=4)


@pytest.mark.parametrize("y_dtype", [F32, BF16])
@pytest.mark.parametrize("R,N,K", [(200, 700, 6016), (140, 2100, 6016)])
def test_product_with_workspaces_of_every_size(R, N, K, y_dtype):
    """Any workspace serves, and from 32 MiB beyond the quantised rows on the result stays the same to the bit."""
    rng = np.random.default_rng(R)
    w, ws = ops._weights(rng, N, K)
    x = ops._activations(rng, R, K, BF16)
    q, xs = ref.quantise(x.float().numpy())
    want, mag = ref.product(q, xs, w, ws)
    tol = ops._product_tol(mag, want, ref.blocks(K), y_dtype)
    need = pk.k_gemm_f8_workspace(K, R, BF16)
    wd, wsd, xd, last = ops._f8(w), torch.from_numpy(ws).cuda(), x.cuda(), None
    for extra in (0, 272, 1 << 20, 4 << 20, 16 << 20, 32 << 20, (32 << 20) + 16, 64 << 20):
        guard = torch.full((need + extra + 256,), 0x55, dtype=torch.uint8, device="cuda")
        y = torch.zeros((R, N), dtype=y_dtype, device="cuda")
        pk.k_gemm_f8(wd, wsd, xd, y, workspace=guard[: need + extra], stream=ops._stream())
        assert (np.abs(y.double().cpu().numpy() - want) <= tol).all(), f"{extra} bytes beyond the quantised rows"
        assert (guard[need + extra:] == 0x55).all(), "written behind the workspace"
        if extra >= 32 << 20:
            assert last is None or torch.equal(y, last)
            last = y


@pytest.mark.parametrize("t_in,t_out", [(F32, F32), (BF16, BF16)])
def test_norm_of_key_heads_alone(t_in, t_out):
    ops._norm_case(np.random.default_rng(6), 9, 0, 4, 64, t_in, t_out)


def test_norm_without_eps():
    """eps = 0: any size of a head whose squares fp32 holds comes out normed."""
    R, hd = 7, 96
    rng = np.random.default_rng(4)
    h = rng.standard_normal((R, 1, hd)) * 2.0 ** np.array([-45, -20, -3, 0, 8, 30, 55])[:, None, None]
    cos, sin = ops._tables(R, hd)
    g = np.ones(hd, dtype=np.float32)
    cu = lambda a: torch.from_numpy(a).cuda()
    q = cu(h.astype(np.float32))
    out = [torch.zeros_like(q), torch.zeros_like(q)]
    pk.k_qk_norm_rope(q, q, cu(g), cu(g), cu(cos), cu(sin), torch.arange(R, dtype=torch.int32, device="cuda"), *out, eps=0.0,
                      stream=ops._stream())
    want, mag = ref.norm_rope(q.double().cpu().numpy(), g.astype(np.float64), 0.0, cos.astype(np.float64), sin.astype(np.float64))
    for o in out:
        assert (np.abs(o.double().cpu().numpy() - want) <= (hd / 2 + 8) * 2.0 ** -23 * mag + 2.0 ** -24 * np.abs(want)).all()


@pytest.mark.parametrize("t_in,t_out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("shift,extra", [(1, 3), (2, 0), (4, 4), (8, 12)])
def test_norm_outputs_with_strides_and_odd_starts(shift, extra, hd, t_in, t_out):
    """Inputs and outputs that start `shift` elements into an allocation, rows `extra` elements apart, both sides alike or not;
    what lies between the rows stays."""
    rng = np.random.default_rng(hd + shift)
    R, nq, nkv, n_pos, eps = 13, 3, 2, 20, 1e-6
    cu = lambda a: torch.from_numpy(a).cuda()

    def rows(heads, dtype, shift, extra):
        ld = heads * hd + extra
        flat = torch.full((shift + R * ld,), 9.0, dtype=dtype, device="cuda")
        return flat, torch.as_strided(flat, (R, heads, hd), (ld, hd, 1), shift)

    cos, sin = ops._tables(n_pos, hd)
    pos = rng.integers(0, n_pos, R).astype(np.int32)
    g = [(1 + 0.3 * rng.standard_normal(hd)).astype(np.float32) for _ in range(2)]
    for o_shift, o_extra in ((shift, extra), (0, 0), (3, 1)):
        ins, outs = [], []
        for heads in (nq, nkv):
            _, v = rows(heads, t_in, shift, extra)
            v.copy_(cu(rng.standard_normal((R, heads, hd)).astype(np.float32)))
            ins.append(v)
            outs.append(rows(heads, t_out, o_shift, o_extra))
        pk.k_qk_norm_rope(ins[0], ins[1], cu(g[0]), cu(g[1]), cu(cos), cu(sin), cu(pos), outs[0][1], outs[1][1], eps=eps,
                          stream=ops._stream())
        for v, (flat, out), w in zip(ins, outs, g):
            want, mag = ref.norm_rope(v.double().cpu().numpy(), w.astype(np.float64), eps, cos[pos].astype(np.float64),
                                      sin[pos].astype(np.float64))
            tol = (hd / 2 + 8) * 2.0 ** -23 * mag + ops.HALF_STEP[t_out] * np.abs(want) + 1e-38
            assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
            out.fill_(9.0)
            assert (flat == 9.0).all(), "written between the rows"
