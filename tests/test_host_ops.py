"""Refusals of the operators of include/spec_ops.h, before anything reaches a GPU."""
import pytest
import torch

import paper_2504_00030_amd as pk
from paper_2504_00030_amd import binding

E = binding.SPEC_EINVAL
P = 1 << 20  # stands for a device pointer: aligned, never read


def _said():
    return pk.load().spec_last_error(None).decode()


def _quant(x=P, dtype=0, ldx=128, R=4, K=128, q=P, scale=P):
    return pk.load().spec_k_quant_f8(x, dtype, ldx, R, K, q, scale, None)


def _gemm(w=P, ws=P, N=32, K=128, x=P, xt=3, ldx=128, xs=P, R=4, y=P, yt=0, ldy=32, work=None, nb=0):
    return pk.load().spec_k_gemm_f8(w, ws, N, K, x, xt, ldx, xs, R, y, yt, ldy, work, nb, None)


def _norm(q=P, ldq=256, nq=2, k=P, ldk=128, nkv=1, dtype=0, hd=128, R=4, gq=P, gk=P, eps=1e-5, c=P, s=P, n_pos=8, pos=P, qo=P,
          ldqo=256, ko=P, ldko=128, ot=0):
    return pk.load().spec_k_qk_norm_rope(q, ldq, nq, k, ldk, nkv, dtype, hd, R, gq, gk, eps, c, s, n_pos, pos, qo, ldqo, ko, ldko, ot, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(q=None), dict(scale=None), dict(dtype=2), dict(dtype=3), dict(dtype=-1), dict(R=-1),
                                 dict(K=0), dict(K=8), dict(K=120), dict(K=2**22 + 16, ldx=2**23), dict(R=2**30 + 1), dict(ldx=127), dict(ldx=-128), dict(x=P + 2), dict(q=P + 8),
                                 dict(scale=P + 2)])
def test_quantiser_refuses(bad):
    assert _quant(**bad) == E
    assert _said().startswith("quant_f8:")


@pytest.mark.parametrize("bad", [dict(w=None), dict(ws=None), dict(x=None), dict(xs=None), dict(y=None), dict(N=0), dict(N=-5), dict(K=0),
                                 dict(K=136), dict(K=2**22 + 16, ldx=2**22 + 16), dict(R=-1), dict(R=2**30 + 1), dict(N=2**30 + 1, ldy=2**31), dict(ldx=129), dict(ldx=100), dict(ldy=31), dict(xt=2), dict(xt=4), dict(yt=3),
                                 dict(yt=2), dict(w=P + 8), dict(x=P + 4), dict(xs=P + 1), dict(y=P + 2), dict(ws=P + 2), dict(nb=-1),
                                 dict(xt=0), dict(xt=0, xs=None), dict(xt=1, xs=None, work=P, nb=527), dict(xt=1, xs=None, work=P + 8, nb=4096),
                                 dict(xt=1, xs=None, work=None, nb=4096), dict(xt=0, xs=None, x=P + 2, work=P, nb=4096)])
def test_product_refuses(bad):
    assert _gemm(**bad) == E
    assert _said().startswith("gemm_f8:")


def test_workspace_sizes_and_refusals():
    f = pk.load().spec_k_gemm_f8_workspace
    assert f(128, 4, 3) == 0 and f(128, 4, 0) == 528 and f(1040, 3, 1) == 132 * 3 * 9
    assert f(14336, 1 << 20, 1) == 132 * (1 << 20) * 112  # beyond 32 bits
    for bad in [(0, 4, 0), (120, 4, 0), (2**22 + 16, 4, 0), (128, -1, 0), (128, 2**30 + 1, 0), (128, 4, 2), (128, 4, 7)]:
        assert f(*bad) == E
    with pytest.raises(pk.SpecError):
        pk.k_gemm_f8_workspace(120, 4, torch.float32)
    with pytest.raises(ValueError):
        pk.k_gemm_f8_workspace(128, 4, torch.float16)


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(gq=None), dict(gk=None), dict(c=None), dict(s=None), dict(pos=None),
                                 dict(qo=None), dict(ko=None), dict(dtype=2), dict(ot=3), dict(hd=0), dict(hd=127), dict(hd=514),
                                 dict(nq=0, nkv=0), dict(nq=-1), dict(nkv=-1), dict(R=-1), dict(n_pos=0), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(ldq=255), dict(ldk=127), dict(ldqo=255), dict(ldko=127), dict(q=P + 2),
                                 dict(ko=P + 1), dict(gq=P + 2), dict(pos=P + 2), dict(c=P + 1), dict(nq=2**31 - 1, nkv=2**31 - 1), dict(R=2**30 + 1), dict(R=2**30, nq=2, nkv=1)])
def test_norm_refuses(bad):
    assert _norm(**bad) == E
    assert _said().startswith("qk_norm_rope:")


def test_calls_without_rows_do_nothing():
    assert _quant(R=0, x=None, q=None, scale=None) == 0
    assert _gemm(R=0, x=None, xs=None, y=None) == 0
    assert _norm(R=0, q=None, k=None, qo=None, ko=None, pos=None) == 0


def test_wrappers_refuse_tensors_that_do_not_fit():
    f8 = torch.float8_e4m3fn
    w, ws, x = torch.zeros((32, 128), dtype=f8), torch.zeros((1, 1)), torch.zeros((4, 128))
    y = torch.zeros((4, 32))
    for bad in [dict(w=w.float()), dict(ws=torch.zeros((1, 2))), dict(x=torch.zeros((4, 144))), dict(y=torch.zeros((3, 32))),
                dict(y=torch.zeros((4, 64))[:, ::2]), dict(x=x.half())]:
        a = dict(w=w, ws=ws, x=x, y=y) | bad
        with pytest.raises(ValueError):
            pk.k_gemm_f8(a["w"], a["ws"], a["x"], a["y"])
    with pytest.raises(ValueError):  # host tensors
        pk.k_gemm_f8(w, ws, x, y)
    with pytest.raises(ValueError):
        pk.k_quant_f8(x, torch.zeros((4, 128), dtype=f8), torch.zeros((4, 1)))
    with pytest.raises(ValueError):
        pk.k_quant_f8(x, torch.zeros((4, 128), dtype=f8), torch.zeros((1, 4)))
    h, g, c = torch.zeros((4, 2, 64)), torch.zeros(64), torch.zeros((8, 32))
    pos = torch.zeros(4, dtype=torch.int32)
    for bad in [dict(g=torch.zeros(32)), dict(c=torch.zeros((8, 64))), dict(pos=pos.long()), dict(o=torch.zeros((4, 2, 32))),
                dict(h=torch.zeros((4, 64, 2)).transpose(1, 2)), dict(o=torch.zeros((4, 2, 64), dtype=torch.bfloat16), o2=h), dict()]:
        a = dict(h=h, g=g, c=c, pos=pos, o=h) | bad
        with pytest.raises(ValueError):
            pk.k_qk_norm_rope(a["h"], a["h"], a["g"], a["g"], a["c"], a["c"], a["pos"], a["o"], a.get("o2", a["o"]))


def test_wrappers_refuse_sizes_beyond_32_bits():
    """Sizes that a 32-bit argument would cut to a small one (tensors without memory)."""
    new = lambda shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="meta")
    f8, long = torch.float8_e4m3fn, 2**32 + 16
    with pytest.raises(ValueError, match="beyond"):
        pk.k_quant_f8(new((long, 16)), new((long, 16), f8), new((1, long)))
    with pytest.raises(ValueError, match="beyond"):
        pk.k_gemm_f8_workspace(128, long, torch.float32)
    for R, N, K in [(long, 32, 16), (4, long, 16), (4, 32, long)]:
        with pytest.raises(ValueError, match="beyond"):
            pk.k_gemm_f8(new((N, K), f8), new(((N + 127) // 128, (K + 127) // 128)), new((R, K)), new((R, N)))
    for R, n_pos in [(long, 8), (4, long)]:
        h, c = new((R, 1, 2)), new((n_pos, 1))
        with pytest.raises(ValueError, match="beyond"):
            pk.k_qk_norm_rope(h, h, new(2), new(2), c, c, new(R, torch.int32), h, h)
