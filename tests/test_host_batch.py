"""Refusals of the operators of include/spec_batch.h, before anything reaches a GPU, and the sizes of their workspaces."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import batch_reference as ref
import paper_2504_00030_amd as pk
from paper_2504_00030_amd import binding, build

E = binding.SPEC_EINVAL
P = 1 << 20  # stands for a device pointer: aligned, never read
NAN, INF = float("nan"), float("inf")


def _said():
    return pk.load().spec_last_error(None).decode()


def _tables(rope=None, rot=64, n_pos=8, c=P, s=P, none=False, **how):
    a = dict(theta=10000.0, scaling=0, factor=4.0, low=1.0, high=4.0, context=8192.0, magnitude=0.0) | how
    r = binding.SpecRope(**a)
    return pk.load().spec_k_rope_tables(None if none else C.byref(r), rot, n_pos, c, s, None)


def _rope(q=P, ldq=256, nq=2, k=P, ldk=128, v=P, ldv=128, nkv=1, dtype=0, hd=128, R=4, c=P, s=P, n_pos=8, rot=64, inter=0, pos=P, slot=P,
          qo=P, ldqo=256, kp=P, vp=P, n_pages=4, page=16, ot=0):
    return pk.load().spec_k_rope_cache(q, ldq, nq, k, ldk, v, ldv, nkv, dtype, hd, R, c, s, n_pos, rot, inter, pos, slot, qo, ldqo, kp, vp,
                                       n_pages, page, ot, None)


def _attn(q=P, ldq=256, nq=4, nkv=2, hd=64, dtype=1, R=3, rows=P, n_seq=2, k=P, v=P, n_pages=8, page=16, pt=P, prefix=500, table=P, tp=20,
          own=P, scale=0.125, out=P, ldo=256, work=P, nb=1 << 30):
    return pk.load().spec_k_attn_shared(q, ldq, nq, nkv, hd, dtype, R, rows, n_seq, k, v, n_pages, page, pt, prefix, table, tp, own, scale, out,
                                        ldo, work, nb, None)


def _verify(p=P, ldp=100, q=P, ldq=100, dtype=0, V=100, start=P, n_seq=2, n_drafts=3, drafted=P, ua=P, un=P, A=P, y=P, work=P, nb=1 << 20):
    return pk.load().spec_k_verify(p, ldp, q, ldq, dtype, V, start, n_seq, n_drafts, drafted, ua, un, A, y, work, nb, None)


@pytest.mark.parametrize("bad", [dict(none=True), dict(c=None), dict(s=None), dict(c=P + 2), dict(s=P + 1), dict(rot=0), dict(rot=63), dict(rot=514),
                                 dict(n_pos=0), dict(n_pos=-1), dict(n_pos=2**28 + 1), dict(scaling=-1), dict(scaling=5), dict(theta=0.0), dict(theta=-1.0),
                                 dict(theta=NAN), dict(theta=INF), dict(scaling=1, factor=0.0), dict(scaling=2, factor=-1.0), dict(scaling=1, factor=NAN),
                                 dict(scaling=3, low=4.0), dict(scaling=3, low=-1.0), dict(scaling=3, high=INF), dict(scaling=3, context=0.0),
                                 dict(scaling=4, low=0.0), dict(scaling=4, theta=1.0), dict(scaling=4, context=NAN), dict(scaling=4, magnitude=-1.0),
                                 dict(scaling=4, magnitude=INF), dict(scaling=1, factor=1e-308, n_pos=2**28), dict(theta=5e-324, rot=512)])
def test_tables_refuse(bad):
    assert _tables(**bad) == E
    assert _said().startswith("rope_tables:")


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(c=None), dict(s=None), dict(pos=None), dict(slot=None), dict(qo=None),
                                 dict(kp=None), dict(vp=None), dict(dtype=2), dict(dtype=3), dict(ot=3), dict(hd=1, rot=2), dict(hd=513), dict(rot=0),
                                 dict(rot=65), dict(rot=130), dict(nq=0, nkv=0), dict(nq=-1), dict(nkv=-1), dict(nq=2**20, ldq=2**40, ldqo=2**40),
                                 dict(R=-1), dict(R=2**30), dict(n_pos=0), dict(ldq=255), dict(ldqo=255), dict(ldk=127), dict(ldv=127), dict(page=4),
                                 dict(page=24), dict(page=0), dict(page=2**21), dict(n_pages=0), dict(n_pages=2**27, page=16), dict(q=P + 2), dict(qo=P + 1),
                                 dict(k=P + 2), dict(v=P + 3), dict(slot=P + 2), dict(pos=P + 2), dict(kp=P + 8), dict(vp=P + 4), dict(c=P + 2)])
def test_rotation_refuses(bad):
    assert _rope(**bad) == E
    assert _said().startswith("rope_cache:")


@pytest.mark.parametrize("bad", [dict(q=None), dict(rows=None), dict(k=None), dict(v=None), dict(pt=None), dict(table=None), dict(own=None), dict(out=None),
                                 dict(work=None), dict(nb=100), dict(nb=-1), dict(dtype=2), dict(dtype=3), dict(nq=3), dict(nq=0), dict(nkv=0), dict(nkv=-2), dict(nq=2**17, R=1, ldq=2**24, ldo=2**24),
                                 dict(hd=4), dict(hd=60), dict(hd=264), dict(R=-1), dict(R=2**30), dict(n_seq=0), dict(n_seq=4097), dict(page=4), dict(page=48),
                                 dict(n_pages=0), dict(n_pages=2**27), dict(prefix=-1), dict(prefix=2**30), dict(tp=-1), dict(tp=2**26), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(scale=3e38), dict(ldq=255), dict(ldo=200), dict(q=P + 1), dict(out=P + 1), dict(k=P + 8),
                                 dict(v=P + 2), dict(rows=P + 2), dict(own=P + 1), dict(table=P + 2), dict(pt=P + 2), dict(work=P + 8)])
def test_attention_refuses(bad):
    assert _attn(**bad) == E
    assert _said().startswith("attn_shared:")


@pytest.mark.parametrize("bad", [dict(p=None), dict(start=None), dict(drafted=None), dict(ua=None), dict(un=None), dict(A=None), dict(y=None), dict(work=None),
                                 dict(nb=10), dict(nb=-1), dict(dtype=2), dict(dtype=3), dict(V=0), dict(V=2**24 + 1, ldp=2**25, ldq=2**25), dict(ldp=99),
                                 dict(ldq=99), dict(n_seq=-1), dict(n_seq=65536), dict(n_drafts=-1), dict(n_drafts=2**31 - 1), dict(p=P + 2), dict(q=P + 1),
                                 dict(start=P + 2), dict(drafted=P + 1), dict(ua=P + 2), dict(un=P + 2), dict(A=P + 2), dict(y=P + 1), dict(work=P + 8)])
def test_verification_refuses(bad):
    assert _verify(**bad) == E
    assert _said().startswith("verify:")


def test_calls_without_work_do_nothing():
    assert _rope(R=0, q=None, k=None, v=None, c=None, s=None, pos=None, slot=None, qo=None, kp=None, vp=None) == 0
    assert _attn(R=0, q=None, out=None, rows=None, own=None, k=None, v=None, pt=None, table=None, work=None, nb=0) == 0
    assert _verify(n_seq=0, n_drafts=0, p=None, q=None, start=None, drafted=None, ua=None, un=None, A=None, y=None, work=None, nb=0) == 0


def test_workspaces():
    f, g = pk.load().spec_k_attn_shared_workspace, pk.load().spec_k_verify_workspace
    assert f(0, 1, 4, 2, 64, 1, 0, 0) == 0 and f(5, 2, 4, 2, 64, 1, 0, 16) == 0
    assert f(9, 2, 4, 2, 64, 1, 4096, 4096) > 0
    assert f(2**20, 64, 32, 8, 128, 0, 4096, 4096) >= 2 * 2**20 * 32 * 130 * 4  # beyond 32 bits
    for bad in [(-1, 1, 4, 2, 64, 1, 0, 0), (1, 0, 4, 2, 64, 1, 0, 0), (1, 1, 4, 3, 64, 1, 0, 0), (1, 1, 4, 2, 65, 1, 0, 0), (1, 1, 4, 2, 64, 2, 0, 0),
                (1, 1, 4, 2, 64, 1, -1, 0), (1, 1, 4, 2, 64, 1, 0, -1), (1, 1, 4, 2, 64, 1, 2**30, 0), (2**30, 1, 4, 2, 64, 1, 0, 0)]:
        assert f(*bad) == E
    assert g(0, 100) == 0 and g(3, 512) == 3 * 20 and g(3, 513) == 3 * 36
    assert g(-1, 100) == E and g(65536, 100) == E and g(1, 0) == E and g(1, 2**24 + 1) == E
    with pytest.raises(pk.SpecError):
        pk.k_attn_shared_workspace(1, 1, 4, 3, 64, torch.bfloat16, 0, 0)
    with pytest.raises(ValueError):
        pk.k_attn_shared_workspace(1, 1, 4, 2, 64, torch.float16, 0, 0)
    with pytest.raises(ValueError, match="beyond"):
        pk.k_attn_shared_workspace(2**32 + 1, 1, 4, 2, 64, torch.bfloat16, 0, 0)
    with pytest.raises(ValueError, match="beyond"):
        pk.k_verify_workspace(2**32, 100)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_wrappers_refuse_tensors_that_do_not_fit():
    t = torch.zeros((8, 32))
    with pytest.raises(ValueError, match="scaling"):
        pk.k_rope_tables(t, t, scaling="other")
    for bad in [(t, t[:4]), (t, t.double()), (t.t(), t.t()), (t, t)]:  # (the last: host tensors)
        with pytest.raises(ValueError):
            pk.k_rope_tables(*bad)
    h, v, pages, pos = torch.zeros((4, 2, 64)), torch.zeros((4, 1, 64)), torch.zeros((3, 1, 16, 64)), _i32(4)
    base = dict(q=h, k=v, v=v, cos=t, sin=t, pos=pos, slot=pos, q_out=h, k_pages=pages, v_pages=pages)
    for bad in [dict(), dict(q=None), dict(q_out=None), dict(k=None), dict(slot=None), dict(v=None), dict(k_pages=None), dict(q=h[:3]), dict(v=h), dict(pos=pos.long()),
                dict(slot=_i32(5)), dict(cos=t.t()), dict(sin=t[:, :16]), dict(k_pages=torch.zeros((3, 2, 16, 64)), v_pages=torch.zeros((3, 2, 16, 64))),
                dict(v_pages=pages.bfloat16()), dict(q_out=h.bfloat16()), dict(q=h.transpose(1, 2)), dict(k=v.bfloat16(), v=v.bfloat16()), dict(q=h.half(), k=v.half(), v=v.half()),
                dict(q=h[0]), dict(k_pages=pages[0], v_pages=pages[0]), dict(q=None, q_out=None, k=None, v=None, slot=None, k_pages=None, v_pages=None)]:
        with pytest.raises(ValueError):
            pk.k_rope_cache(**(base | bad))
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    kv = torch.zeros((3, 1, 16, 64), dtype=torch.bfloat16)
    base = dict(q=q, k_pages=kv, v_pages=kv, row_start=_i32(3), table=_i32(2, 2), own_len=_i32(2), out=q, workspace=None, prefix_table=_i32(2), prefix_len=20)
    for bad in [dict(), dict(q=q[0]), dict(out=q.float()), dict(out=q[:3]), dict(k_pages=kv.float(), v_pages=kv.float()), dict(k_pages=kv[..., :32], v_pages=kv[..., :32]),
                dict(row_start=_i32(2)), dict(table=_i32(3, 2)), dict(table=_i32(2, 2).long()), dict(table=_i32(2, 4)[:, ::2]), dict(own_len=_i32(2).long()),
                dict(prefix_table=None), dict(prefix_table=_i32(1)), dict(prefix_table=_i32(2).float()), dict(prefix_table=_i32(4)[::2]), dict(v_pages=kv[:2])]:
        with pytest.raises(ValueError):
            pk.k_attn_shared(**(base | bad))
    p, d = torch.zeros((5, 100)), torch.zeros((3, 100))
    base = dict(p=p, q=d, draft_start=_i32(3), drafted=_i32(3), u_accept=torch.zeros(3), u_next=torch.zeros(2), n_accepted=_i32(2), next_token=_i32(2), workspace=None)
    for bad in [dict(), dict(p=p[:4]), dict(p=p.t()), dict(q=d[:2]), dict(q=d.bfloat16()), dict(draft_start=_i32(2)), dict(drafted=_i32(3).long()), dict(drafted=_i32(4)),
                dict(u_accept=torch.zeros(2)), dict(u_next=torch.zeros(2).double()), dict(n_accepted=_i32(3)), dict(next_token=_i32(2).long()), dict(u_accept=torch.zeros(6)[::2])]:
        with pytest.raises(ValueError):
            pk.k_verify(**(base | bad))


def test_wrappers_refuse_sizes_beyond_32_bits():
    """Sizes that a 32-bit argument would cut to a small one (tensors without memory)."""
    new = lambda shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="meta")
    long, i32 = 2**32 + 16, torch.int32
    with pytest.raises(ValueError, match="beyond"):
        pk.k_rope_tables(new((long, 2)), new((long, 2)))
    h = new((long, 1, 8))
    with pytest.raises(ValueError, match="beyond"):
        pk.k_rope_cache(h, None, None, new((8, 4)), new((8, 4)), new(long, i32), None, h, None, None)
    q, pages = new((4, 1, 8)), new((long, 1, 8, 8))
    with pytest.raises(ValueError, match="beyond"):
        pk.k_attn_shared(q, pages, pages, new(2, i32), new((1, 1), i32), new(1, i32), q, None)
    with pytest.raises(ValueError, match="beyond"):
        pk.k_verify(new((1, long)), None, new(2, i32), new(0, i32), new(0), new(1), new(1, i32), new(1, i32), None)


# ---- the reference itself, against cases worked out by hand --------------------------------------------------------
def test_reference_frequencies():
    f, size = ref.frequencies(4, 100.0)
    assert np.allclose(f, [1.0, 0.1], rtol=1e-15) and size == 1.0
    f, _ = ref.frequencies(4, 100.0, scaling="linear", factor=4.0)
    assert np.allclose(f, [0.25, 0.025], rtol=1e-15)
    f, _ = ref.frequencies(4, 100.0, scaling="base", factor=4.0)  # slowest pair: 1 / sqrt(100 * 16) = 0.1 / 4
    assert np.allclose(f, [1.0, 0.025], rtol=1e-14)
    # turns over 200 pi positions: 100 and 10; between 4 and 16 turns the second keeps half of itself
    f, _ = ref.frequencies(4, 100.0, scaling="bands", factor=4.0, low=4.0, high=16.0, context=200 * np.pi)
    assert np.allclose(f, [1.0, 0.1 * (0.5 + 0.5 / 4)], rtol=1e-14)
    # pairs that turn 10 and 1 times over 200 pi positions: 1 and 2; pair 1 is kept, pair 2 (and beyond) interpolated
    f, size = ref.frequencies(8, 10000.0, scaling="ramp", factor=4.0, low=1.0, high=10.0, context=200 * np.pi + 1e-6)
    assert np.allclose(f[:2], [1.0, 0.1], rtol=1e-12) and size == 0.1 * np.log(4.0) + 1.0


def test_reference_attention_and_verification():
    k = np.zeros((1, 1, 8, 8))
    v = np.arange(64, dtype=float).reshape(1, 1, 8, 8)
    q = np.zeros((2, 1, 8))
    out, mag, n, _ = ref.attention(q, k, v, [0, 2], np.array([[0]]), [3], np.array([], dtype=int), 0, 1.0, np.zeros((2, 1, 8)))
    assert np.allclose(out[0, 0], v[0, 0, :2].mean(axis=0)) and np.allclose(out[1, 0], v[0, 0, :3].mean(axis=0)) and n[1, 0, 0] == 3
    p = np.array([[0.5, 0.5, 0.0], [0.0, 0.25, 0.75]])
    A, y = ref.verify(p, np.array([[1.0, 0.0, 0.0]]), [0, 1], [0], [0.49], [0.25])
    assert A.tolist() == [1] and y.tolist() == [2]  # u w = 0.25 is not exceeded by 0.25
    A, y = ref.verify(p, np.array([[1.0, 0.0, 0.0]]), [0, 1], [0], [0.5], [0.25])
    assert A.tolist() == [0] and y.tolist() == [1]


# ---- what the compiler made of the attention kernels ---------------------------------------------------------------
def test_attention_kernels_keep_their_registers():
    """No instance spills: a register reloaded from scratch memory in the loop would wait for the copies in flight behind it."""
    path = os.path.join(build.BUILD, "kernels_shared_attention.hip.s")
    if not os.path.exists(path):
        pytest.skip("the library was not built here")
    with open(path) as f:
        asm = f.read()
    names, spills = re.findall(r"\.symbol:\s+(\S+)\.kd", asm), [int(n) for n in re.findall(r"\.vgpr_spill_count:\s+(\d+)", asm)]
    assert len(names) == len(spills) and sum("attn_share_k" in n for n in names) == 18 and sum("attn_split_k" in n for n in names) >= 40
    assert not any(spills), [n for n, s in zip(names, spills) if s]
