"""Operators of include/spec_batch.h against plain 64-bit implementations (tests/batch_reference.py).

Tolerances, derived from the number formats (half a step: fp32 2^-24, bf16 2^-8 of the value).
  tables:   the angle's own rounding, 2^-53 of it, twice (position times frequency, frequency), and 16 steps of the addition
            theorem at 2^-51 each: far below half a step of fp32; 1e-15 (1 + angle) beside that step;
  rotation: two products and a sum in fp32, 2^-24 each: 3 * 2^-24 of the magnitudes of the two terms, then half a step of the
            output type; what does not turn is rounded once;
  attention: a score is a sum of hd products, off by hd 2^-23 A, A = scale sum |q k|; its scaled exponent rounds twice more, 4 * 2^-23 A
            with the scale's own rounding, and exp2 by 2^-23: a weight is off by d = (hd + 4) 2^-23 A + 2^-23 of itself, and so
            are numerator and sum of the weights, 2 d together.  Their sums of n terms, rescaled at most once a term, are off by
            2 n 2^-23 each: 4 n 2^-23.  bf16 rounds every weight in front of the values' product: 2^-8 of the terms.  Joining
            and division: 16 * 2^-23.  All of it relative to sum p |v|, then half a step of the result;
  verification: the tests are exact and whole numbers are equal; draws are taken where the sums' order cannot matter (the tests' u
            lie at least 1e-9 of the mass from a border, sums in 64 bits are off by 1e-11 at most)."""
import numpy as np
import pytest
import torch

import batch_reference as ref
import paper_2504_00030_amd as pk

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _np(t):
    return t.detach().double().cpu().numpy()


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- tables --------------------------------------------------------------------------------------------------------
SCALINGS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
            dict(scaling="bands", factor=8.0, low=1.0, high=4.0, context=8192.0), dict(scaling="ramp", factor=4.0, low=1.0, high=32.0, context=4096.0),
            dict(scaling="ramp", factor=16.0, low=2.0, high=3.0, context=100.0, magnitude=1.5)]


@pytest.mark.parametrize("how", SCALINGS)
@pytest.mark.parametrize("n_pos,rot,theta", [(1, 2, 10000.0), (5, 64, 10000.0), (1037, 14, 500000.0), (300, 128, 500000.0), (4097, 512, 1e6),
                                             (70000, 6, 10000.0)])
def test_tables(n_pos, rot, theta, how):
    if rot == 2 and how.get("scaling") == "base":
        theta = 3.0
    cos = torch.full((n_pos, rot // 2), 7.0, device="cuda")
    sin = torch.full((n_pos, rot // 2), 7.0, device="cuda")
    pk.k_rope_tables(cos, sin, theta=theta, stream=_stream(), **how)
    f, size = ref.frequencies(rot, theta, **how)
    ang = np.arange(n_pos)[:, None] * f[None, :]
    for got, want in ((_np(cos), np.cos(ang) * size), (_np(sin), np.sin(ang) * size)):
        assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + size * 1e-15 * (1 + ang) + 2.0 ** -149).all()


# ---- rotation and cache --------------------------------------------------------------------------------------------
def _rope_case(seed, R, nq, nkv, hd, rot, inter, tx, ty, page, extra=0, shift=0, in_place=False):
    rng = np.random.default_rng(seed)
    width = (nq + 2 * nkv) * hd + extra
    flat = torch.from_numpy(rng.standard_normal(R * width + shift + 8).astype(np.float32)).to(tx).cuda()
    rows = flat[shift: shift + R * width].view(R, width)
    q = rows[:, : nq * hd].unflatten(1, (nq, hd)) if nq else None
    k = rows[:, nq * hd: (nq + nkv) * hd].unflatten(1, (nkv, hd)) if nkv else None
    v = rows[:, (nq + nkv) * hd: (nq + 2 * nkv) * hd].unflatten(1, (nkv, hd)) if nkv else None
    n_pos, n_pages = 37, R // page + 3
    cos = torch.from_numpy(rng.standard_normal((n_pos, rot // 2)).astype(np.float32)).cuda()
    sin = torch.from_numpy(rng.standard_normal((n_pos, rot // 2)).astype(np.float32)).cuda()
    pos = rng.integers(0, n_pos, R)
    slot = rng.permutation(n_pages * page)[:R]
    if R > 3:
        pos[1], pos[2] = -1, n_pos            # padding
        slot[3], slot[R - 1] = -5, n_pages * page  # queries alone
    qo = None if not nq else q if in_place else torch.full((R, nq * hd + extra), 5.0, dtype=ty, device="cuda")[:, : nq * hd].unflatten(1, (nq, hd))
    kp = torch.full((n_pages, nkv, page, hd), 5.0, dtype=ty, device="cuda") if nkv else None
    vp = torch.full((n_pages, nkv, page, hd), 5.0, dtype=ty, device="cuda") if nkv else None
    hq, hk, hv = (_np(t) if t is not None else None for t in (q, k, v))
    q0, k0, v0 = (_np(t) if t is not None else None for t in (qo, kp, vp))
    before = flat.clone()
    pk.k_rope_cache(q, k, v, cos, sin, _int(pos.tolist()), _int(slot.tolist()) if nkv else None, qo, kp, vp, interleaved=inter, stream=_stream())
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(flat, before)
    there = (pos >= 0) & (pos < n_pos)
    at = np.clip(pos, 0, n_pos - 1)
    c, s = _np(cos)[at], _np(sin)[at]
    half = HALF_STEP[ty]

    def near(got, want, mag, what):
        err, tol = np.abs(got - want), (3 * 2.0 ** -24 * mag) * (1 + half) + half * np.abs(want) + 2.0 ** -140
        assert (err <= tol).all(), f"{what}: {np.max(err / tol):.3g} of the tolerance"

    if nq:
        want, mag = ref.rotate(hq, c, s, inter)
        want[~there], mag[~there] = q0[~there], 0.0
        near(_np(qo), want, mag, "q")
    if nkv:
        kept = np.nonzero(there & (slot >= 0) & (slot < n_pages * page))[0]
        want, mag = ref.rotate(hk, c, s, inter)
        wk, wm, wv = k0.copy(), np.zeros_like(k0), v0.copy()
        for r in kept:
            wk[slot[r] // page, :, slot[r] % page], wm[slot[r] // page, :, slot[r] % page] = want[r], mag[r]
            wv[slot[r] // page, :, slot[r] % page] = hv[r]
        near(_np(kp), wk, wm, "k")
        near(_np(vp), wv, 0.0, "v")


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("tx,ty", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("R,nq,nkv,hd,rot,page", [(1, 4, 2, 128, 128, 64), (9, 7, 1, 64, 32, 8), (33, 12, 12, 64, 64, 16), (5, 2, 1, 80, 38, 8),
                                                   (17, 3, 2, 7, 6, 8), (6, 1, 1, 512, 512, 128), (10, 5, 0, 96, 96, 8), (10, 0, 3, 96, 48, 16),
                                                   (4, 1, 1, 2, 2, 8), (70, 20, 5, 32, 16, 32)])
def test_rotation_and_cache(R, nq, nkv, hd, rot, page, tx, ty, inter):
    _rope_case(R * 100 + hd, R, nq, nkv, hd, rot, inter, tx, ty, page)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("tx", [F32, BF16])
@pytest.mark.parametrize("extra,shift", [(8, 0), (4, 4), (3, 0), (1, 1), (2, 5)])
def test_rotation_of_strided_and_oddly_placed_rows(extra, shift, tx, inter):
    _rope_case(extra * 10 + shift, 21, 4, 2, 64, 48, inter, tx, tx, 16, extra=extra, shift=shift)
    _rope_case(extra * 10 + shift, 21, 4, 0, 64, 64, inter, tx, tx, 16, extra=extra, shift=shift, in_place=True)


def test_rotation_with_infinities_and_nan_keeps_them_in_their_rows():
    R, hd = 8, 64
    q = torch.randn((R, 2, hd), device="cuda")
    q[3, 1, 5], q[5, 0, 0] = float("nan"), float("inf")
    cos, sin = torch.ones((4, 32), device="cuda"), torch.full((4, 32), 0.5, device="cuda")
    out = torch.zeros_like(q)
    pk.k_rope_cache(q, None, None, cos, sin, _int([0] * R), None, out, None, None, stream=_stream())
    bad = ~torch.isfinite(out)
    assert bad.nonzero().tolist() == [[3, 1, 5], [3, 1, 37], [5, 0, 0], [5, 0, 32]]


# ---- attention -----------------------------------------------------------------------------------------------------
class Attn:
    """A batch with its cache; the pool's pages that nobody has, and what lies behind the sequences' ends, hold `junk`."""

    def __init__(self, seed, rows, own, prefix, nq, nkv, hd, page, dtype, junk=float("nan"), sharp=1.0, extra_rows=0, spare=1):
        rng = np.random.default_rng(seed)
        self.rng, self.rows, self.own, self.prefix, self.dtype, self.page = rng, rows, own, prefix, dtype, page
        B, R = len(rows), sum(rows) + extra_rows
        n_prefix = (prefix + page - 1) // page
        n_own = (max(own + [0]) + page - 1) // page + spare
        n_pages = n_prefix + B * n_own + 2
        perm = rng.permutation(n_pages)
        self.prefix_table = perm[:n_prefix].astype(np.int32)
        self.table = perm[n_prefix: n_prefix + B * n_own].astype(np.int32).reshape(B, n_own)
        cast = lambda x: torch.from_numpy(x.astype(np.float32)).to(dtype)
        k, v = cast(rng.standard_normal((n_pages, nkv, page, hd)) * sharp), cast(rng.standard_normal((n_pages, nkv, page, hd)))
        used = np.zeros((n_pages, page), dtype=bool)
        for j in range(prefix):
            used[self.prefix_table[j // page], j % page] = True
        for b in range(B):
            for j in range(min(max(own[b], 0), n_own * page)):
                used[self.table[b, j // page], j % page] = True
        hidden = torch.from_numpy(~used)[:, None, :, None]
        self.k, self.v = torch.where(hidden, torch.tensor(junk, dtype=dtype), k), torch.where(hidden, torch.tensor(junk, dtype=dtype), v)
        self.q = cast(rng.standard_normal((R, nq, hd)) * 1.5)
        self.row_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.scale = hd ** -0.5

    def run(self, q=None, out=None, scale=None, work=None):
        R, nq, hd = self.q.shape
        q = self.q.cuda() if q is None else q
        out = torch.full((R, nq, hd), 3.0, dtype=self.dtype, device="cuda") if out is None else out
        n = pk.k_attn_shared_workspace(R, len(self.own), nq, self.k.shape[1], hd, self.dtype, self.prefix, self.table.shape[1] * self.page)
        work = torch.full((max(n, 1),), 0xff, dtype=torch.uint8, device="cuda") if work is None else work  # NaN
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
        pk.k_attn_shared(q, self.k.cuda(), self.v.cuda(), dev(self.row_start), dev(self.table), dev(self.own), out, work,
                         prefix_table=dev(self.prefix_table), prefix_len=self.prefix, scale=scale, stream=_stream())
        torch.cuda.synchronize()
        return out

    def check(self, out=None, scale=None):
        got = _np(self.run(scale=scale) if out is None else out)
        before = np.full(got.shape, 3.0)
        want, mag, n, size = ref.attention(_np(self.q), _np(self.k), _np(self.v), self.row_start, self.table, self.own, self.prefix_table,
                                           self.prefix, self.scale if scale is None else scale, before)
        hd, half = got.shape[2], HALF_STEP[self.dtype]
        rel = 2 * ((hd + 4) * size + 1) * 2.0 ** -23 + (4 * n + 16) * 2.0 ** -23 + (2.0 ** -8 if self.dtype == BF16 else 0.0)
        tol = rel * mag * (1 + half) + half * np.abs(want) + 1e-38
        err = np.abs(got - want)
        assert (err <= tol).all(), f"worst {np.nanmax(err / tol):.3g} of the tolerance at {np.unravel_index(np.argmax(~(err <= tol)), err.shape)}"
        return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [8, 24, 32, 40, 64, 80, 96, 128, 136, 256])
@pytest.mark.parametrize("nq,nkv", [(4, 4), (6, 2), (7, 1)])
def test_attention_head_layouts(nq, nkv, hd, dtype):
    Attn(hd * 10 + nq, [1, 3, 2], [1, 70, 33], 45, nq, nkv, hd, 16, dtype).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [32, 24, 64, 40, 128, 80, 256, 200])
@pytest.mark.parametrize("rows,own,prefix,heads", [
    ([1, 2], [500, 3], 130, 2), ([1, 2], [90, 3], 100, 2),       # up to 16 columns: parts, and through prefix and own positions
    ([5] * 5, [400, 5, 70, 5, 33], 300, 2), ([5] * 5, [100, 5, 70, 5, 33], 90, 2),  # 25 for the prefix, 5 for a sequence
    ([20, 18], [400, 18], 200, 1), ([20, 18], [100, 18], 70, 1),  # up to 32
    ([1] * 40, [300] + [2] * 39, 150, 1),                        # 40 for the prefix, one for a sequence
    ([40], [400], 200, 1), ([70], [200], 200, 1), ([140], [400], 200, 1),  # 64, 128 and 256 that share positions
    ([1] * 100, [20] * 100, 70, 2)])                             # enough of them to go through a prefix that 100 columns share
def test_attention_of_every_width_and_head_size(rows, own, prefix, heads, hd, dtype):
    Attn(hd + sum(rows), rows, own, prefix, heads, heads, hd, 16, dtype).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("prefix", [0, 1, 31, 64, 200])
def test_attention_pages_and_prefixes(prefix, page, dtype):
    Attn(page + prefix, [5, 1, 9, 4], [5, 1, 150, 97], prefix, 4, 2, 64, page, dtype).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix", [
    ([1], [1], 0), ([1], [0], 0), ([1], [0], 1), ([3], [1], 0), ([3], [1], 5), ([2, 0, 3], [0, 9, 2], 0), ([0, 0, 1], [4, 4, 4], 3),
    ([33], [33], 0), ([70], [90], 10), ([1], [1500], 0), ([1], [0], 1500), ([2, 1], [1300, 3], 700), ([1] * 70, list(range(1, 71)), 40),
    ([3, 1, 2] * 30, [9, 1, 130] * 30, 130), ([4, 2], [-3, 6], 9), ([4, 2], [-2**31, 6], 0), ([130, 1], [200, 1], 70), ([1, 0, 2] * 100, [9, 3, 40] * 100, 20)])
def test_attention_lengths(rows, own, prefix, dtype):
    Attn(len(rows) + prefix, rows, own, prefix, 4, 2, 32, 16, dtype).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix,nq,nkv,hd", [([9] * 20, [60] * 20, 300, 8, 2, 128), ([40, 3, 90], [40, 300, 95], 100, 8, 2, 64),
                                                        ([64], [64], 333, 4, 1, 128), ([150], [150], 0, 2, 2, 96), ([30, 30], [30, 64], 64, 7, 1, 256)])
def test_attention_of_many_columns(rows, own, prefix, nq, nkv, hd, dtype):
    Attn(sum(rows), rows, own, prefix, nq, nkv, hd, 32, dtype).check()


@pytest.mark.parametrize("page", [8, 32, 64, 128])
@pytest.mark.parametrize("prefix", [0, 63, 64, 200, 1000])
@pytest.mark.parametrize("rows,own,nq,nkv,hd", [([64], [70], 1, 1, 128), ([33, 40], [40, 300], 4, 2, 64), ([150], [150], 2, 2, 32),
                                                 ([300, 1, 0, 5], [420, 90, 3, 5], 1, 1, 96), ([30, 60], [30, 200], 7, 1, 40)])
def test_attention_of_columns_that_share_positions(rows, own, nq, nkv, hd, prefix, page):
    Attn(sum(rows) + prefix, rows, own, prefix, nq, nkv, hd, page, BF16).check()


@pytest.mark.parametrize("prefix,page", [(0, 64), (64, 64), (70, 16), (300, 128)])
@pytest.mark.parametrize("rows,own,hd", [([64] * 6, [64, 65, 100, 130, 64, 90], 32), ([70] * 5 + [3], [70] * 5 + [200], 16), ([130, 100, 140], [130, 164, 150], 64)])
def test_attention_of_workgroups_that_go_through_prefix_and_own_positions(rows, own, hd, prefix, page):
    a = Attn(sum(own) + prefix, rows, own, prefix, 32, 32, hd, page, BF16, extra_rows=2)
    assert (a.check()[-2:] == 3.0).all()


@pytest.mark.parametrize("rows,hd,prefix,page", [(128, 32, 70, 16), (256, 64, 130, 64)])
def test_attention_of_wide_workgroups_that_go_through_prefix_and_own_positions(rows, hd, prefix, page):
    a = Attn(rows, [rows] * 6, [rows, rows + 1, rows + 70, rows, rows + 3, rows], prefix, 32, 32, hd, page, BF16)
    assert pk.k_attn_shared_workspace(6 * rows, 6, 32, 32, hd, BF16, prefix, a.table.shape[1] * page) == 0  # nothing is left to join
    a.check()


@pytest.mark.parametrize("nq,nkv,hd,prefix", [(4, 4, 32, 200), (2, 2, 128, 100), (32, 32, 64, 130)])
def test_attention_of_columns_that_share_positions_with_bounds_that_make_no_sense(nq, nkv, hd, prefix):
    a = Attn(21, [70, 90], [400, 90], prefix, nq, nkv, hd, 16, BF16, junk=0.25)
    a.own = [2**31 - 1, 90]
    a.check()
    a.table = a.table.copy()
    a.table[0, 3], a.table[1, 1], a.prefix_table[2] = -7, 10**6, a.k.shape[0]
    a.check()
    a.prefix_table[:] = -1
    a.table[0, :] = 2**31 - 1
    a.check()
    for starts in ([-5, 70, 160], [0, 70, 2**31 - 1], [0, 130, 20], [160, 160, 160], [100, 300, -100]):
        a.row_start = np.array(starts, dtype=np.int32)
        a.run()


def test_attention_through_prefix_and_own_positions_with_pages_outside_the_pool():
    a = Attn(22, [64] * 6, [64, 64, 130, 200, 64, 64], 200, 32, 32, 32, 16, BF16, junk=0.25)
    a.table = a.table.copy()
    a.table[3, 2], a.table[2, 0], a.prefix_table[5] = -1, 2**31 - 1, a.k.shape[0]
    a.check()
    a.prefix_table[:] = -1
    a.own = [2**31 - 1, 0, 3, 200, -5, 64]
    a.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("nq,nkv,hd,prefix", [(2, 2, 64, 100), (4, 1, 128, 0), (32, 32, 32, 70), (1, 1, 40, 64)])
def test_attention_of_columns_that_share_positions_keeps_infinities_to_the_rows_that_see_them(nq, nkv, hd, prefix, bad):
    rows, own = [80, 100], [80, 150]
    a, clean = (Attn(12, rows, own, prefix, nq, nkv, hd, 16, BF16) for _ in range(2))
    g = nq // nkv
    seen = np.zeros((sum(rows), nq, hd), dtype=bool)
    for b, j, ch in ((0, 5, 3), (0, 79, 0), (1, 77, 7), (1, 140, 1)):
        a.v[a.table[b, j // 16], 0, j % 16, ch] = bad
        seen[a.row_start[b] + j - (own[b] - rows[b]): a.row_start[b + 1], :g, ch] = True
    a.k[a.table[1, 100 // 16], nkv - 1, 100 % 16, 2] = float("nan")
    seen[a.row_start[1] + 50:, (nkv - 1) * g:, :] = True
    got, want = _np(a.run()), _np(clean.run())
    assert not np.isfinite(got[seen]).any() and np.isfinite(got[~seen]).all()
    assert np.allclose(got[~seen], want[~seen], rtol=2.0 ** -7, atol=2.0 ** -10)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_leaves_rows_of_no_sequence_alone(dtype):
    a = Attn(3, [3, 2], [40, 20], 33, 4, 2, 64, 16, dtype, extra_rows=4)
    got = a.check()
    assert (got[5:] == 3.0).all() and not (got[:5] == 3.0).any()
    a.row_start = np.array([2, 4, 7], dtype=np.int32)  # rows in front of the first sequence as well
    got = a.check()
    assert (got[:2] == 3.0).all() and (got[7:] == 3.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_with_bounds_that_make_no_sense(dtype):
    """Lengths beyond the table, pages outside the pool, row numbers outside the batch: clamped, never followed."""
    a = Attn(4, [3, 2, 4], [500, 64, 30], 40, 4, 2, 32, 16, dtype, junk=0.25)
    a.own = [2**31 - 1, 64, 30]
    a.check()
    a.table = a.table.copy()
    a.table[1, 0], a.table[2, 1], a.prefix_table[1] = -7, 10**6, a.k.shape[0]
    a.check()
    a.prefix_table[:] = -1
    a.table[0, :] = 2**31 - 1
    a.check()
    for starts in ([-5, 3, 5, 9], [0, 3, 5, 2**31 - 1], [0, 7, 2, 9], [9, 9, 9, 9], [5, 5, 100, -100]):
        a.row_start = np.array(starts, dtype=np.int32)
        a.run()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (2, 1, 128), (5, 5, 40)])
def test_attention_keeps_infinities_to_the_rows_that_see_them(nq, nkv, hd, bad, dtype):
    """Values and keys of a drafted position reach the rows from it on, no earlier one and no other sequence."""
    a = Attn(11, [6, 20, 2], [6, 52, 40], 50, nq, nkv, hd, 16, dtype)
    spoilt = {}
    for b, j in ((0, 2), (1, 43), (1, 50)):  # own positions of rows 2 of the first, 11 and 18 of the second sequence
        pg, at = a.table[b, j // 16], j % 16
        a.v[pg, 0, at, 3] = bad
        a.k[pg, 0, at, 1] = float("nan") if b else 0.0
        spoilt[(b, j)] = a.row_start[b] + (j - (a.own[b] - a.rows[b]))
    got = _np(a.run())
    seen = np.zeros(got.shape, dtype=bool)
    g = nq // nkv
    first = spoilt[(0, 2)]
    seen[first: a.row_start[1], :g, 3] = True                 # a value: its channel alone
    seen[spoilt[(1, 43)]: a.row_start[2], :g, :] = True       # a key of NaN: the whole head
    assert not np.isfinite(got[seen]).any()
    clean = Attn(11, [6, 20, 2], [6, 52, 40], 50, nq, nkv, hd, 16, dtype)
    clean.k[a.table[0, 0], 0, 2, 1] = 0.0
    want = _np(clean.run())
    assert np.isfinite(got[~seen]).all()
    tol = 2.0 ** -20 if dtype == F32 else 2.0 ** -7  # (the same sums in another grouping: a rounding of the result apart)
    assert np.allclose(got[~seen], want[~seen], rtol=tol, atol=tol * 0.1)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_with_large_scores(dtype):
    """Scores of hundreds: one position has all the weight, earlier maxima are far below it."""
    Attn(5, [4, 1], [300, 900], 600, 4, 2, 64, 64, dtype, sharp=30.0).check()
    Attn(6, [4, 1], [300, 900], 600, 4, 2, 64, 64, dtype).check(scale=1e-30)
    Attn(7, [4, 1], [30, 90], 60, 4, 2, 64, 64, dtype).check(scale=3.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("extra,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_attention_strides_and_alignment(extra, shift, dtype):
    a = Attn(8, [5, 2], [30, 70], 20, 4, 2, 40, 16, dtype)
    R, nq, hd = a.q.shape
    flat = torch.full((R * (nq * hd + extra) + shift,), float("nan"), dtype=dtype, device="cuda")
    q = flat[shift:].view(R, nq * hd + extra)[:, : nq * hd].unflatten(1, (nq, hd))
    q.copy_(a.q)
    hold = torch.full((R * (nq * hd + extra) + shift,), 3.0, dtype=dtype, device="cuda")
    out = hold[shift:].view(R, nq * hd + extra)[:, : nq * hd].unflatten(1, (nq, hd))
    a.run(q=q, out=out)
    a.check(out=out)
    assert (hold[:shift] == 3.0).all() and (hold[shift:].view(R, -1)[:, nq * hd:] == 3.0).all()


def test_attention_repeats_bit_for_bit():
    for dtype in (F32, BF16):
        for a in (Attn(9, [9] * 12, [100] * 12, 2000, 8, 2, 128, 64, dtype), Attn(9, [200], [300], 700, 8, 2, 128, 64, dtype)):
            first = a.run()
            assert all(torch.equal(first, a.run()) for _ in range(3))


# ---- verification --------------------------------------------------------------------------------------------------
def _rows(rng, n, V, dtype, zeros=0.0):
    x = np.exp(3.0 * rng.standard_normal((n, V)))
    x[rng.random((n, V)) < zeros] = 0.0
    x[:, 0] += 1e-3
    return torch.from_numpy((x / x.sum(axis=1, keepdims=True)).astype(np.float32)).to(dtype)


def _verify(p, q, counts, drafted, ua, un, ld=0):
    B, D, V = len(counts), sum(counts), p.shape[1]
    start = _int(np.concatenate([[0], np.cumsum(counts)]).tolist())

    def strided(t):
        if t is None or not ld:
            return t if t is None else t.cuda()
        wide = torch.full((t.shape[0], V + ld), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, :V] = t.cuda()
        return wide[:, :V]

    A, y = _int([9] * B), _int([9] * B)
    work = torch.full((pk.k_verify_workspace(B, V),), 0xff, dtype=torch.uint8, device="cuda")
    pk.k_verify(strided(p), strided(q), start, _int(drafted.tolist()), torch.from_numpy(ua.astype(np.float32)).cuda(),
                torch.from_numpy(un.astype(np.float32)).cuda(), A, y, work, stream=_stream())
    torch.cuda.synchronize()
    want = ref.verify(_np(p), _np(q) if q is not None else None, start.cpu().numpy(), drafted, ua.astype(np.float32), un.astype(np.float32))
    assert A.tolist() == want[0].tolist()
    assert y.tolist() == want[1].tolist()
    return want


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("V,counts,ld", [(1, [1, 0, 2], 0), (2, [1, 2], 0), (17, [0], 0), (1000, [4, 0, 8, 1], 0), (4096, [3], 8), (4097, [8, 8], 3),
                                         (32000, [4], 0), (50257, [2, 5, 0], 0), (128256, [8, 3], 0), (5000, [70, 130], 1)])
def test_verification(V, counts, ld, given, dtype):
    rng = np.random.default_rng(V + len(counts))
    D, B = sum(counts), len(counts)
    for trial in range(3):
        p, q = _rows(rng, D + B, V, dtype, 0.3), _rows(rng, D, V, dtype, 0.3) if given else None
        if given and trial:  # drafts close to the target, so that some are accepted
            seq = np.repeat(np.arange(B), counts)
            near = _np(p)[np.arange(D) + seq] if D else np.zeros((0, V))
            q = torch.from_numpy((near * (1 + 0.2 * rng.standard_normal(near.shape).clip(-2, 2))).astype(np.float32)).to(dtype)
        rows = _np(p)[np.arange(D) + np.repeat(np.arange(B), counts)] if D else np.zeros((0, V))
        drafted = np.array([rng.choice(V, p=r / r.sum()) for r in rows], dtype=np.int64).reshape(D)
        _verify(p, q, counts, drafted, rng.random(D), rng.random(B), ld)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_verification_at_its_borders(dtype):
    V = 9000
    p = torch.zeros((8, V), dtype=dtype)
    q = torch.zeros((6, V), dtype=dtype)
    # 0: u q == p exactly is no acceptance; the residual is empty, so the draw is from p
    p[0, 5], q[0, 5] = 0.5, 0.5
    # 1: an equal chance everywhere, a draw exactly on a border goes to the next token
    p[1] = 2.0 ** -13
    # 2, 3: accepted at u = 0, then a residual with a single token far back
    p[2, 8999], q[1, 8999] = 0.25, 1.0
    p[3, 4096], p[3, 7], q[2, 7] = 0.5, 0.25, 0.5
    p[4, 1] = 1.0
    counts = [1, 0, 2, 1]
    drafted = np.array([5, 8999, 7, 2, 1, 1][:4])
    p, q = p[:8], q[:4]
    A, y = _verify(p, q, counts, drafted, np.array([1.0, 0.0, 0.9, 0.5]), np.array([0.0, 0.5, 0.999, 0.0]))
    # (sequences 0 .. 3 have rows 0 - 1, 2, 3 - 5 and 6 - 7 of p: the third one's first draft has no chance there, u = 0 or not,
    # and rows 6 and 7 hold no weight at all)
    assert A.tolist() == [0, 0, 0, 0] and y.tolist() == [5, 8999, 4096, 0]
    u = 4096 * 2.0 ** -13 / (V * 2.0 ** -13)
    _verify(p, q, counts, drafted, np.array([1.0, 0.0, 0.9, 0.5]), np.array([1.0, u, 1.0, 1.0]))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_verification_draws_at_the_ends_of_tiles_and_rows(dtype):
    """u of 0 accepts any draft with a chance; residuals of one token, at either side of a tile's end and at the row's."""
    V = 9000
    for places in ([0, 4095, 4096], [8191, 8192, 8999]):
        p, q = torch.zeros((8, V), dtype=dtype), torch.zeros((5, V), dtype=dtype)
        for b, x in enumerate(places):  # two drafts a sequence but the last: the first accepted, the second refused
            k = 2 if b < 2 else 1
            first = 2 * b + b
            p[first, 17], q[2 * b, 17] = 2.0 ** -10, 1.0
            if k == 2:
                p[first + 1, 33], p[first + 1, x], q[2 * b + 1, 33] = 0.25, 0.5, 0.5
            else:
                p[first + 1, x] = 0.5
        drafted = np.array([17, 33, 17, 33, 17])
        for u in (0.0, 0.5, 1.0 - 2.0 ** -24, 1.0):
            A, y = _verify(p, q, [2, 2, 1], drafted, np.array([0.0, 0.9, 0.0, 0.9, 0.0]), np.full(3, u))
            assert A.tolist() == [1, 1, 1] and y.tolist() == places


def test_verification_of_drafts_and_weights_that_make_no_sense():
    V = 5000
    rng = np.random.default_rng(0)
    counts = [2, 2, 1, 1, 1, 1]
    p, q = _rows(rng, 14, V, F32), _rows(rng, 8, V, F32)
    p[4, 100:200], p[0, 3] = float("nan"), -1.0
    p[7] = 0.0                       # no weight anywhere
    p[9] = float("nan")
    q[6, :2500] = float("nan")
    drafted = np.array([-1, 3, V, 2**31 - 1, 4, 5, 6, -2**31])
    _verify(p, q, counts, drafted, np.full(8, 0.999), rng.random(6))
    _verify(p, None, counts, drafted, np.full(8, 0.999), rng.random(6))


def test_verification_with_starts_that_make_no_sense():
    V, B, D = 300, 5, 4
    rng = np.random.default_rng(1)
    p, q = _rows(rng, D + B, V, F32).cuda(), _rows(rng, D, V, F32).cuda()
    A, y = _int([9] * B), _int([9] * B)
    work = torch.zeros(pk.k_verify_workspace(B, V), dtype=torch.uint8, device="cuda")
    ua, un = torch.full((D,), 0.5, device="cuda"), torch.full((B,), 0.5, device="cuda")
    drafted = np.array([1, 2, 3, 4])
    for starts in ([0, 1, 3, 2, 4, 4], [-1, 1, 2, 3, 4, 4], [0, 1, 2, 3, 4, 5], [0, 2**31 - 1, 0, -2**31, 4, 4]):
        pk.k_verify(p, q, _int(starts), _int(drafted.tolist()), ua, un, A, y, work, stream=_stream())
        want = ref.verify(_np(p), _np(q), starts, drafted, np.full(D, 0.5), np.full(B, 0.5))
        assert A.tolist() == want[0].tolist() and y.tolist() == want[1].tolist() and -1 in A.tolist()
