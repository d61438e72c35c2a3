"""Operators of include/spec_batch.h at the edges of what the header allows; tolerances as in test_gpu_batch.py unless stated."""
import numpy as np
import pytest
import torch

import batch_reference as ref
import paper_2504_00030_amd as pk
from test_gpu_batch import BF16, F32, HALF_STEP, Attn, _int, _np, _stream, _verify

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


# ---- attention: tables as a server keeps them ----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix,nq,nkv,hd", [([1], [40], 0, 4, 2, 64), ([3, 20, 1], [70, 300, 0], 100, 4, 1, 128), ([70, 3], [70, 900], 0, 2, 2, 64),
                                                       ([5] * 9, [5, 0, 7, 130, 64, 65, 128, 3, 2], 500, 4, 4, 32), ([130], [140], 300, 2, 1, 80)])
def test_attention_with_tables_far_longer_than_the_sequences(rows, own, prefix, nq, nkv, hd, dtype):
    """Parts are planned for 32000 positions a sequence; most hold none, and the pages named there lie outside the pool."""
    a = Attn(sum(own) + hd, rows, own, prefix, nq, nkv, hd, 16, dtype)
    wide = np.full((len(own), 2000), 2**31 - 1, dtype=np.int32)
    wide[:, : a.table.shape[1]] = a.table
    a.table = wide
    a.check()


def test_attention_of_as_many_sequences_as_there_may_be():
    rng = np.random.default_rng(1)
    rows, own = rng.integers(0, 3, 4096).tolist(), rng.integers(0, 20, 4096).tolist()
    for dtype in (F32, BF16):
        Attn(2, rows, own, 9, 1, 1, 16, 8, dtype, extra_rows=3).check()


# ---- attention: scores of any size ---------------------------------------------------------------------------------
# Scores here are exact: one channel of powers of two (queries) times small whole numbers (keys).  A weight is then off by the two
# roundings of its exponent, 2^-24 of it each (times ln 2; what is left of a weight 2^-a times a is below 0.54), by exp2's 2^-23 and
# by half a step of the reference times the scale, 2^-14 where that is below 2^10 and none beyond; numerator and sum: 2^-12 in all.
SPLIT_AND_SHARED = [([5], [700], 300, 2), ([4], [200], 100, 1), ([20, 3], [60, 400], 100, 1), ([48], [300], 260, 1), ([70], [400], 100, 1),
                    ([150], [300], 300, 1), ([1] * 100, [20] * 100, 70, 2)]


def _near(a, got, scale, n_most):
    want, mag, _, _ = ref.attention(_np(a.q), _np(a.k), _np(a.v), a.row_start, a.table, a.own, a.prefix_table, a.prefix, scale, np.full(got.shape, 3.0))
    half = HALF_STEP[a.dtype]
    rel = 2.0 ** -12 + (4 * n_most + 16) * 2.0 ** -23 + (2.0 ** -8 if a.dtype == BF16 else 0.0)
    err, tol = np.abs(got - want), rel * mag * (1 + half) + half * np.abs(want)
    assert (err <= tol).all(), f"{np.count_nonzero(~(err <= tol))} of {err.size} beyond the tolerance, worst {np.nanmax(err):.3g}"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("order", ["rising", "falling", "any"])
@pytest.mark.parametrize("rows,own,prefix,heads", SPLIT_AND_SHARED)
def test_attention_with_scores_of_any_size(rows, own, prefix, heads, order, dtype):
    """Scores up to 2^127, rows of small and large ones side by side, maxima that repeat."""
    for hd, scale in ((64, None), (40, 0.37), (32, 2.0 ** 40)):  # (the last: scaled, they leave fp32's range)
        a = Attn(sum(rows), rows, own, prefix, heads, heads, hd, 16, dtype, junk=0.0)
        for b, table in [(None, a.prefix_table)] + list(enumerate(a.table)):
            n = prefix if b is None else own[b]
            j = a.rng.integers(-100, 101, n)
            j = j if order == "any" else np.sort(j) if order == "rising" else np.sort(j)[::-1]
            for p in range(n):
                a.k[int(table[p // 16]), :, p % 16] = 0.0
                a.k[int(table[p // 16]), :, p % 16, 3] = float(j[p])
        a.q[:] = 0.0
        powers = torch.tensor([-6, 4, 8, 14, 23, 30, 34, 40, 60, 100, 120])
        at = torch.from_numpy(a.rng.integers(0, len(powers), a.q.shape[:2]))
        a.q[:, :, 3] = torch.where(torch.from_numpy(a.rng.random(a.q.shape[:2]) < 0.3), -1.0, 1.0).to(dtype) * (2.0 ** powers[at].double()).to(dtype)
        got = _np(a.run(scale=scale))
        _near(a, got, hd ** -0.5 if scale is None else scale, prefix + max(own))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix,heads", SPLIT_AND_SHARED)
def test_attention_with_scores_that_differ_by_little_of_their_size(rows, own, prefix, heads, dtype):
    """Scores of 2^24 and an even number below 256, all exact, times 2^-6: weights over a factor of 50 far from zero."""
    a = Attn(sum(rows), rows, own, prefix, heads, heads, 64, 16, dtype, junk=0.0)
    a.k[:] = 0.0
    a.k[..., 0] = 2.0 ** 12
    a.k[..., 1] = torch.from_numpy(2.0 * a.rng.integers(0, 128, a.k.shape[:3])).to(dtype)
    a.q[:] = 0.0
    a.q[..., 0], a.q[..., 1] = 2.0 ** 12, 1.0
    _near(a, _np(a.run(scale=2.0 ** -6)), 2.0 ** -6, prefix + max(own))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix,nq,nkv,hd", [([6, 4], [40, 4], 30, 4, 2, 64), ([4, 2], [4, 70], 0, 2, 2, 40), ([20, 3], [600, 3], 300, 2, 1, 128),
                                                       ([80, 70], [100, 70], 70, 2, 2, 64), ([150, 30], [400, 30], 0, 1, 1, 32), ([70], [90], 200, 4, 1, 96)])
def test_attention_with_infinities_in_keys(rows, own, prefix, nq, nkv, hd, dtype):
    """Scores of plus infinity make their head NaN, those of minus infinity have weight 0; queries of both signs."""
    a = Attn(sum(own) + hd, rows, own, prefix, nq, nkv, hd, 16, dtype)
    spoilt = [(a.table[b], j) for b, n in enumerate(own) for j in (0, n // 2, n - 1)] + [(a.prefix_table, j) for j in range(3, prefix, 100)]
    for table, j in spoilt:
        a.k[int(table[j // 16]), :, j % 16, 3] = -float("inf")  # (minus infinity where the query is positive)
    got, q, k, v = _np(a.run()), _np(a.q), _np(a.k), _np(a.v)
    half, kinds = HALF_STEP[dtype], [0, 0, 0]  # heads that are NaN, zeros, numbers
    for b, n in enumerate(rows):
        for i in range(n):
            at = [(a.prefix_table[j // 16], j % 16) for j in range(prefix)] + [(a.table[b, j // 16], j % 16) for j in range(own[b] - n + i + 1)]
            pages, places = np.array(at).T
            for h in range(nq):
                r = a.row_start[b] + i
                kk, vv, x = k[pages, h // (nq // nkv), places], v[pages, h // (nq // nkv), places], got[r, h]
                s = kk @ q[r, h] * a.scale
                some = s > -np.inf
                kinds[0 if np.isnan(s).any() or (s == np.inf).any() else 1 if not some.any() else 2] += 1
                if np.isnan(s).any() or (s == np.inf).any():
                    assert np.isnan(x).all()
                elif not some.any():
                    assert (x == 0).all()
                else:
                    w = np.exp(s[some] - s[some].max())
                    w /= w.sum()
                    want, mag, m = w @ vv[some], w @ np.abs(vv[some]), len(w)
                    size = (np.abs(kk[some]) @ np.abs(q[r, h])).max() * a.scale
                    rel = 2 * ((hd + 4) * size + 1) * 2.0 ** -23 + (4 * m + 16) * 2.0 ** -23 + (2.0 ** -8 if dtype == BF16 else 0.0)
                    assert (np.abs(x - want) <= rel * mag * (1 + half) + half * np.abs(want)).all()
    assert kinds[0] and kinds[2]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix", [([5], [9], 0), ([3, 1], [700, 4], 300), ([80], [90], 70), ([150], [150], 0)])
def test_attention_of_rows_whose_scores_are_all_minus_infinity(rows, own, prefix, dtype):
    a = Attn(sum(own), rows, own, prefix, 2, 2, 64, 16, dtype, extra_rows=1)
    a.k[..., 7] = -float("inf")
    a.q[..., 7] = a.q[..., 7].abs() + 0.5
    got = _np(a.run())
    assert (got[:-1] == 0).all() and (got[-1] == 3.0).all()


# ---- tables --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("magnitude", [1.0, 3e5])
@pytest.mark.parametrize("every", [30, 62, 7, 1000])
def test_tables_where_cosines_and_sines_vanish(every, magnitude):
    """Half a turn every few positions: what is left there are the angles' and the recurrence's own errors, magnitude * (7e-15 + 1e-15 of
    the angle), beside half a step of fp32.  (The ramp interpolates its second pair here, which turns less than twice over the context.)"""
    n_pos, theta = 4099, 2.0
    factor = theta ** -0.5 * every / np.pi
    cos, sin = torch.zeros((n_pos, 2), device="cuda"), torch.zeros((n_pos, 2), device="cuda")
    pk.k_rope_tables(cos, sin, theta=theta, scaling="ramp", factor=factor, low=2.0, high=3.0, context=1.0, magnitude=magnitude, stream=_stream())
    f, size = ref.frequencies(4, theta, scaling="ramp", factor=factor, low=2.0, high=3.0, context=1.0, magnitude=magnitude)
    assert size == magnitude and abs(f[1] * every - np.pi) < 1e-14
    ang = np.arange(n_pos).astype(np.longdouble)[:, None] * f.astype(np.longdouble)[None, :]
    for got, want in ((_np(cos), np.cos(ang) * magnitude), (_np(sin), np.sin(ang) * magnitude)):
        err = np.abs(got.astype(np.longdouble) - want)
        assert (err <= 2.0 ** -24 * np.abs(want) + magnitude * (7e-15 + 1e-15 * ang)).all(), float((err / magnitude).max())


# ---- verification --------------------------------------------------------------------------------------------------
BORDERS = [1, 7, 8, 63, 64, 100, 511, 512, 513, 4096, 7680, 8191]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail", [0, 808])
def test_verification_draws_exactly_on_borders(tail, dtype):
    """Equal weights 2^-13 and u = x 2^-13, all exact: the sum of the first x weights does not exceed u times all of them, so the draw is
    x; the next smaller u draws x - 1.  Rows of no draft, residuals of a refused draft, and the token left out of a looked-up one."""
    V, n = 8192 + tail, len(BORDERS)
    below = np.nextafter(np.float32(BORDERS) * np.float32(2.0 ** -13), np.float32(0))
    p = torch.zeros((n, V), dtype=dtype)
    p[:, :8192] = 2.0 ** -13
    A, y = _verify(p, None, [0] * n, np.array([], dtype=int), np.array([]), np.float32(BORDERS) * np.float32(2.0 ** -13))
    assert A.tolist() == [0] * n and y.tolist() == BORDERS
    assert _verify(p, None, [0] * n, np.array([], dtype=int), np.array([]), below)[1].tolist() == [x - 1 for x in BORDERS]
    # one draft each, refused: u q = p exactly; the residual is 2^-13 on 8192 tokens again
    p, q = torch.zeros((2 * n, V), dtype=dtype), torch.zeros((n, V), dtype=dtype)
    p[:, :8192], q[:, :8192] = 2.0 ** -12, 2.0 ** -13
    drafted = np.full(n, 5)
    A, y = _verify(p, q, [1] * n, drafted, np.full(n, 2.0), np.float32(BORDERS) * np.float32(2.0 ** -13))
    assert A.tolist() == [0] * n and y.tolist() == BORDERS
    assert _verify(p, q, [1] * n, drafted, np.full(n, 2.0), below)[1].tolist() == [x - 1 for x in BORDERS]
    # looked up: the drafted token, here the first, weighs nothing, 8192 others do
    p = torch.zeros((2 * n, V + 1), dtype=dtype)
    p[:, :8193] = 2.0 ** -13
    A, y = _verify(p, None, [1] * n, np.zeros(n, dtype=int), np.full(n, 2.0 ** -13), np.float32(BORDERS) * np.float32(2.0 ** -13))
    assert A.tolist() == [0] * n and y.tolist() == [x + 1 for x in BORDERS]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_verification_accepts_below_the_border_alone(dtype):
    """u q < p: at u = 0 any p above zero accepts and none at zero does, at u = p / q nothing, at the next smaller u the draft."""
    V = 600
    p, q = torch.zeros((10, V), dtype=dtype), torch.zeros((5, V), dtype=dtype)
    least = 2.0 ** -149 if dtype == F32 else 2.0 ** -133
    for b, (px, qx) in enumerate([(least, 1.0), (0.0, 1.0), (0.25, 0.5), (0.25, 0.5), (0.5, 0.25)]):
        p[2 * b, 300 + b], q[b, 300 + b], p[2 * b, 7], p[2 * b + 1, 9] = px, qx, 1.0, 1.0
    u = np.array([0.0, 0.0, 0.5, 0.0, 1.0], dtype=np.float32)
    u[3] = np.nextafter(np.float32(0.5), np.float32(0))
    A, y = _verify(p, q, [1] * 5, np.arange(300, 305), u, np.zeros(5))
    assert A.tolist() == [1, 0, 0, 1, 1] and y.tolist() == [9, 7, 7, 9, 9]


# ---- attention: weights in two terms -------------------------------------------------------------------------------
@pytest.mark.parametrize("g", [1, 20])  # 16 and 32 columns a workgroup
@pytest.mark.parametrize("hd", [8, 32, 64, 128, 200])
@pytest.mark.parametrize("n", [5, 40, 150])  # (the last in two parts)
def test_attention_of_few_columns_keeps_weights_in_two_terms(n, hd, g):
    """Values that cancel under the weights: what is left of a result shows how exact the weights are.  Two bf16 terms leave 2^-8 of
    2^-8, 2^-16 of a weight, numerator and sum each: 2^-15 of sum p |v| in all; one term would leave far more, which is checked too."""
    a = Attn(n + hd + g, [1, 1], [n, n], 0, 2 * g, 2, hd, 16, BF16)
    a.q = a.q.reshape(2, 2, g, hd)[:, :, :1].repeat(1, 1, g, 1).reshape(2, 2 * g, hd)  # one query for all heads of a cache head
    a.q *= 0.5
    one_term_fails = False
    places = [np.array([(a.table[b, j // 16], j % 16) for j in range(n)]).T for b in range(2)]
    for b, (pages, at) in enumerate(places):
        for h in range(2):
            s = _np(a.k)[pages, h, at] @ _np(a.q)[b, h * g] * a.scale
            w = np.exp(s - s.max())
            order = np.argsort(w)[::-1]
            v = _np(a.v)[pages, h, at]
            for j in (order[0], order[1], order[1]):  # the two heaviest positions take what the others leave
                x = v[j] - (w @ v) / w[j]
                v[j] = _np(torch.from_numpy(x).to(BF16))
            a.v[torch.from_numpy(pages), h, torch.from_numpy(at)] = torch.from_numpy(v).to(BF16)
    got = _np(a.run())
    want, mag, m, size = ref.attention(_np(a.q), _np(a.k), _np(a.v), a.row_start, a.table, a.own, a.prefix_table, 0, a.scale, got)
    rel = 2 * ((hd + 4) * size + 1) * 2.0 ** -23 + (4 * m + 16) * 2.0 ** -23 + 2.0 ** -15
    tol = rel * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    err = np.abs(got - want)
    assert (err <= tol).all(), f"worst {np.max(err / tol):.3g} of the tolerance"
    for b, (pages, at) in enumerate(places):
        for h in range(2):
            s = _np(a.k)[pages, h, at] @ _np(a.q)[b, h * g] * a.scale
            w = _np(torch.from_numpy(np.exp(s - s.max())).to(BF16))
            one_term_fails |= bool((np.abs(w @ _np(a.v)[pages, h, at] / w.sum() - want[b, h * g]) > tol[b, h * g]).any())
    assert one_term_fails


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,own,prefix,heads", SPLIT_AND_SHARED)
def test_attention_with_scales_at_the_ends_of_fp32(rows, own, prefix, heads, dtype):
    """A scale below fp32's normal numbers weighs all positions alike; one near its end leaves the largest score alone."""
    for scale in (1e-42, 1e-38):
        Attn(sum(rows), rows, own, prefix, heads, heads, 64, 16, dtype).check(scale=scale)
    a = Attn(sum(rows), rows, own, prefix, heads, heads, 64, 16, dtype, junk=0.0)
    a.k[:], a.q[:] = 0.0, 0.0
    a.k[..., 5] = torch.from_numpy(a.rng.integers(0, 101, a.k.shape[:3]).astype(np.float32)).to(dtype)
    a.q[..., 5] = torch.from_numpy(np.where(a.rng.random(a.q.shape[:2]) < 0.5, -1.0, 1.0).astype(np.float32)).to(dtype)
    _near(a, _np(a.run(scale=2e38)), 2e38, prefix + max(own))
