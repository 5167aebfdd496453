"""Parity of the residual RMS norm (include/rowops.h) against its formula in 64 bits.

Tolerance.  h, the sum of squares and the products are fp32: y is within 3e-5 relative of its exact value (sums of up to 70000 terms of
one sign, one-ulp square root and division, three products) before its one rounding (half an ulp of the type: 2^-11 or 2^-8 relative, 2^-25 absolute
below binary16's normal numbers).  h itself is one fp32 addition (2^-24) and one rounding.  8 bits: y8 is the e4m3 value nearest to y / scale up to
3e-5 of it: half a step of e4m3 (2^-4 relative, 2^-10 absolute below its normal numbers) and 3e-5; scale is within 3e-5 of max |y| / 448.
"""
import pytest
import torch

import paper_2501_08071_amd as P

pytestmark = pytest.mark.gpu
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
EPS = 1e-6
SLACK = 3e-5


def make(rows, d, dtype, seed=0, mul=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return (r(rows, d) * mul).to(dtype), (r(rows, d) * 3 * mul).to(dtype), (1 + 0.3 * r(d)).to(dtype)


def formula(x, r, w, eps=EPS):
    h = x.double() + (r.double() if r is not None else 0.0)
    return h, h / (h.square().mean(1, keepdim=True) + eps).sqrt() * w.double()


def near(got, ref, dtype):
    return ((got.double() - ref).abs() <= (U[dtype] + SLACK) * ref.abs() + 2.0 ** -25).all()


def check_fp8(y, scale, ref, group):
    rows, d = ref.shape
    size = group or d
    for c in range(-(-d // size)):
        part = ref[:, c * size:(c + 1) * size]
        top = part.abs().amax(1)
        s = torch.where(top == 0, 1.0, top / 448.0)
        got = scale[:, c].double()
        assert ((got - s).abs() <= SLACK * s).all()
        z, y8 = part / s[:, None], y[:, c * size:(c + 1) * size].float().double()
        assert ((y8 - z).abs() <= (2.0 ** -4 + 2 * SLACK) * z.abs() + 2.0 ** -10 + 1e-7).all()
        full = top > 0
        assert (y8.abs().amax(1)[full] == 448.0).all() and (y8[~full] == 0).all()


# every choice of threads a row, with idle lanes and chunks, and lengths that are multiples of nothing; the last ones are read twice
LENGTHS = [1, 2, 7, 8, 9, 63, 64, 65, 72, 120, 127, 128, 129, 136, 256, 500, 512, 520, 1000, 1023, 1024, 1025, 2048, 2049, 4095, 4096, 5001, 8192,
           8193, 16384, 16389, 20000, 32767, 32768, 32769, 70001]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", LENGTHS)
def test_all_forms(d, dtype):
    rows = 37 if d <= 4096 else 5
    x, r, w = make(rows, d, dtype, seed=d)
    for res in (r, None):
        h, ref = formula(x, res, w)
        y, r_out = P.residual_rmsnorm_fwd(x, res, w, EPS)
        assert near(y, ref, dtype)
        assert r_out is None if res is None else ((r_out.double() - h).abs() <= (U[dtype] + 2.0 ** -23) * h.abs() + 2.0 ** -25).all()
        for group in (0, 128):
            y8, scale, r8 = P.residual_rmsnorm_fwd_fp8(x, res, w, EPS, group=group)
            assert y8.dtype == torch.float8_e4m3fn and scale.shape == (rows, -(-d // 128) if group else 1)
            check_fp8(y8, scale, ref, group)
            assert r8 is None if res is None else torch.equal(r8, r_out)


@pytest.mark.parametrize("rows,d", [(70000, 40), (9000, 200), (20000, 513), (4097, 4096)])
def test_more_rows_than_a_grid_holds(rows, d):
    x, r, w = make(rows, d, torch.bfloat16, seed=rows)
    h, ref = formula(x, r, w)
    buf = torch.full((rows * d + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    y, _ = P.residual_rmsnorm_fwd(x, r, w, EPS, y=buf[8:8 + rows * d].view(rows, d))
    assert near(y, ref, torch.bfloat16) and (buf[:8] == 7.0).all() and (buf[8 + rows * d:] == 7.0).all()
    y8, scale, _ = P.residual_rmsnorm_fwd_fp8(x, r, w, EPS, group=128)
    check_fp8(y8, scale, ref, 128)


# 1024 threads a row: 512 workgroups at most; rows past 32768 elements: read twice; short rows: 32 to a workgroup, 2^22 workgroups at most
@pytest.mark.parametrize("rows,d,dtype", [(1100, 16392, torch.bfloat16), (1100, 16389, torch.float16), (1537, 32768, torch.float16), (1100, 32776, torch.bfloat16),
                                          (1537, 32771, torch.float16), (2 ** 27 + 1000, 1, torch.bfloat16), (2 ** 27 + 1000, 8, torch.float16)])
def test_a_workgroup_goes_round_the_rows(rows, d, dtype):
    """More rows than a launch has places for them: the second and third of a workgroup are as right as its first."""
    x, r, w = make(rows, d, dtype, seed=d)
    size = rows * d
    buf = torch.full((size + 16,), 7.0, dtype=dtype, device="cuda")
    y, r_out = P.residual_rmsnorm_fwd(x, r, w, EPS, y=buf[8:8 + size].view(rows, d))
    eight = [(group, P.residual_rmsnorm_fwd_fp8(x, r, w, EPS, group=group)) for group in (0, 128)]
    assert (buf[:8] == 7.0).all() and (buf[8 + size:] == 7.0).all()
    step = max(1, 2 ** 26 // d)
    for a in range(0, rows, step):
        part = slice(a, a + step)
        h, ref = formula(x[part], r[part], w)
        assert near(y[part], ref, dtype)
        assert ((r_out[part].double() - h).abs() <= (U[dtype] + 2.0 ** -23) * h.abs() + 2.0 ** -25).all()
        for group, (y8, scale, r8) in eight:
            check_fp8(y8[part], scale[part], ref, group)
            assert torch.equal(r8[part], r_out[part])


@pytest.mark.parametrize("d", [65, 512, 4099, 16384, 40000])
def test_in_place(d):
    """The residual updated in its own buffer, y over x."""
    x, r, w = make(19, d, torch.float16, seed=d)
    want, want_r = P.residual_rmsnorm_fwd(x, r, w, EPS)
    want8 = P.residual_rmsnorm_fwd_fp8(x, r, w, EPS, group=128)
    r1, x1 = r.clone(), x.clone()
    y, ro = P.residual_rmsnorm_fwd(x1, r1, w, EPS, y=x1, r_out=r1)
    assert y is x1 and ro is r1 and torch.equal(x1, want) and torch.equal(r1, want_r)
    r1 = r.clone()
    y8, s, _ = P.residual_rmsnorm_fwd_fp8(x, r1, w, EPS, group=128, r_out=r1)
    assert torch.equal(y8.view(torch.uint8), want8[0].view(torch.uint8)) and torch.equal(s, want8[1]) and torch.equal(r1, want_r)


@pytest.mark.parametrize("d", [64, 1000, 4096, 33000])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rows_of_zeros_tiny_and_non_finite_values(dtype, d):
    x, _, w = make(8, d, dtype, seed=1)
    r = torch.zeros_like(x)
    x[0] = 0
    x[1], r[1] = 1.5, -1.5                     # sums to zero
    x[2, :d // 2] = 0                          # for wide rows: groups of zeros
    x[3] *= 2.0 ** -10
    x[4, d // 3] = float("nan")
    x[5, d - 1] = float("inf")
    ok = [0, 1, 2, 3, 6, 7]
    _, ref = formula(x, r, w)
    y, _ = P.residual_rmsnorm_fwd(x, r, w, EPS)
    assert near(y[ok], ref[ok], dtype) and torch.isnan(y[4]).all() and torch.isnan(y[5, d - 1]) and (y[5, :d - 1] == 0).all()
    for group in (0, 128):
        y8, s, _ = P.residual_rmsnorm_fwd_fp8(x, r, w, EPS, group=group)
        check_fp8(y8[ok], s[ok], ref[ok], group)
        assert torch.isnan(y8[4].float()).all() and torch.isnan(s[4]).all()
        assert torch.isnan(s[5, -1]) and torch.isnan(y8[5, d - 1].float())
    tiny = torch.full_like(w, 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -120)
    _, ref = formula(x[6:], r[6:], tiny)
    check_fp8(*P.residual_rmsnorm_fwd_fp8(x[6:], r[6:], tiny, EPS)[:2], ref, 0)


def test_streams_shapes_and_eps():
    x, r, w = make(24, 512, torch.bfloat16)
    want, want_r = P.residual_rmsnorm_fwd(x, r, w, 0.5)
    assert near(want, formula(x, r, w, 0.5)[1], torch.bfloat16)
    y, ro = P.residual_rmsnorm_fwd(x.view(2, 3, 4, 512), r.view(2, 3, 4, 512), w, 0.5)
    assert y.shape == (2, 3, 4, 512) and torch.equal(y.view(24, 512), want) and torch.equal(ro.view(24, 512), want_r)
    y8, s, _ = P.residual_rmsnorm_fwd_fp8(x.view(4, 6, 512), None, w, 0.5, group=128)
    assert y8.shape == (4, 6, 512) and s.shape == (4, 6, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, _ = P.residual_rmsnorm_fwd(x, r, w, 0.5, stream=side)
    side.synchronize()
    assert torch.equal(a, want)
    assert P.residual_rmsnorm_fwd(x[:0], r[:0], w, EPS)[0].shape == (0, 512)


@pytest.fixture(params=["short", "long"])
def way(request, monkeypatch):
    from paper_2501_08071_amd import binding
    if request.param == "long":
        class Never:
            def __getattr__(self, name):
                return lambda *a: None
        monkeypatch.setattr(binding, "_fast", Never())
    return request.param


def test_both_ways_agree_and_what_is_refused(way):
    x, r, w = make(6, 300, torch.float16)
    h, ref = formula(x, r, w)
    y, ro = P.residual_rmsnorm_fwd(x, r, w, EPS, r_out=x.clone())
    assert near(y, ref, torch.float16) and P.residual_rmsnorm_fwd(x, None, w, EPS)[1] is None
    y8, s, _ = P.residual_rmsnorm_fwd_fp8(x, r, w, EPS, scale=torch.empty(6, 3, device="cuda"), group=128)
    check_fp8(y8, s, ref, 128)
    f, g = P.residual_rmsnorm_fwd, P.residual_rmsnorm_fwd_fp8
    bad = [(TypeError, lambda: f(x.float(), r.float(), w.float(), EPS)), (ValueError, lambda: f(x, r[:3], w, EPS)), (ValueError, lambda: f(x, r.bfloat16(), w, EPS)),
           (ValueError, lambda: f(x, r, w[:8], EPS)), (ValueError, lambda: f(x, r, w.float(), EPS)), (ValueError, lambda: f(x.cpu(), r, w, EPS)),
           (ValueError, lambda: f(x[:, ::2], r, w, EPS)), (ValueError, lambda: f(x, r, w, EPS, y=y8)), (ValueError, lambda: f(x, r, w, EPS, r_out=s)),
           (P.RowopsError, lambda: f(x, r, w, -1.0)), (P.RowopsError, lambda: f(x, r, w, float("nan"))), (P.RowopsError, lambda: f(x.view(-1)[1:301][None], None, w, EPS)),
           (P.RowopsError, lambda: g(x, r, w, EPS, group=64)), (ValueError, lambda: g(x, r, w, EPS, y=y)), (ValueError, lambda: g(x, r, w, EPS, scale=s)),
           (ValueError, lambda: g(x, r, w, EPS, group=128, scale=s.half()))]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    torch.cuda.synchronize()


def test_a_group_past_32_bits_is_refused(way):
    x, r, w = make(6, 300, torch.float16)
    for group in (2 ** 32, 2 ** 32 + 128, -2 ** 32, 2 ** 40):
        with pytest.raises(ValueError):
            P.residual_rmsnorm_fwd_fp8(x, r, w, EPS, group=group)
    torch.cuda.synchronize()
