"""Group normalisation through the C ABI against the formulas in 64 bits.

Tolerances.  A thread sums at most 144 values in 32 bits (143 x 2^-24 < 2^-16.8 of the sum of their magnitudes at worst), forward about one of them, from which
they are at most twice as far as from their mean on average: SUM = 2^-15.  Sums of threads meet in 64 bits.  Each fp32 operation rounds by 2^-24 relative, a store to a type by eps / 2 of it, and the hardware's exp2 and reciprocal by about
2^-23, the exponent z log2(e) by |z| 2^-24."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_1312_6186_amd import binding as B

DEV = "cuda:0"
TDT = {B.F32: torch.float32, B.BF16: torch.bfloat16}
EPS = 1e-5
SUM = 2.0 ** -15
vp = ctypes.c_void_p


# ---- without a GPU: refusals come before any work on it
def _fwd(x=1 << 20, gamma=1 << 12, beta=1 << 13, y=1 << 24, mean=1 << 14, rstd=1 << 15, n=2, p=9, c=16, g=4, ldx=16, ldy=16, eps=EPS, act=1, dt=B.F32, ws=1 << 16):
    return B.lib().asgd_group_norm_fwd(vp(x), vp(gamma), vp(beta), vp(y), vp(mean), vp(rstd), n, p, c, g, ldx, ldy, ctypes.c_float(eps), act, dt, vp(ws), None)


def _bwd(dy=1 << 20, x=1 << 22, gamma=1 << 12, beta=1 << 13, mean=1 << 14, rstd=1 << 15, dx=1 << 24, dgamma=1 << 17, dbeta=1 << 18, n=2, p=9, c=16, g=4, lddy=16, ldx=16,
         lddx=16, act=1, dt=B.F32, ws=1 << 16):
    return B.lib().asgd_group_norm_bwd(vp(dy), vp(x), vp(gamma), vp(beta), vp(mean), vp(rstd), vp(dx), vp(dgamma), vp(dbeta), n, p, c, g, lddy, ldx, lddx, act, dt,
                                       vp(ws), None)


def test_bad_arguments_are_refused():
    for call in (_fwd, _bwd):
        assert call(dt=5) == B.EINVAL and call(act=3) == B.EINVAL and call(act=-1) == B.EINVAL
        assert call(n=-1) == B.ESHAPE and call(p=-1) == B.ESHAPE and call(c=0) == B.ESHAPE and call(g=0) == B.ESHAPE and call(g=3) == B.ESHAPE and call(g=32) == B.ESHAPE
        assert call(ldx=15) == B.ESHAPE and call(p=(1 << 30) + 1) == B.ESHAPE and call(n=1 << 30, g=4) == B.ESHAPE
        assert call(n=(1 << 22) + 1, p=0, g=4) == B.ESHAPE and call(ldx=(1 << 26) + 1) == B.ESHAPE and call(ldx=(1 << 27) + 1, dt=B.BF16) == B.ESHAPE
        assert call(x=0) == B.EINVAL and call(ws=0) == B.EINVAL
        assert call(x=(1 << 20) + 2) == B.EALIGN and call(x=(1 << 20) + 1, dt=B.BF16) == B.EALIGN and call(gamma=(1 << 12) + 2) == B.EALIGN
        assert call(mean=(1 << 14) + 2) == B.EALIGN and call(ws=(1 << 16) + 8) == B.EALIGN
    for eps in (0.0, -1.0, math.inf, math.nan):
        assert _fwd(eps=eps) == B.EINVAL
    assert _fwd(y=0) == B.EINVAL and _fwd(ldy=8) == B.ESHAPE
    assert _bwd(dy=0) == B.EINVAL and _bwd(dx=0) == B.EINVAL and _bwd(mean=0) == B.EINVAL and _bwd(rstd=0) == B.EINVAL
    assert _bwd(lddy=8) == B.ESHAPE and _bwd(lddx=8) == B.ESHAPE and _bwd(dgamma=(1 << 17) + 2) == B.EALIGN
    assert _fwd(n=0, x=0, y=0, ws=0) == B.OK and _fwd(p=0) == B.OK      # nothing to do


def test_partial_sums_beyond_32_bits_are_refused():
    wide = dict(c=1 << 16, n=1, x=1 << 40, ldx=1 << 16)
    for pixels in (1 << 17, 1 << 18):   # a pixel is a chunk: 2^33 sums of a group, and 2^24 workgroups
        assert _fwd(p=pixels, g=1 if pixels == 1 << 17 else 1 << 14, y=1 << 44, ldy=1 << 16, **wide) == B.ESHAPE and "too large" in B.asgd_last_error()
        assert _bwd(p=pixels, g=1 if pixels == 1 << 17 else 1 << 14, dy=1 << 42, dx=1 << 44, lddy=1 << 16, lddx=1 << 16, **wide) == B.ESHAPE


def test_overlapping_outputs_are_refused():
    x = 1 << 20
    for call, name in ((lambda **k: _fwd(x=x, **k), "y"), (lambda **k: _bwd(x=x, dy=1 << 22, **{("dx" if q == "y" else "lddx" if q == "ldy" else q): v for q, v in k.items()}), "dx")):
        assert call(y=x + 4) == B.EINVAL and "overlap" in B.asgd_last_error()
        assert call(y=x + 64, ldx=16) == B.EINVAL               # a pixel further on
        assert call(y=x, ldx=16, ldy=20) == B.EINVAL            # in place with another stride
        assert call(y=x + 60, ldx=32, ldy=32) == B.EINVAL       # columns that share one
        assert call(y=x - 4, ldx=32, ldy=32) == B.EINVAL
    assert _bwd(dy=x, dx=x + 4) == B.EINVAL


def test_workspace_sizes():
    assert B.asgd_group_norm_workspace_bytes(256, 3025, 96, 8, B.BF16) > 0
    assert B.asgd_group_norm_workspace_bytes(0, 9, 16, 4, B.F32) > 0
    assert B.asgd_group_norm_workspace_bytes(-1, 9, 16, 4, B.F32) == 0 and B.asgd_group_norm_workspace_bytes(1, 9, 16, 4, 9) == 0


class _Call(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("dtype", "act", "batch", "pixels", "channels", "groups")] + [(n, ctypes.c_long) for n in ("ldx", "lddy", "ldo")]


class _Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("vector", "uni", "threads", "regs", "width")]


def _plan(dtype, act, n, p, c, g, bwd):
    """Internal function, by its mangled name."""
    f = B.lib()["_ZN4asgd15group_norm_planERKNS_9GroupNormEb"]
    f.argtypes, f.restype = [ctypes.POINTER(_Call), ctypes.c_bool], _Plan
    return f(ctypes.byref(_Call(dtype, act, n, p, c, g, c, c, c)), bwd)


# images, pixels, channels, groups that between them take every kernel for slabs
SLABS = [(1, 1, 2, 1), (1, 1, 2, 2), (1, 1, 4, 4), (1, 1, 8, 1), (1, 1, 12, 1), (1, 1, 258, 2), (1, 1, 516, 4), (1, 7, 258, 2), (1, 13, 258, 2), (1, 17, 114, 2),
         (1, 17, 228, 4), (1, 18, 114, 2), (1, 29, 132, 4), (1, 33, 114, 2), (1, 33, 228, 4), (1, 36, 114, 2), (1, 66, 114, 2), (1, 85, 24, 1), (1, 145, 124, 4),
         (1, 205, 20, 4), (1, 261, 8, 1), (1, 340, 24, 1), (1, 341, 12, 1), (1, 355, 24, 1), (1, 392, 12, 1), (1, 445, 12, 1), (1, 457, 36, 4), (1, 528, 8, 1),
         (1, 598, 24, 1), (1, 645, 16, 1), (1, 706, 12, 1), (1, 920, 10, 2), (1, 1038, 2, 1), (1, 1048, 16, 1), (1, 1388, 12, 1), (1, 1395, 6, 1), (1, 1549, 24, 1),
         (1, 1554, 6, 1), (1, 1591, 12, 1), (1, 2052, 2, 1), (1, 2057, 4, 4), (1, 2594, 8, 1), (2, 1021, 12, 1), (9, 92, 224, 32), (9, 134, 64, 32), (9, 194, 192, 32),
         (9, 309, 224, 32), (40, 1, 64, 32), (40, 1, 160, 32), (40, 1, 256, 32), (40, 8, 288, 32), (40, 10, 144, 16), (40, 261, 64, 32), (150, 12, 176, 16),
         (150, 65, 516, 4)]


def test_slabs_of_every_kind_are_among_the_cases():
    kinds, threads, ragged = set(), set(), set()
    for n, p, c, g in SLABS:
        for dtype in (B.F32, B.BF16):
            for bwd in (False, True):
                q = _plan(dtype, B.ACT_RELU, n, p, c, g, bwd)
                if q.threads:
                    assert q.width <= q.threads and q.width % q.vector == 0 and (q.width == c or q.width % (c // g) == 0) and q.uni == ((c // g) % q.vector == 0)
                    rows = q.threads // (q.width // q.vector)
                    per = q.vector * (2 if dtype == B.BF16 else 4) // 4
                    assert -(-p // rows) * per <= q.regs                    # an image's pixels fit the registers
                    kinds.add((dtype, bwd, q.vector, q.uni, q.regs))
                    threads.add((dtype, bwd, q.threads))
                    ragged.add((dtype, bwd, c > q.width and c % q.width != 0))
    for dtype in (B.F32, B.BF16):
        for bwd, regs in ((False, (8, 16, 32, 72)), (True, (8, 16, 36, 72))):
            for vector, uni in ((4, 1), (4, 0), (2, 1), (2, 0)) if dtype == B.F32 else ((8, 1), (4, 1), (4, 0)):
                for r in regs:
                    assert (dtype, bwd, vector, uni, r) in kinds, (dtype, bwd, vector, uni, r)
            assert {(dtype, bwd, t) for t in (256, 512, 1024)} <= threads and (dtype, bwd, True) in ragged


# Calls (type, activation, images, pixels, channels, groups, backward) with the us by chunks and in slabs
WAYS = [(B.F32, 1, 8, 784, 8, 2, False, 9.6, 4.6), (B.BF16, 1, 256, 3025, 96, 8, False, 105.0, 74.3), (B.F32, 1, 128, 1024, 32, 8, True, 23.7, 15.7),
        (B.BF16, 1, 128, 729, 256, 32, True, 63.2, 42.2), (B.BF16, 2, 256, 3025, 96, 8, True, 173.3, 142.6), (B.F32, 1, 14, 3404, 14, 2, True, 14.7, 21.8),
        (B.BF16, 1, 33, 7120, 192, 32, True, 111.9, 228.8)]


def test_calls_go_the_faster_way():
    for dtype, act, n, p, c, g, bwd, chunks, slabs in WAYS:
        assert (_plan(dtype, act, n, p, c, g, bwd).threads > 0) == (slabs < chunks), (dtype, act, n, p, c, g, bwd)


# ---- on the GPU
# images, pixels, channels, groups, columns behind the channels, element the tensors start at
CASES = [(1, 1, 1, 1, 0, 0), (2, 1, 8, 2, 0, 0), (1, 3, 8, 8, 0, 0), (3, 7, 5, 5, 0, 0), (2, 49, 20, 4, 4, 0), (2, 50, 37, 1, 0, 0), (1, 2500, 96, 8, 0, 0),
         (4, 169, 384, 32, 0, 0), (2, 9, 4096, 16, 0, 0), (2, 5, 513, 27, 7, 0), (1, 4000, 8, 2, 0, 0), (130, 36, 16, 4, 0, 0), (3, 1000, 24, 2, 8, 0),
         (2, 300, 32, 4, 0, 1), (5, 121, 12, 3, 4, 3), (7, 64, 64, 32, 0, 0), (1, 257, 100, 20, 4, 0), (2, 33, 2056, 8, 0, 0)]
IDS = ["x".join(map(str, c)) for c in CASES]
SLAB_CASES = [(c + (0, 0), i % 3) for i, c in enumerate(SLABS)] + [(c + (0, 0), (i + 1) % 3) for i, c in enumerate(SLABS)]
SLAB_IDS = ["x".join(map(str, c[:4])) + "-%d" % a for c, a in SLAB_CASES]


def _tensor(rows, c, ld, shift, dtype, gen, offset=0.0, scale=1.0, fill=9.0):
    """[rows][c] values in rows of ld elements, the rest filled with a mark; the whole buffer and the view."""
    whole = torch.full((rows * ld + shift + 5,), fill, dtype=TDT[dtype], device=DEV)
    view = whole[shift:shift + rows * ld].view(rows, ld)[:, :c]
    view.copy_(torch.randn(rows, c, generator=gen, device=DEV) * scale + offset)
    return whole, view


def _params(c, dtype, gen):
    gamma = (1 + 0.3 * torch.randn(c, generator=gen, device=DEV)).to(TDT[dtype])
    gamma[::5] *= -1
    return gamma, (0.3 * torch.randn(c, generator=gen, device=DEV)).to(TDT[dtype])


def _workspace(n, p, c, g, dt):
    return torch.empty(B.asgd_group_norm_workspace_bytes(n, p, c, g, dt), dtype=torch.uint8, device=DEV).fill_(255)


def _act64(z, act):
    return z if act == B.ACT_NONE else torch.clamp(z, min=0) if act == B.ACT_RELU else z / (1 + torch.exp(-z))


def _ref_stats(x, n, p, c, g):
    v = x.double().reshape(n, p, g, c // g)
    mean = v.mean(dim=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(dim=(1, 3))
    return mean, 1 / torch.sqrt(var + EPS), torch.sqrt(var)


def _spread(t, n, p, c, g):   # [n][g] -> [n * p][c]
    return t.reshape(n, 1, g, 1).expand(n, p, g, c // g).reshape(n * p, c)


def _check_fwd(x, y, mean, rstd, gamma, beta, n, p, c, g, act, dtype):
    m64, r64, sd = _ref_stats(x, n, p, c, g)
    assert ((mean.double() - m64).abs() <= 2.0 ** -24 * m64.abs() + SUM * sd + 1e-30).all()
    assert ((rstd.double() / r64 - 1).abs() <= SUM).all()
    ga, be = (gamma.double() if gamma is not None else torch.ones(c, device=DEV, dtype=torch.float64)), (beta.double() if beta is not None else 0.0)
    m, r = _spread(m64, n, p, c, g), _spread(r64, n, p, c, g)
    h = (x.double() - m) * r
    z = h * ga + be
    ref = _act64(z, act)
    tol = ga.abs() * (SUM * _spread(sd * r64, n, p, c, g) + h.abs() * SUM + 2.0 ** -23 * (m * r).abs()) + 2.0 ** -22 * z.abs()
    if act == B.ACT_SILU:
        tol = 1.1 * tol + ref.abs() * 2.0 ** -20 * (1 + z.abs())
    tol = tol + torch.finfo(TDT[dtype]).eps / 2 * ref.abs() + 1e-30
    bad = (y.double() - ref).abs() > tol
    assert not bad.any(), ((y.double() - ref).abs() / tol).max().item()


@pytest.mark.gpu
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case, dtype, act):
    _forward(case, dtype, act)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("case,act", SLAB_CASES, ids=SLAB_IDS)
def test_slabs_forward(case, dtype, act):
    _forward(case, dtype, act)


def _forward(case, dtype, act):
    n, p, c, g, pad, shift = case
    gen = torch.Generator(device=DEV).manual_seed(1)
    ld = c + pad
    _, x = _tensor(n * p, c, ld, shift, dtype, gen, 0.4, 1.3)
    yw, y = _tensor(n * p, c, ld, shift, dtype, gen)
    gamma, beta = _params(c, dtype, gen)
    mean, rstd = torch.full((n, g), 7.0, device=DEV), torch.full((n, g), 7.0, device=DEV)
    mark = yw.clone()
    B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, ld, ld, EPS, act, dtype, _workspace(n, p, c, g, dtype))
    _check_fwd(x, y, mean, rstd, gamma, beta, n, p, c, g, act, dtype)
    # nothing but the channels is written
    keep = torch.ones_like(yw, dtype=torch.bool)
    keep[shift:shift + n * p * ld].view(n * p, ld)[:, :c] = False
    assert torch.equal(yw[keep], mark[keep])
    # the same again, without statistics; and in place
    y1 = y.clone()
    B.asgd_group_norm_fwd(x, gamma, beta, y, None, None, n, p, c, g, ld, ld, EPS, act, dtype, _workspace(n, p, c, g, dtype))
    assert torch.equal(y, y1)
    B.asgd_group_norm_fwd(x, gamma, beta, x, None, None, n, p, c, g, ld, ld, EPS, act, dtype, _workspace(n, p, c, g, dtype))
    assert torch.equal(x, y1)


def _ref_bwd(dy, x, gamma, beta, mean, rstd, n, p, c, g, act):
    """dx, dgamma, dbeta for the given mean and rstd, and what each may be off by (but for the store)."""
    ga = gamma.double() if gamma is not None else torch.ones(c, device=DEV, dtype=torch.float64)
    be = beta.double() if beta is not None else torch.zeros(c, device=DEV, dtype=torch.float64)
    m, r = _spread(mean.double(), n, p, c, g), _spread(rstd.double(), n, p, c, g)
    h = (x.double() - m) * r
    z = h * ga + be
    d = dy.double()
    e = torch.zeros_like(z)   # error of dz
    if act == B.ACT_RELU:
        dz = torch.where(z > 0, d, torch.zeros_like(d))
    elif act == B.ACT_SILU:
        s = 1 / (1 + torch.exp(-z))
        dz = d * s * (1 + z * (1 - s))
        e = d.abs() * 2.0 ** -20 * (1 + z * z + (m * r * ga).abs())
    else:
        dz = d
    M = p * (c // g)

    def groups(t):
        return _spread(t.reshape(n, p, g, c // g).sum(dim=(1, 3)), n, p, c, g) / M

    dh = ga * dz
    m1, m2 = groups(dh), groups(dh * h)
    dx = r * (dh - m1 - h * m2)
    t = 2.0 ** -21 * (dh.abs() + m1.abs() + (h * m2).abs()) + SUM * (groups(dh.abs()) + h.abs() * groups((dh * h).abs()))
    t = t + ga.abs() * e + groups(ga.abs() * e) + h.abs() * groups(ga.abs() * e * h.abs())
    return (dx, (dz * h).sum(0), dz.sum(0)), (r * t, SUM * (dz * h).abs().sum(0) + (e * h.abs()).sum(0), SUM * dz.abs().sum(0) + e.sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case, dtype, act):
    _backward(case, dtype, act)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("case,act", SLAB_CASES, ids=SLAB_IDS)
def test_slabs_backward(case, dtype, act):
    _backward(case, dtype, act)


def _backward(case, dtype, act):
    n, p, c, g, pad, shift = case
    gen = torch.Generator(device=DEV).manual_seed(2)
    ld = c + pad
    _, x = _tensor(n * p, c, ld, shift, dtype, gen, 0.4, 1.3)
    _, dy = _tensor(n * p, c, ld, shift, dtype, gen)
    dxw, dx = _tensor(n * p, c, ld, shift, dtype, gen)
    gamma, beta = _params(c, dtype, gen)
    m64, r64, _ = _ref_stats(x, n, p, c, g)
    mean, rstd = m64.float(), r64.float()
    dgamma, dbeta = torch.full((c,), 7.0, device=DEV), torch.full((c,), 7.0, device=DEV)
    mark = dxw.clone()

    def call(to, dg, db):
        B.asgd_group_norm_bwd(dy, x, gamma, beta, mean, rstd, to, dg, db, n, p, c, g, ld, ld, ld, act, dtype, _workspace(n, p, c, g, dtype))

    call(dx, dgamma, dbeta)
    (rx, rg, rb), (tx, tg, tb) = _ref_bwd(dy, x, gamma, beta, mean, rstd, n, p, c, g, act)
    tx = tx + torch.finfo(TDT[dtype]).eps / 2 * rx.abs() + 1e-30
    assert ((dx.double() - rx).abs() <= tx).all(), ((dx.double() - rx).abs() / tx).max().item()
    assert ((dgamma.double() - rg).abs() <= tg + 2.0 ** -23 * rg.abs() + 1e-30).all() and ((dbeta.double() - rb).abs() <= tb + 2.0 ** -23 * rb.abs() + 1e-30).all()
    keep = torch.ones_like(dxw, dtype=torch.bool)
    keep[shift:shift + n * p * ld].view(n * p, ld)[:, :c] = False
    assert torch.equal(dxw[keep], mark[keep])
    # without the parameters' gradients, one of them alone, and in the place of dy and of x
    dx1, dg1, db1 = dx.clone(), dgamma.clone(), dbeta.clone()
    call(dx, None, None)
    assert torch.equal(dx, dx1)
    dgamma.fill_(7.0)
    call(dx, dgamma, None)
    assert torch.equal(dgamma, dg1)
    dbeta.fill_(7.0)
    dy0 = dy.clone()
    call(dy, None, dbeta)
    assert torch.equal(dbeta, db1) and torch.equal(dy, dx1)
    dy.copy_(dy0)
    call(x, None, None)
    assert torch.equal(x, dx1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_no_scale_and_no_shift_are_one_and_zero(dtype):
    n, p, c, g = 3, 77, 24, 3
    gen = torch.Generator(device=DEV).manual_seed(3)
    x, dy = _tensor(n * p, c, c, 0, dtype, gen)[1], _tensor(n * p, c, c, 0, dtype, gen)[1]
    one, zero = torch.ones(c, dtype=TDT[dtype], device=DEV), torch.zeros(c, dtype=TDT[dtype], device=DEV)
    got = []
    for gamma, beta in ((None, None), (one, zero)):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd, dg, db = torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
        ws = _workspace(n, p, c, g, dtype)
        B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, c, c, EPS, B.ACT_RELU, dtype, ws)
        B.asgd_group_norm_bwd(dy, x, gamma, beta, mean, rstd, dx, dg, db, n, p, c, g, c, c, c, B.ACT_RELU, dtype, ws)
        got.append((y, dx, dg, db))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [300.0, -1e4])
@pytest.mark.parametrize("case", [(2, 900, 64, 8), (3, 50, 20, 4)])
def test_values_far_from_zero(case, offset):
    n, p, c, g = case
    gen = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(n * p, c, generator=gen, device=DEV) + offset
    y, mean, rstd = torch.empty_like(x), torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV)
    gamma, beta = _params(c, B.F32, gen)
    B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, c, c, EPS, B.ACT_NONE, B.F32, _workspace(n, p, c, g, B.F32))
    _check_fwd(x, y, mean, rstd, gamma, beta, n, p, c, g, B.ACT_NONE, B.F32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_constant_groups_and_one_outlier(dtype):
    n, p, c, g = 2, 100, 16, 2
    x = torch.full((n * p, c), 3.0, dtype=TDT[dtype], device=DEV)
    x[0, 0] = 1e4                      # the first value of the first group
    gamma, beta = torch.ones(c, dtype=TDT[dtype], device=DEV), torch.full((c,), 0.5, dtype=TDT[dtype], device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV)
    B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, c, c, EPS, B.ACT_NONE, dtype, _workspace(n, p, c, g, dtype))
    _check_fwd(x, y, mean, rstd, gamma, beta, n, p, c, g, B.ACT_NONE, dtype)
    assert (y[p:] == 0.5).all()        # the second image: nothing but its mean


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_values_that_are_not_finite_stay_in_their_group(dtype, act, value):
    n, p, c, g, ld = 3, 40, 24, 2, 32
    gen = torch.Generator(device=DEV).manual_seed(5)
    x, dy = _tensor(n * p, c, ld, 0, dtype, gen, fill=math.nan)[1], _tensor(n * p, c, ld, 0, dtype, gen, fill=math.nan)[1]   # NaN behind the channels, too
    gamma, beta = _params(c, dtype, gen)
    ws = _workspace(n, p, c, g, dtype)

    def both():
        y, dx = torch.zeros(n * p, c, dtype=TDT[dtype], device=DEV), torch.zeros(n * p, c, dtype=TDT[dtype], device=DEV)
        mean, rstd = torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV)
        B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, ld, c, EPS, act, dtype, ws)
        B.asgd_group_norm_bwd(dy, x, gamma, beta, mean, rstd, dx, None, None, n, p, c, g, ld, ld, c, act, dtype, ws)
        return y.reshape(n, p, g, c // g), dx.reshape(n, p, g, c // g)

    clean = both()
    assert all(bool(torch.isfinite(t).all()) for t in clean)
    x[p + 7, 13] = value               # image 1, group 1
    for before, after in zip(clean, both()):
        assert torch.isnan(after[1, :, 1].float()).all()
        after[1, :, 1] = before[1, :, 1]
        assert torch.equal(before, after)


@pytest.mark.gpu
@pytest.mark.parametrize("gamma", [1.0, -1.0, 0.75, -0.0078125, 0.0])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_relu_lets_gradients_through_where_its_input_is_positive(dtype, gamma):
    """dbeta counts the positive inputs: values on the edge, one step to either side of it, and around it, against exact fractions."""
    rng = np.random.default_rng(6)
    for mean, rstd, beta in ((3.0, 1.0, 0.5), (3.0, 1.0, 0.0), (-0.1, 2.7, -1.3), (1e-3, 300.0, 0.25), (0.7, 0.3, -0.40625)):
        mean, rstd = float(np.float32(mean)), float(np.float32(rstd))
        b = float(torch.tensor(beta, dtype=TDT[dtype]))
        edge = mean - b / (rstd * gamma) if gamma else mean
        vals = [edge + k * 2.0 ** -24 * abs(edge) for k in range(-4, 5)] + [float(edge + d) for d in rng.normal(size=50) * 1e-3] + [mean, 0.0, -0.0, 5.0, -5.0]
        x = torch.tensor(vals, dtype=torch.float64).to(torch.float32)
        if dtype == B.F32:
            near = x[:9].numpy()
            x = torch.cat([x, torch.from_numpy(np.nextafter(near, np.float32(np.inf))), torch.from_numpy(np.nextafter(near, np.float32(-np.inf)))])
        x = x.to(TDT[dtype])
        p = x.numel()
        want = sum(Fraction(gamma) * (Fraction(v) - Fraction(mean)) * Fraction(rstd) + Fraction(b) > 0 for v in x.double().tolist())
        t = lambda v: torch.tensor([v], device=DEV)
        xd = x.to(DEV)
        dbeta = torch.empty(1, device=DEV)
        B.asgd_group_norm_bwd(torch.ones_like(xd), xd, t(gamma).to(TDT[dtype]), t(b).to(TDT[dtype]), t(mean), t(rstd), torch.empty_like(xd), None, dbeta, 1, p, 1, 1,
                              1, 1, 1, B.ACT_RELU, dtype, _workspace(1, p, 1, 1, dtype))
        assert dbeta.item() == want, (mean, rstd, beta)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU])
def test_gradients_against_differences(act):
    """Of L = sum(y * dy) along random directions, the differences from the formulas in 64 bits.  The step of 2^-14 costs about its square.  Where a
    ReLU's input z crosses zero within the step, the difference of its output lies between 0 and that of z, and so does the derivative times the step:
    each such element may be off by |dy| |z(+step) - z(-step)| / (2 step)."""
    n, p, c, g = 2, 150, 24, 3
    gen = torch.Generator(device=DEV).manual_seed(7)
    x, dy = (torch.randn(n * p, c, generator=gen, device=DEV) for _ in range(2))
    gamma, beta = _params(c, B.F32, gen)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dgamma, dbeta = torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ws = _workspace(n, p, c, g, B.F32)
    B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, c, c, EPS, act, B.F32, ws)
    B.asgd_group_norm_bwd(dy, x, gamma, beta, mean, rstd, dx, dgamma, dbeta, n, p, c, g, c, c, c, act, B.F32, ws)

    def inputs(xx, ga, be):   # of the activation
        m, r, _ = _ref_stats(xx, n, p, c, g)
        return (xx - _spread(m, n, p, c, g)) * _spread(r, n, p, c, g) * ga + be

    at = [t.double() for t in (x, gamma, beta)]
    for i, grad in enumerate((dx, dgamma, dbeta)):
        for _ in range(3):
            u = torch.randn(at[i].shape, generator=gen, device=DEV).double()
            step = 2.0 ** -14
            lo, hi = list(at), list(at)
            hi[i], lo[i] = at[i] + step * u, at[i] - step * u
            z_hi, z_lo = inputs(*hi), inputs(*lo)
            diff = ((_act64(z_hi, act) - _act64(z_lo, act)) * dy.double()).sum().item() / (2 * step)
            got = (grad.double() * u).sum().item()
            crossing = ((z_hi - z_lo).abs() * dy.double().abs())[(z_hi > 0) != (z_lo > 0)].sum().item() / (2 * step) if act == B.ACT_RELU else 0.0
            assert abs(diff - got) <= 2.0 ** -15 * float(grad.double().norm() * u.norm()) + crossing


@pytest.mark.gpu
def test_columns_of_one_buffer_and_different_strides():
    n, p, c, g = 2, 60, 16, 4
    gen = torch.Generator(device=DEV).manual_seed(8)
    wide = torch.randn(n * p, 48, generator=gen, device=DEV)
    x, y = wide[:, 8:24], wide[:, 24:40]
    other = wide.clone()
    gamma, beta = _params(c, B.F32, gen)
    mean, rstd = torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV)
    ws = _workspace(n, p, c, g, B.F32)
    B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, 48, 48, EPS, B.ACT_SILU, B.F32, ws)
    _check_fwd(x, y, mean, rstd, gamma, beta, n, p, c, g, B.ACT_SILU, B.F32)
    assert torch.equal(wide[:, :24], other[:, :24]) and torch.equal(wide[:, 40:], other[:, 40:])
    dy, dx = torch.randn(n * p, 20, generator=gen, device=DEV), torch.zeros(n * p, 17, device=DEV)
    B.asgd_group_norm_bwd(dy, x, gamma, beta, mean, rstd, dx, None, None, n, p, c, g, 20, 48, 17, B.ACT_SILU, B.F32, ws)
    (rx, _, _), (tx, _, _) = _ref_bwd(dy[:, :c], x, gamma, beta, mean, rstd, n, p, c, g, B.ACT_SILU)
    assert ((dx[:, :c].double() - rx).abs() <= tx + 2.0 ** -24 * rx.abs()).all() and (dx[:, c:] == 0).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    n, p, c, g, ld = 2, 70000, 16, 2, 16384      # 2.3e9 elements apart from first to last
    dtype = B.BF16
    x = torch.empty(n * p * ld, dtype=torch.bfloat16, device=DEV).view(n * p, ld)
    gen = torch.Generator(device=DEV).manual_seed(9)
    x[:, :c] = torch.randn(n * p, c, generator=gen, device=DEV)
    gamma, beta = _params(c, dtype, gen)
    mean, rstd = torch.empty(n, g, device=DEV), torch.empty(n, g, device=DEV)
    ws = _workspace(n, p, c, g, dtype)
    B.asgd_group_norm_fwd(x, gamma, beta, x[:, c:], mean, rstd, n, p, c, g, ld, ld, EPS, B.ACT_RELU, dtype, ws)
    _check_fwd(x[:, :c], x[:, c:2 * c], mean, rstd, gamma, beta, n, p, c, g, B.ACT_RELU, dtype)
    B.asgd_group_norm_bwd(x[:, c:], x, gamma, beta, mean, rstd, x[:, 2 * c:], None, None, n, p, c, g, ld, ld, ld, B.ACT_RELU, dtype, ws)
    (rx, _, _), (tx, _, _) = _ref_bwd(x[:, c:2 * c], x[:, :c], gamma, beta, mean, rstd, n, p, c, g, B.ACT_RELU)
    assert ((x[:, 2 * c:3 * c].double() - rx).abs() <= tx + 2.0 ** -8 * rx.abs()).all()


@pytest.mark.gpu
def test_no_images_and_no_pixels():
    c, g = 16, 4
    for n, p in ((0, 9), (3, 0)):
        dgamma, dbeta = torch.full((c,), 7.0, device=DEV), torch.full((c,), 7.0, device=DEV)
        ws = _workspace(n, p, c, g, B.F32)
        B.asgd_group_norm_fwd(None, None, None, None, None, None, n, p, c, g, c, c, EPS, B.ACT_RELU, B.F32, ws)
        B.asgd_group_norm_bwd(None, None, None, None, None, None, None, dgamma, dbeta, n, p, c, g, c, c, c, B.ACT_RELU, B.F32, ws)
        assert (dgamma == 0).all() and (dbeta == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("case", [(4, 169, 48, 4), (2, 6000, 32, 8)])
def test_captured_calls_replay_and_streams_do_not_meet(case):
    """Forward and backward in one graph, replayed between eager calls on another stream with a workspace of their own."""
    n, p, c, g = case
    dtype = B.BF16
    gen = torch.Generator(device=DEV).manual_seed(10)
    x, dy = _tensor(n * p, c, c, 0, dtype, gen)[1].clone(), _tensor(n * p, c, c, 0, dtype, gen)[1].clone()
    gamma, beta = _params(c, dtype, gen)

    def buffers():
        return (torch.zeros_like(x), torch.zeros_like(x), torch.zeros(n, g, device=DEV), torch.zeros(n, g, device=DEV), torch.zeros(c, device=DEV),
                torch.zeros(c, device=DEV), _workspace(n, p, c, g, dtype))

    def work(b):
        y, dx, mean, rstd, dg, db, ws = b
        B.asgd_group_norm_fwd(x, gamma, beta, y, mean, rstd, n, p, c, g, c, c, EPS, B.ACT_RELU, dtype, ws)
        B.asgd_group_norm_bwd(dy, x, gamma, beta, mean, rstd, dx, dg, db, n, p, c, g, c, c, c, B.ACT_RELU, dtype, ws)

    held, eager = buffers(), buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(held)
    side = torch.cuda.Stream()
    for k in range(4):
        x.mul_(1.25 if k % 2 else -0.5)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            work(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held[:6], eager[:6]))
        for t in held[:6] + eager[:6]:
            t.zero_()
