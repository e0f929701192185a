"""4-bit operands and their products, the root-mean-square norm, log probabilities and clipping through the C boundary, against 64-bit
references (more_operator_refs.py), at the sizes, strides and values where they can go wrong; and a run of them together.

Tolerances are derived, not measured.  A rounding is off by half a step (relative 2^-24 in fp32, 2^-8 in bf16)."""
import numpy as np
import pytest
import torch

import more_operator_refs as M
import operator_refs as R
from gpu_util import DT
from paper_2203_12533_amd import binding as pwb
from paper_2203_12533_amd import inputs as I

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = {False: U, True: 2.0 ** -8}
TINY = 2.0 ** -120
F8 = {"e4m3": pwb.PW_E4M3, "e5m2": pwb.PW_E5M2}


@pytest.fixture(scope="module")
def ctx():
    with pwb.Context(0) as c:
        yield c


def up(n, m):
    return -(-n // m) * m


def act(bf16):
    return torch.bfloat16 if bf16 else torch.float32


def dev(a, dtype=torch.float32, ld=None, fill=0, offset=0):
    """A device array with rows ld apart, `offset` elements into its storage; what lies between the rows is `fill`."""
    a = np.atleast_2d(np.asarray(a))
    ld = a.shape[1] if ld is None else ld
    t = torch.full((a.shape[0] * ld + offset,), fill, dtype=dtype, device="cuda")
    v = t[offset:].view(a.shape[0], ld)
    v[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()
    torch.cuda.synchronize()
    return v


def full(rows, ld, value, dtype=torch.float32, offset=0):
    t = torch.full((rows * ld + offset,), value, dtype=dtype, device="cuda")[offset:].view(rows, ld)
    torch.cuda.synchronize()
    return t


def p(t):
    return t.data_ptr() if t is not None else None


def back(t):
    return t.detach().double().cpu().numpy()


def low(a, bf16):
    """The values a kernel sees."""
    a = np.asarray(a, np.float32)
    return (I.round_to_bf16(a) if bf16 else a).astype(np.float64)


def rnd(seed, *shape):
    return np.random.RandomState(seed).randn(*shape)


def within(got, ref, allow, name="", half_step=0.0):
    bad = R.exceeds(got, ref, allow, half_step)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d off, first at %s: got %r, want %r, allowed %r" % (
            name, bad.sum(), bad.size, i, np.asarray(got)[i], np.asarray(ref)[i], np.broadcast_to(allow, bad.shape)[i]))


# ---- quantisation to 4 bits ------------------------------------------------------------------------------------

def quantize(ctx, x, block, bf16=False, ldx=None, offset=0, rows_out=True, cols_out=True, spare=0):
    rows, cols = x.shape
    xt = dev(x, act(bf16), ldx, fill=float("nan"), offset=offset)
    ldq, ldqt = up(cols, 32) + 32 * spare, up(rows, 32) + 32 * spare
    q, qt = full(rows, ldq // 2, 0xAA, torch.uint8), full(cols, ldqt // 2, 0xAA, torch.uint8)
    s = full(1, pwb.f4_scale_bytes(rows, cols), 0xAA, torch.uint8)
    st = full(1, pwb.f4_scale_bytes(cols, rows), 0xAA, torch.uint8)
    on = lambda t, w: t.data_ptr() if w else None  # noqa: E731
    ctx.f4_quantize(pwb.F4QuantizeArgs(dtype=DT[bf16], block_rows=block, x=p(xt), rows=rows, cols=cols, ldx=xt.shape[1], q=on(q, rows_out),
                                       ldq=ldq if rows_out else 0, q_scale=on(s, rows_out), qt=on(qt, cols_out),
                                       ldqt=ldqt if cols_out else 0, qt_scale=on(st, cols_out)))
    ctx.synchronize()
    return tuple(t.cpu().numpy() for t in (q, s[0], qt, st[0]))


def check_quantized(ctx, x, block, bf16, **kw):
    v = low(x, bf16)
    q, s, qt, st = quantize(ctx, x, block, bf16, **kw)
    for on, got, table, want in ((kw.get("rows_out", True), q, s, v), (kw.get("cols_out", True), qt, st, np.ascontiguousarray(v.T))):
        if not on:
            assert (got == 0xAA).all() and (table == 0xAA).all()
            continue
        codes, byte = M.f4_quantize(want, block)           # 32 x 32 blocks are the same from either side
        packed = M.f4_pack(codes)
        assert np.array_equal(got[:, :packed.shape[1]], packed), np.argwhere(got[:, :packed.shape[1]] != packed)[:5]
        assert np.array_equal(table, M.f4_scale_table(byte))
        assert (got[:, packed.shape[1]:] == 0xAA).all() and got.shape[1] == packed.shape[1] + 16 * kw.get("spare", 0)


@pytest.mark.parametrize("block", [1, 32])
@pytest.mark.parametrize("rows,cols,bf16,kw", [
    (1, 1, False, {}), (1, 200, True, {}), (129, 127, True, {}), (64, 128, False, {}), (300, 257, False, {"ldx": 261, "offset": 3}),
    (70, 520, True, {"ldx": 523, "offset": 1, "spare": 2}), (200, 136, True, {"ldx": 144, "offset": 8, "cols_out": False}),
    (136, 200, False, {"rows_out": False}), (5, 16, True, {"spare": 1}), (257, 385, True, {}), (31, 33, False, {}), (96, 160, True, {})])
def test_f4_quantisation_is_exact(ctx, block, rows, cols, bf16, kw):
    check_quantized(ctx, rnd(rows + cols, rows, cols) * np.exp(2 * rnd(1, rows, 1)) * np.exp(rnd(2, 1, cols)), block, bf16, **kw)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [2, 7, 8, 9, 31, 32, 33, 63, 95, 97, 121, 124, 127, 128, 129, 135, 255])
def test_f4_quantisation_of_any_width(ctx, cols, bf16):
    check_quantized(ctx, rnd(cols, 131, cols) * np.exp(rnd(3, 1, cols)), 1, bf16, ldx=cols + 3, offset=1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("block", [1, 32])
def test_f4_quantisation_of_every_kind_of_value(ctx, block, bf16):
    """Blocks of zeros, of subnormals, of the largest numbers, with a maximum at a border of the scale, ties, NaN and infinities."""
    x = rnd(7, 140, 300).astype(np.float32)
    x[3] = 0.0
    x[4] = -0.0
    x[5, :128] = 1e-42
    x[6, :128] = np.float32(2.0 ** -149)
    x[7, 128:256] = np.finfo(np.float32).max if not bf16 else 3.3895e38
    x[8, 0], x[8, 1:32] = 1.5, np.linspace(-1.4, 1.4, 31)
    x[9, 0], x[9, 1:32] = np.nextafter(np.float32(1.5), np.float32(2)) if not bf16 else 1.5078125, np.linspace(-1.4, 1.4, 31)
    x[10, :8], x[10, 8:32] = M.E2M1, np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, -3.5, 6.0], 2)
    x[11, 5], x[11, 290] = np.nan, np.inf
    x[12, :128] = np.nan
    x[13, 128:256] = -np.inf
    x[20, 7], x[21, 7] = -np.inf, 3e30
    x[64 + 8, 40:60] = 6 * 2.0 ** -127
    x[64 + 9, 40:60] = 2.0 ** -125
    check_quantized(ctx, x, block, bf16)


# ---- products of 4-bit operands --------------------------------------------------------------------------------

def codes(seed, rows, k, spread=7):
    rng = np.random.RandomState(seed)
    return rng.randint(0, 16, (rows, k)).astype(np.uint8), rng.randint(127 - spread, 128 + spread, (rows, k // 32)).astype(np.uint8)


def product(ctx, m, n, k, epilogue=pwb.PW_EPI_STORE, bf16=False, accumulate=0, seed=0, lda=None, ldb=None, ldc=None, bias=True, nan_blocks=(),
            spread=7, exact=False, bias_scale=1.0):
    """Runs one product and checks everything it writes.  Returns C as the bits it has."""
    (a, sa), (b, sb) = codes(seed, m, k, 0 if exact else spread), codes(seed + 10, n, k, 0 if exact else spread)
    if exact:
        sa[:], sb[:] = 127, 127
    for r, blk in nan_blocks:                                # a block without a number in one row of A stays in that row of C
        sa[r, blk] = 255
    va, vb = M.f4_values(a, sa), M.f4_values(b, sb)
    lda, ldb, ldc = lda or k, ldb or k, ldc or up(n, 8)
    at, bt = dev(M.f4_pack(a), torch.uint8, lda // 2, fill=0x77), dev(M.f4_pack(b), torch.uint8, ldb // 2, fill=0x77)
    # what no row or block owns in the tables is a scale that would be seen in any sum
    ta, tb = M.f4_scale_table(sa), M.f4_scale_table(sb)
    for table, s in ((ta, sa), (tb, sb)):
        own = np.zeros(table.size, bool)
        own[M.f4_scale_index(*s.shape)] = True
        table[~own] = 255
    sat, sbt = torch.from_numpy(ta).cuda(), torch.from_numpy(tb).cuda()
    rng = np.random.RandomState(seed + 5)
    bias_v = (bias_scale * rng.randn(n)).astype(np.float32)
    biast = torch.from_numpy(bias_v).cuda()
    aux = c0 = c2 = auxt = None
    ct = full(m, ldc, 7.0, act(bf16))
    if epilogue == pwb.PW_EPI_BIAS_RESIDUAL:
        aux = rng.randn(m, n).astype(np.float32)
        auxt = dev(aux, torch.float32, ldc)
    elif epilogue == pwb.PW_EPI_GELU_BWD:
        aux = low(rng.randn(m, n), True)
        auxt = dev(aux, torch.bfloat16, ldc)
    elif epilogue == pwb.PW_EPI_BIAS_GELU:
        c2 = full(m, ldc, 7.0, act(bf16))
    if accumulate:
        c0 = rng.randn(m, n).astype(np.float32)
        ct[:, :n] = torch.from_numpy(c0).cuda()
    torch.cuda.synchronize()
    has_bias = epilogue in (pwb.PW_EPI_BIAS, pwb.PW_EPI_BIAS_RESIDUAL, pwb.PW_EPI_BIAS_GELU) and bias
    ctx.f4_gemm(pwb.F4GemmArgs(M=m, N=n, K=k, lda=lda, ldb=ldb, ldc=ldc, epilogue=epilogue, out_dtype=DT[bf16], accumulate=accumulate,
                               A=p(at), B=p(bt), a_scale=p(sat), b_scale=p(sbt), bias=p(biast) if has_bias else None, aux=p(auxt), C=p(ct), C2=p(c2)))
    ctx.synchronize()
    ref = va @ vb.T
    # a block's products are added exactly; each of the K / 32 block sums joins the others with an error of at most one unit of 24 bits
    # (2^-23) of a partial sum, which the sum of magnitudes bounds; up to eight waves' sums and the epilogue's additions
    mag = np.abs(va) @ np.abs(vb).T
    allow = 0.0 * mag if exact else (k // 32 + 8 + 4) * 2.0 ** -23 * mag
    if has_bias:                                             # sums may begin with it: then it is part of every partial sum, K / 32 of them
        ref, allow = ref + bias_v, allow + (k // 32 * 2.0 ** -23 + U) * np.abs(bias_v) + U * mag
    if accumulate:
        ref, allow = ref + c0, allow + U * (mag + np.abs(c0))
    if epilogue == pwb.PW_EPI_BIAS_RESIDUAL:
        ref, allow = ref + aux, allow + U * (mag + np.abs(aux) + np.abs(bias_v))
    if epilogue == pwb.PW_EPI_GELU_BWD:
        # gelu' within 2^-20: a handful of fp32 operations on values up to about 2, exp2 and rcp at one unit each
        g = R.gelu_grad(aux)
        ref, allow = ref * g, allow * np.abs(g) + 2.0 ** -20 * np.abs(ref) * (np.abs(g) + 1)
    got = back(ct)
    within(got[:, :n], ref, allow, "C", EPS[bf16])
    assert (got[:, n:] == 7.0).all(), "columns behind N were written"
    if epilogue == pwb.PW_EPI_BIAS_GELU:
        h = R.gelu(ref)
        within(back(c2)[:, :n], h, 1.13 * allow + 2.0 ** -20 * (np.abs(h) + np.abs(ref) * 0.01), "C2", EPS[bf16])
        assert (back(c2)[:, n:] == 7.0).all()
    return ct


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 8, 32), (1, 200, 128), (3, 24, 160), (16, 64, 256), (17, 65, 288), (64, 64, 128), (100, 130, 1056),
                                   (128, 128, 512), (130, 258, 416), (256, 256, 384), (300, 520, 2080), (33, 1000, 4096)])
def test_f4_product(ctx, m, n, k, bf16):
    product(ctx, m, n, k, bf16=bf16, seed=m + n)


EPILOGUES = [(pwb.PW_EPI_STORE, False, 1), (pwb.PW_EPI_BIAS, False, 0), (pwb.PW_EPI_BIAS, True, 0),
             (pwb.PW_EPI_BIAS_RESIDUAL, False, 0), (pwb.PW_EPI_BIAS_GELU, True, 0), (pwb.PW_EPI_BIAS_GELU, False, 0),
             (pwb.PW_EPI_GELU_BWD, True, 0), (pwb.PW_EPI_GELU_BWD, False, 0)]


@pytest.mark.parametrize("epilogue,bf16,accumulate", EPILOGUES)
@pytest.mark.parametrize("m,n,k", [(1, 120, 256), (40, 77, 160), (128, 256, 256), (260, 300, 544), (1500, 1420, 96), (2560, 4096, 256)])
def test_f4_product_epilogues(ctx, m, n, k, epilogue, bf16, accumulate):
    product(ctx, m, n, k, epilogue=epilogue, bf16=bf16, accumulate=accumulate, seed=m)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("k", [32, 128, 224, 256, 416, 1056])
@pytest.mark.parametrize("m,n", [(3, 5000), (260, 300), (500, 1300), (1300, 1100), (1700, 1900), (3100, 2900)])
def test_f4_product_every_tile_and_depth(ctx, m, n, k, bf16):
    """A size for each tile, none of them whole, with a piece of a k tile to several, the last of them partial or not."""
    product(ctx, m, n, k, bf16=bf16, epilogue=pwb.PW_EPI_BIAS, seed=k)


@pytest.mark.parametrize("m,n,k", [(1, 96, 512), (20, 700, 1056), (512, 512, 2048), (700, 900, 160), (1030, 1100, 544), (1500, 1420, 416),
                                   (2570, 4099, 288), (2560, 4096, 768)])
def test_f4_product_sums_are_exact(ctx, m, n, k):
    """Values of one scale: every sum is a multiple of 1/4 below 2^22, whatever the order; a k that is lost or taken twice shows."""
    product(ctx, m, n, k, exact=True, seed=5)


@pytest.mark.parametrize("m,n,k,kw", [(40000, 70, 160, {"bf16": True}), (70, 40000, 160, {"accumulate": 1}), (2560, 4096, 4096, {"bf16": True})])
def test_f4_product_many_tiles(ctx, m, n, k, kw):
    product(ctx, m, n, k, seed=2, **kw)


@pytest.mark.parametrize("m,n,k", [(3, 40, 1056), (300, 520, 416), (3100, 2900, 1056)])
def test_f4_product_beside_a_large_bias(ctx, m, n, k):
    product(ctx, m, n, k, epilogue=pwb.PW_EPI_BIAS, bias_scale=2.0 ** 24)


def test_f4_product_of_rows_far_apart(ctx):
    product(ctx, 3, 40, 160, lda=(1 << 24) + 32, bf16=True)
    product(ctx, 40, 3, 160, ldb=(1 << 24) + 32)
    product(ctx, 70, 40, 416, lda=1 << 24, epilogue=pwb.PW_EPI_BIAS)
    product(ctx, 70, 5000, 96, lda=1 << 24, epilogue=pwb.PW_EPI_BIAS)


def test_f4_product_strides_missing_bias_and_empty_sums(ctx):
    product(ctx, 70, 90, 160, lda=224, ldb=192, ldc=136, epilogue=pwb.PW_EPI_BIAS, bf16=True)
    product(ctx, 33, 40, 128, epilogue=pwb.PW_EPI_BIAS, bias=False)
    product(ctx, 50, 60, 1056, nan_blocks=((0, 3), (49, 32)))
    product(ctx, 1500, 1420, 288, nan_blocks=((0, 8), (200, 0), (1499, 7)), bf16=True)
    product(ctx, 65, 40, 256, spread=60)
    z = torch.zeros(64 * 64, dtype=torch.uint8, device="cuda")
    c, bias = full(5, 8, 3.0), torch.arange(8.0, device="cuda")
    torch.cuda.synchronize()
    k = dict(M=5, N=8, K=0, lda=32, ldb=32, ldc=8, out_dtype=pwb.PW_F32, A=p(z), B=p(z), a_scale=p(z), b_scale=p(z), C=p(c))
    ctx.f4_gemm(pwb.F4GemmArgs(epilogue=pwb.PW_EPI_STORE, accumulate=1, **k))       # nothing to add
    ctx.synchronize()
    assert (back(c) == 3.0).all()
    ctx.f4_gemm(pwb.F4GemmArgs(epilogue=pwb.PW_EPI_BIAS, bias=p(bias), **k))
    ctx.synchronize()
    assert np.array_equal(back(c), np.tile(np.arange(8.0), (5, 1)))


@pytest.mark.parametrize("m,n,k", [(3, 40, 64), (65, 40, 256), (300, 520, 160), (700, 904, 160), (1500, 1424, 160), (2560, 4096, 96)])
def test_f4_product_takes_a_residual_in_place(ctx, m, n, k):
    (a, sa), (b, sb) = codes(1, m, k), codes(2, n, k)
    va, vb = M.f4_values(a, sa), M.f4_values(b, sb)
    res = rnd(9, m, n).astype(np.float32)
    at, bt, c = dev(M.f4_pack(a), torch.uint8), dev(M.f4_pack(b), torch.uint8), dev(res)
    ta, tb = (torch.from_numpy(M.f4_scale_table(s)).cuda() for s in (sa, sb))
    torch.cuda.synchronize()
    ctx.f4_gemm(pwb.F4GemmArgs(M=m, N=n, K=k, lda=k, ldb=k, ldc=n, epilogue=pwb.PW_EPI_BIAS_RESIDUAL, out_dtype=pwb.PW_F32, A=p(at), B=p(bt),
                               a_scale=p(ta), b_scale=p(tb), aux=p(c), C=p(c)))
    ctx.synchronize()
    within(back(c), va @ vb.T + res, (k // 32 + 12) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T + np.abs(res)))


def test_f4_product_repeats_its_bits(ctx):
    for m, n, k in ((260, 300, 2080), (3, 700, 4096), (2560, 4096, 768)):
        x = [product(ctx, m, n, k, seed=3).clone() for _ in range(2)]
        assert torch.equal(x[0], x[1])


# ---- root-mean-square norm -------------------------------------------------------------------------------------

# Additions behind one another in a sum over a row: at most 8 vectors of 4 in a thread, six steps in a wave, 16 waves.
CHAIN = 32 + 6 + 16


def f8_check(h, q, table, fmt, bf16):
    """q against the fp32 values it is the rounding of, if they are known (h is fp32), else against h from 64 bits."""
    rows, cols = h.shape
    wq, e = R.quantize(h, fmt, 1)
    assert np.array_equal(table, R.scale_table(e))
    v = R.decode_table(fmt)
    same = (q[:, :wq.shape[1]] == wq) | (np.isnan(v[q[:, :wq.shape[1]]]) & np.isnan(v[wq]))
    assert same.all(), np.argwhere(~same)[:5]
    assert (q[:, wq.shape[1]:] == 0xAA).all()


def rms_forward(ctx, rows, cols, bf16, y=True, x_out="own", h=True, fmt=None, seed=0, ldx=0, ldh=0, offset=0, eps=1e-5, values=None, spare=0):
    ldx, ldh = ldx or cols, ldh or cols
    x = (rnd(seed, rows, cols) * np.exp(rnd(seed + 1, rows, 1))).astype(np.float32) if values is None else values
    yv = low(rnd(seed + 2, rows, cols), bf16) if y else None
    g = (1 + 0.2 * rnd(seed + 3, cols)).astype(np.float32)
    xt, gt = dev(x, ld=ldx, fill=float("nan"), offset=offset), dev(g, offset=offset)
    yt = dev(yv, act(bf16), ldh, fill=float("nan"), offset=offset) if y else None
    ot = xt if x_out == "same" else full(rows, ldx, 7.0, offset=offset) if x_out == "own" else None
    ht, rt = full(rows, ldh, 7.0, act(bf16), offset=offset) if h else None, full(1, rows + 2, 7.0, offset=1)
    out = None
    if fmt:
        ldq = up(cols, 16) + 16 * spare
        q, s = full(rows, ldq, 0xAA, torch.uint8), full(1, pwb.f8_scale_bytes(rows, cols), 0xAA, torch.uint8)
        out = pwb.F8Out(format=F8[fmt], q=p(q), ldq=ldq, scale=p(s))
    a = pwb.RmsnormArgs(dtype=DT[bf16], rows=rows, cols=cols, ldx=ldx, ldh=ldh, eps=eps, g=p(gt))
    ctx.rmsnorm_fwd(a, p(xt), p(yt), p(ot), p(ht), out, p(rt))
    ctx.synchronize()
    with np.errstate(over="ignore", invalid="ignore"):
        rx, rr, rh = M.rms_fwd((x + yv.astype(np.float32)).astype(np.float64) if y else x.astype(np.float64), None, g.astype(np.float64), eps)
    if ot is not None:
        got = back(ot)
        assert np.array_equal(got[:, :cols], rx, equal_nan=True), "x'"          # one addition, rounded once
        if x_out == "own":
            assert (got[:, cols:] == 7.0).all()
    # squares and their sum: 2^-24 each along a chain, halved by the root; division by the length, eps, root and reciprocal on top
    ar = (CHAIN / 2 + 6) * U
    within(back(rt)[0, :rows], rr, ar * rr, "rstd")
    assert (back(rt)[0, rows:] == 7.0).all()
    if h:
        within(back(ht)[:, :cols], rh, (ar + 3 * U) * np.abs(rh) + TINY, "h", EPS[bf16])
        assert (back(ht)[:, cols:] == 7.0).all()
    if fmt:
        qn, sn = q.cpu().numpy(), s.cpu().numpy()[0]
        if h and not bf16:
            f8_check(back(ht)[:, :cols], qn, sn, fmt, bf16)
        else:                      # the values that q stands for: half a step of the format, and of its smallest step at the block's scale
            e = sn[R.scale_index(rows, -(-cols // 128))].astype(np.int64) - 127
            v = R.values(qn[:, :up(cols, 16)], e, fmt)
            step = np.repeat(2.0 ** e * (2.0 ** -9 if fmt == "e4m3" else 2.0 ** -16), 128, 1)[:, :cols]
            within(v[:, :cols], rh, (ar + 3 * U) * np.abs(rh) * (1 + R.HALF_STEP[fmt]) + step / 2, "q", R.HALF_STEP[fmt])
            assert (qn[:, cols:up(cols, 16)] == 0).all()
    return rx, rr, g, rt


WIDTHS = [1, 3, 61, 64, 127, 129, 255, 256, 257, 500, 512, 513, 1000, 1024, 1025, 2048, 2050, 4096, 5000, 8192, 8200, 16384]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", WIDTHS)
def test_rms_norm_of_any_width(ctx, cols, bf16):
    rms_forward(ctx, 5, cols, bf16, fmt="e4m3", seed=cols, spare=1)
    rms_forward(ctx, 67, cols, bf16, y=False, x_out=None, fmt="e5m2", seed=cols, ldx=cols + 3, ldh=cols + 5, offset=1)
    rms_forward(ctx, 1, cols, bf16, x_out="same", seed=cols)


@pytest.mark.parametrize("rows,cols,kw", [(1, 2048, {}), (6000, 64, {}), (9000, 48, {"x_out": "same"}), (300, 2048, {"h": False}),
                                          (70, 640, {"h": False, "y": False, "x_out": None}), (5000, 1000, {"x_out": "same", "eps": 0.0}),
                                          (2100, 4100, {"y": False}), (3000, 1999, {"x_out": "same"}), (600, 1999, {"x_out": "same"})])
@pytest.mark.parametrize("bf16", [False, True])
def test_rms_norm_of_many_rows(ctx, rows, cols, kw, bf16):
    rms_forward(ctx, rows, cols, bf16, fmt="e4m3", seed=3, **kw)


def test_rms_norm_of_rows_without_a_value_and_with_special_ones(ctx):
    """Zero rows (eps keeps them finite), tiny and large ones, NaN and infinities that stay in their rows."""
    x = rnd(0, 12, 300).astype(np.float32)
    x[1] = 0.0
    x[2] = 1e-30
    x[3] = 3e18 * np.sign(x[3])
    x[4, 7] = np.nan
    x[5, 100] = np.inf
    x[6] = 0.0
    x[6, 299] = 1.0
    rms_forward(ctx, 12, 300, False, y=False, fmt="e4m3", values=x)
    rms_forward(ctx, 12, 300, True, y=False, fmt=None, values=x)
    rms_forward(ctx, 12, 300, False, y=False, fmt="e5m2", values=x)


def rms_backward(ctx, rows, cols, bf16, dres="own", dy=True, dg=True, accumulate=0, seed=0, ldx=0, ldh=0, offset=0, eps=1e-5):
    ldx, ldh = ldx or cols, ldh or cols
    x = (rnd(seed, rows, cols) * np.exp(rnd(seed + 1, rows, 1))).astype(np.float32).astype(np.float64)
    g = (1 + 0.2 * rnd(seed + 3, cols)).astype(np.float32).astype(np.float64)
    dh = low(rnd(seed + 4, rows, cols) * np.exp(rnd(seed + 5, 1, cols)), bf16)
    dr = rnd(seed + 6, rows, cols).astype(np.float32) if dres else None
    r = (1 / np.sqrt((x * x).mean(1) + eps)).astype(np.float32)
    xt, gt, rt = dev(x, ld=ldx, fill=float("nan"), offset=offset), dev(g, offset=offset), dev(r)
    dht = dev(dh, act(bf16), ldh, fill=float("nan"), offset=offset)
    drt = dev(dr, ld=ldx, fill=5.0, offset=offset) if dres else None
    dxt = drt if dres == "same" else full(rows, ldx, 5.0, offset=offset)
    dyt = full(rows, ldh, 7.0, act(bf16), offset=offset) if dy else None
    dg0 = rnd(seed + 7, cols).astype(np.float32)
    dgt = dev(dg0, offset=offset) if dg else None
    ws = full(1, pwb.rmsnorm_bwd_ws_floats(rows, cols) + 1, float("nan"))
    a = pwb.RmsnormArgs(dtype=DT[bf16], rows=rows, cols=cols, ldx=ldx, ldh=ldh, eps=eps, g=p(gt))
    ctx.rmsnorm_bwd(a, p(dht), p(xt), p(rt), p(drt), p(dxt), p(dyt), p(dgt), p(ws) if dg else None, accumulate)
    ctx.synchronize()
    rdx, rdg = M.rms_bwd(x, g, eps, dh, dr)
    # r comes rounded; xh, dh g and their product round, the mean's chain, then a product, a difference, a product, an addition
    r, xh, dhg = r[:, None].astype(np.float64), np.abs(x) * r[:, None], np.abs(dh * g)
    mean = (dhg * xh).mean(1, keepdims=True)
    allow = U * (r * (dhg * 6 + xh * mean * (CHAIN + 12)) + np.abs(rdx)) + (U * np.abs(dr) if dres else 0.0)
    within(back(dxt)[:, :cols], rdx, allow, "dx", U)
    assert (back(dxt)[:, cols:] == 5.0).all()
    if dy:
        within(back(dyt)[:, :cols], rdx, allow + U * np.abs(rdx), "dy", EPS[bf16])
        assert (back(dyt)[:, cols:] == 7.0).all()
    if dg:
        want = rdg + (dg0 if accumulate else 0.0)
        total = (np.abs(dh) * xh).sum(0)              # every row's term passes at most as many additions as there are rows, and 40
        within(back(dgt)[0], want, U * ((rows + 44) * total + np.abs(want)), "dg", U)
    return dxt, dgt


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", WIDTHS)
def test_rms_norm_gradients_of_any_width(ctx, cols, bf16):
    rms_backward(ctx, 5, cols, bf16, seed=cols)
    rms_backward(ctx, 70, cols, bf16, dres=None, accumulate=1, seed=cols, ldx=cols + 3, ldh=cols + 5, offset=1)
    rms_backward(ctx, 1, cols, bf16, dres="same", accumulate=1, seed=cols)


@pytest.mark.parametrize("rows,cols,kw", [(9000, 64, {}), (3000, 500, {"dres": "same"}), (2500, 2048, {"dy": False}), (2500, 1000, {"dg": False}),
                                          (700, 5000, {"accumulate": 1}), (3, 2048, {"accumulate": 1, "dres": None}), (4, 2048, {}), (5, 2048, {}),
                                          (3000, 1999, {"dres": "same"}), (2500, 301, {"dres": "same"}), (300, 9001, {"dres": "same"})])
@pytest.mark.parametrize("bf16", [False, True])
def test_rms_norm_gradients_of_many_rows(ctx, rows, cols, kw, bf16):
    rms_backward(ctx, rows, cols, bf16, seed=1, **kw)


def test_rms_norm_gradients_repeat_their_bits_and_take_no_rows(ctx):
    a, b = rms_backward(ctx, 3000, 1000, True), rms_backward(ctx, 3000, 1000, True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    dg, one = full(1, 11, 3.0, offset=1), full(1, 16, 1.0)
    args = pwb.RmsnormArgs(dtype=0, rows=0, cols=10, ldx=10, ldh=10, eps=1e-5, g=p(one))
    ctx.rmsnorm_fwd(args, p(one), None, None, p(one), None, None)
    ctx.rmsnorm_bwd(args, p(one), p(one), p(one), None, p(one), None, p(dg), None, 1)
    ctx.synchronize()
    assert (back(dg) == 3.0).all() and (back(one) == 1.0).all()
    ctx.rmsnorm_bwd(args, p(one), p(one), p(one), None, p(one), None, p(dg), None, 0)
    ctx.synchronize()
    assert (back(dg)[0, :10] == 0.0).all() and back(dg)[0, 10] == 3.0


# ---- log probabilities -----------------------------------------------------------------------------------------

def shifts(z, scale):
    """d = s (z - max), magnitudes with those that matter nowhere left out, for the bounds."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        m = z.max(1, keepdims=True)
        d = np.abs(scale * (z - np.where(np.isfinite(m), m, 0.0)))
    return np.where(np.isfinite(d), d, 0.0)


def logp_bounds(z, scale):
    """Errors of log p_v, of H; and |d|.  With u = 2^-24: the factor s log2 e is off by 2 u, a shift d by 3 u |d| then, exp2 by 2 u of itself
    and its sum by u per addition: 64 in a thread for each chunk that it sees and 16 where threads meet; log2 by 2 u of itself and of 1."""
    d = shifts(z, scale)
    vocab = z.shape[1]
    with np.errstate(invalid="ignore"):
        pr = np.exp(M.log_softmax(z, scale))
    pr = np.where(np.isfinite(pr), pr, 0.0)
    chain = 64 * -(-vocab // 8192) + 16
    e1, e2 = (pr * d).sum(1, keepdims=True), (pr * d * d).sum(1, keepdims=True)
    big = np.log(vocab) + 1
    lp = U * (4 * d + 3 * e1 + chain + 8 + 4 * big)
    h = U * ((chain + 8) * (2 + e1) + 4 * e2 + 8 * e1 + 4 * big)
    return lp, h[:, 0], d, pr


def logprob(ctx, z, targets, scale=1.0, k=0, bf16=False, ldz=None, offset=0, backward=True, in_place=False, seed=0, parts="both", lddz=None):
    rows, vocab = z.shape
    v = low(z, bf16)
    zt = dev(z, act(bf16), ldz, fill=float("nan"), offset=offset)
    tt = torch.from_numpy(np.asarray(targets, np.int32)).cuda()
    lp, en, st = full(1, rows + 1, 7.0, offset=1), full(1, rows + 1, 7.0, offset=1), full(rows, 2, 7.0)
    ids, tl = (full(rows, k, 7, torch.int32), full(rows, k, 7.0)) if k else (None, None)
    ws = full(1, pwb.logprob_ws_floats(rows, vocab, k) + 1, float("nan"))
    a = pwb.LogprobArgs(dtype=DT[bf16], z=p(zt), ldz=zt.shape[1], rows=rows, vocab=vocab, targets=p(tt), scale=scale)
    ctx.logprob_fwd(a, p(lp), p(en), p(st), k, p(ids), p(tl), p(ws))
    ctx.synchronize()
    s = float(np.float32(scale))
    rlp, rh, rid, rtl = M.logprob_fwd(v, np.asarray(targets), s, k)
    elp, eh, d, pr = logp_bounds(v, s)
    # below -(2 - 2^-24) 2^127 the nearest of fp32's values is -infinity: twice the lowest value has no other
    rlp, rtl = (np.where(r <= -(2 - 2.0 ** -24) * 2.0 ** 127, -np.inf, r) for r in (rlp, rtl))
    t = np.asarray(targets)
    given = (t >= 0) & (t < vocab)
    at = elp[np.arange(rows), np.where(given, t, 0)]
    within(back(lp)[0, :rows], rlp, at, "logp", U)
    within(back(en)[0, :rows], rh, eh, "entropy", U)
    assert back(lp)[0, rows] == back(en)[0, rows] == 7.0
    if k:
        assert np.array_equal(ids.cpu().numpy(), rid), (ids.cpu().numpy()[:3], rid[:3])
        within(back(tl), rtl, np.take_along_axis(elp, np.where(rid < 0, 0, rid), 1), "top", U)
    if not backward:
        return lp, en, st, ids, tl
    dl, de = rnd(seed + 1, rows).astype(np.float32), rnd(seed + 2, rows).astype(np.float32)
    dlt, det = torch.from_numpy(dl).cuda(), torch.from_numpy(de).cuda()
    out = zt if in_place else full(rows, lddz or vocab, 7.0, act(bf16), offset=offset)
    torch.cuda.synchronize()
    with_l, with_h = parts in ("both", "logp"), parts in ("both", "entropy")
    ctx.logprob_bwd(a, p(st), p(en) if with_h else None, p(dlt) if with_l else None, p(det) if with_h else None, p(out), out.shape[1])
    ctx.synchronize()
    dl, de = dl * with_l, de * with_h
    ref = M.logprob_bwd(v, t, dl.astype(np.float64), de.astype(np.float64), s)
    with np.errstate(invalid="ignore"):
        lpv = M.log_softmax(v, s)
    lpv = np.where(np.isfinite(lpv), lpv, 0.0)
    dl, de = np.abs(np.where(given, dl, 0.0))[:, None], np.abs(de)[:, None]
    h = np.abs(np.where(np.isfinite(rh), rh, 0.0))[:, None]
    # an error of log p is one of p, relative; the products and additions of the formula on top; p below 2^-126 may be 0, whatever it is multiplied
    # with then, s (dl + de (|log p| + H)), and so may the result
    hot = np.zeros_like(ref)
    hot[np.arange(rows)[given], t[given]] = 1.0
    allow = s * (pr * (dl * (elp + 8 * U) + de * (elp * (np.abs(lpv) + h + 1) + eh[:, None] + 8 * U * (np.abs(lpv) + h))) + 4 * U * dl * hot) + TINY + 2.0 ** -125 * s * (dl + de * (np.abs(lpv) + h))
    allow = np.where(np.isfinite(allow), allow, 0.0)
    within(back(out)[:, :vocab], ref, allow, "dz", EPS[bf16])
    if not in_place:
        assert (back(out)[:, vocab:] == 7.0).all()
    return out


VOCABS = [1, 2, 7, 64, 100, 255, 1000, 4099, 8192, 8193, 16384, 16391, 32768, 50001]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", VOCABS)
def test_log_probabilities_of_any_vocabulary(ctx, vocab, bf16):
    z = 3 * rnd(vocab, 5, vocab)
    t = np.random.RandomState(1).randint(0, vocab, 5)
    t[2], t[4] = -1, vocab
    logprob(ctx, z, t, 1.0, min(8, vocab), bf16, seed=vocab)
    logprob(ctx, z, t, 0.7, min(32, vocab + 3), bf16, ldz=vocab + 3, offset=1, in_place=True)
    logprob(ctx, z, t, 1.7, 1, bf16, lddz=vocab + 1, offset=1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", [256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 16385, 32769])
def test_log_probabilities_where_one_kernel_takes_over_from_another(ctx, vocab, bf16):
    z = 3 * rnd(vocab, 3, vocab)
    z[1, 0], z[2, vocab - 1] = 40.0, 40.0                     # the likeliest is the first, the last
    logprob(ctx, z, [0, vocab - 1, vocab // 2], 1.0, 9, bf16, seed=vocab)
    logprob(ctx, np.tile(z, (200, 1))[:520], np.arange(520) % vocab, 1.0, 3, bf16, seed=vocab)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,vocab,k", [(300, 500, 4), (600, 9000, 32), (300, 40000, 20), (257, 8200, 0), (1000, 61, 32)])
def test_log_probabilities_of_many_rows(ctx, rows, vocab, k, bf16):
    logprob(ctx, 2 * rnd(rows, rows, vocab), np.random.RandomState(2).randint(-1, vocab, rows), 1.0, k, bf16)


def test_log_probabilities_of_more_rows_than_a_launch_has_threads_for(ctx):
    rows, vocab = (1 << 26) + 5, 3
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, 1 << 25, (1 << 26) - 1, 1 << 26, rows - 1], device="cuda")
    z[at] = torch.arange(at.numel() * vocab, device="cuda").reshape(-1, vocab).remainder(7).to(torch.bfloat16)
    t = torch.ones(rows, dtype=torch.int32, device="cuda")
    lp, en, st = (torch.full((rows, n), 7.0, device="cuda") for n in (1, 1, 2))
    ids, tl = torch.zeros(rows, 1, dtype=torch.int32, device="cuda"), torch.zeros(rows, 1, device="cuda")
    torch.cuda.synchronize()
    a = pwb.LogprobArgs(dtype=pwb.PW_BF16, z=p(z), ldz=vocab, rows=rows, vocab=vocab, targets=p(t), scale=1.0)
    ctx.logprob_fwd(a, p(lp), p(en), p(st), 1, p(ids), p(tl), None)
    ctx.logprob_bwd(a, p(st), p(en), p(st), None, p(z), vocab)             # dlogp: any array of that length
    ctx.synchronize()
    v = np.arange(at.numel() * vocab).reshape(-1, vocab) % 7
    rlp, rh, rid, rtl = M.logprob_fwd(v.astype(np.float64), np.ones(at.numel(), np.int64), 1.0, 1)
    elp, eh, _, _ = logp_bounds(v.astype(np.float64), 1.0)
    within(back(lp[at])[:, 0], rlp, elp[:, 1], "logp", U)
    within(back(en[at])[:, 0], rh, eh, "entropy", U)
    assert np.array_equal(ids[at].cpu().numpy(), rid)
    within(back(tl[at]), rtl, np.take_along_axis(elp, rid, 1), "top", U)
    zeros = torch.ones(rows, dtype=torch.bool, device="cuda")
    zeros[at] = False
    assert torch.isclose(lp[zeros], torch.tensor(-np.log(3.0), dtype=torch.float32, device="cuda"), rtol=1e-5).all()
    assert (ids[zeros] == 0).all() and (st[zeros, 0] == 0).all()


@pytest.mark.parametrize("parts", ["logp", "entropy"])
def test_log_probabilities_with_one_gradient_only(ctx, parts):
    logprob(ctx, 2 * rnd(3, 7, 700), np.arange(7) * 90, 1.3, 0, True, parts=parts)
    logprob(ctx, 2 * rnd(3, 7, 701), np.arange(7) * 90, 1.3, 0, False, parts=parts, in_place=True)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows", [9, 300])
def test_alternatives_where_values_are_alike_or_in_order(ctx, rows, bf16):
    """Rows of one value, of two, ascending, descending, with their largest in one thread's or group's columns, with fewer tokens than
    asked for, with zeros of both signs; the lowest index first among equals, whatever block and thread has it."""
    V = 40000 if rows == 9 else 20000
    z = np.tile(rnd(0, 1, V).astype(np.float32), (rows, 1))
    z[0] = 1.25
    z[1] = np.where(np.arange(V) % 7 == 3, 2.0, -1.0)
    z[2] = np.arange(V) * 0.01
    z[3] = -np.arange(V) * 0.01
    z[4] = -5.0
    z[4, 64:96] = np.arange(32)
    z[5] = -np.inf
    z[5, [5, 17, 12345, V - 1]] = [1.0, 1.0, 3.0, -2.0]
    z[6] = np.where(np.arange(V) % 2 == 0, -0.0, 0.0)
    z[7] = np.where(np.arange(V) % 64 < 8, 4.0 + (np.arange(V) // 64) % 50, -4.0)      # one lane in eight
    z[8] = np.where(np.arange(V) % 8192 < 16, np.arange(V) * 1e-3, -1.0)
    t = np.arange(rows) % V
    for k in (1, 5, 32):
        logprob(ctx, z, t, 1.0, k, bf16, backward=False)


@pytest.mark.parametrize("bf16", [False, True])
def test_log_probabilities_of_masked_rows_and_special_values(ctx, bf16):
    """Masks of -infinity and of the type's lowest value, rows that a mask leaves empty, NaN and +infinity, logits near overflow."""
    V = 9000
    lowest = -3.3895313892515355e38 if bf16 else float(np.finfo(np.float32).min)
    z = 2 * rnd(0, 16, V).astype(np.float32)
    z[0, 100:] = -np.inf
    z[1] = -np.inf
    z[2, 10:8999] = lowest
    z[3] = lowest
    z[4, 4500] = np.nan
    z[5, 77] = np.inf
    z[6] = -np.inf
    z[6, 8999] = np.nan
    z[7] = -np.inf
    z[7, 42] = 1.0
    z[8, :5] = 3e38
    z[9] = 2e38 + 1e35 * z[9]
    z[10] = -2e38 + 1e35 * z[10]
    z[11] = -np.inf
    z[11, 3:9] = lowest
    z[12] = 1e4 + z[12]
    z[13] = -np.inf
    z[13, 1] = np.inf
    z[14] *= 40
    t = np.array([5, 6, 10, 3, 4, 5, 6, 42, 4, 9, 10, 8, 12, 13, int(np.argmax(z[14])), 0])
    logprob(ctx, z, t, 1.0, 7, bf16)
    logprob(ctx, z, t, 2.0, 7, bf16, backward=False)
    t[[0, 7, 11]] = [200, 41, 100]                              # a masked token is the given one
    logprob(ctx, z, t, 0.5, 0, bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", [300, 9000])
def test_log_probabilities_of_rows_far_from_zero(ctx, vocab, bf16):
    """Maxima of any size, several of them in a row, and logits a few steps of the type below: differences are what counts."""
    tops = np.array([s * m for m in (1000.0, 2.0 ** 21, 4.1e6, 5e6, 3e7, 2.0 ** 28, 1e10, 3e14, 1e20, 1e30, 5e37) for s in (1, -1)])
    step = np.exp2(np.floor(np.log2(np.abs(tops))) - (7 if bf16 else 23))
    back_by = np.random.RandomState(3).randint(0, 30, (tops.size, vocab))
    z = low(tops, bf16)[:, None] - np.where(tops < 0, 1, 0.5)[:, None] * step[:, None] * back_by
    t = np.arange(tops.size) * 7
    for k, scale in ((5, 1.0), (0, 0.7), (0, 1e-7), (3, 37.0)):
        z[:, [11, vocab - 1]] = low(tops, bf16)[:, None]
        logprob(ctx, z, t, scale, k, bf16)


def test_log_probabilities_write_what_is_asked_for_and_repeat_their_bits(ctx):
    z = 2 * rnd(0, 40, 5000)
    t = np.arange(40)
    a = logprob(ctx, z, t, 1.0, 9, True, backward=False)
    b = logprob(ctx, z, t, 1.0, 9, True, backward=False)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    zt, en = dev(z, torch.bfloat16), full(1, 40, 7.0)
    args = pwb.LogprobArgs(dtype=pwb.PW_BF16, z=p(zt), ldz=5000, rows=40, vocab=5000, scale=1.0)
    ctx.logprob_fwd(args, None, p(en), None)
    ctx.synchronize()
    assert torch.equal(en[0], a[1][0, :40])
    ids, tl = full(40, 9, 0, torch.int32), full(40, 9, 0.0)
    ctx.logprob_fwd(args, None, None, None, 9, p(ids), p(tl))
    ctx.synchronize()
    assert torch.equal(ids, a[3]) and torch.equal(tl, a[4])
    args.rows = 0
    ctx.logprob_fwd(args, None, p(en), None)


# ---- clipping --------------------------------------------------------------------------------------------------

def clip(ctx, sizes, bf16s, max_norm, std=1.0, in_place=False, skip=(), offset=0, values=None):
    gs = [low(std * rnd(i, n), b) for i, (n, b) in enumerate(zip(sizes, bf16s))] if values is None else values
    make = lambda v, b: torch.full((v.size + offset + 3,), 7.0, dtype=act(b), device="cuda")  # noqa: E731
    gt, ot = [], []
    for i, (v, b) in enumerate(zip(gs, bf16s)):
        t = make(v, b)
        t[offset:offset + v.size] = torch.from_numpy(v.astype(np.float32)).to(act(b)).cuda()
        gt.append(t)
        ot.append(None if i in skip else t if in_place else make(v, b))
    res, ws = full(1, 3, 7.0, offset=1), full(1, pwb.grad_clip_ws_floats(), float("nan"))
    at = lambda t, b: None if t is None else t.data_ptr() + offset * (2 if b else 4)  # noqa: E731
    ts = pwb.grad_tensors([(at(g, b), at(o, b), v.size, DT[b]) for g, o, v, b in zip(gt, ot, gs, bf16s)])
    torch.cuda.synchronize()
    ctx.grad_clip(ts, max_norm, p(res), p(ws))
    ctx.synchronize()
    norm, factor, want = M.clip(gs, float(np.float32(max_norm)))
    r = back(res)[0]
    within(r[:2], np.array([norm, factor]), np.array([norm, factor]) * 2.0 ** -40, "norm, factor", U)
    assert r[2] == 7.0
    for i, (o, w, b) in enumerate(zip(ot, want, bf16s)):
        if o is None:
            assert np.array_equal(back(gt[i])[offset:offset + w.size], gs[i])
            continue
        got = back(o)
        within(got[offset:offset + w.size], w, 1.01 * U * np.abs(w), "g", EPS[b])          # the factor is rounded, then the product
        assert (got[:offset] == 7.0).all() and (got[offset + w.size:] == 7.0).all()
        if factor == 1.0:
            assert np.array_equal(got[offset:offset + w.size], gs[i])
    return r, ot


@pytest.mark.parametrize("sizes,bf16s,max_norm,kw", [
    ([1], [False], 0.5, {}), ([0, 5, 0], [False, True, True], 0.1, {}), ([8192, 8193, 16383, 3], [False, True, False, True], 1.0, {}),
    ([100000], [True], 1e9, {}), ([100000, 70], [False, True], 1e9, {"in_place": True}), ([30000, 20000], [False, True], 2.0, {"in_place": True, "offset": 1}),
    ([30011, 20007], [True, False], 2.0, {"offset": 3}), ([5000, 9000, 17], [False, True, False], 1.0, {"skip": (1,)}),
    ([5000, 9000], [False, False], 1.0, {"skip": (0, 1)}), ([20] * 250, [False, True] * 125, 3.0, {}),
    ([3] * 97 + [200000] + [40] * 100, [False] * 198, 3.0, {}), ([9000] * 96, [True] * 96, 0.0, {}), ([9000000], [False], 10.0, {}),
    ([9000001, 123], [True, True], float("inf"), {})])
def test_gradients_are_clipped_together(ctx, sizes, bf16s, max_norm, kw):
    clip(ctx, sizes, bf16s, max_norm, **kw)


def test_norm_of_values_whose_squares_leave_32_bits(ctx):
    for v in (1e30, 1e-30, 1e-42):
        x = np.full(20000, np.float32(v)).astype(np.float64)
        clip(ctx, [x.size, 100], [False, False], float(np.float32(1.0)), values=[x, x[:100]])
    r, _ = clip(ctx, [5], [False], 1.0, values=[np.zeros(5)])
    assert r[0] == 0.0 and r[1] == 1.0


def test_clipping_of_nothing_of_infinities_and_of_nan(ctx):
    res, ws = full(1, 2, 7.0), full(1, pwb.grad_clip_ws_floats(), float("nan"))
    ctx.grad_clip(pwb.grad_tensors([]), 1.0, p(res), p(ws))
    ctx.synchronize()
    assert back(res)[0].tolist() == [0.0, 1.0]
    g = dev(np.array([1.0, np.inf, -2.0]))
    ctx.grad_clip(pwb.grad_tensors([(p(g), p(g), 3, pwb.PW_F32)]), 1.0, p(res), p(ws))
    ctx.synchronize()
    assert back(res)[0].tolist() == [np.inf, 0.0]
    assert np.array_equal(back(g)[0], [0.0, np.nan, -0.0], equal_nan=True)
    g = dev(np.array([1.0, np.nan, -2.0]))
    ctx.grad_clip(pwb.grad_tensors([(p(g), p(g), 3, pwb.PW_F32)]), 1.0, p(res), p(ws))
    ctx.synchronize()
    assert np.isnan(back(res)).all() and np.isnan(back(g)).all()


def test_clipping_repeats_its_bits(ctx):
    a, b = (clip(ctx, [300000, 1001, 70000], [False, True, False], 1.0) for _ in range(2))
    assert np.array_equal(a[0], b[0]) and all(torch.equal(x, y) for x, y in zip(a[1], b[1]))


# ---- offsets, graphs, two contexts -----------------------------------------------------------------------------

def test_more_operators_at_sizes_past_32_bits_of_offset(ctx):
    """Rows whose offset does not fit 32 bits, in elements and in bytes: the last rows of a strided array."""
    rows, cols, ld = 66000, 40, 1 << 16
    try:
        x = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")     # 8.6 GB, of which little is touched
    except torch.OutOfMemoryError:
        pytest.skip("no room")
    v = x.view(rows, ld)
    vals = low(rnd(0, rows, cols), True)
    v[:, :cols] = torch.from_numpy(vals).cuda().bfloat16()
    q, s = full(rows, 32, 0, torch.uint8), full(1, pwb.f4_scale_bytes(rows, cols), 0, torch.uint8)
    ctx.f4_quantize(pwb.F4QuantizeArgs(dtype=pwb.PW_BF16, block_rows=1, x=p(x), rows=rows, cols=cols, ldx=ld, q=p(q), ldq=64, q_scale=p(s)))
    ctx.synchronize()
    c, _ = M.f4_quantize(vals[-50:])
    assert np.array_equal(q.cpu().numpy()[-50:], M.f4_pack(c))
    en, st, ids, tl = full(1, rows, 0.0), full(rows, 2, 0.0), full(rows, 2, 0, torch.int32), full(rows, 2, 0.0)
    a = pwb.LogprobArgs(dtype=pwb.PW_BF16, z=p(x), ldz=ld, rows=rows, vocab=cols, scale=1.0)
    ctx.logprob_fwd(a, None, p(en), p(st), 2, p(ids), p(tl))
    de = full(1, rows, 1.0)
    ctx.logprob_bwd(a, p(st), p(en), None, p(de), p(x) + 2 * cols, ld)
    ctx.synchronize()
    none = np.full(50, -1)
    _, h, rid, _ = M.logprob_fwd(vals[-50:], none, 1.0, 2)
    assert np.array_equal(ids.cpu().numpy()[-50:], rid)
    _, eh, _, _ = logp_bounds(vals[-50:], 1.0)
    within(back(en)[0, -50:], h, eh, "H", U)
    within(back(v[-50:, cols:2 * cols]), M.logprob_bwd(vals[-50:], none, np.zeros(50), np.ones(50)), 1e-5, "dz", EPS[True])
    g, r = full(1, cols, 1.0), full(1, rows, 0.0)
    small = full(rows, cols, 1.0)
    ctx.rmsnorm_fwd(pwb.RmsnormArgs(dtype=pwb.PW_BF16, rows=rows, cols=cols, ldx=cols, ldh=ld, eps=1e-5, g=p(g)), p(small), p(x), p(small),
                    p(x) + 2 * cols, None, p(r))
    ctx.synchronize()
    rx, rr, rh = M.rms_fwd(1.0 + vals[-50:], None, np.ones(cols), 1e-5)
    within(back(v[-50:, cols:2 * cols]), rh, 64 * U * np.abs(rh), "h", EPS[True])
    del x, v
    torch.cuda.empty_cache()


def test_more_operators_replay_in_a_graph(ctx):
    """All of them, captured and replayed between eager work, against the eager results."""
    side = torch.cuda.Stream()
    with pwb.Context(0, side.cuda_stream) as c:
        n, d, V, k = 2100, 256, 1000, 5
        x, g = torch.randn(n, d, device="cuda"), torch.randn(d, device="cuda")
        w = torch.randn(V, d, device="cuda").bfloat16()
        t = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)
        new = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
        byte = torch.uint8
        xo, h, r = new(n, d), new(n, d, dt=torch.bfloat16), new(n)
        q8, s8 = new(n, d, dt=byte), new(pwb.f8_scale_bytes(n, d), dt=byte)
        q, s, qw, sw = new(n, d // 2, dt=byte), new(pwb.f4_scale_bytes(n, d), dt=byte), new(V, d // 2, dt=byte), new(pwb.f4_scale_bytes(V, d), dt=byte)
        z, lp, en, st, ids, tl = new(n, V, dt=torch.bfloat16), new(n), new(n), new(n, 2), new(n, k, dt=torch.int32), new(n, k)
        dz, ones = new(n, V, dt=torch.bfloat16), torch.ones(n, device="cuda")
        dx, dg, res = new(n, d), new(d), new(2)
        w1, w2, w3 = new(pwb.rmsnorm_bwd_ws_floats(n, d)), new(max(1, pwb.logprob_ws_floats(n, V, k))), new(pwb.grad_clip_ws_floats())
        torch.cuda.synchronize()

        def run():
            a = pwb.RmsnormArgs(dtype=pwb.PW_BF16, rows=n, cols=d, ldx=d, ldh=d, eps=1e-5, g=p(g))
            c.rmsnorm_fwd(a, p(x), p(h), p(xo), p(h), pwb.F8Out(format=pwb.PW_E4M3, q=p(q8), ldq=d, scale=p(s8)), p(r))
            c.f4_quantize(pwb.F4QuantizeArgs(dtype=pwb.PW_BF16, block_rows=1, x=p(h), rows=n, cols=d, ldx=d, q=p(q), ldq=d, q_scale=p(s)))
            c.f4_quantize(pwb.F4QuantizeArgs(dtype=pwb.PW_BF16, block_rows=32, x=p(w), rows=V, cols=d, ldx=d, q=p(qw), ldq=d, q_scale=p(sw)))
            c.f4_gemm(pwb.F4GemmArgs(M=n, N=V, K=d, lda=d, ldb=d, ldc=V, epilogue=0, out_dtype=pwb.PW_BF16, A=p(q), B=p(qw), a_scale=p(s), b_scale=p(sw), C=p(z)))
            b = pwb.LogprobArgs(dtype=pwb.PW_BF16, z=p(z), ldz=V, rows=n, vocab=V, targets=p(t), scale=1.0)
            c.logprob_fwd(b, p(lp), p(en), p(st), k, p(ids), p(tl), p(w2))
            c.logprob_bwd(b, p(st), p(en), p(ones), p(ones), p(dz), V)
            c.rmsnorm_bwd(a, p(h), p(xo), p(r), None, p(dx), None, p(dg), p(w1))
            c.grad_clip(pwb.grad_tensors([(p(dx), p(dx), n * d, 0), (p(dz), p(dz), n * V, 1), (p(dg), p(dg), d, 0)]), 1.0, p(res), p(w3))
        outs = (xo, h, r, q8, s8, q, s, qw, sw, z, lp, en, st, ids, tl, dz, dx, dg, res)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        for i in range(3):
            x.copy_(torch.randn(n, d, device="cuda"))
            for o in outs:
                o.zero_()
            torch.cuda.synchronize()
            run()
            c.synchronize()
            want = [o.clone() for o in outs]
            for o in outs:
                o.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outs)), i


def test_two_contexts_at_the_same_time(ctx):
    """Calls on two streams with workspaces of their own, one of them the program's current one."""
    side = torch.cuda.Stream()
    n, d = 3000, 700
    with pwb.Context(0, side.cuda_stream) as other:
        sets = []
        for i, c in enumerate((ctx, other)):
            x, dh, g = torch.randn(n, d, device="cuda"), torch.randn(n, d, device="cuda"), torch.ones(d, device="cuda")
            r = 1 / torch.sqrt((x * x).mean(1) + 1e-5)
            sets.append((c, x, dh, g, r, torch.zeros(n, d, device="cuda"), torch.zeros(d, device="cuda"), torch.zeros(2, device="cuda"),
                         torch.zeros(pwb.rmsnorm_bwd_ws_floats(n, d), device="cuda"), torch.zeros(pwb.grad_clip_ws_floats(), device="cuda")))
        torch.cuda.synchronize()
        for _ in range(20):
            for c, x, dh, g, r, dx, dg, res, w1, w2 in sets:
                c.rmsnorm_bwd(pwb.RmsnormArgs(dtype=0, rows=n, cols=d, ldx=d, ldh=d, eps=1e-5, g=p(g)), p(dh), p(x), p(r), None, p(dx), None, p(dg), p(w1))
                c.grad_clip(pwb.grad_tensors([(p(dx), None, n * d, 0), (p(dg), None, d, 0)]), 1.0, p(res), p(w2))
        ctx.synchronize()
        other.synchronize()
        for c, x, dh, g, r, dx, dg, res, w1, w2 in sets:
            rdx, rdg = M.rms_bwd(back(x), np.ones(d), 1e-5, back(dh))
            assert np.linalg.norm(back(dx) - rdx) < 1e-6 * np.linalg.norm(rdx)
            assert np.linalg.norm(back(dg) - rdg) < 1e-5 * np.linalg.norm(rdg)
            got = np.sqrt((back(dx) ** 2).sum() + (back(dg) ** 2).sum())
            assert abs(back(res)[0] - got) < 1e-6 * got


# ---- together --------------------------------------------------------------------------------------------------

def test_a_step_on_a_head_in_few_bits(ctx):
    """A policy-gradient step on an output layer: x' = x + y, h = norm(x'), logits = h W with h and W in 4 bits, log probabilities of
    given tokens and entropy, back through the same 4-bit products to x, y, g and W, clipping, Adam.  Every stage is held to its formula on the
    values that its inputs have on the device (64 bits), so that no rounding in front of it is in its bound."""
    n, d, V, k = 200, 256, 700, 4
    rng = np.random.RandomState(0)
    t = lambda v, dt=torch.float32: torch.from_numpy(np.ascontiguousarray(v)).to(dt).cuda()  # noqa: E731
    x, y, g = t(rng.randn(n, d), torch.float32), t(rng.randn(n, d), torch.bfloat16), t(1 + 0.1 * rng.randn(d), torch.float32)
    W = t(0.1 * rng.randn(d, V))                              # [in][out], the master copy
    tok = t(rng.randint(-1, V, n), torch.int32)
    dlp, den = t(rng.randn(n) / n, torch.float32), t(0.01 * rng.randn(n) / n, torch.float32)
    new = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731

    def quant(v, block=1):
        rows, cols = v.shape
        o = {"rows": rows, "cols": cols, "q": new(rows, up(cols, 32) // 2, dt=torch.uint8), "s": new(pwb.f4_scale_bytes(rows, cols), dt=torch.uint8),
             "qt": new(cols, up(rows, 32) // 2, dt=torch.uint8), "st": new(pwb.f4_scale_bytes(cols, rows), dt=torch.uint8)}
        torch.cuda.synchronize()
        ctx.f4_quantize(pwb.F4QuantizeArgs(dtype=DT[v.dtype == torch.bfloat16], block_rows=block, x=p(v), rows=rows, cols=cols, ldx=cols, q=p(o["q"]),
                                           ldq=up(cols, 32), q_scale=p(o["s"]), qt=p(o["qt"]), ldqt=up(rows, 32), qt_scale=p(o["st"])))
        ctx.synchronize()
        return o

    def side(o, turned):
        q, s, rows, cols = (o["qt"], o["st"], o["cols"], o["rows"]) if turned else (o["q"], o["s"], o["rows"], o["cols"])
        b = q.cpu().numpy()
        c = np.stack([b & 15, b >> 4], -1).reshape(rows, -1)
        return q, s, rows, up(cols, 32), M.f4_values(c, s.cpu().numpy()[M.f4_scale_index(rows, up(cols, 32) // 32)])

    def mul(a, b, bf16):
        (qa, sa, m, K, va), (qb, sb, nn, K2, vb) = a, b
        assert K == K2
        c = new(m, up(nn, 8), dt=act(bf16))
        torch.cuda.synchronize()
        ctx.f4_gemm(pwb.F4GemmArgs(M=m, N=nn, K=K, lda=K, ldb=K, ldc=c.shape[1], epilogue=0, out_dtype=DT[bf16], A=p(qa), B=p(qb), a_scale=p(sa),
                                   b_scale=p(sb), C=p(c)))
        ctx.synchronize()
        within(back(c)[:, :nn], va @ vb.T, (K // 32 + 12) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T), "product", EPS[bf16])
        return c

    xo, h, r = new(n, d), new(n, d, dt=torch.bfloat16), new(n)
    torch.cuda.synchronize()
    ra = pwb.RmsnormArgs(dtype=pwb.PW_BF16, rows=n, cols=d, ldx=d, ldh=d, eps=1e-5, g=p(g))
    ctx.rmsnorm_fwd(ra, p(x), p(y), p(xo), p(h), None, p(r))
    qh, qW = quant(h), quant(W, 32)
    z = mul(side(qh, False), side(qW, True), True)            # [n][V up to 8]
    lp, en, st, ids, tl = new(n), new(n), new(n, 2), new(n, k, dt=torch.int32), new(n, k)
    torch.cuda.synchronize()
    la = pwb.LogprobArgs(dtype=pwb.PW_BF16, z=p(z), ldz=z.shape[1], rows=n, vocab=V, targets=p(tok), scale=1.0)
    ctx.logprob_fwd(la, p(lp), p(en), p(st), k, p(ids), p(tl))
    ctx.synchronize()
    zv, tv = back(z)[:, :V], tok.cpu().numpy()
    rlp, rh, rid, _ = M.logprob_fwd(zv, tv, 1.0, k)
    elp, eh, _, _ = logp_bounds(zv, 1.0)
    within(back(lp), rlp, elp.max(1), "logp", U)
    within(back(en), rh, eh, "entropy", U)
    assert np.array_equal(ids.cpu().numpy(), rid)
    ctx.logprob_bwd(la, p(st), p(en), p(dlp), p(den), p(z), z.shape[1])      # in place
    ctx.synchronize()
    dz = M.logprob_bwd(zv, tv, back(dlp), back(den))
    within(back(z)[:, :V], dz, 1e-5 * np.abs(dz) + 1e-9, "dz", EPS[True])
    qd = quant(z[:, :V].contiguous())
    dW = mul(side(qh, True), side(qd, True), False)           # [d][V]
    dh = mul(side(qd, False), side(qW, False), True)          # [n][d]
    dx, dg, ws = new(n, d), new(d), new(max(1, pwb.rmsnorm_bwd_ws_floats(n, d)))
    torch.cuda.synchronize()
    ctx.rmsnorm_bwd(ra, p(dh), p(xo), p(r), None, p(dx), None, p(dg), p(ws))
    ctx.synchronize()
    rdx, rdg = M.rms_bwd(back(xo), back(g), 1e-5, back(dh))
    assert np.linalg.norm(back(dx) - rdx) < 1e-6 * np.linalg.norm(rdx) and np.linalg.norm(back(dg) - rdg) < 1e-5 * np.linalg.norm(rdg)
    dWd = dW[:, :V].contiguous()
    before = [back(dWd), back(dg)]
    res, w2 = new(2), new(pwb.grad_clip_ws_floats())
    torch.cuda.synchronize()
    ctx.grad_clip(pwb.grad_tensors([(p(dWd), p(dWd), d * V, 0), (p(dg), p(dg), d, 0)]), 1e-3, p(res), p(w2))
    m1, m2 = new(d, V), new(d, V)
    torch.cuda.synchronize()
    W0 = back(W)
    ctx.op("adam", p(W), p(m1), p(m2), p(dWd), None, d * V, 1e-2, 0.9, 0.999, 1e-8, 1)
    ctx.synchronize()
    norm, factor, want = M.clip(before, float(np.float32(1e-3)))
    assert factor < 1.0 and abs(back(res)[0] - norm) < 1e-6 * norm
    within(back(dWd), want[0], 2 * U * np.abs(want[0]), "clipped", U)
    step = W0 - back(W)
    gr = back(dWd)
    assert np.allclose(step, 1e-2 * gr / (np.abs(gr) + 1e-8), rtol=1e-3, atol=1e-7)
    # the gradient of W is the one of the loss through the values that the products had: differences along a direction, in 64 bits
    vh, vW = side(qh, False)[4], side(qW, True)[4].T

    def loss(w):
        l, e, _, _ = M.logprob_fwd(vh @ w, tv, 1.0, 0)
        return (l * back(dlp)).sum() + (e * back(den)).sum()
    u = vh.T @ M.logprob_bwd(vh @ vW, tv, back(dlp), back(den))
    v = u / np.linalg.norm(u)
    num = (loss(vW + 1e-5 * v) - loss(vW - 1e-5 * v)) / 2e-5
    assert abs(num - np.linalg.norm(u)) < 1e-5 * abs(num)
    # dz in 4 bits is off by a quarter of a value at most and by half of 2^-1 / sqrt(3) of it in the mean square: 15 %
    assert np.linalg.norm(before[0] - u) < 0.2 * np.linalg.norm(u)
