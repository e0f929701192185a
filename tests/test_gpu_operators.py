"""8-bit operands and their products, dropout and the gated recurrence through the C boundary, against 64-bit references
(operator_refs.py), at the sizes, strides and values where they can go wrong; and a run of them together.

Tolerances are derived, not measured.  A rounding is off by half a step (relative 2^-24 in fp32, 2^-8 in bf16)."""
import ctypes as C

import numpy as np
import pytest
import torch

import operator_refs as R
from gpu_util import DT
from paper_2203_12533_amd import binding as pwb
from paper_2203_12533_amd import inputs as I

pytestmark = pytest.mark.gpu

F8 = {"e4m3": pwb.PW_E4M3, "e5m2": pwb.PW_E5M2}
EPS = {False: 2.0 ** -24, True: 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    with pwb.Context(0) as c:
        yield c


def up(n, m):
    return -(-n // m) * m


def dev(a, dtype=torch.float32, ld=None, fill=None, offset=0):
    """A device array with rows ld apart, `offset` elements into its storage; what lies between the rows is `fill`.  -> (holder, address)"""
    a = np.atleast_2d(np.asarray(a))
    ld = a.shape[1] if ld is None else ld
    t = torch.full((a.shape[0] * ld + offset,), 0 if fill is None else fill, dtype=dtype, device="cuda")
    v = t[offset:].view(a.shape[0], ld)
    v[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()
    torch.cuda.synchronize()
    return v, v.data_ptr()


def back(t):
    return t.detach().double().cpu().numpy()


def act(bf16):
    return torch.bfloat16 if bf16 else torch.float32


def low(a, bf16):
    """The values a kernel sees."""
    a = np.asarray(a, np.float32)
    return (I.round_to_bf16(a) if bf16 else a).astype(np.float64)


def rnd(seed, *shape):
    return np.random.RandomState(seed).randn(*shape)


def within(got, ref, allow, name=""):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, name
    assert np.array_equal(np.isnan(got), np.isnan(ref)), name
    fin = np.isfinite(ref)
    assert np.array_equal(got[~fin & ~np.isnan(ref)], ref[~fin & ~np.isnan(ref)]), name
    d = np.abs(got - ref)[fin]
    a = np.broadcast_to(allow, ref.shape)[fin]
    if d.size:
        i = int(np.argmax(d - a))
        assert d[i] <= a[i], f"{name}: off by {d[i]:.3e}, allowed {a[i]:.3e} (largest difference {d.max():.3e})"


# ---- quantisation ----------------------------------------------------------------------------------------------

def quantize(ctx, x, fmt, block, bf16=False, ldx=None, offset=0, rows_out=True, cols_out=True, spare=0):
    rows, cols = x.shape
    xt, px = dev(x, act(bf16), ldx, fill=float("nan"), offset=offset)
    ldq, ldqt = up(cols, 16) + 16 * spare, up(rows, 16) + 16 * spare
    q = torch.full((rows, ldq), 0xAA, dtype=torch.uint8, device="cuda")
    qt = torch.full((cols, ldqt), 0xAA, dtype=torch.uint8, device="cuda")
    s = torch.full((pwb.f8_scale_bytes(rows, cols),), 0xAA, dtype=torch.uint8, device="cuda")
    st = torch.full((pwb.f8_scale_bytes(cols, rows),), 0xAA, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    p = lambda t, on: t.data_ptr() if on else None  # noqa: E731
    ctx.f8_quantize(pwb.F8QuantizeArgs(dtype=DT[bf16], format=F8[fmt], block_rows=block, x=px, rows=rows, cols=cols,
                                       ldx=xt.shape[1], q=p(q, rows_out), ldq=ldq if rows_out else 0, q_scale=p(s, rows_out),
                                       qt=p(qt, cols_out), ldqt=ldqt if cols_out else 0, qt_scale=p(st, cols_out)))
    ctx.synchronize()
    return tuple(t.cpu().numpy() for t in (q, s, qt, st))


def same_codes(got, want, fmt, name):
    v = R.decode_table(fmt)
    same = (got == want) | (np.isnan(v[got]) & np.isnan(v[want]))
    assert same.all(), (name, np.argwhere(~same)[:5], got[~same][:5], want[~same][:5])


def check_quantized(ctx, x, fmt, block, bf16, **kw):
    v = low(x, bf16)
    q, s, qt, st = quantize(ctx, x, fmt, block, bf16, **kw)
    spare = kw.get("spare", 0)
    if kw.get("rows_out", True):
        wq, e = R.quantize(v, fmt, block)
        same_codes(q[:, :wq.shape[1]], wq, fmt, "q")
        assert np.array_equal(s, R.scale_table(e))
        assert (q[:, wq.shape[1]:] == 0xAA).all() and q.shape[1] == wq.shape[1] + 16 * spare
    else:
        assert (q == 0xAA).all() and (s == 0xAA).all()
    if kw.get("cols_out", True):
        if block == 1:
            wq, e = R.quantize(np.ascontiguousarray(v.T), fmt, 1)
        else:                                      # 128 x 128 blocks are the same from either side
            wq, e = R.quantize(np.ascontiguousarray(v.T), fmt, 128)
        same_codes(qt[:, :wq.shape[1]], wq, fmt, "qt")
        assert np.array_equal(st, R.scale_table(e))
        assert (qt[:, wq.shape[1]:] == 0xAA).all()
    else:
        assert (qt == 0xAA).all() and (st == 0xAA).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,cols,bf16,kw", [
    (1, 1, False, {}), (1, 200, True, {}), (129, 127, True, {}), (64, 128, False, {}), (300, 257, False, {"ldx": 261, "offset": 3}),
    (70, 520, True, {"ldx": 523, "offset": 1, "spare": 2}), (200, 136, True, {"ldx": 144, "offset": 8, "cols_out": False}),
    (136, 200, False, {"rows_out": False}), (5, 16, True, {"spare": 1})])
def test_quantisation_is_exact(ctx, fmt, block, rows, cols, bf16, kw):
    x = rnd(rows + cols, rows, cols) * np.exp(2 * rnd(1, rows, 1)) * np.exp(rnd(2, 1, cols))
    check_quantized(ctx, x, fmt, block, bf16, **kw)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [2, 7, 8, 9, 121, 122, 123, 124, 125, 126, 127, 128, 129, 135, 255])
def test_quantisation_of_any_width(ctx, cols, bf16):
    """Every number of columns left over behind whole groups of eight, at rows that start anywhere; what lies behind a row is NaN."""
    check_quantized(ctx, rnd(cols, 131, cols) * np.exp(rnd(3, 1, cols)), "e4m3", 1, bf16, ldx=cols + 3, offset=1)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
def test_quantisation_of_every_kind_of_value(ctx, fmt, block):
    """Blocks of zeros, of subnormals, with the largest numbers, whose maximum sits at a border of the scale, ties between
    neighbouring values, NaN and infinities in some rows and columns."""
    x = rnd(7, 140, 300).astype(np.float32)
    x[3] = 0.0
    x[4] = -0.0
    x[5, :128] = 1e-42
    x[6, :128] = np.float32(2.0 ** -149)
    x[7, 128:256] = np.finfo(np.float32).max
    x[8, 0], x[8, 1:128] = 1.75, np.linspace(-1.7, 1.7, 127)
    x[9, 0], x[9, 1:128] = np.nextafter(np.float32(1.75), np.float32(2)), np.linspace(-1.7, 1.7, 127)
    grid = R.decode_table(fmt)[:128]
    grid = grid[np.isfinite(grid)]
    mid = ((grid[1:] + grid[:-1]) / 2)[-100:]
    x[10, :mid.size], x[10, mid.size:128] = mid, R.TOP[fmt]
    x[11, 5], x[11, 290] = np.nan, np.inf
    x[12, :128] = np.nan
    x[13, 128:256] = -np.inf
    x[20, 7], x[21, 7] = -np.inf, 3e30
    check_quantized(ctx, x, fmt, block, False)


# ---- products --------------------------------------------------------------------------------------------------

def operand(seed, rows, k, fmt, block=1):
    x = rnd(seed, rows, k) * np.exp(rnd(seed + 1, rows, 1)) * np.exp(0.5 * rnd(seed + 2, 1, k))
    q, e = R.quantize(x, fmt, block)
    return q[:, :k], R.scale_table(e), R.values(q[:, :k], e, fmt)


def product(ctx, M, N, K, fa="e4m3", fb="e4m3", epilogue=pwb.PW_EPI_STORE, bf16=False, accumulate=0, seed=0, lda=None, ldb=None,
            ldc=None, block=1, bias=True, nan_rows=()):
    """Runs one product and checks everything it writes.  Returns C as the bits it has."""
    a, sa, va = operand(seed, M, K, fa)
    b, sb, vb = operand(seed + 10, N, K, fb, block)
    va, vb = va.copy(), vb.copy()
    for r in nan_rows:                                       # NaN in one row of A stays in that row of C
        a[r, K // 2], va[r, K // 2] = 0x7F, np.nan
    lda, ldb, ldc = lda or up(K, 16), ldb or up(K, 16), ldc or up(N, 8)
    at, pa = dev(a, torch.uint8, lda, fill=0x7F)             # NaN behind the rows: must not be read into a sum
    bt, pb = dev(b, torch.uint8, ldb, fill=0x7F)
    sat, sbt = torch.from_numpy(sa).cuda(), torch.from_numpy(sb).cuda()
    rng = np.random.RandomState(seed + 5)
    bias_v = rng.randn(N).astype(np.float32)
    biast = torch.from_numpy(bias_v).cuda()
    aux = c0 = c2 = auxt = None
    ct = torch.full((M, ldc), 7.0, dtype=act(bf16), device="cuda")
    if epilogue == pwb.PW_EPI_BIAS_RESIDUAL:
        aux = rng.randn(M, N).astype(np.float32)
        auxt, _ = dev(aux, torch.float32, ldc)
    elif epilogue == pwb.PW_EPI_GELU_BWD:
        aux = low(rng.randn(M, N), True)
        auxt, _ = dev(aux, torch.bfloat16, ldc)
    elif epilogue == pwb.PW_EPI_BIAS_GELU:
        c2 = torch.full((M, ldc), 7.0, dtype=act(bf16), device="cuda")
    if accumulate:
        c0 = rng.randn(M, N).astype(np.float32)
        ct[:, :N] = torch.from_numpy(c0).cuda()
    torch.cuda.synchronize()
    has_bias = epilogue in (pwb.PW_EPI_BIAS, pwb.PW_EPI_BIAS_RESIDUAL, pwb.PW_EPI_BIAS_GELU) and bias
    ctx.f8_gemm(pwb.F8GemmArgs(a_format=F8[fa], b_format=F8[fb], M=M, N=N, K=K, lda=lda, ldb=ldb, ldc=ldc, epilogue=epilogue,
                               out_dtype=DT[bf16], accumulate=accumulate, A=pa, B=pb, a_scale=sat.data_ptr(), b_scale=sbt.data_ptr(),
                               bias=biast.data_ptr() if has_bias else None, aux=auxt.data_ptr() if auxt is not None else None,
                               C=ct.data_ptr(), C2=c2.data_ptr() if c2 is not None else None))
    ctx.synchronize()
    ref = va @ vb.T
    # K products (exact in fp32) added in some order: each addition is off by 2^-24 of a partial sum, which the sum of
    # magnitudes bounds; K additions and the ones of the epilogue
    mag = np.abs(va) @ np.abs(vb).T
    allow = (K + 4) * 2.0 ** -24 * mag
    if bf16:                 # the 8-bit pipe: seven of eight products each cut off 2^-13 under the eighth
        allow = allow + 7 * 2.0 ** -13 * mag
    if has_bias:
        ref, allow = ref + bias_v, allow + 2.0 ** -24 * np.abs(bias_v)
    if accumulate:
        ref, allow = ref + c0, allow + 2.0 ** -24 * np.abs(c0)
    if epilogue == pwb.PW_EPI_BIAS_RESIDUAL:
        ref, allow = ref + aux, allow + 2.0 ** -24 * np.abs(aux)
    if epilogue == pwb.PW_EPI_GELU_BWD:
        # gelu' within 2^-20: a handful of fp32 operations on values up to about 2, exp2 and rcp at one unit each
        g = R.gelu_grad(aux)
        ref, allow = ref * g, allow * np.abs(g) + 2.0 ** -20 * np.abs(ref) * (np.abs(g) + 1)
    # the rounding of what is stored; on top of an error of the value itself
    store = lambda r, al: al + EPS[bf16] * (np.abs(r) + al)  # noqa: E731
    got = back(ct)
    within(got[:, :N], ref, store(ref, allow), "C")
    assert (got[:, N:] == 7.0).all(), "columns behind N were written"
    fin = np.isfinite(ref)
    # and as a whole: rounding errors of random signs, so the norm of the error is far below the sum of the bounds
    err = np.linalg.norm((got[:, :N] - ref)[fin]) / np.linalg.norm(ref[fin])
    assert err < (4e-3 if bf16 else 1e-5), err
    if epilogue == pwb.PW_EPI_BIAS_GELU:
        h = R.gelu(ref)
        within(back(c2)[:, :N], h, store(h, 1.13 * allow + 2.0 ** -20 * (np.abs(h) + np.abs(ref) * 0.01)), "C2")
    return ct


SHAPES = [(1, 8, 16), (1, 200, 128), (3, 24, 144), (16, 64, 256), (17, 65, 272), (64, 64, 128), (100, 130, 1008), (128, 128, 512),
          (130, 258, 400), (256, 256, 384), (300, 520, 2064), (33, 1000, 4096)]


@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_f8_product(ctx, M, N, K, fa, fb):
    product(ctx, M, N, K, fa, fb, seed=M + N)


EPILOGUES = [(pwb.PW_EPI_STORE, False, 1), (pwb.PW_EPI_STORE, True, 0), (pwb.PW_EPI_BIAS, False, 0), (pwb.PW_EPI_BIAS, True, 0),
             (pwb.PW_EPI_BIAS_RESIDUAL, False, 0), (pwb.PW_EPI_BIAS_GELU, True, 0), (pwb.PW_EPI_BIAS_GELU, False, 0),
             (pwb.PW_EPI_GELU_BWD, True, 0), (pwb.PW_EPI_GELU_BWD, False, 0)]


@pytest.mark.parametrize("epilogue,bf16,accumulate", EPILOGUES)
@pytest.mark.parametrize("M,N,K", [(1, 120, 256), (40, 77, 144), (128, 256, 256), (260, 300, 528), (300, 1033, 272)])
def test_f8_product_epilogues(ctx, M, N, K, epilogue, bf16, accumulate):
    product(ctx, M, N, K, epilogue=epilogue, bf16=bf16, accumulate=accumulate, seed=M, block=128)


@pytest.mark.parametrize("M,N,K,kw", [
    (1500, 1420, 400, {"bf16": True}), (1500, 1420, 400, {"fa": "e5m2", "epilogue": pwb.PW_EPI_BIAS_RESIDUAL}),
    (1408, 1536, 272, {"fb": "e5m2"}), (3100, 3900, 272, {"bf16": True, "epilogue": pwb.PW_EPI_BIAS}),
    (3100, 3900, 144, {"bf16": True, "epilogue": pwb.PW_EPI_GELU_BWD, "fa": "e5m2"}),
    (2560, 4096, 384, {"bf16": True, "epilogue": pwb.PW_EPI_BIAS_GELU, "block": 128}), (2560, 4096, 128, {"bf16": True}),
    (2570, 4099, 272, {"epilogue": pwb.PW_EPI_BIAS}), (40000, 70, 144, {"bf16": True}), (70, 40000, 144, {"accumulate": 1})])
def test_f8_product_many_tiles(ctx, M, N, K, kw):
    product(ctx, M, N, K, seed=2, **kw)


@pytest.mark.parametrize("bf16,fa,fb", [(True, "e4m3", "e4m3"), (True, "e5m2", "e4m3"), (False, "e4m3", "e5m2")])
@pytest.mark.parametrize("K", [16, 128, 240, 400, 1040])
@pytest.mark.parametrize("M,N", [(3, 5000), (260, 300), (500, 1300), (1300, 1100), (1700, 1900), (2100, 2600)])
def test_f8_product_every_tile_and_depth(ctx, M, N, K, bf16, fa, fb):
    """A size for each tile, none of them whole, with one to nine k tiles, the last of them partial or not."""
    product(ctx, M, N, K, fa, fb, bf16=bf16, epilogue=pwb.PW_EPI_BIAS, seed=K, block=128)


@pytest.mark.parametrize("K", [16, 256, 272, 528])
def test_f8_product_largest_tile_and_depth(ctx, K):
    product(ctx, 3000, 3100, K, bf16=True, seed=K)


def test_f8_product_of_rows_far_apart(ctx):
    product(ctx, 3, 40, 144, lda=(1 << 23) + 16, bf16=True)
    product(ctx, 40, 3, 144, ldb=(1 << 23) + 16)
    product(ctx, 70, 5, 400, lda=1 << 23, epilogue=pwb.PW_EPI_BIAS)


def test_f8_product_strides_missing_bias_and_empty_sums(ctx):
    product(ctx, 70, 90, 144, lda=208, ldb=176, ldc=136, epilogue=pwb.PW_EPI_BIAS, bf16=True)
    product(ctx, 33, 40, 128, epilogue=pwb.PW_EPI_BIAS, bias=False)
    product(ctx, 50, 60, 1040, nan_rows=(0, 49))
    a = torch.zeros(64 * 64, dtype=torch.uint8, device="cuda")
    c, bias = torch.full((5, 8), 3.0, device="cuda"), torch.arange(8.0, device="cuda")
    torch.cuda.synchronize()
    k = dict(M=5, N=8, K=0, lda=16, ldb=16, ldc=8, out_dtype=pwb.PW_F32, A=a.data_ptr(), B=a.data_ptr(), a_scale=a.data_ptr(),
             b_scale=a.data_ptr(), C=c.data_ptr())
    ctx.f8_gemm(pwb.F8GemmArgs(epilogue=pwb.PW_EPI_STORE, accumulate=1, **k))       # nothing to add
    ctx.synchronize()
    assert (back(c) == 3.0).all()
    ctx.f8_gemm(pwb.F8GemmArgs(epilogue=pwb.PW_EPI_BIAS, bias=bias.data_ptr(), **k))
    ctx.synchronize()
    assert np.array_equal(back(c), np.tile(np.arange(8.0), (5, 1)))


def test_f8_product_takes_extreme_scales_and_a_residual_in_place(ctx):
    """Scales far apart that meet in one product, and C over aux."""
    M, N, K = 65, 40, 256
    a, sa, va = operand(1, M, K, "e4m3")
    b, sb, vb = operand(2, N, K, "e4m3")
    ea = np.clip(np.random.RandomState(0).randint(-60, 60, (M, 2)), -127, 127)
    eb = np.random.RandomState(1).randint(-40, 40, (N, 2))
    va, vb = R.values(a, ea, "e4m3"), R.values(b, eb, "e4m3")
    at, bt = torch.from_numpy(a).cuda(), torch.from_numpy(np.ascontiguousarray(b)).cuda()
    sat, sbt = torch.from_numpy(R.scale_table(ea)).cuda(), torch.from_numpy(R.scale_table(eb)).cuda()
    res = rnd(9, M, N).astype(np.float32)
    c = torch.from_numpy(res).cuda()
    torch.cuda.synchronize()
    ctx.f8_gemm(pwb.F8GemmArgs(M=M, N=N, K=K, lda=K, ldb=K, ldc=N, epilogue=pwb.PW_EPI_BIAS_RESIDUAL, out_dtype=pwb.PW_F32, A=at.data_ptr(),
                               B=bt.data_ptr(), a_scale=sat.data_ptr(), b_scale=sbt.data_ptr(), aux=c.data_ptr(), C=c.data_ptr()))
    ctx.synchronize()
    within(back(c), va @ vb.T + res, (K + 4) * 2.0 ** -24 * (np.abs(va) @ np.abs(vb).T + np.abs(res)))


def test_f8_product_repeats_its_bits(ctx):
    x = [product(ctx, 260, 300, 2064, seed=3).clone() for _ in range(3)]
    assert torch.equal(x[0], x[1]) and torch.equal(x[0], x[2])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,N", [(1, 40), (40, 70), (300, 200), (300, 2050), (1000, 760), (1500, 4096), (4096, 4096)])
def test_products_over_nothing(ctx, M, N, bf16):
    """K = 0: the bias alone, in every tile; with PW_EPI_STORE zeros, or what was there where the output accumulates."""
    ldc = up(N, 8)
    bias = torch.randn(ldc, device="cuda")
    c = torch.full((M, ldc), 7.0, dtype=act(bf16), device="cuda")
    q, s = torch.zeros(64, dtype=torch.uint8, device="cuda"), torch.zeros(64, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def run(epilogue, accumulate):
        c.fill_(7.0)
        torch.cuda.synchronize()
        ctx.f8_gemm(pwb.F8GemmArgs(M=M, N=N, K=0, lda=0, ldb=0, ldc=ldc, epilogue=epilogue, out_dtype=pwb.PW_BF16 if bf16 else pwb.PW_F32,
                                   accumulate=accumulate, A=q.data_ptr(), B=q.data_ptr(), a_scale=s.data_ptr(), b_scale=s.data_ptr(),
                                   bias=bias.data_ptr(), C=c.data_ptr()))
        ctx.synchronize()
        assert (c[:, N:] == 7.0).all()
        return c[:, :N]

    assert (run(pwb.PW_EPI_BIAS, 0) == bias[:N].to(act(bf16))).all()
    assert (run(pwb.PW_EPI_STORE, 0) == 0).all()
    if not bf16:
        assert (run(pwb.PW_EPI_STORE, 1) == 7.0).all()


# ---- dropout ---------------------------------------------------------------------------------------------------

def dropout(ctx, rows, cols, bf16, out_bf16, p, res=True, bias=True, seed=(1 << 40) + 17, site=3, step=11, step_dev=None, ldx=None,
            ldy=None, offset=0, accumulate=0):
    x, dy = rnd(rows, rows, cols), rnd(cols, rows, cols)
    b, r = rnd(3, cols).astype(np.float32), rnd(4, rows, cols).astype(np.float32)
    ldx, ldy = ldx or cols, ldy or cols
    xt, px = dev(x, act(bf16), ldx, offset=offset)
    dyt, pdy = dev(dy, act(out_bf16), ldy, offset=offset)
    bt, pb = dev(b)
    rt, pr = dev(r, torch.float32, ldy, offset=offset)
    y, py = dev(np.full((rows, cols), 7.0), act(out_bf16), ldy, fill=7.0, offset=offset)
    dx, pdx = dev(np.full((rows, cols), 7.0), act(bf16), ldx, fill=7.0, offset=offset)
    db0 = rnd(5, cols).astype(np.float32)
    dbt, pdb = dev(db0)
    ws = torch.full((max(1, pwb.dropout_bwd_ws_floats(rows, cols)),), float("nan"), device="cuda")
    torch.cuda.synchronize()
    a = pwb.DropoutArgs(dtype=DT[bf16], out_dtype=DT[out_bf16], rows=rows, cols=cols, ldx=ldx, ldy=ldy, p=p, seed=seed, site=site,
                        step=step, step_dev=step_dev.data_ptr() if step_dev is not None else None)
    ctx.dropout_fwd(a, px, pb if bias else None, pr if res else None, py)
    ctx.dropout_bwd(a, pdy, pdx, pdb if bias else None, ws.data_ptr() if bias else None, accumulate)
    ctx.synchronize()
    keep, scale = R.dropout_keep(rows, cols, p, seed, site, step + (int(step_dev.item()) if step_dev is not None else 0))
    v = low(x, bf16) + (b if bias else 0)
    k = np.where(keep, v * scale, 0.0)
    ref = k + (r if res else 0)
    # x + bias, its product with the scale (itself rounded), the residual's addition: 2^-24 each of what they yield
    within(back(y)[:, :cols], ref, 3 * 2.0 ** -24 * np.abs(k) + EPS[out_bf16] * np.abs(ref) * (1 + 1e-6), "y")
    g = np.where(keep, low(dy, out_bf16) * scale, 0.0)
    within(back(dx)[:, :cols], g, (2 * 2.0 ** -24 + EPS[bf16] * (1 + 1e-6)) * np.abs(g), "dx")
    assert (back(y)[:, cols:] == 7.0).all() and (back(dx)[:, cols:] == 7.0).all()
    if bias:
        want = g.sum(0) + (db0 if accumulate else 0)
        within(back(dbt)[0], want, (rows + 4) * 2.0 ** -24 * (np.abs(g).sum(0) + np.abs(db0)), "dbias")
    else:
        assert np.array_equal(back(dbt)[0], db0.astype(np.float64))
    return y, dx, dbt


@pytest.mark.parametrize("bf16,out_bf16,res", [(True, False, True), (True, True, False), (False, False, True), (True, False, False),
                                               (False, False, False)])
@pytest.mark.parametrize("rows,cols,p", [(1, 1, 0.5), (1, 8, 0.1), (3, 7, 0.9), (37, 1003, 0.3), (1000, 24, 0.25), (64, 512, 0.0),
                                         (5, 130, 1.0), (300, 520, 2.0 ** -17), (9, 4099, 0.999)])
def test_dropout(ctx, rows, cols, p, bf16, out_bf16, res):
    dropout(ctx, rows, cols, bf16, out_bf16, p, res=res)


def test_dropout_strides_offsets_and_adding_gradients(ctx):
    dropout(ctx, 40, 100, True, False, 0.2, ldx=107, ldy=101, offset=3)
    dropout(ctx, 40, 96, True, True, 0.2, res=False, ldx=104, ldy=99, offset=1, accumulate=1)
    dropout(ctx, 700, 2048, False, False, 0.4, accumulate=1)
    dropout(ctx, 20, 64, True, False, 0.2, bias=False)
    dropout(ctx, 50000, 9, False, False, 0.5)                # more rows than one launch has row blocks for


def test_dropout_leaves_no_trace_of_what_it_drops_and_works_in_place(ctx):
    rows, cols = 33, 136
    keep, scale = R.dropout_keep(rows, cols, 0.5, 5, 6, 7)
    x = np.where(keep, rnd(1, rows, cols), np.where(rnd(2, rows, cols) > 0, np.nan, np.inf)).astype(np.float32)
    xt, px = dev(x)
    a = pwb.DropoutArgs(dtype=pwb.PW_F32, out_dtype=pwb.PW_F32, rows=rows, cols=cols, ldx=cols, ldy=cols, p=0.5, seed=5, site=6, step=7)
    ctx.dropout_fwd(a, px, None, None, px)                   # y over x
    ctx.synchronize()
    want = np.where(keep, np.nan_to_num(x) * scale, 0.0)
    assert np.array_equal(back(xt), want)                    # 1 / (1 - 0.5) = 2: exact
    res = rnd(3, rows, cols).astype(np.float32)
    rt, pr = dev(res)
    x2, px2 = dev(np.where(keep, 1.0, np.nan))
    ctx.dropout_fwd(a, px2, None, pr, pr)                    # y over res
    ctx.dropout_bwd(a, px2, px2)                             # dx over dy
    ctx.synchronize()
    assert np.array_equal(back(rt), np.where(keep, np.float32(res + np.float32(2)), res).astype(np.float64))
    assert np.array_equal(back(x2), np.where(keep, 2.0, 0.0))


def test_dropout_step_on_the_device_wraps_and_replays_draw_anew(ctx):
    step = torch.tensor([5], dtype=torch.int32, device="cuda")
    dropout(ctx, 30, 72, True, False, 0.5, step=2 ** 32 - 3, step_dev=step)      # 2^32 - 3 + 5 wraps to 2
    side = torch.cuda.Stream()
    with pwb.Context(0, side.cuda_stream) as c:
        rows, cols = 64, 256
        x = torch.ones(rows, cols, device="cuda")
        y = torch.zeros_like(x)
        dx, db = torch.zeros_like(x), torch.zeros(cols, device="cuda")
        ws = torch.empty(max(1, pwb.dropout_bwd_ws_floats(rows, cols)), device="cuda")
        a = pwb.DropoutArgs(dtype=pwb.PW_F32, out_dtype=pwb.PW_F32, rows=rows, cols=cols, ldx=cols, ldy=cols, p=0.25, seed=1, site=2, step=0,
                            step_dev=step.data_ptr())
        torch.cuda.synchronize()

        def both():
            c.dropout_fwd(a, x.data_ptr(), None, None, y.data_ptr())
            c.dropout_bwd(a, y.data_ptr(), dx.data_ptr(), db.data_ptr(), ws.data_ptr())
            step.add_(1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
        step.fill_(100)
        torch.cuda.synchronize()
        for k in range(4):
            graph.replay()
            torch.cuda.synchronize()
            keep, scale = R.dropout_keep(rows, cols, 0.25, 1, 2, 100 + k)
            s = float(np.float32(scale))
            assert np.allclose(back(y), np.where(keep, s, 0.0), rtol=2.0 ** -23, atol=0)
            assert np.allclose(back(dx), np.where(keep, s * s, 0.0), rtol=2.0 ** -22, atol=0)
            assert np.allclose(back(db), back(dx).sum(0), rtol=2.0 ** -18, atol=0)
            torch.randn(1000, device="cuda").sum().item()    # the program's own work between replays


# ---- gated recurrence ------------------------------------------------------------------------------------------

def scan(ctx, B, T, D, bf16, lens=None, seed=0, shift=1.0, h0=True, dh=True, packed=True, ld_extra=0, offset=0, backward=True,
         f=None, x=None, poison=True, aliases=False):
    f = rnd(seed, B * T, D) * 1.5 + shift if f is None else f
    x = rnd(seed + 1, B * T, D) if x is None else x
    dy, h0v, dhv = rnd(seed + 2, B * T, D), rnd(seed + 3, B, D).astype(np.float32), rnd(seed + 4, B, D).astype(np.float32)
    fv, xv, dyv = (low(a, bf16).reshape(B, T, D) for a in (f, x, dy))
    if lens is not None and poison:                          # what lies behind the end of a sequence must not matter
        f, x, dy = (np.array(a, np.float64) for a in (f, x, dy))
        for b in range(B):
            for a in (f, x, dy):
                a.reshape(B, T, D)[b, max(0, min(T, lens[b])):] = np.nan
    es = 2 if bf16 else 4
    ld = (2 * D if packed else D) + ld_extra
    if packed:
        fx, pf = dev(np.concatenate([f, x], 1).reshape(B * T, 2 * D), act(bf16), ld, offset=offset)
        px = pf + D * es
    else:
        ft, pf = dev(f.reshape(B * T, D), act(bf16), ld, offset=offset)
        xt, px = dev(x.reshape(B * T, D), act(bf16), ld, offset=offset)
    dyt, pdy = dev(dy.reshape(B * T, D), act(bf16), D + ld_extra, offset=offset)
    y, py = dev(np.full((B * T, D), 7.0), act(bf16), D + ld_extra, fill=7.0, offset=offset)
    dfx, pd = dev(np.full((B * T, 2 * D), 7.0), act(bf16), 2 * D + ld_extra, fill=7.0, offset=offset)
    h0t, ph0 = dev(h0v)
    dht, pdh = dev(dhv)
    he, phe = (h0t, ph0) if aliases else dev(np.full((B, D), 7.0))
    dh0, pdh0 = (dht, pdh) if aliases else dev(np.full((B, D), 7.0))
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    states = torch.full((max(1, pwb.scan_state_floats(B, T, D)),), float("nan"), device="cuda")
    ws = torch.full((max(2, pwb.scan_ws_floats(B, T, D)),), float("nan"), device="cuda")
    torch.cuda.synchronize()
    a = pwb.ScanArgs(dtype=DT[bf16], f=pf, x=px, ldf=ld, ldx=ld, B=B, T=T, D=D, h0=ph0 if h0 else None,
                     lens=lt.data_ptr() if lt is not None else None)
    ctx.scan_fwd(a, py, D + ld_extra, phe, states.data_ptr() if backward else None, ws.data_ptr())
    if backward:
        if aliases:                                          # the forward call has put h_end where h0 was
            ctx.synchronize()
        ctx.scan_bwd(a, pdy, D + ld_extra, pdh if dh else None, states.data_ptr(), pd, 2 * D + ld_extra, pd + D * es, 2 * D + ld_extra,
                     pdh0, ws.data_ptr())
    ctx.synchronize()
    h0r, dhr = h0v.astype(np.float64) * h0, dhv.astype(np.float64) * dh
    ry, rhe = R.scan_fwd(fv, xv, h0r, lens)
    # Gates are good to a few units in the last place (exp2 of a rounded argument, |f| up to 8: 2^-24 (2 + |f|); rcp, a product),
    # call it 16 * 2^-24; every step adds that much of the state, and a step's error fades by a_t: over 1 / (1 - a) steps at
    # most, or T.
    z = R._sigmoid(-fv)
    n_eff = min(max(T, 1), 1 / z.min()) if T else 1.0
    hmax = max(np.abs(xv).max() if T else 0, np.abs(h0r).max())
    tol = 16 * 2.0 ** -24 * (n_eff + 1) * hmax
    got_y = back(y)
    within(got_y[:, :D].reshape(B, T, D), ry, tol + EPS[bf16] * (np.abs(ry) + tol), "y")
    within(back(he), rhe, tol, "h_end")
    assert (got_y[:, D:] == 7.0).all()
    if T and bf16 is False:
        err = np.linalg.norm(got_y[:, :D].reshape(B, T, D) - ry) / max(np.linalg.norm(ry), 1e-30)
        assert err < 1e-5 or np.linalg.norm(ry) == 0
    if not backward:
        return [y, he]
    rdf, rdx, rdh0 = R.scan_bwd(fv, xv, h0r, dyv, dhr, lens)
    gmax = (np.abs(dyv).max() if T else 0) * n_eff + np.abs(dhr).max()
    gtol = 16 * 2.0 ** -24 * (n_eff + 1) * gmax              # the same recurrence, of values up to gmax
    got = back(dfx)
    within(got[:, D:2 * D].reshape(B, T, D), rdx, gtol + EPS[bf16] * (np.abs(rdx) + gtol), "dx")
    dft = 0.25 * (gtol * 2 * hmax + gmax * tol + 8 * 2.0 ** -24 * gmax * 2 * hmax)
    within(got[:, :D].reshape(B, T, D), rdf, dft + EPS[bf16] * (np.abs(rdf) + dft), "df")
    within(back(dh0), rdh0, gtol, "dh0")
    assert (got[:, 2 * D:] == 7.0).all()
    if T and bf16 is False:
        for name, g, r in (("df", got[:, :D], rdf), ("dx", got[:, D:2 * D], rdx)):
            # gradients through closed gates reach 1e-87 in 64 bits: fp32 has nothing under 2^-149, and a factor under 2^-126
            # may be taken as zero, so each value may be off by 2^-126 (times gmax, hmax < 2^6) whatever it is
            n = np.linalg.norm(r)
            assert np.linalg.norm(g.reshape(B, T, D) - r) <= 1e-5 * n + 2.0 ** -114 * np.sqrt(r.size), name
    return [y, he, dfx, dh0]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,T,D", [(1, 1, 1), (8, 1, 200), (2, 2, 63), (1, 7, 64), (3, 8, 66), (2, 9, 30), (2, 16, 128), (1, 17, 65), (2, 100, 31),
                                   (1, 255, 34), (2, 256, 64), (1, 257, 70), (3, 300, 20), (1, 1000, 130), (1, 4097, 8), (2, 2000, 3)])
def test_recurrence_forward_and_backward(ctx, B, T, D, bf16):
    scan(ctx, B, T, D, bf16, seed=T)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("T,lens", [(1, [0, 1, 1]), (40, [0, 40, 17]), (300, [256, 1, 299]), (1030, [0, 513, 1030]), (520, [-3, 900, 255])])
def test_recurrence_of_padded_batches(ctx, T, lens, bf16):
    scan(ctx, 3, T, 70, bf16, lens=lens, seed=T)


@pytest.mark.parametrize("bf16", [False, True])
def test_recurrence_layouts_and_missing_states(ctx, bf16):
    scan(ctx, 2, 50, 64, bf16, packed=False, ld_extra=3, offset=1)
    scan(ctx, 2, 50, 64, bf16, ld_extra=2, offset=1)             # pairs that start on an odd element
    scan(ctx, 2, 600, 64, bf16, h0=False, dh=False)
    scan(ctx, 1, 2000, 64, bf16, h0=False, dh=True, packed=False)
    scan(ctx, 1, 700, 40, bf16, backward=False)
    scan(ctx, 600, 5, 16, bf16)                                  # many short sequences: one segment


@pytest.mark.parametrize("lens", [None, [800, 0, 31, 770]])
def test_recurrence_of_more_blocks_than_units(ctx, lens):
    """260 blocks of 64 channels: 256 of whole sequences, the others' sequences in segments."""
    B, T, D = 65, 800, 250
    assert 0 < pwb.scan_ws_floats(B, T, D) < 2 * 64 * 4 * 5
    scan(ctx, B, T, D, True, lens=None if lens is None else (lens * 17)[:B], seed=3)


def test_recurrence_step_of_more_blocks_than_a_launch_takes(ctx):
    """65535 sequences of one step and 4160 channels: 4259775 blocks.  Rows from both ends and around the launches' border."""
    B, D = 65535, 4160
    g = torch.Generator(device="cuda").manual_seed(4)
    f, x = (torch.randn(B, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    y = torch.full_like(f, 7.0)
    torch.cuda.synchronize()
    assert pwb.scan_ws_floats(B, 1, D) == 0
    a = pwb.ScanArgs(dtype=pwb.PW_BF16, f=f.data_ptr(), x=x.data_ptr(), ldf=D, ldx=D, B=B, T=1, D=D)
    ctx.scan_fwd(a, y.data_ptr(), D, None, None, None)
    ctx.synchronize()
    border = (1 << 22) // 65
    rows = torch.tensor(list(range(40)) + list(range(border - 20, border + 20)) + list(range(B - 40, B)), device="cuda")
    want = torch.sigmoid(-f[rows].double()) * x[rows].double()
    # half a step of bf16 (2^-8) for the output, 2^-20 for what fp32 adds before it
    assert ((y[rows].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -120).all()
    assert (y != 7.0).all()


def test_recurrence_states_in_place(ctx):
    """h_end over h0 and dh0 over dh_end, in one segment and in several."""
    for B, T, D in ((4, 1, 64), (1, 3000, 64), (5, 33, 70)):
        scan(ctx, B, T, D, True, aliases=True)


def test_recurrence_of_closed_and_open_gates(ctx):
    """Gates that saturate either way: the state stays exactly, or is exactly the input."""
    B, T, D = 2, 400, 64
    x = rnd(1, B * T, D).astype(np.float32)
    out = scan(ctx, B, T, D, False, f=np.full((B * T, D), 200.0), x=x, seed=9)
    h0 = rnd(12, B, D).astype(np.float32)
    assert np.array_equal(back(out[0]).reshape(B, T, D), np.broadcast_to(h0[:, None].astype(np.float64), (B, T, D)))
    out = scan(ctx, B, T, D, False, f=np.full((B * T, D), -200.0), x=x, seed=9)
    assert np.array_equal(back(out[0]), x.astype(np.float64))


def test_recurrence_of_nothing(ctx):
    h0, he = dev(rnd(1, 3, 10))[0], torch.full((3, 10), 7.0, device="cuda")
    t = torch.zeros(64, device="cuda")
    torch.cuda.synchronize()
    a = pwb.ScanArgs(dtype=pwb.PW_F32, f=t.data_ptr(), x=t.data_ptr(), ldf=10, ldx=10, B=3, T=0, D=10, h0=h0.data_ptr())
    ctx.scan_fwd(a, t.data_ptr(), 10, he.data_ptr(), None, None)
    ctx.synchronize()
    assert torch.equal(he, h0)
    ctx.scan_bwd(a, t.data_ptr(), 10, None, None, t.data_ptr(), 10, t.data_ptr(), 10, he.data_ptr(), None)
    ctx.synchronize()
    assert (back(he) == 0).all() and (back(t) == 0).all()


def test_recurrence_repeats_its_bits_and_decodes_step_by_step(ctx):
    one, two = scan(ctx, 1, 3000, 66, True, seed=5), scan(ctx, 1, 3000, 66, True, seed=5)
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    B, T, D = 3, 20, 70
    f, x = (torch.from_numpy(rnd(s, B, T, D).astype(np.float32)).cuda() for s in (1, 2))
    h = torch.zeros(B, D, device="cuda")
    y, whole = torch.zeros(B, T, D, device="cuda"), torch.zeros(B, T, D, device="cuda")
    torch.cuda.synchronize()
    a = pwb.ScanArgs(dtype=pwb.PW_F32, f=f.data_ptr(), x=x.data_ptr(), ldf=D, ldx=D, B=B, T=T, D=D)
    ctx.scan_fwd(a, whole.data_ptr(), D, None, None, None)
    for t in range(T):                                           # one token of every sequence at a time, state in place
        a = pwb.ScanArgs(dtype=pwb.PW_F32, f=f.data_ptr() + 4 * t * D, x=x.data_ptr() + 4 * t * D, ldf=T * D, ldx=T * D, B=B, T=1, D=D,
                         h0=h.data_ptr())
        ctx.scan_fwd(a, y.data_ptr() + 4 * t * D, T * D, h.data_ptr(), None, None)
    ctx.synchronize()
    # the order of compositions differs: a few roundings of values of up to 4
    within(back(y), back(whole), 64 * 2.0 ** -24 * 4)
    assert torch.equal(h, y[:, -1])


def test_operators_replay_in_a_graph(ctx):
    """Quantisation, a product and both passes of a recurrence over several segments, captured and replayed between eager
    work, against the eager results."""
    side = torch.cuda.Stream()
    with pwb.Context(0, side.cuda_stream) as c:
        B, T, D = 1, 2048, 64
        x = torch.randn(B * T, D, device="cuda").bfloat16()
        w = torch.randn(2 * D, D, device="cuda").bfloat16()
        q, s = torch.zeros(T, D, dtype=torch.uint8, device="cuda"), torch.zeros(pwb.f8_scale_bytes(T, D), dtype=torch.uint8, device="cuda")
        wq, wsc = torch.zeros(2 * D, D, dtype=torch.uint8, device="cuda"), torch.zeros(pwb.f8_scale_bytes(2 * D, D), dtype=torch.uint8, device="cuda")
        fx = torch.zeros(T, 2 * D, dtype=torch.bfloat16, device="cuda")
        y, dfx = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, 2 * D, dtype=torch.bfloat16, device="cuda")
        he, dh0 = torch.zeros(B, D, device="cuda"), torch.zeros(B, D, device="cuda")
        st = torch.zeros(pwb.scan_state_floats(B, T, D), device="cuda")
        ws = torch.zeros(pwb.scan_ws_floats(B, T, D), device="cuda")
        assert ws.numel() > 0
        torch.cuda.synchronize()

        def run():
            c.f8_quantize(pwb.F8QuantizeArgs(dtype=pwb.PW_BF16, format=pwb.PW_E4M3, block_rows=1, x=x.data_ptr(), rows=T, cols=D, ldx=D,
                                             q=q.data_ptr(), ldq=D, q_scale=s.data_ptr()))
            c.f8_quantize(pwb.F8QuantizeArgs(dtype=pwb.PW_BF16, format=pwb.PW_E4M3, block_rows=128, x=w.data_ptr(), rows=2 * D, cols=D,
                                             ldx=D, q=wq.data_ptr(), ldq=D, q_scale=wsc.data_ptr()))
            c.f8_gemm(pwb.F8GemmArgs(M=T, N=2 * D, K=D, lda=D, ldb=D, ldc=2 * D, epilogue=pwb.PW_EPI_STORE, out_dtype=pwb.PW_BF16,
                                     A=q.data_ptr(), B=wq.data_ptr(), a_scale=s.data_ptr(), b_scale=wsc.data_ptr(), C=fx.data_ptr()))
            a = pwb.ScanArgs(dtype=pwb.PW_BF16, f=fx.data_ptr(), x=fx.data_ptr() + 2 * D, ldf=2 * D, ldx=2 * D, B=B, T=T, D=D)
            c.scan_fwd(a, y.data_ptr(), D, he.data_ptr(), st.data_ptr(), ws.data_ptr())
            c.scan_bwd(a, y.data_ptr(), D, he.data_ptr(), st.data_ptr(), dfx.data_ptr(), 2 * D, dfx.data_ptr() + 2 * D, 2 * D,
                       dh0.data_ptr(), ws.data_ptr())
        outs = (q, s, wq, wsc, fx, y, he, dfx, dh0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        for k in range(3):
            x.copy_(torch.randn(B * T, D, device="cuda"))
            torch.cuda.synchronize()
            run()
            c.synchronize()
            want = [t.clone() for t in outs]
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, t) for p, t in zip(want, outs)), k


def test_sizes_past_32_bits_of_offset(ctx):
    """Rows whose offset does not fit 32 bits, in elements and in bytes: the last rows of a strided array."""
    rows, cols, ld = 66000, 40, 1 << 16
    try:
        x = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")     # 8.6 GB, of which little is touched
    except torch.OutOfMemoryError:
        pytest.skip("no room")
    v = x.view(rows, ld)
    vals = rnd(0, rows, cols)
    v[:, :cols] = torch.from_numpy(vals).cuda().bfloat16()
    v[:, cols:2 * cols] = torch.from_numpy(vals[::-1].copy()).cuda().bfloat16()
    lowv = low(vals, True)
    torch.cuda.synchronize()
    y = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    a = pwb.DropoutArgs(dtype=pwb.PW_BF16, out_dtype=pwb.PW_BF16, rows=rows, cols=cols, ldx=ld, ldy=cols, p=0.5, seed=1, site=0, step=0)
    ctx.dropout_fwd(a, x.data_ptr(), None, None, y.data_ptr())
    ctx.synchronize()
    keep, _ = R.dropout_keep(rows, cols, 0.5, 1, 0, 0)
    assert np.array_equal(back(y), np.where(keep, 2 * lowv, 0.0))
    s = torch.zeros(pwb.f8_scale_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    q = torch.zeros(rows, 48, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ctx.f8_quantize(pwb.F8QuantizeArgs(dtype=pwb.PW_BF16, format=pwb.PW_E4M3, block_rows=1, x=x.data_ptr(), rows=rows, cols=cols, ldx=ld,
                                       q=q.data_ptr(), ldq=48, q_scale=s.data_ptr()))
    ctx.synchronize()
    wq, _ = R.quantize(lowv[-50:], "e4m3", 1)
    same_codes(q.cpu().numpy()[-50:], wq, "e4m3", "q")
    he = torch.zeros(1, cols, device="cuda")
    ws = torch.zeros(max(2, pwb.scan_ws_floats(1, rows, cols)), device="cuda")
    torch.cuda.synchronize()
    a = pwb.ScanArgs(dtype=pwb.PW_BF16, f=x.data_ptr(), x=x.data_ptr() + 2 * cols, ldf=ld, ldx=ld, B=1, T=rows, D=cols)
    ctx.scan_fwd(a, y.data_ptr(), cols, he.data_ptr(), None, ws.data_ptr())
    ctx.synchronize()
    tail = 400                                                   # a state from before these steps has faded below 2^-24 of it
    ry, rh = R.scan_fwd(lowv[None, -tail:], lowv[::-1][None, -tail:], np.zeros((1, cols)))
    assert (np.cumprod(R._sigmoid(lowv[-tail:]), 0)[-1] * 8 < 2.0 ** -24).all()
    within(back(he), rh, 64 * 2.0 ** -24 * 5)
    del x, v
    torch.cuda.empty_cache()


# ---- together --------------------------------------------------------------------------------------------------

class _Quantized:
    def __init__(self, ctx, x, fmt, block=1):
        rows, cols = x.shape
        z = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.rows, self.cols, self.fmt = rows, cols, fmt
        self.q, self.s = z(rows, up(cols, 16)), z(pwb.f8_scale_bytes(rows, cols))
        self.qt, self.st = z(cols, up(rows, 16)), z(pwb.f8_scale_bytes(cols, rows))
        torch.cuda.synchronize()
        ctx.f8_quantize(pwb.F8QuantizeArgs(dtype=DT[x.dtype == torch.bfloat16], format=F8[fmt], block_rows=block, x=x.data_ptr(), rows=rows,
                                           cols=cols, ldx=cols, q=self.q.data_ptr(), ldq=up(cols, 16), q_scale=self.s.data_ptr(),
                                           qt=self.qt.data_ptr(), ldqt=up(rows, 16), qt_scale=self.st.data_ptr()))

    def side(self, turned):
        """(bytes, scales, rows, K, format)"""
        return (self.qt, self.st, self.cols, up(self.rows, 16), self.fmt) if turned else (self.q, self.s, self.rows, up(self.cols, 16), self.fmt)


def _mul(ctx, a, b, out_bf16, epilogue=pwb.PW_EPI_STORE, bias=None):
    (qa, sa, M, K, fa), (qb, sb, N, K2, fb) = a, b
    assert K == K2
    c = torch.zeros(M, up(N, 8), dtype=act(out_bf16), device="cuda")
    torch.cuda.synchronize()
    ctx.f8_gemm(pwb.F8GemmArgs(a_format=F8[fa], b_format=F8[fb], M=M, N=N, K=K, lda=K, ldb=K, ldc=c.shape[1], epilogue=epilogue,
                               out_dtype=DT[out_bf16], A=qa.data_ptr(), B=qb.data_ptr(), a_scale=sa.data_ptr(), b_scale=sb.data_ptr(),
                               bias=bias.data_ptr() if bias is not None else None, C=c.data_ptr()))
    return c


def test_a_recurrent_residual_block_forward_and_backward(ctx):
    """x_out = x + dropout(scan(a W_fx + b_fx) W_o + b_o) with every product in 8 bits: the whole block against 64 bits without any
    rounding.  An e4m3 rounding is off by 2^-4 at most and by 2^-4 / sqrt(12) * 1.5 = 2.7 % in the mean square, an e5m2 one by twice
    that; the longest path here passes three products of two such operands, forward and backward, which add up in the mean
    square to less than 3 * sqrt(2.7^2 + 5.4^2) = 18 %.  Each stage by itself is held to a rounding in the tests above."""
    B, T, d, p = 2, 136, 128, 0.1
    n = B * T
    rng = np.random.RandomState(0)
    a, x = low(rng.randn(n, d), True), rng.randn(n, d).astype(np.float32)
    wfx, wo = low(0.1 * rng.randn(d, 2 * d), True), low(0.1 * rng.randn(d, d), True)
    bfx, bo = rng.randn(2 * d).astype(np.float32) * 0.2, rng.randn(d).astype(np.float32) * 0.2
    dout = rng.randn(n, d).astype(np.float32)
    t = lambda v, dt=torch.float32: torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(dt).cuda()  # noqa: E731
    ad, xd, bfxd, bod, doutd = t(a, torch.bfloat16), t(x), t(bfx), t(bo), t(dout)
    qa, qwfx, qwo = _Quantized(ctx, ad, "e4m3"), _Quantized(ctx, t(wfx, torch.bfloat16), "e4m3", 128), _Quantized(ctx, t(wo, torch.bfloat16), "e4m3", 128)
    fx = _mul(ctx, qa.side(False), qwfx.side(True), True, pwb.PW_EPI_BIAS, bfxd)
    h = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    states = torch.zeros(pwb.scan_state_floats(B, T, d), device="cuda")
    ws = torch.zeros(max(2, pwb.scan_ws_floats(B, T, d), pwb.dropout_bwd_ws_floats(n, d)), device="cuda")
    torch.cuda.synchronize()
    sa = pwb.ScanArgs(dtype=pwb.PW_BF16, f=fx.data_ptr(), x=fx.data_ptr() + 2 * d, ldf=2 * d, ldx=2 * d, B=B, T=T, D=d)
    ctx.scan_fwd(sa, h.data_ptr(), d, None, states.data_ptr(), ws.data_ptr())
    qh = _Quantized(ctx, h, "e4m3")
    u = _mul(ctx, qh.side(False), qwo.side(True), True)
    out = torch.zeros(n, d, device="cuda")
    torch.cuda.synchronize()
    da = pwb.DropoutArgs(dtype=pwb.PW_BF16, out_dtype=pwb.PW_F32, rows=n, cols=d, ldx=d, ldy=d, p=p, seed=77, site=1, step=2)
    ctx.dropout_fwd(da, u.data_ptr(), bod.data_ptr(), xd.data_ptr(), out.data_ptr())
    # backward
    du, dbo = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(d, device="cuda")
    torch.cuda.synchronize()
    ctx.dropout_bwd(da, doutd.data_ptr(), du.data_ptr(), dbo.data_ptr(), ws.data_ptr())
    qdu = _Quantized(ctx, du, "e5m2")
    dwo = _mul(ctx, qh.side(True), qdu.side(True), False)
    dh = _mul(ctx, qdu.side(False), qwo.side(False), True)
    dfx = torch.zeros(n, 2 * d, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    ctx.scan_bwd(sa, dh.data_ptr(), d, None, states.data_ptr(), dfx.data_ptr(), 2 * d, dfx.data_ptr() + 2 * d, 2 * d, None, ws.data_ptr())
    qdfx = _Quantized(ctx, dfx, "e5m2")
    dwfx = _mul(ctx, qa.side(True), qdfx.side(True), False)
    dact = _mul(ctx, qdfx.side(False), qwfx.side(False), True)
    ctx.synchronize()
    # 64 bits
    keep, scale = R.dropout_keep(n, d, p, 77, 1, 2)
    rfx = a @ wfx + bfx
    rf, rx = rfx[:, :d].reshape(B, T, d), rfx[:, d:].reshape(B, T, d)
    rh, _ = R.scan_fwd(rf, rx, np.zeros((B, d)))
    rh2 = rh.reshape(n, d)
    ru = rh2 @ wo
    branch = np.where(keep, (ru + bo) * scale, 0.0)
    rdu = np.where(keep, dout * scale, 0.0)
    rdh = rdu @ wo.T
    rdf, rdx, _ = R.scan_bwd(rf, rx, np.zeros((B, d)), rdh.reshape(B, T, d), np.zeros((B, d)))
    rdfx = np.concatenate([rdf.reshape(n, d), rdx.reshape(n, d)], 1)
    rel = lambda g, r: np.linalg.norm(back(g) - r) / np.linalg.norm(r)  # noqa: E731
    assert np.linalg.norm(back(out) - x - branch) / np.linalg.norm(branch) < 0.18
    assert rel(dbo, rdu.sum(0)) < 1e-5
    for name, g, r in (("fx", fx, rfx), ("h", h, rh2), ("u", u, ru), ("dwo", dwo, rh2.T @ rdu), ("dh", dh, rdh), ("dfx", dfx, rdfx),
                       ("dwfx", dwfx, a.T @ rdfx), ("da", dact, rdfx @ wfx.T)):
        assert rel(g, r) < 0.18, (name, rel(g, r))
    # and the gradient of the whole block is the one of its loss: central differences along directions, in 64 bits
    def loss(wfx_, wo_):
        q = a @ wfx_ + bfx
        hh, _ = R.scan_fwd(q[:, :d].reshape(B, T, d), q[:, d:].reshape(B, T, d), np.zeros((B, d)))
        return (np.where(keep, (hh.reshape(n, d) @ wo_ + bo) * scale, 0.0) * dout).sum()
    for name, g, i in (("dwfx", back(dwfx), 0), ("dwo", back(dwo), 1)):
        s, v = 1e-5, g / np.linalg.norm(g)
        w = [wfx, wo]
        plus, minus = [m + s * v if k == i else m for k, m in enumerate(w)], [m - s * v if k == i else m for k, m in enumerate(w)]
        num = (loss(*plus) - loss(*minus)) / (2 * s)
        assert abs(num - np.linalg.norm(g)) < 0.18 * np.linalg.norm(g), name
