"""Ends of the ranges that the header promises for the 8-bit operands and the recurrence, and sharper bounds than those of
test_gpu_operators.py: special values in bf16, scale bytes at either end, sums that every pipe forms exactly, infinite states,
and an error bound of its own for every element of a recurrence."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import operator_refs as R
import test_gpu_operators as G
from gpu_util import DT
from paper_2203_12533_amd import binding as pwb

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ctx():
    with pwb.Context(0) as c:
        yield c


# ---- the measured cases ----------------------------------------------------------------------------------------

def test_a_pass_comes_after_its_inputs_and_before_its_readers():
    """perf/operators.py without a synchronisation, behind work that keeps the stream of the inputs busy for a while."""
    spec = importlib.util.spec_from_file_location("perf_operators", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.own = True
    before = torch.cuda.current_stream()
    try:
        case = {"family": "quant", "rows": 333, "cols": 500, "dtype": "bf16", "format": "e5m2", "block": 1, "both": True}
        m.run(m.prepare(case, 1))
        torch.cuda.synchronize()
        want = {k: v.clone() for k, v in m.run(m.prepare(case, 2)).items()}
        torch.cuda.synchronize()
        w = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            w = w @ w * 1e-2
        got = {k: v.view(torch.uint8).clone() for k, v in m.run(m.prepare(case, 2)).items()}
        assert torch.cuda.current_stream() == m._stream
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k].view(torch.uint8)) for k in want)
    finally:
        torch.cuda.synchronize()
        if m._context is not None:
            m._context.close()
        torch.cuda.set_stream(before)


# ---- quantisation ----------------------------------------------------------------------------------------------

BF16_MAX = float.fromhex("0x1.fep127")


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
def test_bf16_quantisation_of_every_kind_of_value(ctx, fmt, block):
    """As in fp32, with values that bf16 holds: zeros, subnormals, the largest numbers, maxima at a border of the scale, ties, scales
    clamped at 2^-127, and NaN or infinities in either half of a word and in either row of a pair of rows."""
    x = G.low(G.rnd(7, 140, 300), True)
    x[3] = 0.0
    x[4] = -0.0
    x[5, :128] = 2.0 ** -133 * np.arange(1, 129)                  # subnormal in bf16: steps of 2^-133
    x[6, :128] = 2.0 ** -133
    x[7, 128:256] = BF16_MAX
    x[8, 128:256] = -BF16_MAX
    x[8, 0], x[8, 1:128] = 1.75, G.low(np.linspace(-1.7, 1.7, 127), True)
    x[9, 0], x[9, 1:128] = 1.75 + 2.0 ** -7, G.low(np.linspace(-1.7, 1.7, 127), True)
    grid = R.decode_table(fmt)[:128]
    grid = grid[np.isfinite(grid)]
    mid = ((grid[1:] + grid[:-1]) / 2)[-100:]
    x[10, :mid.size], x[10, mid.size:128] = mid, R.TOP[fmt]       # ties, of at most five bits
    x[11, :128] = mid[:128].repeat(2)[:128] * 2.0 ** -100
    x[11, 0] = R.TOP[fmt] * 2.0 ** -100
    for row, col, v in ((20, 4, np.nan), (23, 5, np.nan), (24, 138, np.inf), (27, 139, -np.inf), (30, 270, -np.inf), (33, 299, np.nan),
                        (130, 0, np.inf), (139, 1, np.nan)):
        x[row, col] = v
        x[row, (col + 1) % 300], x[row ^ 1, col] = 3e30, -5e-30   # its neighbours are ordinary
    x[40, :128] = np.nan
    x[41, 128:256] = np.inf
    x[42:44, 250:] = -np.inf
    x[44, :128] = 2.0 ** -119 * np.linspace(0.01, 1.75, 128)      # around where the scale stops at 2^-127
    x[45, :128] = 2.0 ** -119 * np.linspace(0.01, 1.76, 128)
    x[46, :128] = 2.0 ** -112 * np.linspace(0.01, 1.75, 128)
    x[47, :128] = 2.0 ** -125 * np.linspace(-1, 1.75, 128)
    G.check_quantized(ctx, x, fmt, block, True)
    G.check_quantized(ctx, x[:, :77], fmt, block, True, ldx=81, offset=1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantisation_around_the_smallest_scale(ctx, fmt, bf16):
    """Blocks whose scale is 2^-127 or next to it, each row a factor of two above the one before."""
    x = G.rnd(3, 40, 256) * 2.0 ** (np.arange(40) - 140.0)[:, None]
    G.check_quantized(ctx, x, fmt, 1, bf16)


# ---- products --------------------------------------------------------------------------------------------------

TILES = [(3, 200), (40, 200), (260, 300), (500, 1300), (1300, 1100), (1700, 1900), (2100, 2600), (2304, 4096), (2300, 4090)]


def multiply(ctx, a, ea, b, eb, fa, fb, bf16, M, N, K):
    """C of operands given as bytes and scale exponents (128 stands for the byte 255)."""
    at, bt = (torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in (a, b))
    sa, sb = (torch.from_numpy(R.scale_table(e)).cuda() for e in (ea, eb))
    ldc = G.up(N, 8)
    c = torch.full((M, ldc), 7.0, dtype=G.act(bf16), device="cuda")
    torch.cuda.synchronize()
    ctx.f8_gemm(pwb.F8GemmArgs(a_format=G.F8[fa], b_format=G.F8[fb], M=M, N=N, K=K, lda=K, ldb=K, ldc=ldc, epilogue=pwb.PW_EPI_STORE,
                               out_dtype=DT[bf16], A=at.data_ptr(), B=bt.data_ptr(), a_scale=sa.data_ptr(), b_scale=sb.data_ptr(),
                               C=c.data_ptr()))
    ctx.synchronize()
    assert (c[:, N:] == 7.0).all()
    return G.back(c[:, :N])


def scaled(q, e, fmt):
    """The operand's values in 64 bits; a block with the byte 255 is NaN, its zeros too."""
    with np.errstate(invalid="ignore"):
        return R.decode_table(fmt)[q] * np.where(e == 128, np.nan, 2.0 ** np.minimum(e, 127))[:, np.arange(q.shape[1]) // 128]


def times(va, vb):
    with np.errstate(invalid="ignore", over="ignore"):
        return va @ vb.T


SMALL = {"e4m3": [0x38, 0xB8, 0x40, 0xC0, 0x00, 0x80], "e5m2": [0x3C, 0xBC, 0x40, 0xC0, 0x00, 0x80]}      # 1, -1, 2, -2, 0, -0


@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,N", TILES)
def test_sums_that_every_pipe_forms_exactly(ctx, M, N, bf16, fa, fb):
    """Operands of 0, 1, 2 with scales of 1, 2 and 4 for each row and block: all products and sums are whole numbers under 2^13, so
    nothing is cut off or rounded before the output is: every element is the one nearest to the result, in every tile."""
    K = 400
    rng = np.random.RandomState(M + N)
    a, b = (np.array(SMALL[f], np.uint8)[rng.randint(0, 6, (n, K))] for n, f in ((M, fa), (N, fb)))
    ea, eb = rng.randint(0, 3, (M, 4)), rng.randint(0, 3, (N, 4))
    ref = times(scaled(a, ea, fa), scaled(b, eb, fb))
    assert np.abs(ref).max() < 2 ** 13
    assert np.array_equal(multiply(ctx, a, ea, b, eb, fa, fb, bf16, M, N, K), G.low(ref, bf16))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("M,N", TILES)
def test_scale_bytes_at_both_ends(ctx, M, N, fmt, bf16):
    """Bytes 0, 1, 253, 254 in single rows of either operand against scales that bring the result back into range, over zeros in the
    other blocks; 255 makes its row (its column) NaN, over zeros too."""
    K = 272
    rng = np.random.RandomState(M)
    a, b = (np.array(SMALL[fmt], np.uint8)[rng.randint(0, 6, (n, K))] for n in (M, N))
    ea, eb = np.zeros((M, 3), int), np.zeros((N, 3), int)
    # (byte - 127) of a row; with numbers of at most 2 on the other side at 2^0 .. 2^4 every product is a normal fp32 number
    rows = rng.permutation(M)[:6] if M >= 6 else np.arange(M)
    for r, e in zip(rows, (-127, 126, 128, -126, 127, 128)):
        ea[r] = 0 if e == 128 else e
        if e == 128:
            ea[r, rng.randint(3)] = 128
        if e == -127:
            a[r] &= 0x80                        # +-2 only: 1 * 2^-127 is below what the bf16 pipe holds exactly
            a[r] |= 0x40
        if e in (126, 127):                     # one product: a sum would leave the range
            a[r] = 0
            a[r, 5] = SMALL[fmt][0]
    b[:, 5] = SMALL[fmt][1]
    cols = rng.permutation(N)[:2]
    eb[cols[0], 2] = 128
    b[cols[1]], eb[cols[1], 1] = 0, 128         # a column of zeros
    va, vb = scaled(a, ea, fmt), scaled(b, eb, fmt)
    ref, mag = times(va, vb), times(np.abs(va), np.abs(vb))
    got = multiply(ctx, a, ea, b, eb, fmt, fmt, bf16, M, N, K)
    # whole numbers of the smallest scale: exact up to the output's rounding; a result under 2^-126 may be taken as zero
    tiny = np.abs(ref) < 2.0 ** -126
    G.within(got, ref, np.where(tiny, 2.0 ** -126, G.EPS[bf16] * np.abs(ref)), "C")
    assert np.isnan(ref[:, cols]).all() and (M < 6 or np.isnan(ref[rows[[2, 5]]]).all()) and np.isfinite(mag).any()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,N", TILES)
def test_nan_and_infinite_operands(ctx, M, N, bf16):
    """NaN (either format) and infinities (e5m2) stay in their row or column and follow the formula there; in the last, partial
    block of k too."""
    K = 400
    rng = np.random.RandomState(N)
    a = np.array(SMALL["e4m3"][:4], np.uint8)[rng.randint(0, 4, (M, K))]
    b = np.array(SMALL["e5m2"], np.uint8)[rng.randint(0, 6, (N, K))]
    a[0, 7], a[M - 1, K - 1] = 0x7F, 0xFF
    cols = rng.permutation(N)[:7]
    for c, (k, v) in zip(cols, ((0, 0x7C), (K - 1, 0xFC), (200, 0x7D), (130, 0xFF), (131, 0x7C), (255, 0xFC), (256, 0x7E))):
        b[c, k] = v
    b[cols[4], 140] = 0xFC                      # two infinities: a sum of one sign, or NaN
    ea, eb = rng.randint(-2, 3, (M, 4)), rng.randint(-2, 3, (N, 4))
    ref = times(scaled(a, ea, "e4m3"), scaled(b, eb, "e5m2"))
    got = multiply(ctx, a, ea, b, eb, "e4m3", "e5m2", bf16, M, N, K)
    G.within(got, ref, G.EPS[bf16] * np.abs(ref), "C")
    keep = np.setdiff1d(np.arange(N), cols)
    assert np.isfinite(got[1:M - 1][:, keep]).all() and (M < 4 or np.isinf(ref[1:M - 1][:, cols]).any())


@pytest.mark.parametrize("M,N", TILES)
def test_a_residual_in_place_in_every_tile(ctx, M, N):
    """C over aux, with a bias: whole numbers, equal to the last bit; columns behind N stay."""
    K, ldc = 144, G.up(N, 8) + 8
    rng = np.random.RandomState(M)
    a, b = (np.array(SMALL["e4m3"], np.uint8)[rng.randint(0, 6, (n, K))] for n in (M, N))
    ea, eb = rng.randint(0, 3, (M, 2)), rng.randint(0, 3, (N, 2))
    bias, res = rng.randint(-50, 50, N).astype(np.float32), rng.randint(-1000, 1000, (M, N)).astype(np.float32)
    at, bt, sa, sb, bt32 = (torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in (a, b, R.scale_table(ea), R.scale_table(eb), bias))
    c = torch.full((M, ldc), 7.0, device="cuda")
    c[:, :N] = torch.from_numpy(res).cuda()
    torch.cuda.synchronize()
    ctx.f8_gemm(pwb.F8GemmArgs(M=M, N=N, K=K, lda=K, ldb=K, ldc=ldc, epilogue=pwb.PW_EPI_BIAS_RESIDUAL, out_dtype=pwb.PW_F32, A=at.data_ptr(),
                               B=bt.data_ptr(), a_scale=sa.data_ptr(), b_scale=sb.data_ptr(), bias=bt32.data_ptr(), aux=c.data_ptr(), C=c.data_ptr()))
    ctx.synchronize()
    assert np.array_equal(G.back(c[:, :N]), times(scaled(a, ea, "e4m3"), scaled(b, eb, "e4m3")) + bias + res) and (c[:, N:] == 7.0).all()


# ---- dropout ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols,ld,offset", [(1, 5, 5, 1), (300, 77, 83, 3), (9000, 200, 201, 1)])
def test_dropout_of_bf16_rows_in_place(ctx, rows, cols, ld, offset):
    """y over x and dx over dy where rows start anywhere; what lies between the rows stays."""
    keep, _ = R.dropout_keep(rows, cols, 0.5, 9, 1, 2)
    x = G.low(G.rnd(1, rows, cols), True)
    t, p = G.dev(x, torch.bfloat16, ld, fill=7.0, offset=offset)
    a = pwb.DropoutArgs(dtype=pwb.PW_BF16, out_dtype=pwb.PW_BF16, rows=rows, cols=cols, ldx=ld, ldy=ld, p=0.5, seed=9, site=1, step=2)
    ctx.dropout_fwd(a, p, None, None, p)
    ctx.synchronize()
    assert np.array_equal(G.back(t)[:, :cols], np.where(keep, 2 * x, 0.0)) and (G.back(t)[:, cols:] == 7.0).all()
    ctx.dropout_bwd(a, p, p)
    ctx.synchronize()
    assert np.array_equal(G.back(t)[:, :cols], np.where(keep, 4 * x, 0.0)) and (G.back(t)[:, cols:] == 7.0).all()


# ---- gated recurrence ------------------------------------------------------------------------------------------

def recur(ctx, f, x, h0, dy, dh, lens, bf16):
    """-> y, h_end, df, dx, dh0 of f, x, dy [B, T, D] (values that the type holds)."""
    B, T, D = f.shape
    dt = G.act(bf16)
    flat = lambda v: torch.from_numpy(np.ascontiguousarray(v, np.float32)).reshape(B * T, D).to(dt).cuda()  # noqa: E731
    ft, xt, dyt = flat(f), flat(x), flat(dy)
    h0t, dht = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (h0, dh))
    lt = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    y, df, dx = (torch.full((B * T, D), 7.0, dtype=dt, device="cuda") for _ in range(3))
    he, dh0 = (torch.full((B, D), 7.0, device="cuda") for _ in range(2))
    states = torch.full((max(1, pwb.scan_state_floats(B, T, D)),), float("nan"), device="cuda")
    ws = torch.full((max(2, pwb.scan_ws_floats(B, T, D)),), float("nan"), device="cuda")
    torch.cuda.synchronize()
    a = pwb.ScanArgs(dtype=DT[bf16], f=ft.data_ptr(), x=xt.data_ptr(), ldf=D, ldx=D, B=B, T=T, D=D, h0=h0t.data_ptr(),
                     lens=lt.data_ptr() if lt is not None else None)
    ctx.scan_fwd(a, y.data_ptr(), D, he.data_ptr(), states.data_ptr(), ws.data_ptr())
    ctx.scan_bwd(a, dyt.data_ptr(), D, dht.data_ptr(), states.data_ptr(), df.data_ptr(), D, dx.data_ptr(), D, dh0.data_ptr(), ws.data_ptr())
    ctx.synchronize()
    return tuple(G.back(v).reshape(s) for v, s in ((y, f.shape), (he, h0.shape), (df, f.shape), (dx, f.shape), (dh0, h0.shape)))


NAMES = ("y", "h_end", "df", "dx", "dh0")


def check_recurrence(ctx, f, x, h0, dy, dh, lens, bf16, names=NAMES):
    f, x, dy = (G.low(v, bf16) for v in (f, x, dy))
    h0, dh = (np.asarray(v, np.float32).astype(np.float64) for v in (h0, dh))
    n = None if lens is None else np.array(lens)
    with np.errstate(invalid="ignore", over="ignore"):
        (y, he), (df, dx, dh0) = R.scan_fwd(f, x, h0, n), R.scan_bwd(f, x, h0, dy, dh, n)
        ey, eh, edf, edx, edh = R.scan_bounds(f, x, h0, dy, dh, n)
    got = dict(zip(NAMES, recur(ctx, f, x, h0, dy, dh, lens, bf16)))
    half = G.EPS[bf16]
    for name, ref, allow in (("y", y, ey), ("h_end", he, eh), ("df", df, edf), ("dx", dx, edx), ("dh0", dh0, edh)):
        if name not in names:
            continue
        bad = R.exceeds(got[name], ref, allow, 0.0 if name in ("h_end", "dh0") else half)
        at = np.argwhere(bad)[:3]
        assert not bad.any(), (name, bad.mean(), [(tuple(i), got[name][tuple(i)], ref[tuple(i)]) for i in at])
    return y, he, df, dx, dh0


RUNS = [(1, 1, 1, None), (8, 1, 200, None), (2, 9, 30, None), (1, 17, 65, None), (2, 256, 64, None), (1, 257, 70, None), (1, 1000, 130, None),
        (1, 4097, 8, None), (2, 2000, 3, None), (3, 1030, 70, [0, 513, 1030]), (3, 520, 70, [-3, 900, 255]), (1, 3000, 66, None),
        (2, 600, 64, None), (65, 800, 250, None), (65, 800, 250, "mixed"), (3, 16384, 64, [16384, 9000, 77])]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,T,D,lens", RUNS)
def test_every_element_of_a_recurrence(ctx, B, T, D, lens, bf16):
    lens = ([800, 0, 31, 770] * 17)[:B] if lens == "mixed" else lens
    rng = np.random.RandomState(T + D)
    f, x, dy = rng.randn(B, T, D) * 1.5 + 1, rng.randn(B, T, D), rng.randn(B, T, D)
    check_recurrence(ctx, f, x, rng.randn(B, D), dy, rng.randn(B, D), lens, bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("size", [20.0, 60.0, 80.0])
def test_gates_far_from_zero(ctx, size, bf16):
    """Gates near 0 or 1, each to the precision that the bound gives it."""
    rng = np.random.RandomState(int(size))
    B, T, D = 2, 700, 66
    f = np.where(rng.rand(B, T, D) < 0.5, 1.0, -1.0) * size * (0.9 + 0.1 * rng.rand(B, T, D))
    check_recurrence(ctx, f, rng.randn(B, T, D), rng.randn(B, D), rng.randn(B, T, D), rng.randn(B, D), None, bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shift", [-6.0, -2.0, 0.0, 3.0])
@pytest.mark.parametrize("B,T,D,lens", [(4, 1, 66, None), (2, 40, 66, None), (1, 300, 70, None), (3, 1030, 70, [0, 513, 1030]), (1, 4097, 64, None),
                                        (1, 16384, 34, None)])
def test_infinite_states_inputs_and_gradients(ctx, B, T, D, lens, shift, bf16):
    """An infinity stays one whatever the gates behind it (their product over a tile is far below the smallest number), meets another
    of either sign as the formula has it, and what lies in front of it is finite."""
    rng = np.random.RandomState((T + int(shift)) % 2 ** 32)
    f, x, dy = rng.randn(B, T, D) + shift, rng.randn(B, T, D), rng.randn(B, T, D)
    h0, dh = rng.randn(B, D), rng.randn(B, D)
    h0[:, 0], h0[:, 1], h0[:, 2] = np.inf, -np.inf, np.nan
    dh[:, 3], dh[:, 4], dh[:, 5] = np.inf, -np.inf, np.nan
    for c in range(6, 14):                               # somewhere in the sequence
        x[:, rng.randint(T), c] = np.inf if c % 2 else -np.inf
    for c in range(12, 20):
        dy[:, rng.randint(T), c] = np.inf if c % 2 else -np.inf
    x[:, T // 3, 20], x[:, T // 2, 20] = np.inf, -np.inf
    x[:, T // 3, 21], dy[:, T // 2, 21] = np.nan, np.nan
    f[:, T // 2, 22] = np.nan
    y, he, df, dx, dh0 = check_recurrence(ctx, f, x, h0, dy, dh, lens, bf16)
    assert np.isinf(he[:, :2]).all() and np.isinf(dh0[:, 3:5]).all()
    assert np.isfinite(y[:, :, 23:]).all() and np.isfinite(df[:, :, 23:]).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("size", [90.0, 100.0, 200.0, 600.0])
def test_infinities_and_gates_beyond_what_fp32_holds(ctx, size, bf16):
    """Gates of 1e-39 to 1e-260: an infinite state passes them, and an infinite input."""
    rng = np.random.RandomState(int(size))
    B, T, D = 2, 600, 66
    f = np.where(rng.rand(B, T, D) < 0.5, 1.0, -1.0) * size
    x, h0, dh = rng.randn(B, T, D), rng.randn(B, D), rng.randn(B, D)
    h0[:, 0], h0[:, 1], dh[:, 2], dh[:, 3] = np.inf, -np.inf, np.inf, -np.inf
    for c in range(4, 24):
        x[:, rng.randint(T), c] = np.inf if c % 2 else -np.inf
    _, he, _, _, dh0 = check_recurrence(ctx, f, x, h0, rng.randn(B, T, D), dh, None, bf16, ("y", "h_end", "dx", "dh0"))
    assert np.isinf(he[:, :2]).all() and np.isinf(he[:, 4:24]).all() and np.isinf(dh0[:, 2:4]).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("T", [1, 40, 3000])
def test_gates_that_are_shut_or_open_for_good(ctx, T, bf16):
    """f of either infinity: the state is the input, or stays; no more than 2^-125 of anything else comes through, within what a gate
    is rounded by (exp2 and the reciprocal by one unit in the last place each, the product: 5 * 2^-24 < 2^-21)."""
    rng = np.random.RandomState(T)
    B, D = 2, 66
    f, x, dy = np.where(np.arange(D) % 2, np.inf, -np.inf) * np.ones((B, T, D)), G.low(rng.randn(B, T, D), bf16), rng.randn(B, T, D)
    x[:, ::3] = 0.0
    h0, dh = rng.randn(B, D), rng.randn(B, D)
    y, he, df, dx, dh0 = recur(ctx, f, x, h0, G.low(dy, bf16), dh, None, bf16)
    h0, dh = (v.astype(np.float32).astype(np.float64) for v in (h0, dh))
    dy = G.low(dy, bf16)
    shut = 2.0 ** -125 * (1 + 2.0 ** -21)
    least = shut * 8                                             # of states and gradients of up to 8
    live = x[:, :, ::2] != 0
    assert np.array_equal(y[:, :, ::2][live], x[:, :, ::2][live]) and (np.abs(y[:, :, ::2][~live]) <= least).all()
    assert np.array_equal(he[:, 1::2], h0[:, 1::2]) and np.array_equal(y[:, :, 1::2], np.broadcast_to(G.low(h0, bf16)[:, None, 1::2], (B, T, D // 2)))
    total = np.abs(dy).sum(1) + np.abs(dh)
    assert (np.abs(df) <= least * total[:, None]).all() and (np.abs(dx[:, :, 1::2]) <= shut * total[:, None, 1::2]).all()
    assert (np.abs(dh0[:, ::2]) <= shut * total[:, ::2]).all()
    want = dh[:, 1::2] + dy[:, :, 1::2].sum(1)
    assert (np.abs(dh0[:, 1::2] - want) <= 2.0 ** -24 * 2 * T * total[:, 1::2]).all()
