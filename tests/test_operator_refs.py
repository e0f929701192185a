"""The references that the GPU tests of the 8-bit operands, dropout and the recurrence use, against published values and
finite differences; and what the library refuses, checked on the host before anything reaches a GPU."""
import os
import subprocess
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_refs as R  # noqa: E402
from paper_2203_12533_amd import binding as pwb  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_philox_reproduces_the_published_known_answers():
    """Known-answer vectors of Philox4x32-10 that its authors publish."""
    for ctr, key, want in [([0] * 4, [0] * 2, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
                           ([0xffffffff] * 4, [0xffffffff] * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
                           ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
                            "d16cfe09 94fdcceb 5001e420 24126ea1")]:
        assert " ".join("%08x" % int(v) for v in R.philox(ctr, key)) == want


def test_dropout_reference_keeps_the_share_it_says():
    keep, scale = R.dropout_keep(300, 1003, 0.3, 99, 5, 7)
    n = keep.size
    assert abs(keep.mean() - 1 / scale) < 5 * np.sqrt(0.21 / n)             # five standard deviations
    other, _ = R.dropout_keep(300, 1003, 0.3, 99, 5, 8)
    assert 0.5 < (keep == other).mean() < 0.66                              # 0.58 expected of independent masks
    assert R.dropout_keep(3, 9, 0.0, 1, 2, 3)[0].all() and not R.dropout_keep(3, 9, 1.0, 1, 2, 3)[0].any()
    small, _ = R.dropout_keep(300, 11, 0.3, 99, 5, 7)
    assert np.array_equal(small, keep[:, :11])                              # a mask does not depend on the width


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantisation_reference(fmt):
    v = R.decode_table(fmt)
    fin = np.isfinite(v[:128])
    assert v[:128][fin].max() == R.TOP[fmt] and np.array_equal(R.nearest_code(v[:128][fin], fmt), np.arange(128)[fin])
    rng = np.random.RandomState(3)
    x = rng.randn(130, 300) * np.exp(3 * rng.randn(130, 1))
    for block in (1, 128):
        q, e = R.quantize(x, fmt, block)
        back = R.values(q, e, fmt)[:, :300]
        peak = np.repeat(np.stack([[np.abs(x[r // block * block:r // block * block + block, b:b + 128]).max() for b in range(0, 300, 128)]
                                   for r in range(130)]), 128, 1)[:, :300]
        tiny = {"e4m3": 2.0 ** -10, "e5m2": 2.0 ** -17}[fmt]                # half the smallest step, in units of the scale
        assert (np.abs(back - x) <= np.maximum(R.HALF_STEP[fmt] * np.abs(x), tiny * 2 * peak / R.TOP[fmt])).all()
        assert np.array_equal(R.scale_table(e)[R.scale_index(*e.shape)], e + 127)
    q, e = R.quantize(np.array([[0.0, -0.0, np.nan, np.inf, -np.inf, 3.0]]), fmt)
    d = R.decode_table(fmt)[q[0, :6]]
    assert d[0] == 0 and np.signbit(d[1]) and np.isnan(d[2]) and d[5] * 2.0 ** e[0, 0] == 3.0
    assert (np.isnan(d[3]) and np.isnan(d[4])) if fmt == "e4m3" else (d[3] == np.inf and d[4] == -np.inf)


@pytest.mark.parametrize("lens", [None, [7, 0, 3]])
def test_recurrence_gradients_against_differences(lens):
    rng = np.random.RandomState(1)
    B, T, D = 3, 7, 4
    lens = None if lens is None else np.array(lens)
    f, x, dy = rng.randn(3, B, T, D)
    h0, dh = rng.randn(2, B, D)
    df, dx, dh0 = R.scan_bwd(f, x, h0, dy, dh, lens)

    def loss(f, x, h0):
        y, h = R.scan_fwd(f, x, h0, lens)
        return (y * dy).sum() + (h * dh).sum()
    for i, g in enumerate((df, dx, dh0)):
        args = [f, x, h0]
        for _ in range(8):
            u, s = rng.randn(*g.shape), 1e-5
            plus, minus = [a + s * u * (k == i) if k == i else a for k, a in enumerate(args)], \
                [a - s * u * (k == i) if k == i else a for k, a in enumerate(args)]
            num = (loss(*plus) - loss(*minus)) / (2 * s)
            assert abs(num - (g * u).sum()) < 1e-7 * (1 + abs(num))         # s^2 of third derivatives, 1e-16 / s of rounding


REFUSALS = r'''
#include <cstdio>
#include <cmath>
#include "kernels.hpp"
using namespace pw;
static int bad = 0;
static void expect(const char* what, hipError_t got, hipError_t want) {
  if (got != want) { std::printf("%s: %d\n", what, (int)got); ++bad; }
}
int main() {
  void* const P = (void*)(uintptr_t)4096;
  uint8_t* const S = (uint8_t*)P;
  float* const F = (float*)P;
  const hipError_t no = hipErrorInvalidValue, ok = hipSuccess;
  #define REFUSE(call, base, change) { auto a = base; a.change; expect(#change, call, no); }
  #define ACCEPT(call, base, change) { auto a = base; a.change; expect(#change, call, ok); }
  // quantisation
  const F8QuantizeArgs q0{kF32, kE4M3, 1, P, 8, 100, 100, P, 112, S, P, 16, S};
  #define Q launch_f8_quantize(nullptr, a)
  ACCEPT(Q, q0, rows = 0) ACCEPT(Q, q0, cols = 0)
  REFUSE(Q, q0, dtype = kI32) REFUSE(Q, q0, format = 2) REFUSE(Q, q0, format = -1) REFUSE(Q, q0, block_rows = 64) REFUSE(Q, q0, x = nullptr)
  REFUSE(Q, q0, rows = -1) REFUSE(Q, q0, cols = -1) REFUSE(Q, q0, ldx = 99) REFUSE(Q, q0, ldq = 104) REFUSE(Q, q0, ldq = 96)
  REFUSE(Q, q0, ldqt = 0) REFUSE(Q, q0, ldqt = 24) REFUSE(Q, q0, q_scale = S + 2) REFUSE(Q, q0, qt_scale = S + 1) REFUSE(Q, q0, q_scale = nullptr) REFUSE(Q, q0, qt_scale = nullptr)
  REFUSE(Q, q0, q = (char*)P + 8) REFUSE(Q, q0, qt = (char*)P + 4) REFUSE(Q, q0, x = (char*)P + 2) REFUSE(Q, q0, rows = 128LL * 65535 + 1)
  REFUSE(Q, q0, cols = (1LL << 30) + 1)
  { auto a = q0; a.q = a.qt = nullptr; expect("no output", Q, no); }
  expect("bytes", (hipError_t)(f8_scale_bytes(65, 129) != 256 || f8_scale_bytes(-1, 4) != -1 || f8_scale_bytes(0, 4) != 0 ||
                               f8_scale_bytes(4, (1LL << 30) + 1) != -1), ok);
  // products
  GemmF8Args g0{};
  g0.M = 8; g0.N = 8; g0.K = 16; g0.lda = g0.ldb = 16; g0.ldc = 8; g0.epilogue = kEpiStore; g0.out_dtype = kF32;
  g0.A = g0.B = P; g0.a_scale = g0.b_scale = S; g0.C = P;
  #define G launch_gemm_f8(nullptr, a)
  ACCEPT(G, g0, M = 0) ACCEPT(G, g0, N = 0)
  REFUSE(G, g0, A = nullptr) REFUSE(G, g0, B = nullptr) REFUSE(G, g0, C = nullptr) REFUSE(G, g0, a_scale = nullptr) REFUSE(G, g0, b_scale = nullptr)
  REFUSE(G, g0, a_format = 2) REFUSE(G, g0, b_format = -1) REFUSE(G, g0, K = 8) REFUSE(G, g0, K = 32) REFUSE(G, g0, K = -16) REFUSE(G, g0, M = -1)
  REFUSE(G, g0, lda = 24) REFUSE(G, g0, ldb = 8) REFUSE(G, g0, ldc = 12) REFUSE(G, g0, N = 9) REFUSE(G, g0, M = (1LL << 30) + 1)
  REFUSE(G, g0, A = (char*)P + 8) REFUSE(G, g0, C = (char*)P + 8) REFUSE(G, g0, bias = (float*)((char*)P + 4)) REFUSE(G, g0, a_scale = S + 2)
  REFUSE(G, g0, epilogue = kEpiAdam) REFUSE(G, g0, epilogue = -1) REFUSE(G, g0, epilogue = kEpiBiasResidual) REFUSE(G, g0, epilogue = kEpiGeluBwd)
  REFUSE(G, g0, epilogue = kEpiBiasGelu) REFUSE(G, g0, out_dtype = kI32)
  REFUSE(G, g0, M = (1LL << 26) + 1) REFUSE(G, g0, N = (1LL << 26) + 8)
  { auto a = g0; a.M = a.N = a.ldc = 1LL << 26; expect("more tiles than a launch has", G, no); a.lda = 1LL << 24; expect("nor apart", G, no); }
  { auto a = g0; a.out_dtype = kBF16; a.accumulate = 1; expect("bf16 accumulate", G, no); }
  { auto a = g0; a.epilogue = kEpiBias; a.accumulate = 1; expect("bias accumulate", G, no); }
  { auto a = g0; a.epilogue = kEpiBiasResidual; a.aux = P; a.out_dtype = kBF16; expect("bf16 residual", G, no); }
  // dropout
  const DropoutArgs d0{kBF16, kF32, 4, 5, 5, 5, 0.5f, 1, 2, 3, nullptr};
  #define DF launch_dropout_fwd(nullptr, a, P, F, F, P)
  #define DB launch_dropout_bwd(nullptr, a, P, P, F, F, 0)
  ACCEPT(DF, d0, rows = 0) ACCEPT(DF, d0, cols = 0) ACCEPT(DB, d0, cols = 0)
  REFUSE(DF, d0, p = -0.1f) REFUSE(DF, d0, p = 1.5f) REFUSE(DF, d0, p = NAN) REFUSE(DB, d0, p = NAN) REFUSE(DF, d0, dtype = kI32)
  REFUSE(DF, d0, out_dtype = kI32) REFUSE(DF, d0, out_dtype = kBF16) REFUSE(DF, d0, rows = -1) REFUSE(DF, d0, cols = -1) REFUSE(DF, d0, ldx = 4)
  REFUSE(DF, d0, ldy = 4) REFUSE(DB, d0, ldx = 4) REFUSE(DF, d0, rows = (1LL << 31) + 1) REFUSE(DF, d0, cols = (1LL << 24) + 1)
  REFUSE(DF, d0, step_dev = (uint32_t*)((char*)P + 1))
  { auto a = d0; a.dtype = kF32; a.out_dtype = kBF16; expect("f32 to bf16", launch_dropout_fwd(nullptr, a, P, F, nullptr, P), no); }
  { auto a = d0; expect("null x", launch_dropout_fwd(nullptr, a, nullptr, F, F, P), no); expect("null y", launch_dropout_fwd(nullptr, a, P, F, F, nullptr), no);
    expect("odd y", launch_dropout_fwd(nullptr, a, P, F, F, (char*)P + 2), no); a.rows = 100000; expect("no ws", launch_dropout_bwd(nullptr, a, P, P, F, nullptr, 0), no); a.rows = 4;
    expect("null dy", launch_dropout_bwd(nullptr, a, nullptr, P, F, F, 0), no); expect("null dx", launch_dropout_bwd(nullptr, a, P, nullptr, F, F, 0), no); }
  expect("ws", (hipError_t)(dropout_bwd_ws_floats(-1, 4) != -1 || dropout_bwd_ws_floats(0, 4) != 0 || dropout_bwd_ws_floats(4, 1LL << 40) != -1 || dropout_bwd_ws_floats(100000, 5) <= 0), ok);
  // recurrence
  const ScanArgs s0{kBF16, P, P, 8, 8, 2, 4, 8, nullptr, nullptr};
  #define SF launch_scan_fwd(nullptr, a, P, 8, nullptr, nullptr, nullptr)
  #define SB launch_scan_bwd(nullptr, a, P, 8, nullptr, F, P, 8, P, 8, nullptr, nullptr)
  ACCEPT(SF, s0, B = 0) ACCEPT(SF, s0, D = 0) ACCEPT(SB, s0, B = 0)
  REFUSE(SF, s0, dtype = kI32) REFUSE(SF, s0, f = nullptr) REFUSE(SF, s0, x = nullptr) REFUSE(SF, s0, ldf = 7) REFUSE(SB, s0, ldx = 7)
  REFUSE(SF, s0, B = -1) REFUSE(SF, s0, T = -1) REFUSE(SB, s0, D = -1) REFUSE(SF, s0, B = 65536) REFUSE(SF, s0, f = (char*)P + 1)
  REFUSE(SF, s0, h0 = (float*)((char*)P + 2)) REFUSE(SF, s0, lens = (int32_t*)((char*)P + 1)) REFUSE(SF, s0, D = (1 << 24) + 1)
  REFUSE(SF, s0, D = (1 << 21) + 1) REFUSE(SF, s0, ldf = (1 << 21) + 1) REFUSE(SB, s0, ldx = (1 << 21) + 1)
  { auto a = s0; const int64_t far = (1 << 21) + 1; expect("far y", launch_scan_fwd(nullptr, a, P, far, nullptr, nullptr, nullptr), no);
    expect("far dy", launch_scan_bwd(nullptr, a, P, far, nullptr, F, P, 8, P, 8, nullptr, nullptr), no);
    expect("far df", launch_scan_bwd(nullptr, a, P, 8, nullptr, F, P, far, P, 8, nullptr, nullptr), no);
    expect("far dx", launch_scan_bwd(nullptr, a, P, 8, nullptr, F, P, 8, P, far, nullptr, nullptr), no); }
  { auto a = s0; expect("null y", launch_scan_fwd(nullptr, a, nullptr, 8, nullptr, nullptr, nullptr), no);
    expect("short ldy", launch_scan_fwd(nullptr, a, P, 7, nullptr, nullptr, nullptr), no);
    expect("no states", launch_scan_bwd(nullptr, a, P, 8, nullptr, nullptr, P, 8, P, 8, nullptr, nullptr), no);
    expect("no dy", launch_scan_bwd(nullptr, a, nullptr, 8, nullptr, F, P, 8, P, 8, nullptr, nullptr), no);
    expect("short lddf", launch_scan_bwd(nullptr, a, P, 8, nullptr, F, P, 7, P, 8, nullptr, nullptr), no);
    a.T = 4096; a.B = 1;
    expect("no ws", launch_scan_fwd(nullptr, a, P, 8, nullptr, nullptr, nullptr), no);
    expect("odd ws", launch_scan_fwd(nullptr, a, P, 8, nullptr, nullptr, F + 1), no); }
  expect("sizes", (hipError_t)(scan_ws_floats(-1, 1, 1) != -1 || scan_state_floats(1, -1, 1) != -1 || scan_ws_floats(2, 0, 8) != 0 ||
                               scan_state_floats(2, 0, 8) != 0 || scan_state_floats(2, 1, 8) != 16 || scan_ws_floats(1, 4096, 8) <= 0), ok);
  std::printf("%d\n", bad);
  return bad != 0;
}
'''


def test_what_the_launchers_refuse(tmp_path):
    """Every refusal happens on the host: this program never reaches a GPU, with or without one."""
    src, exe = tmp_path / "refusals.cpp", tmp_path / "refusals"
    src.write_text(REFUSALS)
    here = os.path.dirname(pwb.LIB_PATH)
    subprocess.check_call(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(here, "csrc"), str(src),
                           "-L", here, "-lpw", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath," + here, "-Wl,-rpath,/opt/rocm/lib", "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_calls_without_a_context_or_arguments_are_refused():
    lib = pwb.lib()
    for name, args in (("f8_quantize", [None]), ("f8_gemm", [None]), ("dropout_fwd", [None] * 5), ("dropout_bwd", [None] * 5 + [0]),
                       ("scan_fwd", [None, None, 0, None, None, None]),
                       ("scan_bwd", [None, None, 0, None, None, None, 0, None, 0, None, None])):
        assert getattr(lib, "pw_op_" + name)(None, *args) == pwb.PW_ERR_INVALID, name


def test_argument_structures_match_the_header(tmp_path):
    import ctypes as C
    structs = [("pw_f8_quantize_args", pwb.F8QuantizeArgs), ("pw_f8_gemm_args", pwb.F8GemmArgs), ("pw_dropout_args", pwb.DropoutArgs),
               ("pw_scan_args", pwb.ScanArgs)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "pw.h"', 'int main(void) {']
    for c, py in structs:
        lines.append('printf("%%zu ", sizeof(%s));' % c)
        lines += ['printf("%%zu ", offsetof(%s, %s));' % (c, f[0]) for f in py._fields_]
    (tmp_path / "s.c").write_text("\n".join(lines + ["return 0;}"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "s")], text=True).split()]
    want = [n for _, py in structs for n in [C.sizeof(py)] + [getattr(py, f[0]).offset for f in py._fields_]]
    assert got == want


def bf16(a):
    from paper_2203_12533_amd import inputs as I
    return I.round_to_bf16(np.asarray(a, np.float32)).astype(np.float64)


@pytest.mark.parametrize("B,T,D,lens", [(1, 1000, 130, None), (1, 4097, 8, None), (2, 2000, 3, None), (3, 1030, 70, [0, 513, 1030]), (1, 3000, 66, None),
                                        (3, 520, 70, [-3, 900, 255]), (2, 600, 64, None), (5, 800, 25, None)])
def test_recurrence_bounds_reject_mistakes(B, T, D, lens):
    """The allowances for bf16 outputs let through results in fp32 and reject zeros, flipped signs, and a state or a gradient that is
    lost where tiles of 256 steps or segments of them meet."""
    rng = np.random.RandomState(T)
    f, x, dy = (bf16(v) for v in (rng.randn(B, T, D) * 1.5 + 1, rng.randn(B, T, D), rng.randn(B, T, D)))
    h0, dh = rng.randn(2, B, D).astype(np.float32).astype(np.float64)
    lens = None if lens is None else np.array(lens)
    y, he = R.scan_fwd(f, x, h0, lens)
    df, dx, dh0 = R.scan_bwd(f, x, h0, dy, dh, lens)
    ey, eh, edf, edx, edh = R.scan_bounds(f, x, h0, dy, dh, lens)
    half = R.HALF_STEP["bf16"]
    # fp32, step by step
    n = np.full(B, T) if lens is None else np.clip(lens, 0, T)
    h, hs, f4, x4, dy4 = h0.astype(np.float32), [], f.astype(np.float32), x.astype(np.float32), dy.astype(np.float32)
    one = np.float32(1)
    for t in range(T):
        hs.append(h)
        on = (t < n)[:, None]
        h = np.where(on, (h + np.exp(-f4[:, t]) * x4[:, t]) / (one + np.exp(-f4[:, t])), h).astype(np.float32)
    y4 = np.stack(hs[1:] + [h], 1) * (np.arange(T) < n[:, None])[:, :, None]
    assert not R.exceeds(bf16(y4), y, ey, half).any() and not R.exceeds(h, he, eh).any()
    r, df4, dx4 = dh.astype(np.float32), np.zeros((B, T, D), np.float32), np.zeros((B, T, D), np.float32)
    for t in reversed(range(T)):
        on = (t < n)[:, None]
        a, z, g = one / (one + np.exp(-f4[:, t])), one / (one + np.exp(f4[:, t])), dy4[:, t] + r
        df4[:, t], dx4[:, t] = np.where(on, g * (hs[t] - x4[:, t]) * a * z, 0), np.where(on, g * z, 0)
        r = np.where(on, a * g, r).astype(np.float32)
    assert not R.exceeds(bf16(df4), df, edf, half).any() and not R.exceeds(bf16(dx4), dx, edx, half).any()
    assert not R.exceeds(r, dh0, edh).any()
    # mistakes
    for ref, allow in ((y, ey), (df, edf), (dx, edx)):
        live = ref != 0
        for wrong in (np.zeros_like(ref), -ref):
            assert R.exceeds(bf16(wrong), ref, allow, half)[live].mean() > 0.99
    for cut in range(256, T, 256):
        b = int(np.argmax(n))
        if n[b] <= cut:
            continue
        late = [v[b:b + 1, cut:n[b]] for v in (f, x, dy)]
        early = [v[b:b + 1, :cut] for v in (f, x, dy)]
        zero = np.zeros((1, D))
        wrong_y = R.scan_fwd(late[0], late[1], zero)[0]
        assert R.exceeds(bf16(wrong_y), y[b:b + 1, cut:n[b]], ey[b:b + 1, cut:n[b]], half).any()
        wrong_df, _, _ = R.scan_bwd(late[0], late[1], zero, late[2], dh[b:b + 1])
        assert R.exceeds(bf16(wrong_df), df[b:b + 1, cut:n[b]], edf[b:b + 1, cut:n[b]], half).any()
        for wrong, ref, allow in zip(R.scan_bwd(early[0], early[1], h0[b:b + 1], early[2], zero), (df, dx), (edf, edx)):
            assert R.exceeds(bf16(wrong), ref[b:b + 1, :cut], allow[b:b + 1, :cut], half).any()


def test_exceeds_tells_infinities_and_nan_apart():
    ref = np.array([1.0, np.inf, -np.inf, np.nan, 0.0])
    assert not R.exceeds(ref, ref, 0.0).any()
    for i, v in ((0, np.nan), (0, np.inf), (1, np.nan), (1, -np.inf), (1, 3e38), (2, np.inf), (3, 0.0), (3, np.inf), (4, np.nan), (4, 1e-30)):
        got = ref.copy()
        got[i] = v
        assert R.exceeds(got, ref, 0.0).tolist() == [k == i for k in range(5)]
