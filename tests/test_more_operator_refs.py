"""The references of more_operator_refs.py against hand-made values and differences, and what the launchers of these operators refuse (CPU)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import more_operator_refs as M
from paper_2203_12533_amd import binding as pwb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_f4_reference_by_hand():
    x = np.zeros((2, 33))
    x[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -6.0]
    x[1, 0], x[1, 32] = 6.0000001, np.nan
    c, b = M.f4_quantize(x)
    assert c.shape == (2, 64) and c[0, :8].tolist() == [0, 2, 2, 4, 4, 6, 6, 15]
    assert b.tolist() == [[127, 0], [128, 255]] and c[1, 0] == 5 and not c[1, 32:].any()
    assert M.f4_values(c, b)[0, :8].tolist() == [0, 1, 1, 2, 2, 4, 4, -6] and np.isnan(M.f4_values(c, b)[1, 32:]).all()
    assert M.f4_pack(c)[0, :4].tolist() == [0x20, 0x42, 0x64, 0xF6]
    i = M.f4_scale_index(65, 5)
    assert np.unique(i).size == 65 * 5 and i.max() < M.f4_scale_table(np.zeros((65, 5), np.uint8)).size == pwb.f4_scale_bytes(65, 129)
    assert i[17, 2] == 2 * 64 + 4 + 1 and i[64, 4] == (128 + 64) * 4


def test_f4_reference_is_the_nearest_of_all_values():
    y = np.random.RandomState(0).uniform(-6, 6, 1000)
    v = np.concatenate([M.E2M1, -M.E2M1])
    got = v[M.f4_nearest(y)]
    assert np.array_equal(np.abs(y - got), np.abs(y[:, None] - v).min(1))


def differences(f, args, grads, tol=1e-7):
    """Directional derivatives of a scalar f against its gradients: s^2 of third derivatives, 1e-16 / s of rounding."""
    rng = np.random.RandomState(3)
    for i, g in enumerate(grads):
        for _ in range(6):
            u, s = rng.randn(*g.shape), 1e-5
            plus, minus = ([a + w * s * u if k == i else a for k, a in enumerate(args)] for w in (1, -1))
            num = (f(*plus) - f(*minus)) / (2 * s)
            assert abs(num - (g * u).sum()) < tol * (1 + abs(num))


@pytest.mark.parametrize("residual", [False, True])
def test_rms_gradients_against_differences(residual):
    rng = np.random.RandomState(0)
    x, dh, dres, g = rng.randn(4, 6), rng.randn(4, 6), rng.randn(4, 6), rng.randn(6)
    dx, dg = M.rms_bwd(x, g, 1e-2, dh, dres if residual else None)

    def loss(x, g):
        xo, _, h = M.rms_fwd(x, None, g, 1e-2)
        return (h * dh).sum() + ((xo * dres).sum() if residual else 0.0)
    differences(loss, [x, g], [dx, dg])


@pytest.mark.parametrize("scale", [1.0, 0.6, 2.5])
def test_logprob_gradients_against_differences(scale):
    rng = np.random.RandomState(1)
    z, t = rng.randn(5, 9), np.array([0, 8, -1, 4, 9])
    dl, de = rng.randn(5), rng.randn(5)

    def loss(z):
        lp, h, _, _ = M.logprob_fwd(z, t, scale)
        return (lp * dl).sum() + (h * de).sum()
    differences(loss, [z], [M.logprob_bwd(z, t, dl, de, scale)])


def test_logprob_reference_of_masked_rows():
    inf = np.inf
    z = np.array([[1.0, -inf, 1.0], [-inf, -inf, -inf], [0.0, inf, 0.0], [np.nan, 0.0, 0.0], [-inf, 2.0, -inf]])
    t = np.array([1, 0, 0, 1, 1])
    lp, h, ids, best = M.logprob_fwd(z, t, 1.0, 3)
    assert lp[0] == -inf and lp[1] == -inf and np.isnan(lp[2:4]).all() and lp[4] == 0.0
    assert np.isclose(h[0], np.log(2)) and h[1] == 0.0 and np.isnan(h[2:4]).all() and h[4] == 0.0
    assert ids.tolist() == [[0, 2, -1], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1], [1, -1, -1]] and best[0, 2] == -inf and np.isnan(best[2]).all()
    dz = M.logprob_bwd(z, t, np.ones(5), np.ones(5))
    assert np.isfinite(dz[[0, 1, 4]]).all() and not dz[1].any() and np.isnan(dz[2:4]).all() and dz[0, 1] == 1.0


def test_clip_reference():
    n, f, g = M.clip([np.array([3.0]), np.array([4.0])], 1.0)
    assert n == 5.0 and f == 0.2 and np.allclose([v[0] for v in g], [0.6, 0.8])
    assert M.clip([np.array([3.0])], 3.0)[1] == 1.0


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
  int32_t* const I = (int32_t*)P;
  auto off = [&](int n) { return (void*)((char*)P + n); };
  auto foff = [&](int n) { return (float*)((char*)P + n); };
  const hipError_t no = hipErrorInvalidValue, ok = hipSuccess;
  #define REFUSE(call, base, change) { auto a = base; a.change; expect(#call " " #change, call, no); }
  #define ACCEPT(call, base, change) { auto a = base; a.change; expect(#call " " #change, call, ok); }
  // quantisation
  const F4QuantizeArgs q0{kF32, 1, P, 8, 100, 100, P, 128, S, P, 32, S};
  #define Q launch_f4_quantize(nullptr, a)
  ACCEPT(Q, q0, rows = 0) ACCEPT(Q, q0, cols = 0)
  REFUSE(Q, q0, dtype = kI32) REFUSE(Q, q0, block_rows = 64) REFUSE(Q, q0, block_rows = 0) REFUSE(Q, q0, x = nullptr)
  REFUSE(Q, q0, rows = -1) REFUSE(Q, q0, cols = -1) REFUSE(Q, q0, ldx = 99) REFUSE(Q, q0, ldq = 112) REFUSE(Q, q0, ldq = 96)
  REFUSE(Q, q0, ldqt = 0) REFUSE(Q, q0, ldqt = 48) REFUSE(Q, q0, q_scale = S + 8) REFUSE(Q, q0, qt_scale = S + 4) REFUSE(Q, q0, q_scale = nullptr) REFUSE(Q, q0, qt_scale = nullptr)
  REFUSE(Q, q0, q = off(8)) REFUSE(Q, q0, qt = off(4)) REFUSE(Q, q0, x = off(2)) REFUSE(Q, q0, rows = 128LL * 65535 + 1)
  REFUSE(Q, q0, cols = (1LL << 30) + 1)
  { auto a = q0; a.q = a.qt = nullptr; expect("no output", Q, no); }
  expect("bytes", (hipError_t)(f4_scale_bytes(65, 129) != 1024 || f4_scale_bytes(-1, 4) != -1 || f4_scale_bytes(0, 4) != 0 ||
                               f4_scale_bytes(4, (1LL << 30) + 1) != -1), ok);
  // products
  GemmF4Args g0{};
  g0.M = 8; g0.N = 8; g0.K = 32; g0.lda = g0.ldb = 32; g0.ldc = 8; g0.epilogue = kEpiStore; g0.out_dtype = kF32;
  g0.A = g0.B = P; g0.a_scale = g0.b_scale = S; g0.C = P;
  #define G launch_gemm_f4(nullptr, a)
  ACCEPT(G, g0, M = 0) ACCEPT(G, g0, N = 0)
  REFUSE(G, g0, A = nullptr) REFUSE(G, g0, B = nullptr) REFUSE(G, g0, C = nullptr) REFUSE(G, g0, a_scale = nullptr) REFUSE(G, g0, b_scale = nullptr)
  REFUSE(G, g0, K = 16) REFUSE(G, g0, K = 64) REFUSE(G, g0, K = -32) REFUSE(G, g0, M = -1)
  REFUSE(G, g0, lda = 48) REFUSE(G, g0, ldb = 16) REFUSE(G, g0, ldc = 12) REFUSE(G, g0, N = 9) REFUSE(G, g0, M = (1LL << 26) + 1) REFUSE(G, g0, N = (1LL << 26) + 8)
  REFUSE(G, g0, A = off(8)) REFUSE(G, g0, C = off(8)) REFUSE(G, g0, bias = foff(4)) REFUSE(G, g0, a_scale = S + 4) REFUSE(G, g0, b_scale = S + 8)
  REFUSE(G, g0, epilogue = kEpiAdam) REFUSE(G, g0, epilogue = -1) REFUSE(G, g0, epilogue = kEpiBiasResidual) REFUSE(G, g0, epilogue = kEpiGeluBwd)
  REFUSE(G, g0, epilogue = kEpiBiasGelu) REFUSE(G, g0, out_dtype = kI32)
  { auto a = g0; a.M = a.N = a.ldc = 1LL << 26; expect("more tiles than a launch has", G, no); a.lda = 1LL << 25; expect("nor apart", G, no); }
  { auto a = g0; a.out_dtype = kBF16; a.accumulate = 1; expect("bf16 accumulate", G, no); }
  { auto a = g0; a.epilogue = kEpiBias; a.accumulate = 1; expect("bias accumulate", G, no); }
  { auto a = g0; a.epilogue = kEpiBiasResidual; a.aux = P; a.out_dtype = kBF16; expect("bf16 residual", G, no); }
  // norm
  const RmsnormArgs r0{kBF16, 4, 10, 10, 10, 1e-5f, F};
  const F8Out none{}, f8{kE4M3, P, 16, S};
  #define RF launch_rmsnorm_fwd(nullptr, a, F, P, F, P, f8, F)
  #define RB launch_rmsnorm_bwd(nullptr, a, P, F, F, F, F, P, F, F, 0)
  ACCEPT(RF, r0, rows = 0)
  REFUSE(RF, r0, dtype = kI32) REFUSE(RF, r0, rows = -1) REFUSE(RF, r0, rows = 1LL << 31) REFUSE(RF, r0, cols = 0) REFUSE(RF, r0, cols = 16385) REFUSE(RF, r0, ldx = 9)
  REFUSE(RF, r0, ldh = 9) REFUSE(RF, r0, eps = -1.f) REFUSE(RF, r0, eps = NAN) REFUSE(RF, r0, g = nullptr) REFUSE(RF, r0, g = foff(2)) REFUSE(RF, r0, rows = (1LL << 30) + 1)
  REFUSE(RB, r0, dtype = kI32) REFUSE(RB, r0, ldx = 9) REFUSE(RB, r0, ldh = 9) REFUSE(RB, r0, cols = 16385) REFUSE(RB, r0, g = nullptr)
  { const auto a = r0;
    expect("no x", launch_rmsnorm_fwd(nullptr, a, nullptr, P, F, P, none, F), no);
    expect("no output", launch_rmsnorm_fwd(nullptr, a, F, P, F, nullptr, none, F), no);
    expect("odd x", launch_rmsnorm_fwd(nullptr, a, foff(2), P, F, P, none, F), no);
    expect("odd y", launch_rmsnorm_fwd(nullptr, a, F, off(1), F, P, none, F), no);
    expect("odd x_out", launch_rmsnorm_fwd(nullptr, a, F, P, foff(1), P, none, F), no);
    expect("odd h", launch_rmsnorm_fwd(nullptr, a, F, P, F, off(1), none, F), no);
    expect("odd rstd", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, none, foff(2)), no);
    expect("format", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, F8Out{2, P, 16, S}, F), no);
    expect("no scale", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, F8Out{kE4M3, P, 16, nullptr}, F), no);
    expect("odd scale", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, F8Out{kE4M3, P, 16, S + 2}, F), no);
    expect("odd q", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, F8Out{kE4M3, off(8), 16, S}, F), no);
    expect("short ldq", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, F8Out{kE4M3, P, 0, S}, F), no);
    expect("odd ldq", launch_rmsnorm_fwd(nullptr, a, F, P, F, P, F8Out{kE4M3, P, 24, S}, F), no);
    expect("no dh", launch_rmsnorm_bwd(nullptr, a, nullptr, F, F, F, F, P, F, F, 0), no);
    expect("no x", launch_rmsnorm_bwd(nullptr, a, P, nullptr, F, F, F, P, F, F, 0), no);
    expect("no rstd", launch_rmsnorm_bwd(nullptr, a, P, F, nullptr, F, F, P, F, F, 0), no);
    expect("no dx", launch_rmsnorm_bwd(nullptr, a, P, F, F, F, nullptr, P, F, F, 0), no);
    expect("odd dres", launch_rmsnorm_bwd(nullptr, a, P, F, F, foff(2), F, P, F, F, 0), no);
    expect("odd dy", launch_rmsnorm_bwd(nullptr, a, P, F, F, F, F, off(1), F, F, 0), no);
    expect("odd dg", launch_rmsnorm_bwd(nullptr, a, P, F, F, F, F, P, foff(2), F, 0), no); }
  { auto a = r0; a.rows = 10000; expect("no ws", launch_rmsnorm_bwd(nullptr, a, P, F, F, F, F, P, F, nullptr, 0), no);
    expect("odd ws", launch_rmsnorm_bwd(nullptr, a, P, F, F, F, F, P, F, foff(4), 0), no); }
  expect("ws", (hipError_t)(rmsnorm_bwd_ws_floats(-1, 4) != -1 || rmsnorm_bwd_ws_floats(4, 0) != -1 || rmsnorm_bwd_ws_floats(4, 16385) != -1 ||
                            rmsnorm_bwd_ws_floats(0, 5) != 0 || rmsnorm_bwd_ws_floats(1LL << 31, 5) != -1 || rmsnorm_bwd_ws_floats(10000, 5) <= 0), ok);
  // log probabilities
  const LogprobArgs l0{kBF16, P, 10, 4, 10, I, 1.f};
  #define LF launch_logprob_fwd(nullptr, a, F, F, F, 3, I, F, F)
  #define LB launch_logprob_bwd(nullptr, a, F, F, F, F, P, 10)
  ACCEPT(LF, l0, rows = 0) ACCEPT(LB, l0, rows = 0)
  REFUSE(LF, l0, dtype = kI32) REFUSE(LF, l0, z = nullptr) REFUSE(LF, l0, z = off(1)) REFUSE(LF, l0, rows = -1) REFUSE(LF, l0, rows = 1LL << 31) REFUSE(LF, l0, vocab = 0)
  REFUSE(LF, l0, vocab = (1LL << 28) + 1) REFUSE(LF, l0, ldz = 9) REFUSE(LF, l0, targets = nullptr) REFUSE(LF, l0, targets = (int32_t*)off(2)) REFUSE(LF, l0, scale = 0.f)
  REFUSE(LF, l0, scale = -1.f) REFUSE(LF, l0, scale = NAN) REFUSE(LF, l0, scale = INFINITY)
  REFUSE(LB, l0, dtype = kI32) REFUSE(LB, l0, z = nullptr) REFUSE(LB, l0, ldz = 9) REFUSE(LB, l0, targets = nullptr) REFUSE(LB, l0, scale = 0.f) REFUSE(LB, l0, vocab = 11)
  { const auto a = l0;
    expect("k", launch_logprob_fwd(nullptr, a, F, F, F, 33, I, F, F), no);
    expect("k", launch_logprob_fwd(nullptr, a, F, F, F, -1, I, F, F), no);
    expect("no ids", launch_logprob_fwd(nullptr, a, F, F, F, 3, nullptr, F, F), no);
    expect("no top", launch_logprob_fwd(nullptr, a, F, F, F, 3, I, nullptr, F), no);
    expect("ids without k", launch_logprob_fwd(nullptr, a, F, F, F, 0, I, F, F), no);
    expect("nothing", launch_logprob_fwd(nullptr, a, nullptr, nullptr, nullptr, 0, nullptr, nullptr, F), no);
    expect("odd logp", launch_logprob_fwd(nullptr, a, foff(2), F, F, 3, I, F, F), no);
    expect("odd entropy", launch_logprob_fwd(nullptr, a, F, foff(2), F, 3, I, F, F), no);
    expect("odd stats", launch_logprob_fwd(nullptr, a, F, F, foff(4), 3, I, F, F), no);
    expect("odd ids", launch_logprob_fwd(nullptr, a, F, F, F, 3, (int32_t*)off(2), F, F), no);
    expect("odd top", launch_logprob_fwd(nullptr, a, F, F, F, 3, I, foff(2), F), no);
    expect("no stats", launch_logprob_bwd(nullptr, a, nullptr, F, F, F, P, 10), no);
    expect("odd stats", launch_logprob_bwd(nullptr, a, foff(4), F, F, F, P, 10), no);
    expect("no entropy", launch_logprob_bwd(nullptr, a, F, nullptr, F, F, P, 10), no);
    expect("no dz", launch_logprob_bwd(nullptr, a, F, F, F, F, nullptr, 10), no);
    expect("odd dz", launch_logprob_bwd(nullptr, a, F, F, F, F, off(1), 10), no);
    expect("short lddz", launch_logprob_bwd(nullptr, a, F, F, F, F, P, 9), no);
    expect("odd dlogp", launch_logprob_bwd(nullptr, a, F, F, foff(2), F, P, 10), no); }
  expect("ws", (hipError_t)(logprob_ws_floats(-1, 4, 0) != -1 || logprob_ws_floats(4, 0, 0) != -1 || logprob_ws_floats(4, 4, 33) != -1 ||
                            logprob_ws_floats(4, 4, -1) != -1 || logprob_ws_floats(0, 4, 3) != 0), ok);
  // clipping
  const GradTensor t0{P, P, 5, kF32};
  #define C launch_grad_clip(nullptr, &a, 1, 1.f, F, F)
  REFUSE(C, t0, g = nullptr) REFUSE(C, t0, g = off(2)) REFUSE(C, t0, out = off(2)) REFUSE(C, t0, n = -1) REFUSE(C, t0, n = (1LL << 40) + 1) REFUSE(C, t0, dtype = kI32)
  { const auto a = t0;
    expect("count", launch_grad_clip(nullptr, &a, -1, 1.f, F, F), no);
    expect("count", launch_grad_clip(nullptr, &a, (1 << 20) + 1, 1.f, F, F), no);
    expect("none", launch_grad_clip(nullptr, nullptr, 1, 1.f, F, F), no);
    expect("max", launch_grad_clip(nullptr, &a, 1, -1.f, F, F), no);
    expect("max", launch_grad_clip(nullptr, &a, 1, NAN, F, F), no);
    expect("no result", launch_grad_clip(nullptr, &a, 1, 1.f, nullptr, F), no);
    expect("odd result", launch_grad_clip(nullptr, &a, 1, 1.f, foff(2), F), no);
    expect("no ws", launch_grad_clip(nullptr, &a, 1, 1.f, F, nullptr), no);
    expect("odd ws", launch_grad_clip(nullptr, &a, 1, 1.f, F, foff(4)), no); }
  { const GradTensor two[2] = {{P, P, 1LL << 39, kF32}, {P, P, (1LL << 39) + 1, kF32}}; expect("too many", launch_grad_clip(nullptr, two, 2, 1.f, F, F), no); }
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


def run_on_the_host(tmp_path, body):
    """A program over the launchers; `expect` as in REFUSALS."""
    src, exe = tmp_path / "more.cpp", tmp_path / "more"
    src.write_text("#include <string>" + REFUSALS[:REFUSALS.index("  // quantisation")] + body + '  std::printf("%d\\n", bad);\n  return bad != 0;\n}\n')
    here = os.path.dirname(pwb.LIB_PATH)
    subprocess.check_call(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(here, "csrc"), str(src),
                           "-L", here, "-lpw", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath," + here, "-Wl,-rpath,/opt/rocm/lib", "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_a_gradient_in_place_has_the_rows_of_the_logits(tmp_path):
    """With another stride a row of the gradient would lie on logits that another workgroup has still to read."""
    run_on_the_host(tmp_path, r'''
  const LogprobArgs a{kBF16, P, 12, 4, 10, I, 1.f};
  expect("closer", launch_logprob_bwd(nullptr, a, F, F, F, F, P, 10), no);
  expect("further apart", launch_logprob_bwd(nullptr, a, F, F, F, F, P, 16), no);
  LogprobArgs none = a; none.rows = 0;
  expect("the same", launch_logprob_bwd(nullptr, none, F, F, F, F, P, 12), ok);
''')


def test_a_scale_whose_base_2_form_overflows_is_refused(tmp_path):
    """s log2 e has to be a number: 0 times infinity would make the likeliest token's shift NaN."""
    run_on_the_host(tmp_path, r'''
  LogprobArgs a{kBF16, P, 10, 4, 10, I, 3e38f};
  expect("forward", launch_logprob_fwd(nullptr, a, F, F, F, 3, I, F, F), no);
  expect("backward", launch_logprob_bwd(nullptr, a, F, F, F, F, P, 10), no);
  a.scale = 0x1.000002p127f; expect("just above", launch_logprob_fwd(nullptr, a, F, F, F, 3, I, F, F), no);
  a.scale = 0x1p127f; a.rows = 0; expect("the largest", launch_logprob_fwd(nullptr, a, F, F, F, 3, I, F, F), ok);
  a.scale = 1e-30f; expect("a small one", launch_logprob_fwd(nullptr, a, F, F, F, 3, I, F, F), ok);
''')


def test_sizes_of_the_product_tests_reach_the_kernels_that_they_are_for(tmp_path):
    """Where the choice of a kernel changes, sizes here and in the GPU tests have to follow."""
    import test_gpu_more_operator_edges as edges
    want = [(1, 200, 128, 0, "direct, 4 waves"), (3, 5000, 256, 0, "direct, 4 waves"), (33, 1000, 4096, 0, "direct, 8 waves"), (70, 5000, 96, 1 << 24, "32 x 64"),
            (70, 5000, 96, (1 << 24) + 32, "direct, 4 waves"), (260, 300, 1056, 0, "direct, 4 waves"), (300, 520, 2080, 0, "32 x 64"), (500, 1300, 1056, 0, "64 x 64"),
            (700, 900, 160, 0, "64 x 64"), (1030, 1100, 544, 0, "128 x 64"), (1300, 1100, 256, 0, "128 x 64"), (1500, 1420, 288, 0, "128 x 128"),
            (1700, 1900, 1056, 0, "128 x 128"), (40000, 70, 160, 0, "128 x 128"), (70, 40000, 160, 0, "128 x 128"),
            (2560, 4096, 256, 0, "128 x 128"), (3100, 2900, 256, 0, "128 x 128"), (3100, 2900, 416, 0, "256 x 256"), (2570, 4099, 288, 0, "256 x 256"),
            (2560, 4096, 4096, 0, "256 x 256")]
    want += [(m, n, k, 0, "256 x 256") for m, n, k in edges.STREAM] + [(4900, 4701, 288, 0, "256 x 256"), (9000, 4700, 288, 0, "256 x 256")]
    lines = ["  struct { int64_t m, n, k, ld; const char* name; } const want[] = {"]
    lines += ['    {%d, %d, %d, %d, "%s"},' % w for w in want]
    lines += ["  };", "  for (const auto& w : want) {", "    GemmF4Args a{}; a.M = w.m; a.N = w.n; a.K = w.k; a.lda = w.ld ? w.ld : w.k; a.ldb = w.k;",
              "    const char* got = gemm_f4_kernel(a);",
              '    if (std::string(got) != w.name) { std::printf("%ld x %ld x %ld: %s, not %s\\n", (long)w.m, (long)w.n, (long)w.k, got, w.name); ++bad; }', "  }\n"]
    run_on_the_host(tmp_path, "\n".join(lines))
    tiles = [(m, n, -(-m // 256) * -(-n // 256)) for m, n, _ in edges.STREAM]
    assert any(t > 256 and m % 256 == n % 256 == 0 for m, n, t in tiles) and any(t > 256 and m % 256 and n % 256 for m, n, t in tiles)   # several to a workgroup


def test_calls_without_a_context_or_arguments_are_refused():
    lib = pwb.lib()
    for name, args in (("f4_quantize", [None]), ("f4_gemm", [None]), ("rmsnorm_fwd", [None] * 7), ("rmsnorm_bwd", [None] * 9 + [0]),
                       ("logprob_fwd", [None] * 4 + [0] + [None] * 3), ("logprob_bwd", [None] * 6 + [0]), ("grad_clip", [None, 0, 1.0, None, None])):
        assert getattr(lib, "pw_op_" + name)(None, *args) == pwb.PW_ERR_INVALID, name


def test_argument_structures_match_the_header(tmp_path):
    structs = [("pw_f4_quantize_args", pwb.F4QuantizeArgs), ("pw_f4_gemm_args", pwb.F4GemmArgs), ("pw_rmsnorm_args", pwb.RmsnormArgs),
               ("pw_f8_out", pwb.F8Out), ("pw_logprob_args", pwb.LogprobArgs), ("pw_grad_tensor", pwb.GradTensor)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "pw.h"', 'int main(void) {']
    for c, py in structs:
        lines.append('printf("%%zu ", sizeof(%s));' % c)
        lines += ['printf("%%zu ", offsetof(%s, %s));' % (c, f[0]) for f in py._fields_]
    (tmp_path / "s.c").write_text("\n".join(lines + ["return 0;}"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "s")], text=True).split()]
    want = [n for _, py in structs for n in [C.sizeof(py)] + [getattr(py, f[0]).offset for f in py._fields_]]
    assert got == want
