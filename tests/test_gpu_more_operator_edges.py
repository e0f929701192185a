"""Ends of the ranges that the header promises for the 4-bit products, log probabilities and clipping: the signs of log probabilities and
entropies, sums over long rows, the largest and smallest scales, every epilogue of the product whose workgroups take tiles in turn, and arrays that no cache holds.

Tolerances are derived, not measured.  A rounding is off by half a step (relative 2^-24 in fp32, 2^-8 in bf16)."""
import numpy as np
import pytest
import torch

import test_gpu_more_operators as G
from gpu_util import DT
from paper_2203_12533_amd import binding as pwb

pytestmark = pytest.mark.gpu

U = G.U
p = G.p


@pytest.fixture(scope="module")
def ctx():
    with pwb.Context(0) as c:
        yield c


# ---- log probabilities: signs ----------------------------------------------------------------------------------

@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,vocab,scale", [(600, 1, 1.0), (600, 2, 0.7), (600, 130, 1.0), (200, 3000, 1.3), (600, 9000, 1.0), (40, 40000, 1.0),
                                              (40, 40000, 37.0)])
def test_log_probabilities_are_at_most_zero_and_entropies_at_least(ctx, rows, vocab, scale, bf16):
    """Rows with one token that is nearly certain, its logit of any size: the sum of the others is at, far below and above a rounding of
    1.  A NaN in a row still shows."""
    rng = np.random.RandomState(vocab)
    top = rng.uniform(1, 100, rows) * np.where(np.arange(rows) % 2, 1, -1) * 10.0 ** rng.randint(-2, 4, rows)
    z = top[:, None] - (rng.uniform(8, 30, (rows, 1)) + rng.rand(rows, vocab)) / scale
    t = rng.randint(0, vocab, rows)
    z[np.arange(rows), t] = top
    z[7, 0] = np.nan
    k = min(3, vocab)
    lp, en, st, ids, tl = G.logprob(ctx, z, t, scale, k, bf16, backward=False)
    lp, en, st, tl = G.back(lp)[0, :rows], G.back(en)[0, :rows], G.back(st), G.back(tl)
    ok = np.arange(rows) != 7
    assert (lp[ok] <= 0).all() and (tl[ok] <= 0).all(), (lp[ok].max(), tl[ok].max())
    assert (en[ok] >= 0).all() and (st[ok, 1] >= 0).all(), (en[ok].min(), st[ok, 1].min())
    assert np.isnan(lp[7]) and np.isnan(en[7]) and np.isnan(tl[7]).all() and np.isnan(st[7, 1])


# ---- log probabilities: long rows ------------------------------------------------------------------------------

def check_long_rows(ctx, levels, at, scale, bf16):
    """Rows of `levels` [rows, L] in the order that `at` [vocab] tells: sums over the L values are the reference."""
    rows, vocab = levels.shape[0], at.size
    levels = G.low(levels, bf16)
    dt = G.act(bf16)
    where = torch.from_numpy(at).cuda()
    z = torch.empty(rows, vocab, dtype=dt, device="cuda")
    for r in range(rows):
        z[r] = torch.from_numpy(levels[r]).to(dt).cuda()[where]
    del where
    n = np.bincount(at, minlength=levels.shape[1]).astype(np.float64)
    s = float(np.float32(scale))
    d = s * (levels - levels.max(1, keepdims=True))
    e = n * np.exp(d)
    S, T = e.sum(1), (e * d).sum(1)
    first = [int(np.argmax(at == level)) for level in range(levels.shape[1])]
    targets = np.array([first[r % len(first)] for r in range(rows)])
    dt_target = d[np.arange(rows), np.arange(rows) % len(first)]
    tt = torch.from_numpy(targets.astype(np.int32)).cuda()
    lp, en, st = G.full(1, rows, 7.0), G.full(1, rows, 7.0), G.full(rows, 2, 7.0)
    ws = G.full(1, pwb.logprob_ws_floats(rows, vocab, 0) + 1, float("nan"))
    a = pwb.LogprobArgs(dtype=DT[bf16], z=p(z), ldz=vocab, rows=rows, vocab=vocab, targets=p(tt), scale=scale)
    torch.cuda.synchronize()
    ctx.logprob_fwd(a, p(lp), p(en), p(st), 0, None, None, p(ws))
    ctx.synchronize()
    # as test_gpu_more_operators.logp_bounds has them, but the chain does not grow with the row: 32 additions in a part of it, and where
    # parts, threads and segments meet 32 more
    e1, e2 = -T / S, (e * d * d).sum(1) / S
    big, chain = np.log(vocab) + 1, 64
    G.within(G.back(lp)[0], dt_target - np.log(S), U * (4 * np.abs(dt_target) + 3 * e1 + chain + 8 + 4 * big), "logp", U)
    G.within(G.back(en)[0], np.log(S) - T / S, U * ((chain + 8) * (2 + e1) + 4 * e2 + 8 * e1 + 4 * big), "entropy", U)


@pytest.mark.parametrize("bf16,rows,vocab", [(True, 256, 1 << 22), (False, 256, 1 << 21), (True, 3, (1 << 27) + 5), (False, 3, 1 << 26), (False, 300, 50001)])
def test_log_probabilities_of_long_rows_of_few_values(ctx, bf16, rows, vocab):
    """Equal terms round the same way again and again, as logits in few bits do."""
    rng = np.random.RandomState(1)
    levels = 3 * rng.randn(rows, 1) - np.arange(8) * rng.uniform(0.01, 0.6, (rows, 1))
    check_long_rows(ctx, levels, rng.randint(0, 8, vocab).astype(np.uint8).astype(np.int64), 1.0, bf16)


@pytest.mark.parametrize("rows,vocab", [(256, 1 << 20), (2, 1 << 24)])
def test_log_probabilities_of_long_rows_far_from_zero(ctx, rows, vocab):
    """Rows that are read again with differences from their largest value."""
    rng = np.random.RandomState(2)
    levels = 1e11 - 8192.0 * np.arange(8) * (1 + np.arange(rows) % 5)[:, None]
    check_long_rows(ctx, levels, rng.randint(0, 8, vocab), 1e-4, False)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("scale", [2.0 ** 127, 1e30, 1e-30, 2.0 ** -126, 1e-44])
def test_log_probabilities_at_the_ends_of_the_scale(ctx, scale, bf16):
    z = 3 * G.rnd(5, 20, 700)
    z[3:6] = 0.0
    z[4, 10] = -1.0
    G.logprob(ctx, z, np.arange(20) * 30, scale, 4, bf16, backward=False)


# ---- arrays that no cache holds --------------------------------------------------------------------------------

@pytest.mark.parametrize("bf16,rows", [(True, 5000), (False, 2600)])
def test_log_probabilities_past_the_caches_are_those_of_parts(ctx, bf16, rows):
    """More than 256 MB of logits: rows read past the caches, rows left in them and the border between; the same bits as calls of fewer rows have."""
    vocab, k, part = 33001, 5, 900                            # parts of more rows than a call has for which kernels are others
    z = 2 * torch.randn(rows, vocab, device="cuda")
    z = z.to(G.act(bf16))
    t = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
    dl, de = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    new = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731

    def outputs():
        return new(rows), new(rows), new(rows, 2), new(rows, k, dt=torch.int32), new(rows, k), torch.zeros_like(z)

    def run(out, first, n, dz=None):
        lp, en, st, ids, tl, own = out
        dz = own if dz is None else dz
        at = lambda x: x[first:].data_ptr()  # noqa: E731
        a = pwb.LogprobArgs(dtype=DT[bf16], z=at(z), ldz=vocab, rows=n, vocab=vocab, targets=at(t), scale=1.25)
        ctx.logprob_fwd(a, at(lp), at(en), at(st), k, at(ids), at(tl))
        ctx.logprob_bwd(a, at(st), at(en), at(dl), at(de), at(dz), vocab)
    whole, parts = outputs(), outputs()
    torch.cuda.synchronize()
    run(whole, 0, rows)
    for first in range(0, rows, part):
        run(parts, max(0, min(first, rows - part)), part)
    ctx.synchronize()
    for name, x, y in zip(("logp", "entropy", "stats", "ids", "top", "dz"), whole, parts):
        assert torch.equal(x, y), name
    zd = z[-3:].double()                                      # and they are the right ones
    lsm = torch.log_softmax(1.25 * zd, 1)
    assert torch.allclose(whole[0][-3:].double(), lsm.gather(1, t[-3:].long()[:, None])[:, 0], rtol=0, atol=1e-5)
    run(whole, 0, rows, dz=z)
    ctx.synchronize()
    assert torch.equal(z, parts[5])


def test_clipping_past_the_caches_and_of_many_groups(ctx):
    """More chunks than blocks in both launches, more tensors than a launch takes, and 256 MB from the end inside of a tensor."""
    sizes = [60000001, 40000003] + [1000 + 17 * i for i in range(100)] + [50000005, 100000007]
    kinds = [torch.float32, torch.bfloat16] + [torch.bfloat16 if i % 2 else torch.float32 for i in range(100)] + [torch.float32, torch.bfloat16]
    g = [(torch.randn(n, device="cuda") * (1 + i % 3)).to(dt) for i, (n, dt) in enumerate(zip(sizes, kinds))]
    total = sum(float((x.double() ** 2).sum()) for x in g)
    res, ws = G.full(1, 2, 0.0), G.full(1, pwb.grad_clip_ws_floats(), float("nan"))

    def run(outs, max_norm):
        ts = pwb.grad_tensors([(x.data_ptr(), o.data_ptr(), x.numel(), DT[x.dtype == torch.bfloat16]) for x, o in zip(g, outs)])
        torch.cuda.synchronize()
        ctx.grad_clip(ts, max_norm, p(res), p(ws))
        ctx.synchronize()
        norm, factor = G.back(res)[0]
        assert abs(norm - total ** 0.5) <= (U + 2.0 ** -40) * norm
        assert abs(factor - min(1.0, float(np.float32(max_norm)) / total ** 0.5)) <= (U + 2.0 ** -40) * factor
        return factor
    before = [x.clone() for x in g]
    for max_norm in (100.0, 1e9):
        outs = [torch.zeros_like(x) for x in g]
        f = run(outs, max_norm)
        for x, o in zip(g, outs):                             # one product in 32 bits, which bf16 rounds
            assert torch.equal(o, (x.float() * f).to(x.dtype))
        del outs
    assert run(g, 1e9) == 1.0
    assert all(torch.equal(x, b) for x, b in zip(g, before))
    f = run(g, 100.0)
    assert f < 1.0 and all(torch.equal(x, (b.float() * f).to(x.dtype)) for x, b in zip(g, before))


# ---- products whose workgroups take output tiles in turn -------------------------------------------------------

# Whole tiles of 256 x 256 and ragged ones, one to a workgroup and several, two k tiles and more, the last of them whole or not.
STREAM = [(2560, 4096, 288), (3100, 2900, 544), (5120, 4352, 288), (4900, 4700, 800)]


@pytest.mark.parametrize("epilogue,bf16,accumulate", G.EPILOGUES)
@pytest.mark.parametrize("m,n,k", STREAM)
def test_f4_product_epilogues_of_tiles_in_turn(ctx, m, n, k, epilogue, bf16, accumulate):
    G.product(ctx, m, n, k, epilogue=epilogue, bf16=bf16, accumulate=accumulate, seed=m)


@pytest.mark.parametrize("m,n,k,bf16", [(2560, 4096, 512, True), (5120, 4352, 512, False), (4900, 4701, 544, True), (4900, 4701, 544, False), (9000, 4700, 288, False)])
def test_f4_product_sums_of_tiles_in_turn_are_exact(ctx, m, n, k, bf16):
    """fp32: every sum is a multiple of 1/4 below 2^22; bf16 rounds it once."""
    G.product(ctx, m, n, k, exact=True, seed=7, bf16=bf16)


def test_f4_product_of_tiles_in_turn_keeps_its_blocks_apart(ctx):
    """Blocks without a number stay in their rows, rows and tables apart, no bias where none is given, and a bias that outweighs the sums."""
    G.product(ctx, 4900, 4701, 288, nan_blocks=((0, 8), (255, 0), (256, 8), (4899, 7)), bf16=True)
    G.product(ctx, 4900, 4700, 544, lda=576, ldb=640, ldc=4736, epilogue=pwb.PW_EPI_BIAS, bf16=True)
    G.product(ctx, 4900, 4700, 288, epilogue=pwb.PW_EPI_BIAS_GELU, bf16=True, bias=False)
    G.product(ctx, 4900, 4700, 800, epilogue=pwb.PW_EPI_BIAS, bias_scale=2.0 ** 24)


@pytest.mark.parametrize("m,n,k", [(2560, 4096, 288), (3100, 2904, 288), (5120, 4352, 288), (4900, 4704, 800)])
def test_f4_product_of_tiles_in_turn_takes_a_residual_in_place(ctx, m, n, k):
    G.test_f4_product_takes_a_residual_in_place(ctx, m, n, k)
