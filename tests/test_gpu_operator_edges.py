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
