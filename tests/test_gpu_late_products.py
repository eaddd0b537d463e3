"""A CTA that gives up waiting for its products marks the call, starts no more of them and ends: attention over the
4-bit cache in a build where every wait counts as one that gave up (after it has ended), without any fault.
"""
import math

import pytest

from paper_2608_26004_gb300 import asymspec as A
from paper_2608_26004_gb300 import build
from paper_2608_26004_gb300 import serving as S
from tests.test_gpu_attend4 import check, inputs, some_rows

pytestmark = pytest.mark.gpu

CASES = [  # lens, Q, heads, kv heads, D
    ([5], 1, 8, 8, 128),
    ([700, 0, 3000, 64], 1, 16, 4, 64),
    ([500, 9000], 8, 32, 8, 128),
    ([900], 9, 16, 4, 256),
]


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    assert _torch.cuda.is_available(), "the gpu tests need a CUDA device"
    build.build_cuda()
    return _torch


@pytest.fixture(scope="module")
def late(torch, tmp_path_factory):
    path = str(tmp_path_factory.mktemp("late") / "libasymspec_late.so")
    return build.build_cuda(force=True, target=path, defines=("ASYMSPEC_TEST_LATE_PRODUCTS=1",))


def test_a_call_that_gave_up_says_so_and_the_next_one_is_right(torch, late, monkeypatch):
    for seed, (lens, Q, heads, kv, D) in enumerate(CASES):
        B = len(lens)
        x = inputs(torch, lens, Q, heads, kv, D, "bfloat16", 16, seed)
        attend, err = S.Cache4Attend(B, Q, heads, kv, D), torch.zeros(1, device="cuda", dtype=torch.int32)
        with monkeypatch.context() as m:
            m.setattr(A, "LIB_PATH", late)
            for module in (A, S):
                m.setattr(module, "_lib", None)
            S.lib()
            for _ in range(3):  # (tensor memory that a call kept would be missing from the ones after it)
                attend(*x, error_word=err)
            torch.cuda.synchronize()
            assert int(err) == A.DATA_TIMEOUT
        err.zero_()
        out, lse = attend(*x, error_word=err)
        assert int(err) == 0
        check(torch, x, out, lse, some_rows(B, Q, heads, seed))


@pytest.mark.parametrize("lens,Q,heads,kv,D", [
    *CASES,
    ([500, 9000, 40, 129] * 30, 8, 32, 8, 128),  # several items a CTA, 32 rows
    ([300, 1, 2000] * 40, 8, 16, 4, 64),         # 32 rows of 64
    ([400, 700] * 30, 4, 32, 4, 256),            # 32 rows of 256
    ([200, 64] * 200, 1, 16, 4, 128),            # 4 rows
])
def test_results_of_a_call_that_gave_up_are_nan(torch, late, monkeypatch, lens, Q, heads, kv, D):
    """Without an error word, too: no number is left that could be taken for a result."""
    B = len(lens)
    x = inputs(torch, lens, Q, heads, kv, D, "bfloat16", 16, 3)
    attend = S.Cache4Attend(B, Q, heads, kv, D)
    out, lse = torch.zeros_like(x[0]), torch.zeros(B, Q, heads, device="cuda")
    with monkeypatch.context() as m:
        m.setattr(A, "LIB_PATH", late)
        for module in (A, S):
            m.setattr(module, "_lib", None)
        S.lib()
        attend(*x, out=out, lse=lse)
        torch.cuda.synchronize()
    assert out.isnan().all() and lse.isnan().all()
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    out, lse = attend(*x, error_word=err)
    assert int(err) == 0
    check(torch, x, out, lse, some_rows(B, Q, heads, 3))
