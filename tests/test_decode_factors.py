"""The norm's branch without power-of-two factors: their bound K is then not looked at,
whatever it is."""
import numpy as np
import pytest

import decode_cases as R
from test_decode_abi import NORM, RAN, host_library
from test_layers_abi import caller
from test_linear_gpu import dev, fq, host, say  # noqa: F401
from paper_2111_13824_amd import binding as B

BOUNDS = (-1, -2 ** 31, -33, 0, 7, 99, 2 ** 31 - 1)


def test_the_kernel_gets_a_bound_that_it_can_shift_by(tmp_path):
    lib = B.load(host_library(str(tmp_path / "libhost.so")))
    one = caller(lib, "rmsnorm_int8", **NORM, s_out=0.5, zp=0, bits=8, h=1, y=1)
    rows = caller(lib, "rmsnorm_rows_int8", **NORM, bits=8, h=1, y=1, scales=1)
    for call in (one, rows):
        for K in BOUNDS:
            assert call(alpha=None, K=K) == RAN and lib.fq_test_norm_bound() == 0
            assert call(x=None, K=K) == RAN and lib.fq_test_norm_bound() == 0
        for K in (0, 3, 7):
            assert call(K=K) == RAN and lib.fq_test_norm_bound() == K


@pytest.mark.gpu
@pytest.mark.parametrize("C", (40, 701, 1024))
def test_a_branch_without_factors(fq, C):  # noqa: F811
    a = R.norm_inputs(5, C, seed=C)
    branch = dict(zp_x=2, m_x=1.5)
    one = R.norm(a["r"], a["gamma"], 1.0, 0.05, x=a["x"], **branch)
    rows = R.norm(a["r"], a["gamma"], 1.0, x=a["x"], **branch)
    for K in BOUNDS:
        say("no factors", C, K)
        args = (dev(a["r"]), dev(a["gamma"]), 1.0)
        on = dict(x=dev(a["x"]), K=K, **branch)
        for got, want in zip(fq.rmsnorm_int8(*args, 0.05, **on), one):
            assert np.array_equal(host(got), want)
        for got, want in zip(fq.rmsnorm_rows_int8(*args, **on), rows):
            assert np.array_equal(host(got), want)
