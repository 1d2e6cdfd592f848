"""How the 4-bit product is cut, asked on the host."""
import ctypes as C
import random

import pytest

from paper_2511_14450_b200 import hyperion as hyp
from tests import test_gpu_low_bit_paths as gpu


def test_the_gpu_tests_reach_every_path():
    missing = gpu.WANTED - set().union(*(gpu.paths(c) for c in gpu.CASES))
    assert not missing, missing


def test_plan_refusals():
    plan = (C.c_int32 * 8)()
    call = lambda m, n, k, t, e, p=plan: hyp.lib().hyp_op_gemm_mx4_plan(m, n, k, t, e, p)
    assert call(8, 128, 128, 3, 3) == hyp.HYP_OK
    for bad in ((0, 128, 128, 3, 3), ((1 << 26) + 1, 128, 128, 3, 3), (8, 0, 128, 3, 3), (8, 128, 60, 3, 3), (8, 128, 128, 0, 3), (8, 128, 128, 4, 3),
                (8, 128, 128, 3, -1), (8, 128, 128, 3, 4), (8, 128, 128, 3, 3, None)):
        assert call(*bad) == hyp.HYP_EINVAL, bad
    assert call(8, 1 << 30, 1 << 20, 3, 3) == hyp.HYP_ECAPACITY
    with pytest.raises(hyp.HyperionError):
        hyp.hyp_op_gemm_mx4_plan(8, 128, 128, 4, 3)


def test_plans_of_any_size_fit():
    """Every cut leaves a ring of two stages at least, all of K to some share, and CTAs that cover tokens and rows."""
    rng = random.Random(5)
    for _ in range(4000):
        m, n, k = (int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 16)), 8 * int(2 ** rng.uniform(0, 12)))
        terms, epi = rng.randint(1, 3), rng.randrange(4)
        p, kb = hyp.hyp_op_gemm_mx4_plan(m, n, k, terms, epi), (k + 127) // 128
        assert p["stages"] >= 2 and p["per_sm"] >= 1 and 1 <= p["shares"] <= 8 and (p["shares"] == 1 or p["shares"] <= kb // 4)
        tiles = 1 if epi == hyp.HYP_EPI_SWIGLU_BF16 else p["row_tiles"]
        assert p["ctas"] == -(-n // (128 * tiles)) * p["token_tiles"] * p["shares"]
        assert p["chunks"] == 0 if p["own_terms"] else p["chunks"] in (1, 2)
        assert p == hyp.hyp_op_gemm_mx4_plan(m, n, k, terms, epi)
