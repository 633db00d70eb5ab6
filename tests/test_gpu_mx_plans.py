"""Every kernel of the microscaled product, in every form that a plan gives it, for each pair of formats, result and sums."""
import pytest
import torch

from paper_2405_16256_amd import binding as hh
from tests.mx_plans import BF16, BF16_FAST, F32, FEW, MANY_128, PAIRS, SHARES, SIZES, check

pytestmark = pytest.mark.gpu
HOWS = (BF16, F32, BF16_FAST)


@pytest.fixture(scope="module")
def ctx():
    c = hh.hh_ctx_create(0)
    yield c
    torch.cuda.synchronize()
    hh.hh_ctx_destroy(c)


@pytest.mark.parametrize("fa,fb", PAIRS)
@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("m,n,k", [s for sizes in SHARES.values() for s in sizes])
def test_shares_of_k(ctx, m, n, k, how, fa, fb):
    check(ctx, m, n, k, fa, fb, how, extra=3)


@pytest.mark.parametrize("fa,fb", PAIRS)
@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("m,n,k", [*SIZES.values(), MANY_128, *(s for sizes in SHARES.values() for s in sizes)])
def test_what_is_there_is_added_to(ctx, m, n, k, how, fa, fb):
    check(ctx, m, n, k, fa, fb, how, accumulate=True, extra=n % 4 + 1)


@pytest.mark.parametrize("fa,fb", PAIRS)
@pytest.mark.parametrize("m,n,k", FEW)
def test_few_rows(ctx, m, n, k, fa, fb):
    for how in HOWS:
        check(ctx, m, n, k, fa, fb, how, extra=m % 3)
        check(ctx, m, n, k, fa, fb, how, accumulate=True)
