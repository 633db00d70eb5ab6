"""Plans of the microscaled product, and its refusals of sums that are not named.  Runs without a GPU."""
import re

import pytest

from paper_2405_16256_amd import binding as hh
from tests.mx_plans import BF16, BF16_FAST, E2M1, E4M3, F32, FEW, MANY_128, PAIRS, ROWS_16, ROWS_32, SHARES, SIZES, TILES_128, plan


def test_sums_that_are_not_named_are_refused():
    q, a = hh.make_mx(1 << 20, 1 << 20), 1 << 20
    for sums in (-1, 2):
        cfg = hh.make_mx_product_cfg(4, 40, 100, E4M3, E2M1, sums=sums)
        for call in (lambda: hh.hh_mx_product_sizes(cfg), lambda: hh.hh_mx_product(None, cfg, q, q, a, 0, a)):
            with pytest.raises(hh.HHError) as e:
                call()
            assert e.value.code == hh.HH_ERR_INVALID_ARG and "sums" in str(e.value)


def test_a_size_for_each_kernel():
    for kernel, s in SIZES.items():
        for fa, fb in PAIRS:
            for how in (BF16, F32, BF16_FAST):
                assert plan(*s, fa, fb, how)[0] == kernel, (s, fa, fb, how)


def test_sizes_in_shares_of_k():
    """Tiles of each size, for each pair of formats, result and sums."""
    for fa, fb in PAIRS:
        for how in (BF16, F32, BF16_FAST):
            for kernel, sizes in SHARES.items():
                plans = [plan(*s, fa, fb, how) for s in sizes]
                assert {p[0] for p in plans} == {kernel} and max(p[1] for p in plans) > 1, (kernel, plans, fa, fb, how)


def test_a_size_of_more_tiles_of_128_than_compute_units():
    m, n, _ = MANY_128
    assert -(-m // 128) * -(-n // 128) > 256
    for fa, fb in PAIRS:
        for how in (BF16, F32, BF16_FAST):
            assert plan(*MANY_128, fa, fb, how) == (TILES_128, 1), (fa, fb, how)


def test_sizes_of_few_rows():
    """Both kernels with every number of waves (up to 4 units of 256 k: 4, up to 8: 8, more: 16), a wave with one unit and with several."""
    seen = set()
    for m, n, k in FEW:
        kernel, _ = plan(m, n, k, E4M3, E2M1, BF16)
        units = -(-k // 256)
        waves = 4 if units <= 4 else 8 if units <= 8 else 16
        assert kernel == (ROWS_16 if m <= 16 else ROWS_32)
        seen.add((kernel, waves, units > waves))
    assert seen == {(kernel, waves, False) for kernel in (ROWS_16, ROWS_32) for waves in (4, 8, 16)} | {(kernel, 16, True) for kernel in (ROWS_16, ROWS_32)}


def test_fast_sums_change_plans_of_tiles_with_an_e4m3_operand_alone():
    """Elsewhere a call with fast sums is the call without."""
    for m in (1, 16, 32, 33, 2000, 4096):
        for fa, fb in PAIRS:
            plans = [plan(m, 4096, 4096, fa, fb, how) for how in (BF16, BF16_FAST)]
            if m <= 32 or (fa, fb) == (E2M1, E2M1):
                assert plans[0] == plans[1]
    assert plan(2000, 2600, 8192, E4M3, E4M3, BF16) == plan(2000, 2600, 8192, E4M3, E4M3, F32)


def test_tiles_of_128_are_built_in_the_forms_that_are_launched():
    """Of mixed formats with three stages alone; of two that are alike with two stages and with three."""
    from paper_2405_16256_amd import build
    from tests.test_kernel_resources import code_objects, kernels
    with open(build.LIB, "rb") as f:
        names = [k[".name"] for elf in code_objects(f.read()) for k in kernels(elf)]
    stages = {}
    for n in names:
        m = re.search(r"k_product_tilesILi(\d)ELi(\d)ELb(\d)E([ft])Li(\d+)ELi128ELi128ELi2ELi2ELi(\d)E", n)
        if m:
            stages.setdefault((int(m[1]), int(m[2])), set()).add(int(m[6]))
    assert stages == {p: {2, 3} if p[0] == p[1] else {3} for p in PAIRS}
