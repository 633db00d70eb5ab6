"""Which kernel a microscaled product takes, asked of the library without a GPU, sizes that reach each of them, and packed operands made on the
GPU for them."""
import torch

from paper_2405_16256_amd import binding as hh
from paper_2405_16256_amd import glue as L

E4M3, E2M1 = hh.HH_MX_E4M3, hh.HH_MX_E2M1
PAIRS = [(a, b) for a in (E4M3, E2M1) for b in (E4M3, E2M1)]
BF16, F32, BF16_FAST = range(3)        # result and sums
ROWS_16, ROWS_32, TILES_64, TILES_128, TILES_256 = range(5)
# a size for each kernel of the product, whatever the formats
SIZES = {ROWS_16: (7, 35, 1000), ROWS_32: (23, 70, 1100), TILES_64: (70, 130, 513), TILES_128: (2697, 715, 48), TILES_256: (516, 13083, 36)}

# with shares of k: each number of them that tiles of 64 take, and tiles of 128 and 256; rows and columns that are odd
SHARES = {TILES_64: [(513, 497, 2189), (45, 85, 2730), (35, 35, 1738), (33, 65, 8010)], TILES_128: [(851, 1179, 9505)], TILES_256: [(2131, 1967, 14112)]}

# tiles of 128, more of them than compute units: another number of stages where the formats are alike
MANY_128 = (2409, 2124, 261)

# few rows, four, eight and sixteen waves, each with one unit of 256 k and with several; no row or column more than there is room for, and all
FEW = [(m, n, k) for m in (1, 7, 16, 17, 23, 31, 32) for n, k in ((33, 31), (19, 1000), (70, 1100), (48, 2048), (65, 2300), (35, 9001))]


def plan(m, n, k, fa, fb, how):
    """-> (kernel, shares of k)"""
    v = hh.lib.hh_internal_mx_plan(m, n, k, fa, fb, how)
    return v // 100, v % 100


def cfg(m, n, k, fa, fb, how, ldc=None):
    return hh.make_mx_product_cfg(m, n, k, fa, fb, hh.HH_F32 if how == F32 else hh.HH_BF16, ldc, hh.HH_MX_SUMS_FAST if how == BF16_FAST else hh.HH_MX_SUMS_F32)


def table(fmt):
    """The numbers of a format by their code, NaN where a code is none."""
    if fmt == E2M1:
        half = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    else:
        half = torch.tensor([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)], dtype=torch.float64)
        half[127] = float("nan")
    return torch.cat((half, -half)).to(L.DEV)


class Operand:
    """A packed tensor of codes [rows, k] (one a byte) and scales [rows, blocks of 32], with its values in fp64."""

    def __init__(self, codes, scales, fmt):
        rows, k = codes.shape
        width = -(-k // 256) * 256
        full = torch.zeros(rows, width, dtype=torch.uint8, device=L.DEV)
        full[:, :k] = codes
        self.scales = torch.zeros(rows, width // 32, dtype=torch.uint8, device=L.DEV)
        self.scales[:, :scales.shape[1]] = scales
        power = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [float("nan")], dtype=torch.float64, device=L.DEV)
        self.values = (table(fmt)[full.long()] * power[self.scales.long()].repeat_interleave(32, dim=1))[:, :k]
        self.codes = (full[:, 0::2] | (full[:, 1::2] << 4)).contiguous() if fmt == E2M1 else full
        self.struct = hh.make_mx(self.codes, self.scales)


def product(ctx, a, b, m, n, k, fa, fb, how, old=None, extra=0):
    """a b^T (+ old) [m, n] as the library forms it, in fp64; `extra` columns and two rows behind it stay as they are, and so does what lies
    behind the workspace."""
    f32 = how == F32
    c = torch.full((m + 2, n + extra), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device=L.DEV)
    if old is not None:
        c[:m, :n] = old
    p = cfg(m, n, k, fa, fb, how, n + extra)
    ws = torch.full((hh.hh_mx_product_sizes(p) + 256,), 0xA5, dtype=torch.uint8, device=L.DEV)
    hh.hh_mx_product(ctx, p, a.struct, b.struct, c, old is not None, ws, L.stream_ptr())
    torch.cuda.synchronize()
    assert bool((c[m:] == 7.0).all()) and bool((c[:, n:] == 7.0).all()) and bool((ws[-256:] == 0xA5).all())
    return c[:m, :n].double()


def drawn(gen, rows, k, fmt):
    """A packed tensor of any numbers of the format under scales of 2^-3 .. 2^3."""
    codes = torch.randint(0, 256 if fmt == E4M3 else 16, (rows, k), dtype=torch.uint8, device=L.DEV, generator=gen)
    if fmt == E4M3:
        codes[codes % 128 == 127] = 0
    return Operand(codes, torch.randint(124, 131, (rows, (k + 31) // 32), dtype=torch.uint8, device=L.DEV, generator=gen), fmt)


def check(ctx, m, n, k, fa, fb, how, accumulate=False, extra=0, seed=0):
    """One product of drawn operands against fp64.  The sum: k products, each added with an error of at most 2^-23 of the sum of magnitudes so
    far; fast with an E4M3 operand and more than 32 rows, each of the 64 products of an instruction cut at 2^-16 of the largest of them, 2^-10
    of the sum of their magnitudes.  Then half a step of the result's type, and one of fp32 where the old value is added."""
    gen = torch.Generator(device=L.DEV).manual_seed(seed + m + 3 * n + 5 * k)
    a, b = drawn(gen, m, k, fa), drawn(gen, n, k, fb)
    want, size = a.values @ b.values.T, a.values.abs() @ b.values.T.abs()
    old = None
    if accumulate:   # as large as the sums are
        old = torch.randn(m, n, device=L.DEV, generator=gen) * float(want.std())
        old = old if how == F32 else old.bfloat16()
        want += old.double()
    got = product(ctx, a, b, m, n, k, fa, fb, how, old, extra)
    fast = how == BF16_FAST and m > 32 and E4M3 in (fa, fb)
    half = 2.0 ** -24 if how == F32 else 2.0 ** -8
    bound = (2.0 ** -10 if fast else 2.0 ** -23 * k) * size + half * want.abs()
    if accumulate:
        bound += 2.0 ** -23 * (old.double().abs() + want.abs())
    bad = (got - want).abs() > bound
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())
    # Roundings of either sign grow with the root of their number.  The result's own: each at most half a step of its value, so half in the norm too;
    # evenly spread, with results that begin at any place between two powers of two, half (0.54 / 3)^0.5 = 0.43 in the mean.  Over 100 results
    # (of 2^14, which are weighed by their size) the root of the mean square is off by a twentieth of that: 0.58 is seven such deviations off.
    sums = 2.0 ** -12 if fast else 2.0 ** -22 * k ** 0.5
    error = float((got - want).norm() / want.norm())
    assert error <= sums + half * (0.58 if m * n >= 1 << 14 else 1.0), (error, sums)
