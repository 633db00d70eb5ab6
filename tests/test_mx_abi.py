"""hh_mx.h: host-side sizes, refusals before any GPU work, and pins of the fp64 definitions that the GPU tests compare with.  Runs without a GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import mx_oracle as O
from paper_2405_16256_amd import binding as hh

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, ODD = 1 << 20, (1 << 20) + 4          # addresses: aligned, aligned to four bytes
BAD, SHAPE, MIS = hh.HH_ERR_INVALID_ARG, hh.HH_ERR_UNSUPPORTED_SHAPE, hh.HH_ERR_MISALIGNED
Q = hh.make_mx(A, A)


def refused(code, call, *args, say="", **kw):
    with pytest.raises(hh.HHError) as e:
        call(*args, **kw)
    assert e.value.code == code and say in str(e.value), e.value


def test_structs_are_those_of_the_header(tmp_path):
    structs = {n: getattr(hh, n) for n in ("hh_dropout_cfg", "hh_mx_tensor", "hh_add_norm_cfg", "hh_mx_product_cfg")}
    lines = ["#include <stdio.h>", '#include "hh_mx.h"', "int main(void) {"]
    for n, s in structs.items():
        lines.append('printf("%s %%zu", sizeof(%s));' % (n, n))
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (n, f) for f, _ in s._fields_] + ['printf("\\n");']
    lines += ['printf("names %d %d %d %d\\n", HH_MX_NONE, HH_MX_E4M3, HH_MX_E2M1, HH_MX_PAD); return 0; }']
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(line.split(" ", 1) for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for n, s in structs.items():
        assert [int(t) for t in out[n].split()] == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_], n
    assert [int(t) for t in out["names"].split()] == [hh.HH_MX_NONE, hh.HH_MX_E4M3, hh.HH_MX_E2M1, hh.HH_MX_PAD]


# ------------------------------------------------------------------ sizes
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 256), (7, 257), (333, 2050)])
def test_packed_sizes(rows, k):
    width = -(-k // 256) * 256
    assert hh.hh_mx_sizes(hh.HH_MX_E4M3, rows, k) == (rows * width, rows * width // 32)
    assert hh.hh_mx_sizes(hh.HH_MX_E2M1, rows, k) == (rows * width // 2, rows * width // 32)
    codes, scales = O.quantise(np.zeros((rows, k)), O.E2M1)
    assert O.in_memory(codes, O.E2M1).nbytes == rows * width // 2 and scales.nbytes == rows * width // 32


def test_norm_workspace():
    small, large = (hh.hh_add_norm_sizes(hh.make_add_norm_cfg(r, 4096)) for r in (3, 1 << 20))
    assert 3 * 4096 * 4 <= small <= 3 * 4096 * 4 + 256
    assert large <= 1024 * 4096 * 4          # however many rows there are


# ------------------------------------------------------------------ refusals
def test_dropout_refuses():
    d = hh.make_dropout(0.1, 1)

    def call(drop=d, rows=2, cols=8, dtype=hh.HH_BF16, x=A, ldx=8, y=A, ldy=8):
        hh.hh_dropout(None, drop, rows, cols, dtype, x, ldx, y, ldy)
    refused(BAD, call, say="ctx")
    refused(BAD, call, drop=None, say="drop")
    for p in (-0.1, 1.1, float("nan")):
        refused(BAD, call, drop=hh.make_dropout(p, 1), say="drop.p")
    refused(MIS, call, drop=hh.make_dropout(0.1, 1, 0, ODD), say="drop.step")
    refused(BAD, call, dtype=2, say="dtype")
    for kw in (dict(rows=0), dict(cols=0), dict(rows=-1)):
        refused(BAD, call, **kw)
    refused(BAD, call, ldx=7, say="ldx")
    refused(BAD, call, ldy=7, say="ldy")
    refused(BAD, call, ldy=9, say="another ld")
    for n in ("x", "y"):
        refused(BAD, call, say=n, **{n: None})
        refused(MIS, call, say=n, **{n: ODD})
    refused(SHAPE, call, rows=1 << 30, cols=17, ldx=17, ldy=17)
    refused(SHAPE, call, rows=1 << 31, cols=1, ldx=8, ldy=8)


def test_packing_refuses():
    def quantise(rows=4, cols=40, dtype=hh.HH_BF16, x=A, ldx=40, fmt=hh.HH_MX_E4M3, by_row=Q, by_column=Q):
        hh.hh_mx_quantise(None, rows, cols, dtype, x, ldx, fmt, by_row, by_column)

    def values(rows=4, k=40, fmt=hh.HH_MX_E4M3, q=Q, dtype=hh.HH_BF16, y=A, ldy=40):
        hh.hh_mx_values(None, rows, k, fmt, q, dtype, y, ldy)
    for call, ld, ptr, packed in ((quantise, "ldx", "x", ("by_row", "by_column")), (values, "ldy", "y", ("q",))):
        refused(BAD, call, say="ctx")
        refused(BAD, call, dtype=2, say="dtype")
        for f in (0, 3):
            refused(BAD, call, fmt=f, say="format")
        refused(BAD, call, rows=0)
        refused(BAD, call, say=ld, **{ld: 39})
        refused(BAD, call, say=ptr, **{ptr: None})
        refused(MIS, call, say=ptr, **{ptr: ODD})
        for n in packed:
            for bad, code in ((hh.make_mx(None, A), BAD), (hh.make_mx(A, None), BAD), (hh.make_mx(ODD, A), MIS), (hh.make_mx(A, ODD), MIS)):
                refused(code, call, say=n, **{n: bad})
    refused(BAD, quantise, by_row=None, by_column=None, say="NULL")
    refused(BAD, values, q=None, say="q")
    refused(SHAPE, quantise, rows=1 << 28, cols=40)                          # as padded by row
    refused(SHAPE, quantise, rows=40, cols=1 << 28, ldx=1 << 28)             # as padded by column
    for f in (0, 3):
        refused(BAD, hh.hh_mx_sizes, f, 4, 4, say="format")
    for r, k in ((0, 4), (4, 0), (-1, 4)):
        refused(BAD, hh.hh_mx_sizes, hh.HH_MX_E4M3, r, k)
    refused(SHAPE, hh.hh_mx_sizes, hh.HH_MX_E4M3, 1 << 40, 1 << 40)


def test_add_norm_refuses():
    def fwd(cfg=None, drop=None, x=A, b=A, g=A, h=A, xn=A, q=None, **kw):
        hh.hh_add_norm_fwd(None, cfg or hh.make_add_norm_cfg(**{**dict(rows=4, hidden=40), **kw}), drop, x, b, g, h, xn, q)

    def bwd(cfg=None, drop=None, h=A, g=A, dxn=A, dh=A, dx=A, db=A + 16, dg=A, workspace=A, **kw):
        hh.hh_add_norm_bwd(None, cfg or hh.make_add_norm_cfg(**{**dict(rows=4, hidden=40), **kw}), drop, h, g, dxn, dh, dx, db, dg, 0, workspace)
    for call, pointers, optional in ((fwd, ("x", "g", "b", "xn", "h"), ("b", "xn")), (bwd, ("h", "g", "dxn", "dx", "dh", "db", "dg", "workspace"), ("dh", "db", "dg"))):
        refused(BAD, call, say="ctx")
        for kw, code in ((dict(rows=0), BAD), (dict(hidden=0), BAD), (dict(hidden=-8), BAD), (dict(dtype=2), BAD), (dict(eps=-1.0), BAD),
                         (dict(eps=float("nan")), BAD), (dict(format=3), BAD), (dict(hidden=32769), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE),
                         (dict(rows=1 << 21, hidden=32768), SHAPE)):
            refused(code, call, **kw)
        for p in (-0.1, 1.1):
            refused(BAD, call, drop=hh.make_dropout(p, 1), say="drop.p")
        for n in pointers:
            refused(MIS, call, say=n, **{n: ODD})
            if n not in optional:
                refused(BAD, call, say=n, **{n: None})
    refused(BAD, fwd, b=None, say="h is x")
    refused(BAD, fwd, xn=None, say="xn and q")
    refused(BAD, fwd, q=Q, say="HH_MX_NONE")
    refused(BAD, fwd, format=hh.HH_MX_E4M3, say="q")
    refused(MIS, fwd, format=hh.HH_MX_E4M3, q=hh.make_mx(ODD, A), say="q")
    refused(BAD, bwd, db=A, say="db is dx")
    assert hh.lib.hh_add_norm_sizes(None, None) == BAD


def test_product_refuses():
    good = dict(m=4, n=40, k=100, a_format=hh.HH_MX_E4M3, b_format=hh.HH_MX_E2M1)

    def call(a=Q, b=Q, c=A, workspace=A, **kw):
        hh.hh_mx_product(None, hh.make_mx_product_cfg(**{**good, **kw}), a, b, c, 0, workspace)

    def sizes(**kw):
        hh.hh_mx_product_sizes(hh.make_mx_product_cfg(**{**good, **kw}))
    refused(BAD, call, say="ctx")
    for kw, code in ((dict(m=0), BAD), (dict(n=0), BAD), (dict(k=0), BAD), (dict(k=-1), BAD), (dict(a_format=0), BAD), (dict(b_format=3), BAD), (dict(dtype=2), BAD),
                     (dict(ldc=39), BAD), (dict(m=1 << 24, k=256), SHAPE), (dict(n=1 << 25, k=256), SHAPE), (dict(m=1 << 18, n=1 << 18), SHAPE)):
        refused(code, call, **kw)
        refused(code, sizes, **kw)
    for n in ("a", "b"):
        refused(BAD, call, say=n, **{n: None})
        refused(BAD, call, say=n, **{n: hh.make_mx(A, None)})
        refused(MIS, call, say=n, **{n: hh.make_mx(A, ODD)})
    refused(BAD, call, c=None, say="c")
    refused(MIS, call, c=ODD, say="c")
    assert hh.lib.hh_mx_product_sizes(None, None) == BAD


# ------------------------------------------------------------------ plans of the product
def test_every_kernel_of_the_product_is_tested():
    """The sizes of the GPU tests reach each kernel, whole and in shares of k, with one workgroup on a compute unit and with several."""
    def plan(m, n, k, fa, fb, f32):
        v = hh.lib.hh_internal_mx_plan(m, n, k, fa, fb, int(f32))
        return v // 100, v % 100
    from tests import test_gpu_mx as G
    sizes = [s for t in (G.test_product, G.test_larger_products) for mark in t.pytestmark if mark.name == "parametrize" and mark.args[0] == "m,n,k" for s in mark.args[1]]
    seen = {plan(m, n, k, fa, fb, f32) for m, n, k in sizes for fa in (1, 2) for fb in (1, 2) for f32 in (0, 1)}
    assert {k for k, _ in seen} == set(range(5)) and {k for k, s in seen if s > 1} == {2, 3, 4}, seen
    many = {plan(m, n, k, 1, 1, 0)[0] for m, n, k in sizes if -(-m // 128) * -(-n // 128) > 256}
    assert 3 in {plan(*s, 1, 1, 0)[0] for s in sizes} and many, many
    for m in (1, 16, 17, 32, 33):      # rows of their own up to 32
        assert plan(m, 4096, 4096, 1, 2, 0)[0] == (0 if m <= 16 else 1 if m <= 32 else 2)


# ------------------------------------------------------------------ pins of the definitions
def test_generator_gives_its_authors_known_answers():
    """Counter, key and result as published with the generator."""
    def words(*args):
        return [int(w) for w in O.philox([np.uint64(c) for c in args[:4]], args[4:])]
    assert words(0, 0, 0, 0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert words(f, f, f, f, f, f) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words(0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344, 0xA4093822, 0x299F31D0) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_its_share():
    for p in (0.0625, 0.5, 0.9):
        k = O.kept(400, 500, p, 12345, 7)
        assert abs(k.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / k.size)       # five deviations
        for other in (O.kept(400, 500, p, 12345, 8), O.kept(400, 500, p, 12346, 7)):
            both = (k & other).mean()
            assert abs(both - (1 - p) ** 2) < 6 * np.sqrt((1 - p) ** 2 / k.size)
    assert O.kept(3, 9, 0.0, 1, 1).all() and not O.kept(3, 9, 1.0, 1, 1).any()


@pytest.mark.parametrize("fmt", (O.E4M3, O.E2M1))
def test_packing_is_the_nearest_number(fmt):
    """Against a search over all numbers of the format, value by value, and against numbers worked by hand."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 70)) * np.exp2(rng.integers(-20, 20, (3, 70)).astype(float))
    codes, scales = O.quantise(x, fmt)
    got = O.values(codes, scales, 70, fmt)
    every = np.concatenate((O.numbers(fmt), -O.numbers(fmt)))
    for r in range(3):
        for b in range(3):
            block = x[r, 32 * b:32 * b + 32]
            e = int(np.floor(np.log2(np.abs(block).max()))) - O.TOP[fmt]
            assert scales[r, b] == e + 127
            for j, v in enumerate(block):
                assert abs(got[r, 32 * b + j] - v) == np.abs(every * 2.0 ** e - v).min()
    assert (codes[:, 70:] == 0).all() and (scales[:, 3:] == 0).all()
    one = np.zeros((1, 32))
    one[0, :6] = (6, 5, 2.5, 1.25, 0.25, -7) if fmt == O.E2M1 else (448, 18, 17, 19, 2.0 ** -10, -500)
    want = (6, 4, 2, 1, 0, -6) if fmt == O.E2M1 else (448, 18, 16, 20, 0, -448)      # ties to even, saturation
    assert O.quantise(one, fmt)[1][0, 0] == 127 and tuple(O.rounded(one, fmt)[0, :6]) == want
    assert len(O.numbers(fmt)) == (127 if fmt == O.E4M3 else 8) and O.numbers(fmt)[-1] == (448 if fmt == O.E4M3 else 6)


def test_norm_gradient_is_that_of_differences():
    rng = np.random.default_rng(2)
    h, g, dxn, dh = rng.standard_normal((2, 11)), rng.standard_normal(11), rng.standard_normal((2, 11)), rng.standard_normal((2, 11))
    dx, dg = O.norm_grad(h, g, 1e-3, dxn, dh)

    def f(h, g):
        return np.sum(dxn * O.norm(h, g, 1e-3)) + np.sum(dh * h)
    s = 1e-6
    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = s
        assert abs((f(h + e, g) - f(h - e, g)) / (2 * s) - dx[i]) < 1e-7
    for i in range(11):
        e = np.zeros_like(g)
        e[i] = s
        assert abs((f(h, g + e) - f(h, g - e)) / (2 * s) - dg[i]) < 1e-7
