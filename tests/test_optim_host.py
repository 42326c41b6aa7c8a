"""CPU: refusals of the optimizer's plan that need no GPU, the settings' layout, and the 8-bit form of moments in
the oracle against its definition through fp32 bit patterns."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import optim as O
from paper_2210_17357_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2210_17357_amd import build
        build.build()
    return B.lib()


def test_settings_layout(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "lgreco.h"', 'int main(void) {',
             'printf("size %zu\\n", sizeof(lgreco_adamw_t));', 'printf("block %d\\n", LGRECO_OPTIM_BLOCK);',
             'printf("types %d%d%d\\n", LGRECO_F32, LGRECO_BF16, LGRECO_F16);']
    lines += ['printf("%s %%zu\\n", offsetof(lgreco_adamw_t, %s));' % (f, f) for f, _ in B.AdamW._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0;", "}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")], check=True)
    out = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(out["size"]) == C.sizeof(B.AdamW) and int(out["block"]) == B.OPTIM_BLOCK == O.BLOCK
    assert out["types"] == "%d%d%d" % (B.F32, B.BF16, B.F16)
    for f, _ in B.AdamW._fields_:
        assert int(out[f]) == getattr(B.AdamW, f).offset


def create(lib, layers, L, lr_scale=None, decay_scale=None):
    o = C.c_void_p(1)
    a = [None if x is None else np.ascontiguousarray(x, np.float32) for x in (lr_scale, decay_scale)]
    st = lib.lgreco_optim_create(C.byref(o), None if layers is None else C.addressof(layers), L, *(None if x is None else x.ctypes.data for x in a))
    assert st == B.OK or not o.value
    return st


def test_refused_tables_and_factors(lib):
    ok = B.layer_table([0, 10], [10, 5], [0, 0], [0, 0])
    assert lib.lgreco_optim_create(None, C.addressof(ok), 2, None, None) == B.EINVAL
    assert create(lib, None, 2) == B.EINVAL and create(lib, ok, 0) == B.EINVAL and create(lib, ok, -1) == B.EINVAL
    for offs, numels in (([0, 9], [10, 5]), ([-1, 10], [1, 5]), ([0, 10], [0, 5]), ([0, 10], [10, 1 << 31]), ([0, (1 << 58) + 1], [1, 1])):
        assert create(lib, B.layer_table(offs, numels, [0, 0], [0, 0]), 2) == B.EINVAL, (offs, numels)
    for bad in (-1.0, np.nan, np.inf):
        assert create(lib, ok, 2, [1.0, bad]) == B.EINVAL and create(lib, ok, 2, None, [bad, 1.0]) == B.EINVAL
    many = 1 << 14                                     # more workgroups than one launch is given: 2^14 layers of 2^30 elements
    offs = np.arange(many, dtype=np.int64) << 30
    assert create(lib, B.layer_table(offs, np.full(many, 1 << 30), np.zeros(many), np.zeros(many)), many) == B.ENOSPACE
    assert lib.lgreco_optim_destroy(None) == B.EINVAL and lib.lgreco_optim_blocks(None) == -1
    assert lib.lgreco_optim_last_hip_error(None) == b""


def bits_decode(code, x, top):
    """The header's definition: the fp32 number with the bits code << 19, times 2^(x - top)."""
    return float(np.array([code << 19], np.uint32).view(np.float32)[0]) * 2.0 ** (x - top)


def test_codes_in_the_oracle_are_the_headers():
    for octaves, top in ((O.OCTAVES_M, 7), (O.OCTAVES_V, 15)):
        codes = np.arange(128 if top == 7 else 256)
        for x in (0, 1, 100, 127, 254, 255):
            got = O.decode(codes, np.full(codes.size, x), octaves)
            assert got.tolist() == [bits_decode(int(c), x, top) for c in codes]
            assert np.array_equal(O.rounded(got, x, octaves), got)              # on the grid, and kept
            mid = (got[1:] + got[:-1]) / 2
            even = np.where(codes[1:] % 2 == 0, got[1:], got[:-1])
            assert np.array_equal(O.rounded(mid, x, octaves), even)             # ties to even codes


def test_exponents_in_the_oracle_are_the_bits():
    rng = np.random.default_rng(0)
    bits = np.concatenate([rng.integers(0, 0x7F800000, 4000), np.arange(0, 300), 0x780000 + np.arange(-3, 4), 0x800000 + np.arange(-3, 4),
                           (np.arange(1, 255)[:, None] * (1 << 23) + 0x780000 + np.arange(-1, 2)).reshape(-1), [0x7F7FFFFF]])
    for b in bits:
        v = float(np.array([b], np.uint32).view(np.float32)[0])
        assert O.exponent(np.array([v])) == (int(b) + 0x7FFFF) >> 23, hex(int(b))
        assert O.rounded(np.array([v]), O.exponent(np.array([v])), O.OCTAVES_M)[0] <= bits_decode(127, O.exponent(np.array([v])), 7)


def test_step_in_the_oracle_against_differences():
    """The first step from zero moments moves every parameter by the rate against its gradient's sign, and decay shrinks it."""
    g = np.array([3.0, -0.5, 1e-3, 0.0])
    p, m, v = O.step(g, np.full(4, 2.0), np.zeros(4), np.zeros(4), 1, 0.1, 0.9, 0.99, 1e-12, 0.5, 1.0)
    assert np.allclose(p, 2.0 - 0.1 * 0.5 * 2.0 - 0.1 * np.sign(g), atol=1e-9)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.01 * g * g)
    assert O.clip(4.0, 1.0, 1.0) == pytest.approx(0.5, rel=1e-5) and O.clip(4.0, 1.0, 3.0) == 1.0 and O.clip(4.0, 0.5, 0.0) == 0.5
