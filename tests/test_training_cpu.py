"""Host side of the training and quantised-buffer calls: argument structures, the coefficients of a step, refusals that need
no device."""
import ctypes
import math
import os
import re
import subprocess
from fractions import Fraction

import numpy as np
import pytest

import paper_2512_14628_amd as pkg
from paper_2512_14628_amd import binding
from tests.ref_e4m3 import rounding_numbers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_argument_structures_have_the_layout_the_binding_fills(tmp_path):
    header = open(os.path.join(ROOT, "include", "hsadmm.h")).read()
    for c_name, cls in (("hsadmm_adamw_args_t", binding._AdamwArgs), ("hsadmm_adamw_coef_t", binding._AdamwCoef)):
        fields = [name for name, _ in cls._fields_]
        src = ["#include <stdio.h>", "#include <stddef.h>", '#include "hsadmm.h"', "int main(void) {",
               '  printf("%%zu\\n", sizeof(%s));' % c_name]
        src += ['  printf("%%zu\\n", offsetof(%s, %s));' % (c_name, f) for f in fields]
        c, exe = tmp_path / (c_name + ".c"), tmp_path / c_name
        c.write_text("\n".join(src + ["  return 0;", "}"]))
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)])
        out = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
        assert out == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]
        body = header[:header.index("} %s;" % c_name)]
        body = re.sub(r"/\*.*?\*/", "", body[body.rindex("typedef struct {"):], flags=re.S)
        assert re.findall(r"([A-Za-z_0-9]+);", body) == fields
    consts = {"HSADMM_TYPE_F32": pkg.TYPE_F32, "HSADMM_TYPE_BF16": pkg.TYPE_BF16, "HSADMM_TYPE_F16": pkg.TYPE_F16,
              "HSADMM_MX_FP8": pkg.MX_FP8, "HSADMM_MX_FP4": pkg.MX_FP4}
    for name, value in consts.items():
        assert int(re.search(r"#define %s +(\d+)" % name, header).group(1)) == value


def test_coefficients_against_exact_arithmetic():
    """decay, step_size and root within half a step of fp32 plus what fp64 loses: 1 - beta^t loses up to 2^-52 / (1 - beta)
    of its value (beta_2 = 0.999: 2^-42), the power and the root a few units of fp64."""
    for lr, b1, b2, wd, t in ((1e-3, 0.9, 0.999, 0.01, 1), (1e-3, 0.9, 0.999, 0.01, 7), (0.1, 0.0, 0.0, 0.0, 1),
                              (3e-4, 0.95, 0.99, 0.1, 100000), (0.0, 0.9, 0.999, 0.0, 2 ** 40)):
        decay, step, root, noise = pkg.hsadmm_adamw_coefficients(lr, b1, b2, wd, t, 0xFFFFFFFF)
        f = Fraction
        p1, p2 = (f(0) if t > 10 ** 5 else f(b) ** t for b in (b1, b2))
        want = (1 - f(lr) * f(wd), f(lr) / (1 - p1), 1 / math.sqrt(1 - p2))
        for got, w in zip((decay, step, root), want):
            assert float(np.float32(got)) == got
            assert abs(f(got) - f(w)) <= f(w) * f(2 ** -24 + 2 ** -40), (lr, t)
        assert noise == 0xFFFFFFFF
    for bad in ((-1e-3, 0.9, 0.999, 0, 1), (float("nan"), 0.9, 0.999, 0, 1), (float("inf"), 0.9, 0.999, 0, 1),
                (1e-3, 1.0, 0.999, 0, 1), (1e-3, -0.1, 0.999, 0, 1), (1e-3, 0.9, 1.0, 0, 1), (1e-3, 0.9, float("nan"), 0, 1),
                (1e-3, 0.9, 0.999, -1, 1), (1e-3, 0.9, 0.999, 0, 0), (1e-3, 0.9, 0.999, 0, -5), (1e39, 0.9, 0.999, 0, 1),
                (1e25, 1 - 2.0 ** -53, 0.999, 0, 1), (1e30, 0.9, 0.999, 1e30, 1)):
        with pytest.raises(pkg.HsadmmError) as e:
            pkg.hsadmm_adamw_coefficients(*bad)
        assert e.value.code == -1
    assert pkg.load_library().hsadmm_adamw_coefficients(1e-3, 0.9, 0.999, 0.0, 1, 0, None) == -1


def test_calls_without_a_plan_are_refused():
    lib = pkg.load_library()
    assert lib.hsadmm_gradient_norms(None, None, 1, 0, 1.0, None, None, None, 0, None) == -1
    assert lib.hsadmm_plan_state_blocks(None, None) == -1
    assert lib.hsadmm_compact_mx(None, None, None, None, 0, None, None, None, None, None, 0, None) == -1
    assert lib.hsadmm_expand_mx(None, None, None, 1, 0, None, None, None, None, None, 0, None) == -1
    args = binding._AdamwArgs()
    args.struct_bytes = ctypes.sizeof(binding._AdamwArgs)
    assert lib.hsadmm_adamw(None, ctypes.byref(args)) == -1
    args.struct_bytes -= 8
    assert lib.hsadmm_adamw(ctypes.c_void_p(1), ctypes.byref(args)) == -1      # another size: nothing is read from it
    assert lib.hsadmm_adamw(ctypes.c_void_p(1), None) == -1


def test_rounding_numbers_are_even_and_independent_from_step_to_step():
    """65536 numbers: mean and variance of an even spread, correlations of an element's numbers of two steps, of its
    neighbours and of two replicas, each within five standard deviations (2^-8 for a correlation, 2^-8 / sqrt(12) for a mean)."""
    n = 1 << 16
    limit = 5 * 2.0 ** -8
    series = [rounding_numbers(n, 2, (t * 0x9E3779B9) & 0xFFFFFFFF) for t in range(3)]
    unit = [(u - (0.5 - 2.0 ** -21)) * math.sqrt(12) for u in series]
    for u in unit:
        assert np.abs(u.mean(1)).max() < limit and np.abs((u ** 2).mean(1) - 1).max() < limit
        assert abs((u[0] * u[1]).mean()) < limit
        for k in (4, 8, 256):
            assert abs((u[0][k:] * u[0][:-k]).mean()) < limit
    for a, b in ((0, 1), (1, 2), (0, 2)):
        assert abs((unit[a][0] * unit[b][0]).mean()) < limit
    # with a plain counter for noise as well
    a, b = (rounding_numbers(n, 1, t)[0] for t in (1000, 1001))
    assert abs(((a - 0.5) * (b - 0.5)).mean() * 12) < limit
