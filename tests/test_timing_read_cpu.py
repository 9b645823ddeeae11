"""hsadmm_kernel_timing_read as C programs see it: compiled now, it says how long their arrays are."""
import os
import subprocess

import paper_2512_14628_amd as pkg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_program_compiled_now_passes_the_length_of_its_arrays(tmp_path):
    src, exe = tmp_path / "read.c", tmp_path / "read"
    src.write_text("""
#include <stdio.h>
#include "hsadmm.h"
static int seen = -1;
int hsadmm_kernel_timing_read_n(hsadmm_plan_t* p, double* ms, int64_t* n, int32_t count)
{ (void)p; (void)ms; (void)n; seen = count; return 0; }
int main(void)
{
    double ms[HSADMM_KERNEL_COUNT]; int64_t n[HSADMM_KERNEL_COUNT];
    if (hsadmm_kernel_timing_read((hsadmm_plan_t*)0, ms, n) != 0) return 1;
    printf("%d %d", seen, HSADMM_KERNEL_COUNT);
    return 0;
}
""")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    seen, count = subprocess.check_output([str(exe)], text=True).split()
    assert seen == count


def test_refusals_without_a_plan():
    lib = pkg.load_library()
    assert lib.hsadmm_kernel_timing_read_n(None, None, None, 0) == -1
    assert lib.hsadmm_kernel_timing_read(None, None, None) == -1
