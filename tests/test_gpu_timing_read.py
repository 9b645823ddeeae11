"""Timing records never leave the caller's arrays, whatever the number of kernels a later library has."""
import ctypes

import pytest
import torch

import paper_2512_14628_amd as pkg
import workloads as wk
from paper_2512_14628_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def recorded(plan):
    """An update (one of the kernels that came last) and a projection on the record."""
    n = plan.arena_elems
    W, G, M, V, U, Z = (torch.zeros(n, device=DEV) for _ in range(6))
    mask = torch.zeros(plan.groups_total, dtype=torch.uint8, device=DEV)
    key = torch.zeros(plan.groups_total, dtype=torch.float64, device=DEV)
    ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device=DEV)
    pkg.hsadmm_kernel_timing_enable(plan, True)
    pkg.hsadmm_adamw(plan, [W], [G], [M], [V], lr=1e-3)
    pkg.hsadmm_project(plan, [W], U, Z, None, mask, key, ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("n,call", [(29, "old"), (0, "n"), (5, "n"), (binding.KERNEL_COUNT, "n"), (binding.KERNEL_COUNT + 7, "n")])
def test_only_the_callers_entries_are_written(n, call):
    """`old`: the function that programs compiled against 2.1 call with arrays of the 29 kernels of that version."""
    wl = wk.custom_workload([(8, 8, 9, wk.MODE_FILTER, 4)], R=1, seed=0)
    plan = pkg.Plan(wl.table())
    recorded(plan)
    lib = pkg.load_library()
    room = binding.KERNEL_COUNT + 16
    ms, count = (ctypes.c_double * room)(*[-1.0] * room), (ctypes.c_int64 * room)(*[-1] * room)
    args = (plan.handle, ms, count)
    assert (lib.hsadmm_kernel_timing_read(*args) if call == "old" else lib.hsadmm_kernel_timing_read_n(*args, n)) == 0
    assert all(x >= 0 for x in ms[:n]) and all(x >= 0 for x in count[:n])
    assert all(x == -1 for x in ms[n:]) and all(x == -1 for x in count[n:])
    names = [lib.hsadmm_kernel_name(i).decode() for i in range(binding.KERNEL_COUNT)]
    launches = dict(zip(names, count[:n]))
    assert sum(launches.values()) >= (1 if n > 28 else 0) and launches.get("adamw", 1) == 1
    assert sum(count[binding.KERNEL_COUNT:n]) == 0
    assert all(launches == 0 for _, launches in pkg.hsadmm_kernel_timing_read(plan).values())    # the record was cleared
    assert lib.hsadmm_kernel_timing_read_n(plan.handle, ms, count, -1) == -1
    plan.close()
