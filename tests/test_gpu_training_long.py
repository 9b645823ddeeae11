"""8-bit optimizer states over thousands of steps, next to 32-bit states under the same gradients."""
import pytest
import torch

import paper_2512_14628_amd as pkg
import workloads as wk
from tests.ref_e4m3 import E4M3

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_moments_of_8_bits_stay_near_those_of_32_over_thousands_of_steps():
    """No `noise` is given: rounding numbers come from the step.  The second moment settles at most 3 / 16 above its value and
    never below it (tests/test_training_noise_cpu.py derives this; the mean of 65536 elements of a spread of a half: five
    standard deviations are 0.01).  The first moment is not biased: |m8 - m32| has a mean of zero; of 65536 elements whose
    deviation is at most V^0.5 (m's own is 0.23 V^0.5) the mean lies within 5 / 256 V^0.5."""
    wl = wk.custom_workload([(64, 1024, 1, wk.MODE_FILTER, 8)], R=1, seed=0)
    plan = pkg.Plan(wl.table())
    n, blocks = plan.arena_elems, plan.state_blocks
    gen = torch.Generator(device=DEV).manual_seed(1)
    W32, W8, M32, V32 = (torch.zeros(n, device=DEV) for _ in range(4))
    M8, V8 = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    Ms, Vs = (torch.zeros(blocks, device=DEV) for _ in range(2))
    table = torch.from_numpy(E4M3).to(DEV).float()
    steps = 3000
    for t in range(1, steps + 1):
        G = torch.randn(n, generator=gen, device=DEV)
        how = dict(lr=1e-3, step=t, beta_two=0.999)
        pkg.hsadmm_adamw(plan, [W32], [G], [M32], [V32], **how)
        pkg.hsadmm_adamw(plan, [W8], [G], [M8], [V8], state_bits=8, M_scale=[Ms], V_scale=[Vs], **how)
    each = lambda s: s.repeat_interleave(256)[:n]                       # noqa: E731
    v8, m8 = (table[V8.long()] * each(Vs)).double().square(), (table[M8.long()] * each(Ms)).double()
    ratio = float(v8.mean() / V32.double().mean())
    assert 0.99 < ratio < 1.19 + 0.01, ratio
    assert abs(float((m8 - M32.double()).mean())) < 5 / 256 * float(V32.double().mean()) ** 0.5
    # weights walk by m / r.  A rounding of m is off by its own variance, at most step * distance = (m / 8) (0.1 |g - m|), about
    # 0.25 V^0.5 / 8 * 0.1 V^0.5 = 0.003 V, and stays in m for ten steps: 0.3 of what a gradient adds (V).  1 / r^2 is 1 + 3 * 0.2^2 =
    # 1.12 times as large on average for a root whose deviation is a fifth.  Squares of the lengths thus agree to 1.3 * 1.12, the
    # lengths to 1.21; nothing makes the walk shorter but a second moment that is 0.19 too large, by 0.92 at most.
    a, b = float(W8.double().norm()), float(W32.double().norm())
    assert 0.9 < a / b < 1.23, (a, b)
    plan.close()
