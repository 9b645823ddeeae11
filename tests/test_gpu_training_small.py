"""AdamW with second moments below fp32's normal range, and an eps that does not hide them."""
import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
import workloads as wk

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E = 2.0 ** -24


@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-18])
def test_the_first_step_of_gradients_whose_squares_are_tiny(eps):
    """Gradients of 1e-23 to 1e-15: second moments from zero over single units of 2^-149 to 1e-33.  The weights' step from the
    moments as they were stored: a root, a fused product and sum, a reciprocal of two units, a product and a fused end, each half a
    unit of 2^-23 (E) but for the reciprocal (2 E) and the root (here 2 E); three constants rounded once."""
    wl = wk.custom_workload([(64, 1024, 1, wk.MODE_FILTER, 8)], R=1, seed=0)
    plan = pkg.Plan(wl.table())
    n = plan.arena_elems
    rng = np.random.default_rng(0)
    g = (10.0 ** rng.uniform(-23, -15, n) * rng.choice([-1, 1], n)).astype(np.float32)
    W, M, V = (torch.zeros(n, device=DEV) for _ in range(3))
    pkg.hsadmm_adamw(plan, [W], [torch.from_numpy(g).to(DEV)], [M], [V], lr=1e-3, eps=eps, beta_one=0.9, beta_two=0.999, step=1)
    w, m, v = (x.cpu().numpy().astype(np.float64) for x in (W, M, V))
    g2 = g.astype(np.float64) ** 2
    # (the square and the product with 1 - beta_2 round once each, to multiples of 2^-149 at the low end)
    assert (np.abs(v - (1 - 0.999) * g2) <= 3 * E * v + 1.5 * 2.0 ** -149).all()
    assert ((v > 0) & (v < 2.0 ** -126)).sum() > n // 8 and (v == 0).any()
    root = 1 / np.sqrt(1 - 0.999)
    want = -1e-3 / (1 - 0.9) * m / (np.sqrt(v) * root + eps)
    assert (np.abs(w - want) <= 12 * E * np.abs(want)).all(), float(np.max(np.abs(w / want - 1)))
    plan.close()


def test_roots_of_8_bits_are_cut_from_the_right_root():
    """A block whose second moments are all one tiny number: its scale is that number's root / 448 (the root, the division and
    the constant round by 2 E, 2 E and E)."""
    wl = wk.custom_workload([(1, 256 * 24, 1, wk.MODE_FILTER, 1)], R=1, seed=0)
    plan = pkg.Plan(wl.table())
    n, blocks = plan.arena_elems, plan.state_blocks
    of_block = (10.0 ** np.linspace(-21, -16, blocks)).astype(np.float32)
    W, Ms, Vs = torch.zeros(n, device=DEV), torch.zeros(blocks, device=DEV), torch.zeros(blocks, device=DEV)
    M, V = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    G = torch.from_numpy(np.repeat(of_block, 256)[:n]).to(DEV)
    pkg.hsadmm_adamw(plan, [W], [G], [M], [V], state_bits=8, M_scale=[Ms], V_scale=[Vs], lr=1e-3, eps=1e-30)
    v = np.float32(1.0 - 0.999) * (of_block * of_block)                      # fp32, each operation rounded as the kernel's
    assert ((v > 0) & (v < np.float32(2.0 ** -126))).sum() >= 6
    want = np.sqrt(v.astype(np.float64)) / 448
    got = Vs.cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= 5 * E * want).all(), got / want
    plan.close()


@pytest.mark.parametrize("layers,elems,groups", [(160, 900, 4), (1100, 900, 1), (160, 8000, 1), (20, 8192, 4)])
def test_replicas_are_shared_out_by_the_work_there_is(layers, elems, groups):
    """With the pull, 16 replicas are taken in fours unless 1024 stretches of 1024 elements hold anything, in however many
    layers; the grid has eight stretches for every 8192 elements of a layer, or what it has of them."""
    pitch = elems + -elems % 4
    t = {"elem_off": pitch * np.arange(layers, dtype=np.int64), "c_out": np.ones(layers, np.int32),
         "c_in": np.full(layers, elems, np.int32), "khw": np.ones(layers, np.int32), "mode": np.ones(layers, np.int32),
         "k": np.ones(layers, np.int32)}
    plan = pkg.Plan(t)
    n, R = plan.arena_elems, 16
    arenas = [torch.zeros(n, device=DEV) for _ in range(3 * R)]
    G, Z = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
    pkg.hsadmm_kernel_timing_enable(plan, True)
    pkg.hsadmm_adamw(plan, arenas[:R], [G] * R, arenas[R:2 * R], arenas[2 * R:], Z=Z, U=Z, rho=torch.ones(layers, device=DEV),
                     lr=0.25, step=1)
    assert pkg.hsadmm_kernel_grids(plan)["adamw"] == layers * -(-elems // 8192) * 8 * groups
    w = torch.stack(arenas[:R])
    inside = (torch.arange(n, device=DEV) % pitch) < elems
    # the first step is lr against the gradient's sign: a dozen roundings of 2 E on 0.25, eps is 1e-8 of it
    assert float((w[:, inside] + 0.25).abs().max()) < 8 * E and not w[:, ~inside].any()
    plan.close()


def test_a_call_per_replica_takes_each_replicas_own_dual():
    """Eq. (7) with u_ij: R calls of one replica; and with the same dual for all they are the one call's bits."""
    wl = wk.custom_workload([(40, 33, 9, wk.MODE_FILTER, 8), (7, 5, 1, wk.MODE_FILTER, 2)], R=1, seed=0)
    plan = pkg.Plan(wl.table())
    n, R = plan.arena_elems + -plan.arena_elems % 64, 3              # (replicas are rows: each of them aligned)
    gen = torch.Generator(device=DEV).manual_seed(2)
    W, U = torch.randn(R, n, generator=gen, device=DEV), torch.randn(R, n, generator=gen, device=DEV)
    G, Z = torch.zeros(n, device=DEV), torch.randn(n, generator=gen, device=DEV)
    rho = torch.tensor([0.5, 0.25], device=DEV)

    def steps(duals, at_once):
        w, m, v = W.clone(), torch.zeros_like(W), torch.zeros_like(W)
        how = dict(Z=Z, rho=rho, lr=1e-2, beta_one=0.0, step=1)
        if at_once:
            pkg.hsadmm_adamw(plan, list(w), [G] * R, list(m), list(v), U=duals, **how)
        else:
            for r in range(R):
                pkg.hsadmm_adamw(plan, [w[r]], [G], [m[r]], [v[r]], U=duals[r], **how)
        return w, m, v

    _, m, _ = steps(U, False)
    for i, l in enumerate(wl.layers):
        on = slice(l.elem_off, l.elem_off + l.n)
        # beta_1 = 0: the first moment is the pull.  A difference, a sum and a product round
        d = W[:, on].double() - Z[on].double()
        want = float(rho[i]) * (d + U[:, on].double())
        assert ((m[:, on].double() - want).abs() <= 3 * E * float(rho[i]) * (d.abs() + U[:, on].double().abs())).all()
    one, each = steps(U[0], True), steps([U[0]] * R, False)
    for x, y in zip(one, each):
        assert torch.equal(x.view(torch.int32), y.view(torch.int32))
    plan.close()
