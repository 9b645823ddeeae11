"""Quantised packed buffers and the update in the forms that the sizes of the other tests do not reach: packing of more positions than the
chip holds at once, several launches of a call, runs of channels, index mappings that a step has left."""
import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
import workloads as wk
from tests.test_gpu_mx import B, C, DEV, F, FORMATS, N, SHAPES, Case, buffers, dev, packing, random_mask

pytestmark = pytest.mark.gpu

# More than 2^22 packed positions, from which on a thread packs four fours instead of two: rows of whole words and of any length,
# columns one by one and in runs of nine, both constraints, small layers of every mode in between (tiles of several layers), an
# unconstrained layer at the end.
LARGE = [(700, 1152, 1, F, 500), (3, 5, 1, F, 2), (16, 16, 9, C, 7), (300, 256, 9, F, 280), (7, 3, 9, F, 3), (999, 1025, 1, F, 900),
         (5, 31, 1, C, 30), (10, 64, 1, N, 10), (1500, 515, 1, C, 500), (24, 20, 9, B, 9, 8), (256, 255, 9, C, 200), (31, 17, 1, B, 30, 5),
         (1000, 640, 1, B, 800, 600), (2, 2, 1, F, 1), (256, 130, 9, B, 250, 120), (1000, 513, 1, N, 1000)]


@pytest.mark.parametrize("keep", [None, 1.0])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
def test_written_codes_of_more_positions_than_the_chip_holds(fmt, two, keep):
    case = Case(LARGE, seed=2)
    z, v = case.arena(2.0), case.arena(2.0) if two else None
    mask = random_mask(case.wl, case.rng, keep)
    own = packing(case.wl, random_mask(case.wl, case.rng), case.align)[1][-1]
    assert own > 2 ** 22                                       # what the plan's own selection packs, by which the form is chosen
    pkg.hsadmm_kernel_timing_enable(case.plan, True)
    case.write(z, v, dev(mask), fmt)
    assert pkg.hsadmm_kernel_grids(case.plan)["gather_mx"] == -(-own // 4096)            # 4096 positions to a workgroup: the wide form
    with np.errstate(invalid="ignore"):
        case.check_written(z + v if two else z, mask, fmt)
    case.close()


def expanded(case, nodes, places, mask, M):
    """The mean on kept elements, +0 elsewhere, 7 in the padding."""
    want = np.full(case.wl.n_arena, 7.0, np.float32)
    for li, (l, p) in enumerate(zip(case.wl.layers, places)):
        want[l.elem_off:l.elem_off + l.n] = 0.0
        acc = nodes[0][2][li]
        for node in nodes[1:]:
            acc = acc + node[2][li]
        want[p] = acc * np.float32(1.0 / M)
    return want


@pytest.mark.parametrize("fmt", FORMATS)
def test_read_back_of_a_large_plan(fmt):
    case = Case(LARGE, seed=4)
    mask = random_mask(case.wl, case.rng)
    places, nodes = buffers(case, mask, fmt, 2)
    want = expanded(case, nodes, places, mask, 2)
    dst, vd, zi = torch.full((case.wl.n_arena,), 7.0, device=DEV), case.arena(1.0), case.arena(1.0)
    dvd = dev(vd)
    pkg.hsadmm_expand_mx(case.plan, [dev(c) for c, _, _ in nodes], [dev(s) for _, s, _ in nodes], fmt, dev(mask), dst, dev(zi), dvd,
                         case.ws)
    assert np.array_equal(dst.cpu().numpy().view(np.uint32), want.view(np.uint32))
    on = ~np.isnan(vd)
    assert np.array_equal(dvd.cpu().numpy()[on].view(np.uint32), (vd + (zi - want))[on].view(np.uint32))
    case.close()


@pytest.mark.parametrize("most", [1, 4, 12, 40])
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
def test_reading_in_several_launches(fmt, dual, most, monkeypatch):
    monkeypatch.setenv("HSADMM_GRID_MOST", str(most))
    case = Case(SHAPES + LARGE[:3], seed=6)
    mask = random_mask(case.wl, case.rng)
    places, nodes = buffers(case, mask, fmt, 3)
    want = expanded(case, nodes, places, mask, 3)
    vd, zi = case.arena(1.0), case.arena(1.0)
    dst, dvd = torch.full((case.wl.n_arena,), 7.0, device=DEV), dev(vd)
    pkg.hsadmm_kernel_timing_enable(case.plan, True)
    pkg.hsadmm_expand_mx(case.plan, [dev(c) for c, _, _ in nodes], [dev(s) for _, s, _ in nodes], fmt, dev(mask), dst,
                         dev(zi) if dual else None, dvd if dual else None, case.ws)
    items = sum(-(-l.n // 8192) for l in case.wl.layers)
    assert pkg.hsadmm_kernel_timing_read(case.plan)["scatter_mx"][1] == -(-items // max(1, most // 4))
    assert np.array_equal(dst.cpu().numpy().view(np.uint32), want.view(np.uint32))
    if dual:
        on = ~np.isnan(vd)
        assert np.array_equal(dvd.cpu().numpy()[on].view(np.uint32), (vd + (zi - want))[on].view(np.uint32))
    case.close()


@pytest.mark.parametrize("most", [1, 64, 200])
@pytest.mark.parametrize("R,bits,prox", [(1, 32, False), (5, 8, True), (3, 8, False)])
def test_updates_in_several_launches(R, bits, prox, most, monkeypatch):
    """The same bits as in one launch."""
    wl = wk.custom_workload(SHAPES + LARGE[:3], R=R, seed=0)
    n = wl.n_arena
    results = []
    for limit in (None, most):
        if limit:
            monkeypatch.setenv("HSADMM_GRID_MOST", str(limit))
        plan = pkg.Plan(wl.table())
        gen = torch.Generator(device=DEV).manual_seed(3)
        rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)      # noqa: E731
        W, G = [rand(n) for _ in range(R)], [rand(n) for _ in range(R)]
        state = torch.uint8 if bits == 8 else torch.float32
        M, V = ([torch.zeros(n, dtype=state, device=DEV) for _ in range(R)] for _ in range(2))
        more = {}
        if bits == 8:
            more = {k: [torch.zeros(plan.state_blocks, device=DEV) for _ in range(R)] for k in ("M_scale", "V_scale")}
        if prox:
            more.update(Z=rand(n), U=rand(n), rho=torch.full((plan.n_layers,), 0.1, device=DEV))
        pkg.hsadmm_kernel_timing_enable(plan, True)
        for t in (1, 2):
            pkg.hsadmm_adamw(plan, W, G, M, V, state_bits=bits, lr=1e-2, step=t, **more)
        results.append([x.clone().view(torch.uint8) for x in W + M + V + more.get("M_scale", []) + more.get("V_scale", [])])
        launches = pkg.hsadmm_kernel_timing_read(plan)["adamw"][1]
        assert launches == 2 if limit is None else launches > 2
        plan.close()
    assert all(torch.equal(x, y) for x, y in zip(*results))


@pytest.mark.parametrize("fmt", FORMATS)
def test_plans_with_runs_of_channels(fmt):
    """Channels in runs (a convolution through its matrix view): any mask of theirs packs and reads back as another plan's."""
    shapes = [(40, 27 * 9, 1, C, 50), (16, 24, 9, F, 9), (33, 20 * 9, 1, B, 20, 35), (12, 31, 1, C, 7)]
    case = Case(shapes, seed=8)
    t = dict(case.wl.table(), span=np.array([9, 0, 9, 0], np.int32), k_coarse=np.array([10, 0, 6, 0], np.int32))
    nested = pkg.Plan(t, pack_align_elems=32)
    plain, case.plan = case.plan, nested
    W = case.arena(0.0)
    out = [torch.zeros(case.wl.n_arena, device=DEV) for _ in range(2)]
    mask = torch.zeros(nested.groups_total, dtype=torch.uint8, device=DEV)
    z = torch.zeros(case.wl.n_arena, device=DEV)
    on = ~np.isnan(W)
    case.ws = torch.zeros(max(nested.workspace_bytes, plain.workspace_bytes), dtype=torch.uint8, device=DEV)
    # under the selection the nested projection makes, its mappings and its mask, and under a mask of any counts
    pkg.hsadmm_project(nested, [dev(np.where(on, W, 0))], torch.zeros(case.wl.n_arena, device=DEV), z, None, mask, None, case.ws)
    selected = mask.cpu().numpy()
    for m, given in ((selected, None), (selected, mask), (random_mask(case.wl, case.rng, 0.4), "own")):
        given = dev(m) if isinstance(given, str) else given
        case.codes.fill_(0xAB)
        case.scales.fill_(0xCD)
        case.kept.fill_(-1)
        case.write(W, None, given, fmt)
        case.check_written(W, m, fmt)
        for plan, dst, how in ((nested, out[0], None), (plain, out[1], dev(m))):
            dst.fill_(7.0)
            pkg.hsadmm_expand_mx(plan, [case.codes], [case.scales], fmt, how, dst, None, None, case.ws)
        assert torch.equal(out[0].view(torch.int32), out[1].view(torch.int32))
        assert not out[0][torch.from_numpy(on).to(DEV)].isnan().any()
    plain.close()
    case.close()


STEPS = {
    "filters in one launch": [(64, 48, 9, F, 20), (10, 64, 1, N, 10), (33, 31, 1, F, 20)],
    "channels in one launch": [(128, 64, 9, C, 20), (128, 256, 1, C, 100), (10, 64, 1, N, 10)],
    "several launches": [(16, 16, 9, F, 8), (40, 24, 1, C, 7), (24, 20, 9, B, 9, 8), (10, 64, 1, N, 10), (31, 17, 1, B, 30, 5)],
}


@pytest.mark.parametrize("pack", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shapes", list(STEPS.values()), ids=list(STEPS))
def test_mappings_a_step_has_left(shapes, fmt, weighted, pack):
    """mask NULL straight behind hsadmm_step: what the same calls give that are handed its mask."""
    case = Case(shapes, seed=9)
    plan, n = case.plan, case.wl.n_arena
    clean = lambda x: dev(np.nan_to_num(x))                          # noqa: E731
    W, U, Z, Zg, Vd = [clean(case.arena(0.0)) for _ in range(2)], clean(case.arena(0.0)), *(clean(case.arena(0.0)) for _ in range(3))
    mask = torch.zeros(plan.groups_total, dtype=torch.uint8, device=DEV)
    more = {}
    if weighted:
        a, b = pkg.hsadmm_node_coefficients([0.05] * plan.n_layers, [0.02] * plan.n_layers, 1e-4, 2, 2)
        more = dict(Zg=Zg, Vd=Vd, coef=torch.tensor([x for ab in zip(a, b) for x in ab], device=DEV))
    if pack:
        more.update(packed=torch.zeros(plan.packed_capacity_elems, device=DEV), layer_off=torch.zeros_like(case.off),
                    kept_idx=torch.zeros_like(case.kept))
    pkg.hsadmm_step(plan, W, U=U, Z=Z, mask=mask, workspace=case.ws, **more)
    pkg.hsadmm_compact_mx(plan, Z, Vd, None, fmt, case.codes, case.scales, case.off, case.kept, case.ws)
    left = torch.full((n,), 7.0, device=DEV)
    pkg.hsadmm_expand_mx(plan, [case.codes], [case.scales], fmt, None, left, None, None, case.ws)
    case.check_written((Z + Vd).cpu().numpy(), mask.cpu().numpy(), fmt)
    given, ws = torch.full((n,), 7.0, device=DEV), torch.zeros_like(case.ws)
    pkg.hsadmm_expand_mx(plan, [case.codes], [case.scales], fmt, mask, given, None, None, ws)
    assert torch.equal(left.view(torch.int32), given.view(torch.int32))
    case.close()


@pytest.mark.parametrize("fmt,step", [(pkg.MX_FP8, 2.0 ** -4), (pkg.MX_FP4, 2.0 ** -2)])
def test_an_exchange_of_two_nodes_is_within_half_a_step_of_the_exact_mean(fmt, step):
    """Per element: half a step of each node's value (2^-4 or 2^-2 of it), or half its block's smallest code, halved by the mean; three
    roundings of fp32."""
    case = Case(seed=12)
    mask = random_mask(case.wl, case.rng)
    places, off, _ = packing(case.wl, mask, 32)
    n, bufs, room, mean = case.wl.n_arena, [], np.zeros(case.wl.n_arena), np.zeros(case.wl.n_arena)
    for _ in range(2):
        z, v = case.arena(1.0), case.arena(1.0)
        case.write(z, v, dev(mask), fmt)
        bufs.append((case.codes.clone(), case.scales.clone()))
        s = case.scales.cpu().numpy()
        for p, o in zip(places, off):
            c = z[p].astype(np.float64) + v[p]
            small = np.ldexp(2.0 ** -9 if fmt == pkg.MX_FP8 else 0.5, s[o // 32 + np.arange(p.size) // 32].astype(int) - 127)
            mean[p] += c / 2
            room[p] += np.maximum(np.abs(c) * step, small / 2) / 2 + 3 * 2.0 ** -24 * (np.abs(z[p]) + np.abs(v[p]))
    dst = torch.zeros(n, device=DEV)
    pkg.hsadmm_expand_mx(case.plan, [c for c, _ in bufs], [s for _, s in bufs], fmt, dev(mask), dst, None, None, case.ws)
    got = dst.cpu().numpy().astype(np.float64)
    on = np.concatenate(places)
    assert (np.abs(got - mean)[on] <= room[on] * (1 + 1e-6)).all()
    case.close()
