"""The training and quantised-buffer calls as a node's program uses them: local steps between two steps of the consensus, the
exchange in eight or four bits, in a captured graph, from several streams and host threads, and at the largest offsets."""
import threading

import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
import workloads as wk
from tests.ref_e4m3 import E2M1, E4M3

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
N, F, C, B = wk.MODE_NONE, wk.MODE_FILTER, wk.MODE_CHANNEL, wk.MODE_BOTH
SHAPES = [(16, 3, 9, F, 8), (32, 16, 9, F, 13), (33, 32, 1, C, 15), (24, 33, 9, B, 13, 21), (40, 77, 1, F, 17), (10, 40, 1, N, 10)]


class Node:
    """A node's arenas: two replicas that are trained towards targets of their own, states in 8 bits, bf16 gradients."""

    def __init__(self, wl, plan, seed, z0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        n, R = wl.n_arena, 2
        rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)               # noqa: E731
        self.target = z0 + 0.3 * rand(R, n)
        self.W = (z0 + 0.01 * rand(R, n)).contiguous()
        self.G = torch.zeros(R, n, dtype=torch.bfloat16, device=DEV)
        self.low = torch.zeros_like(self.G)
        blocks = pkg.hsadmm_plan_state_blocks(plan)
        self.M, self.V = (torch.zeros(R, n, dtype=torch.uint8, device=DEV) for _ in range(2))
        self.Ms, self.Vs = (torch.zeros(R, blocks, device=DEV) for _ in range(2))
        self.U, self.Z, self.Vd, self.Zg = torch.zeros(n, device=DEV), z0.clone(), torch.zeros(n, device=DEV), z0.clone()
        self.mask = torch.zeros(plan.groups_total, dtype=torch.uint8, device=DEV)
        self.scale = torch.zeros(R, device=DEV)
        self.norm = torch.zeros(R, dtype=torch.float64, device=DEV)
        self.ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device=DEV)
        cap = plan.packed_capacity_elems
        self.codes = torch.zeros(cap, dtype=torch.uint8, device=DEV)
        self.scales = torch.zeros(cap // 32, dtype=torch.uint8, device=DEV)
        self.off = torch.zeros(plan.n_layers + 1, dtype=torch.int64, device=DEV)
        self.kept = torch.zeros(plan.groups_total, dtype=torch.int32, device=DEV)

    def state(self):
        return [getattr(self, k) for k in ("W", "M", "V", "Ms", "Vs", "low", "U", "Z", "Vd", "Zg", "mask", "codes", "scales")]

    def train(self, plan, rho, coef):
        torch.sub(self.W, self.target, out=self.W_diff)
        self.G.copy_(self.W_diff)
        pkg.hsadmm_gradient_norms(plan, list(self.G), 5.0, self.norm, self.scale, self.ws, grad_type=pkg.TYPE_BF16)
        pkg.hsadmm_adamw(plan, list(self.W), list(self.G), list(self.M), list(self.V), state_bits=8, M_scale=list(self.Ms),
                         V_scale=list(self.Vs), W_low=list(self.low), grad_type=pkg.TYPE_BF16, Z=self.Z, U=self.U, rho=rho,
                         grad_scale=self.scale, coef=coef)

    def project(self, plan, coef):
        pkg.hsadmm_step(plan, list(self.W), U=self.U, Zg=self.Zg, Vd=self.Vd, coef=coef, Z=self.Z, mask=self.mask,
                        workspace=self.ws)


@pytest.mark.parametrize("fmt", [pkg.MX_FP8, pkg.MX_FP4])
def test_outer_iterations_in_a_captured_graph(fmt):
    """Three outer iterations of two nodes: clipped AdamW steps with the pull, the projection, the exchange of quantised
    buffers under the union of the masks, the dual update.  A graph of an iteration, replayed with new coefficients each
    time, gives the same bits as the calls one by one; and the exchange gives what the fp32 calls give, to half a code's step."""
    wl = wk.custom_workload(SHAPES, R=2, seed=1)
    wl.n_arena += -wl.n_arena % 64
    plan = pkg.Plan(wl.table(), pack_align_elems=32)
    L = plan.n_layers
    inside = torch.zeros(wl.n_arena, device=DEV)
    for l in wl.layers:
        inside[l.elem_off:l.elem_off + l.n] = 1
    z0 = torch.randn(wl.n_arena, generator=torch.Generator(device=DEV).manual_seed(0), device=DEV) * 0.1 * inside
    a, b = pkg.hsadmm_node_coefficients([0.05] * L, [0.02] * L, 1e-4, 2, 2)
    node_coef = torch.tensor([x for ab in zip(a, b) for x in ab], device=DEV)
    rho = torch.full((L,), 0.05, device=DEV)
    coef = [torch.zeros(4, device=DEV) for _ in range(2)]                  # of the two local steps of an iteration
    runs = [[Node(wl, plan, 10 + i, z0) for i in range(2)] for _ in range(2)]
    union = [torch.zeros_like(runs[0][0].mask) for _ in runs]
    for nodes in runs:
        for node in nodes:
            node.W_diff = torch.zeros_like(node.W)

    def put(step):
        for i, c in enumerate(coef):
            values = np.array(list(pkg.hsadmm_adamw_coefficients(0.02, 0.9, 0.999, 0.01, 2 * step + i + 1))[:3] + [0], np.float32)
            values.view(np.uint32)[3] = (step * 977 + i) * 0x9E3779B1 & 0xFFFFFFFF
            c.copy_(torch.from_numpy(values).to(DEV))

    def iteration(nodes, union):
        for node in nodes:
            for c in coef:
                node.train(plan, rho, c)
            node.project(plan, node_coef)
        pkg.hsadmm_mask_or(plan, [n.mask for n in nodes], union)
        for node in nodes:
            pkg.hsadmm_compact_mx(plan, node.Z, node.Vd, union, fmt, node.codes, node.scales, node.off, node.kept, node.ws)
        for node in nodes:
            pkg.hsadmm_expand_mx(plan, [n.codes for n in nodes], [n.scales for n in nodes], fmt, None, node.Zg, node.Z, node.Vd,
                                 node.ws)

    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    put(0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        iteration(runs[0], union[0])
    scratch = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device=DEV)
    start = (runs[1][0].W - runs[1][0].target).norm()
    for t in range(4):
        put(t)
        before = [(n.Vd.clone()) for n in runs[1]]
        torch.cuda.synchronize()
        graph.replay()
        iteration(runs[1], union[1])
        torch.cuda.synchronize()
        for x, y in zip(runs[0], runs[1]):
            for i, (p, q) in enumerate(zip(x.state(), y.state())):
                assert torch.equal(p.view(torch.uint8), q.view(torch.uint8)), (t, i)
        # the same exchange through fp32 buffers
        bufs, steps = [], []
        for node, vd in zip(runs[1], before):
            packed = torch.zeros(plan.packed_capacity_elems, device=DEV)
            pkg.hsadmm_compact_sum(plan, node.Z, vd, union[1], packed, node.off, node.kept, scratch)
            bufs.append(packed)
            one = torch.zeros(wl.n_arena, device=DEV)
            pkg.hsadmm_expand_mx(plan, [node.codes], [node.scales], fmt, union[1], one, None, None, scratch)
            exact = torch.zeros(wl.n_arena, device=DEV)
            pkg.hsadmm_expand(plan, packed, union[1], exact, scratch)
            steps.append((one - exact).abs())
            # half a step: 2^-4 (2^-2) of the value, or half the smallest code of a block whose largest it is at least
            assert float((one - exact).abs().max()) <= float(exact.abs().max()) * (2.0 ** -4 if fmt == pkg.MX_FP8 else 2.0 ** -2)
        mean, z = torch.zeros(plan.packed_capacity_elems, device=DEV), torch.zeros(wl.n_arena, device=DEV)
        total = int(runs[1][0].off[-1])
        pkg.hsadmm_average(plan, bufs, total, mean)
        vd = before[0].clone()
        pkg.hsadmm_expand_dual(plan, mean, union[1], z, runs[1][0].Z, vd, scratch)
        room = (steps[0] + steps[1]) / 2 + 2.0 ** -22 * z.abs() + 1e-30
        assert ((z - runs[1][0].Zg).abs() <= room).all()
        assert ((vd - runs[1][0].Vd).abs() <= room + 2.0 ** -22 * (vd.abs() + runs[1][0].Z.abs() + z.abs())).all()
        assert all(torch.isfinite(x.float()).all() for x in (runs[1][0].W, runs[1][0].Zg, runs[1][0].Vd))
    assert (runs[1][0].W - runs[1][0].target).norm() != start
    plan.close()


def test_two_host_threads_on_two_streams():
    """Two threads train and exchange on one plan, each with buffers, a workspace and a stream of its own, at once; the
    results are those of one after the other."""
    wl = wk.custom_workload([(256, 256, 9, F, 100), (300, 256, 1, C, 77), (128, 300, 9, F, 40)], R=2, seed=2)
    wl.n_arena += -wl.n_arena % 64
    plan = pkg.Plan(wl.table(), pack_align_elems=32)
    z0 = torch.randn(wl.n_arena, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    rho = torch.full((plan.n_layers,), 0.1, device=DEV)
    values = np.array(list(pkg.hsadmm_adamw_coefficients(0.02, 0.9, 0.999, 0.01, 1))[:3] + [0], np.float32)
    coef = torch.from_numpy(values).to(DEV)
    results = []
    for together in (False, True):
        nodes = [Node(wl, plan, 20 + i, z0) for i in range(2)]
        for node in nodes:
            node.W_diff = torch.zeros_like(node.W)
            node.mask.fill_(1)
        torch.cuda.synchronize()

        def work(node, stream):
            with torch.cuda.stream(stream):
                for _ in range(5):
                    node.train(plan, rho, coef)
                    pkg.hsadmm_compact_mx(plan, node.W[0], None, node.mask, pkg.MX_FP8, node.codes, node.scales, node.off,
                                          node.kept, node.ws)
                    pkg.hsadmm_expand_mx(plan, [node.codes], [node.scales], pkg.MX_FP8, None, node.Zg, None, None, node.ws)

        streams = [torch.cuda.Stream() for _ in nodes]
        threads = [threading.Thread(target=work, args=a) for a in zip(nodes, streams)]
        for th in threads:
            th.start()
            if not together:
                th.join()
                torch.cuda.synchronize()
        for th in threads:
            th.join()
        torch.cuda.synchronize()
        results.append([x.clone() for node in nodes for x in node.state()])
    for x, y in zip(*results):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    plan.close()


def quantised(c, fmt):
    """fp32 values (a whole number of blocks) as the formats hold them, in torch in 64 bits."""
    b = c.double().view(-1, 32)
    top = 448.0 if fmt == pkg.MX_FP8 else 6.0
    e = torch.ceil(torch.log2(b.abs().amax(1) / top)).clamp(min=-127)
    e = torch.where(b.abs().amax(1) > top * torch.exp2(e), e + 1, e)
    e = torch.where(b.abs().amax(1) <= top * torch.exp2(e - 1), e - 1, e).clamp(min=-127)
    y = b / torch.exp2(e)[:, None]
    bits, least = (3, -6) if fmt == pkg.MX_FP8 else (1, 0)
    step = torch.exp2(torch.clamp(torch.frexp(y)[1] - 1, min=least).double() - bits)
    return (torch.round(y / step) * step * torch.exp2(e)[:, None]).view(-1).float()


@pytest.mark.parametrize("rows,row_len,mode,kept", [
    (71500, 30000, F, [0, 1, 35000, 71498, 71499]),            # the last elements of a layer of nearly 2^31, whole words
    (71000, 30001, F, [0, 2, 40000, 70998, 70999]),            # ... rows that start anywhere
    (3, 5000003, F, [0, 2]),                                   # a row longer than 2^22
    (2, 4300001, C, [0, 5, 4194303, 4194304, 4300000]),        # channels beyond 2^22
    (3, 4300000, B, [1, 4194305, 4299999])])
def test_layers_of_nearly_two_gibi_elements_and_rows_beyond_four_mebi(rows, row_len, mode, kept):
    """Kept groups at both ends of a layer; a small layer of another mode before it."""
    first = 40
    t = {"elem_off": np.array([0, first], np.int64), "c_out": np.array([5, rows], np.int32),
         "c_in": np.array([8, row_len], np.int32), "khw": np.array([1, 1], np.int32), "mode": np.array([N, mode], np.int32),
         "k": np.array([5, max(1, min(len(kept), rows))], np.int32), "k_in": np.array([0, len(kept)], np.int32)}
    plan = pkg.Plan(t, pack_align_elems=32)
    n = first + rows * row_len
    groups = {F: rows, C: row_len, B: rows + row_len}[mode]
    mask = torch.zeros(5 + groups, dtype=torch.uint8, device=DEV)
    row_at = torch.tensor(kept if mode == F else list(range(rows)) if mode == C else [0, 2], device=DEV)
    col_at = torch.arange(row_len, device=DEV) if mode == F else torch.tensor(kept, device=DEV)
    if mode == F:
        mask[5 + row_at] = 1
    elif mode == C:
        mask[5 + col_at] = 1
    else:
        mask[5 + row_at] = 1
        mask[5 + rows + col_at] = 1
    place = (first + row_at[:, None] * row_len + col_at[None, :]).reshape(-1)
    src = torch.empty(n, device=DEV)
    src[:first] = torch.randn(first, device=DEV)
    src[place] = torch.randn(place.numel(), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    size = place.numel()
    room = plan.packed_capacity_elems
    ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device=DEV)
    off = torch.zeros(3, dtype=torch.int64, device=DEV)
    kept_idx = torch.zeros(plan.groups_total, dtype=torch.int32, device=DEV)
    for fmt in (pkg.MX_FP8, pkg.MX_FP4):
        codes = torch.zeros(room, dtype=torch.uint8, device=DEV)
        scales = torch.zeros(room // 32, dtype=torch.uint8, device=DEV)
        pkg.hsadmm_compact_mx(plan, src, None, mask, fmt, codes, scales, off, kept_idx, ws)
        assert off.tolist() == [0, 64, 64 + -(-size // 32) * 32]
        want = quantised(torch.cat((src[place], torch.zeros(-size % 32, device=DEV))), fmt)[:size]
        c = codes[64:64 + size] if fmt == pkg.MX_FP8 else torch.stack((codes & 15, codes >> 4), -1).view(-1)[64:64 + size]
        table = torch.from_numpy(E4M3 if fmt == pkg.MX_FP8 else E2M1).to(DEV)
        s = torch.exp2(scales[2:2 + -(-size // 32)].double() - 127).repeat_interleave(32)[:size]
        assert torch.equal((table[c.long()] * s).float(), want)
        dst = torch.full((n,), 5.0, device=DEV)
        pkg.hsadmm_expand_mx(plan, [codes], [scales], fmt, None, dst, None, None, ws)
        assert torch.equal(dst[place], want)
        dst[place] = 0
        assert int(torch.count_nonzero(dst[first:])) == 0
        del dst, codes, scales
    plan.close()


def test_an_arena_beyond_four_gibi_elements():
    far = 2 ** 32 + 4096
    t = {"elem_off": np.array([0, far], np.int64), "c_out": np.array([6, 40], np.int32), "c_in": np.array([50, 33], np.int32),
         "khw": np.array([1, 9], np.int32), "mode": np.array([F, C], np.int32), "k": np.array([3, 20], np.int32)}
    plan = pkg.Plan(t, pack_align_elems=32)
    n = far + 40 * 33 * 9
    src, dst = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    spans = [(0, 300), (far, 40 * 33 * 9)]
    for o, m in spans:
        src[o:o + m] = torch.randn(m, device=DEV)
    mask = torch.zeros(6 + 33, dtype=torch.uint8, device=DEV)
    mask[[1, 2, 5]] = 1
    mask[6 + torch.arange(0, 33, 2)] = 1
    ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device=DEV)
    room = plan.packed_capacity_elems
    codes, scales = torch.zeros(room, dtype=torch.uint8, device=DEV), torch.zeros(room // 32, dtype=torch.uint8, device=DEV)
    off, kept = torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(39, dtype=torch.int32, device=DEV)
    pkg.hsadmm_compact_mx(plan, src, None, mask, pkg.MX_FP8, codes, scales, off, kept, ws)
    pkg.hsadmm_expand_mx(plan, [codes], [scales], pkg.MX_FP8, mask, dst, None, None, ws)
    keep0 = (mask[:6, None].bool() & torch.ones(6, 50, dtype=torch.bool, device=DEV)).view(-1)
    keep1 = mask[6:].bool()[None, :, None].expand(40, 33, 9).reshape(-1)
    for (o, m), keep in zip(spans, (keep0, keep1)):
        x = src[o:o + m][keep]
        want = torch.zeros(m, device=DEV)
        want[keep] = quantised(torch.cat((x, x.new_zeros(-x.numel() % 32))), pkg.MX_FP8)[:x.numel()]
        assert torch.equal(dst[o:o + m], want)
    plan.close()
