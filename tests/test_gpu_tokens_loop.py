"""A language model's training step made of the calls together, as a program runs them: embedding, dropout, loss, the gradients back
through all of them, their norm, and AdamW, whose rounded weights the next step reads.  Every stage is checked against its formulas in
64 bits on the inputs it had on the device; the same steps are replayed from a graph."""
import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
from tests import ref_tokens as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = pkg.TYPE_F32, pkg.TYPE_BF16, pkg.TYPE_F16
P_DROP, SEED, SCALE = 0.25, 0xDEADBEEF12345, 6.0


class Model:
    """An embedding of V rows and a head over the classes; tied: one layer is both.  A layer in front keeps them off the arena's start."""

    def __init__(self, kind, n, V, D, tied, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.kind, self.n, self.V, self.D, self.tied = kind, n, V, D, tied
        self.dtype = ref.TYPES[kind]
        off, size = 16, V * D + (-V * D) % 8
        offs = [0, off] + ([] if tied else [off + size])
        L = len(offs)
        self.plan = pkg.Plan({"elem_off": offs, "c_out": [4] + [V] * (L - 1), "c_in": [4] + [D] * (L - 1), "khw": [1] * L,
                              "mode": [0] * L, "k": [4] + [V] * (L - 1)})
        self.first, self.last, self.offs = 1, L - 1, offs
        elems = self.plan.arena_elems
        self.W = (torch.randn(elems, generator=gen) * D ** -0.5).to(DEV)
        self.low = self.W.to(self.dtype) if kind != F32 else None
        self.G = torch.zeros(elems, dtype=self.dtype, device=DEV)
        self.M, self.Vv = torch.zeros(elems, device=DEV), torch.zeros(elems, device=DEV)
        rows = lambda: torch.zeros((n, D), dtype=self.dtype, device=DEV)          # noqa: E731
        self.x0, self.x1, self.dx1, self.dx0 = rows(), rows(), rows(), rows()
        self.ids = torch.zeros(n, dtype=torch.int64, device=DEV)
        self.labels = torch.zeros(n, dtype=torch.int64, device=DEV)
        self.loss, self.total = torch.zeros(n, device=DEV), torch.zeros(2, device=DEV)
        self.norm, self.factor = torch.zeros(1, dtype=torch.float64, device=DEV), torch.zeros(1, device=DEV)
        self.call = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.coef = torch.zeros(16, dtype=torch.uint8, device=DEV)
        self.ws = torch.zeros(max(self.plan.workspace_bytes, pkg.hsadmm_embedding_workspace(self.plan, 1, n),
                                  pkg.hsadmm_softmax_loss_workspace(self.plan, self.last, n, kind, True)), dtype=torch.uint8, device=DEV)
        self.loss_scale = 256.0 if kind == F16 else 1.0

    def batch(self, step):
        gen = torch.Generator().manual_seed(100 + step)
        ids = torch.randint(0, self.V, (self.n + 1,), generator=gen)
        ids[:self.n // 4] = 3                                                    # (one token many times)
        labels = ids[1:].clone()
        labels[torch.rand(self.n, generator=gen) < 0.2] = -100
        ids[torch.rand(self.n + 1, generator=gen) < 0.05] = -1
        self.ids.copy_(ids[:-1])
        self.labels.copy_(labels)
        self.call.fill_(step)
        decay, size, root, noise = pkg.hsadmm_adamw_coefficients(1e-2, 0.9, 0.99, 0.01, step + 1, 0)
        raw = np.array([decay, size, root], np.float32).tobytes() + np.uint32(noise).tobytes()
        self.coef.copy_(torch.frombuffer(bytearray(raw), dtype=torch.uint8))

    def layer(self, arena, l):
        return arena[self.offs[l]:self.offs[l] + self.V * self.D].view(self.V, self.D)

    def step(self, watch=lambda stage: None):
        p, kind, weights = self.plan, self.kind, self.W if self.low is None else self.low
        pkg.hsadmm_embedding(p, self.first, weights, self.ids, self.x0, scale=SCALE, type=kind, index_bits=64)
        watch("embedding")
        pkg.hsadmm_dropout(p, self.x0, self.x1, P_DROP, SEED, 0, type=kind, call_device=self.call)
        watch("dropout")
        pkg.hsadmm_softmax_loss(p, self.last, weights, self.x1, self.labels, workspace=self.ws, loss=self.loss, total=self.total, dX=self.dx1,
                                G=self.G, scale=self.loss_scale, type=kind, index_bits=64)
        watch("loss")
        pkg.hsadmm_dropout(p, self.dx1, self.dx0, P_DROP, SEED, 0, type=kind, call_device=self.call)
        watch("dropout back")
        pkg.hsadmm_embedding_gradient(p, self.first, self.ids, self.dx0, self.G, self.ws, scale=SCALE, accumulate=self.tied, type=kind,
                                      index_bits=64)
        watch("embedding back")
        pkg.hsadmm_gradient_norms(p, [self.G], 1.0 * self.loss_scale, self.norm, self.factor, self.ws, grad_type=kind)
        if self.loss_scale != 1.0:
            self.factor.mul_(1.0 / self.loss_scale)
        pkg.hsadmm_adamw(p, [self.W], [self.G], [self.M], [self.Vv], grad_type=kind, W_low=None if self.low is None else [self.low],
                         grad_scale=self.factor, coef=self.coef)
        watch("update")

    def state(self):
        return [t.clone() for t in (self.W, self.G, self.M, self.Vv, self.loss, self.total, self.dx0, self.norm)]


def check_stages(m):
    held = {}

    def watch(stage):
        torch.cuda.synchronize()
        kind, weights = m.kind, m.W if m.low is None else m.low
        kept, factor = ref.dropout_kept(m.n * m.D, P_DROP, SEED, int(m.call))
        kept = torch.from_numpy(kept).view(m.n, m.D).to(DEV)
        if stage == "embedding":
            ref.close(m.x0, *ref.embedding_reference(kind, m.layer(weights, m.first), m.ids, SCALE), stage)
        elif stage == "dropout":
            ref.close(m.x1, *ref.dropout_reference(kind, m.x0, kept, factor), stage)
        elif stage == "loss":
            want = ref.loss_reference(kind, m.x1, m.layer(weights, m.last), m.labels, True, m.loss_scale)
            ref.close(m.loss, *want["loss"], "loss")
            ref.close(m.total[0], *want["total"], "total")
            ref.close(m.dx1, *want["dX"], "dX")
            value, bound = want["G"]
            ref.close(m.layer(m.G, m.last), value, ref.rounded(kind, value, bound), "G of the head")
            held["G"] = m.layer(m.G, m.first).clone()
        elif stage == "dropout back":
            ref.close(m.dx0, *ref.dropout_reference(kind, m.dx1, kept, factor), stage)
        elif stage == "embedding back":
            value, bound = ref.embedding_gradient_reference(m.V, m.dx0, m.ids, SCALE)
            if m.tied:
                value, bound = value + held["G"].double(), bound + ref.U * (value.abs() + held["G"].double().abs())
            ref.close(m.layer(m.G, m.first), value, ref.rounded(kind, value, bound), "G of the embedding")
            held["norm"] = m.G.double().norm()
        else:
            # (sums of squares in 64 bits: 2^-53 a term)
            assert abs(m.norm[0] - held["norm"]) <= 1e-12 * held["norm"]
            if m.low is not None:
                assert torch.equal(m.low[:m.plan.arena_elems], m.W.to(m.dtype))

    return watch


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("n,V,D", [(70, 131, 24), (300, 600, 71)])
def test_steps_stage_by_stage(kind, tied, n, V, D):
    print("steps", kind, tied, n, V, D, flush=True)
    m = Model(kind, n, V, D, tied)
    for step in range(3):
        m.batch(step)
        m.step(check_stages(m))


@pytest.mark.parametrize("kind,tied", [(F32, True), (BF16, True), (BF16, False)])
def test_captured_steps_give_the_eager_ones_bits(kind, tied):
    eager, graphed = (Model(kind, 300, 600, 72, tied) for _ in range(2))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        graphed.step()
    for step in range(4):
        for m in (eager, graphed):
            m.batch(step)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b), step


def test_two_models_on_two_streams():
    """Calls of two models in flight at once, each with a workspace of its own, give what each gives alone."""
    alone, together = ([Model(BF16, 200 + 60 * i, 500, 64, True, seed=i) for i in range(2)] for _ in range(2))
    streams = [torch.cuda.Stream() for _ in together]
    for step in range(3):
        for m in alone:
            m.batch(step)
            m.step()
            torch.cuda.synchronize()
        for m in together:
            m.batch(step)
        torch.cuda.synchronize()
        for m, s in zip(together, streams):
            with torch.cuda.stream(s):
                m.step()
        torch.cuda.synchronize()
        for a, b in zip(alone, together):
            for x, y in zip(a.state(), b.state()):
                assert torch.equal(x, y)


def test_the_models_gradient_against_differences():
    """The whole step's gradient in fp32 along random directions of the weights against differences of the loss in 64 bits, the
    masks taken as they fall.  Its bound: what the stages' bounds add up to along the direction is below 2^-15 of the terms here
    (sums of fewer than 2^9 terms of 2^-24 each), the difference's own error (h = 1e-4) below 1e-6 of a third derivative of order 10."""
    m = Model(F32, 60, 90, 16, True, seed=4)
    m.batch(0)
    W0 = m.W.clone()
    pkg.hsadmm_embedding(m.plan, 1, m.W, m.ids, m.x0, scale=SCALE, index_bits=64)
    m.step()
    torch.cuda.synchronize()
    kept, factor = ref.dropout_kept(m.n * m.D, P_DROP, SEED, 0)
    kept = torch.from_numpy(kept).view(m.n, m.D).to(DEV).double() * factor
    token, target = (m.ids >= 0), ((m.labels >= 0) & (m.labels < m.V))
    w0 = m.layer(W0, 1).double()
    gen = torch.Generator().manual_seed(8)

    def loss(w):
        x = torch.where(token[:, None], w[m.ids.clamp(min=0)], 0.0) * SCALE * kept
        return torch.nn.functional.cross_entropy((x @ w.T)[target], m.labels[target])

    for _ in range(4):
        d = torch.randn(w0.shape, generator=gen, dtype=torch.float64).to(DEV)
        h = 1e-4
        slope = (loss(w0 + h * d) - loss(w0 - h * d)) / (2 * h)
        g = m.layer(m.G, 1).double()
        assert abs((g * d).sum() - slope) <= 2.0 ** -15 * (g * d).abs().sum() + 1e-5
