"""hsadmm_softmax_loss against its formulas in 64 bits (tests/ref_tokens.py derives the bounds)."""
import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
from tests import ref_tokens as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = pkg.TYPE_F32, pkg.TYPE_BF16, pkg.TYPE_F16
NAMES = {F32: "fp32", BF16: "bf16", F16: "fp16"}


def say(*what):
    print(*what, flush=True)


class Case:
    """A table of three layers, the middle one with V rows of D weights; arenas hold NaN everywhere else, and activations lie in rows
    with a gap of NaN.  Inputs differ with the seed."""

    def __init__(self, kind, n, D, V, seed=0, pad=0, share=0.2, index_bits=64, before=12):
        gen = torch.Generator().manual_seed(seed)
        self.kind, self.n, self.D, self.V, self.bits = kind, n, D, V, index_bits
        dtype = ref.TYPES[kind]
        self.off = before + (-before) % 4
        size = V * D
        after = self.off + size + (-size) % 4
        self.plan = pkg.Plan({"elem_off": [0, self.off, after], "c_out": [1, V, 2], "c_in": [self.off, D, 3], "khw": [1, 1, 2],
                              "mode": [0, 0, 0], "k": [1, V, 2]})
        nan = float("nan")

        def arena():
            return torch.full((self.plan.arena_elems,), nan, dtype=dtype, device=DEV)

        def rows(width):
            return torch.full((n + 2, width + pad), nan, dtype=dtype, device=DEV)

        w = torch.randn((V, D), generator=gen) * (1.5 / D ** 0.5)
        x = torch.randn((n, D), generator=gen) * 2
        self.W, self.G = arena(), arena()
        self.layer(self.W).copy_(w.to(dtype))
        self.all_x, self.all_dx = rows(D), rows(D)
        self.X, self.dX = self.all_x[:n, :D], self.all_dx[:n, :D]
        self.X.copy_(x.to(dtype))
        y = torch.randint(0, V, (n,), generator=gen)
        none = torch.rand(n, generator=gen) < share
        y[none] = torch.tensor([-100, -1, V, V + 7])[torch.randint(0, 4, (int(none.sum()),), generator=gen)]
        self.labels = y.to(torch.int64 if index_bits == 64 else torch.int32).to(DEV)
        self.loss, self.lse = (torch.full((n + 1,), nan, device=DEV) for _ in range(2))
        self.total = torch.full((3,), nan, device=DEV)

    def layer(self, arena):
        return arena[self.off:self.off + self.V * self.D].view(self.V, self.D)

    def run(self, mean=True, scale=1.0, accumulate=False, outputs=("loss", "lse", "total", "dX", "G"), stream=None, ws=None):
        nbytes = pkg.hsadmm_softmax_loss_workspace(self.plan, 1, self.n, self.kind, "dX" in outputs or "G" in outputs)
        if ws is None:
            ws = torch.full((nbytes + 512,), 255, dtype=torch.uint8, device=DEV)        # (NaN wherever it is read unwritten)
        give = {"loss": self.loss[:self.n], "lse": self.lse[:self.n], "total": self.total[:2], "dX": self.dX, "G": self.G}
        pkg.hsadmm_softmax_loss(self.plan, 1, self.W, self.X, self.labels, workspace=ws, workspace_bytes=nbytes, mean=mean, scale=scale,
                                accumulate=accumulate, type=self.kind, index_bits=self.bits, stream=stream,
                                **{k: give[k] for k in outputs})
        torch.cuda.synchronize()
        if ws.numel() == nbytes + 512:
            assert (ws[nbytes:] == 255).all()
        return self

    def check(self, mean=True, scale=1.0, before=None, outputs=("loss", "lse", "total", "dX", "G")):
        want = ref.loss_reference(self.kind, self.X, self.layer(self.W), self.labels.long(), mean, scale)
        for name in outputs:
            if name == "total":
                ref.close(self.total[0], *want["total"], "total")
                target = ((self.labels >= 0) & (self.labels < self.V)).sum()
                assert self.total[1] == target
            elif name == "G":
                value, bound = want["G"]
                if before is not None:
                    value, bound = value + before.double(), bound + ref.U * (value.abs() + before.double().abs())
                ref.close(self.layer(self.G), value, ref.rounded(self.kind, value, bound), "G")
            elif name == "dX":
                ref.close(self.dX, *want["dX"], "dX")
            else:
                ref.close(getattr(self, name)[:self.n], *want[name], name)
        # nothing else was written: gaps, rows behind the last, other layers
        assert torch.isnan(self.all_dx[self.n:]).all() and torch.isnan(self.all_dx[:, self.D:]).all()
        assert torch.isnan(self.G[:self.off]).all() and torch.isnan(self.G[self.off + self.V * self.D:]).all()
        assert torch.isnan(self.loss[self.n:]).all() and torch.isnan(self.lse[self.n:]).all() and torch.isnan(self.total[2:]).all()
        return self


SIZES = [(1, 1, 1), (1, 8, 3), (2, 5, 7), (3, 64, 128), (31, 65, 129), (32, 72, 257), (33, 64, 10), (64, 63, 64), (129, 100, 300), (200, 45, 1001),
         (257, 136, 515), (300, 1441, 700), (1000, 24, 2050)]


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", SIZES)
def test_loss_and_gradients(kind, n, D, V):
    say("loss", NAMES[kind], n, D, V)
    scale = 1024.0 if kind == F16 else 1.0
    Case(kind, n, D, V, seed=n + D + V, pad=(n * 3) % 9).run(scale=scale).check(scale=scale)


@pytest.mark.parametrize("kind,n,D,V", [(BF16, 4096, 96, 4100), (BF16, 4100, 4096, 300), (F16, 300, 4096, 4096), (BF16, 4096, 4104, 4096)])
def test_large_tiles(kind, n, D, V):
    """Sizes that fill the chip with tiles of 256 by 256 in one or more of the products."""
    say("loss", NAMES[kind], n, D, V)
    Case(kind, n, D, V, seed=1, pad=8, share=0.05).run(mean=False).check(mean=False)


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(20, 40, 1500), (20, 41, 1500), (300, 72, 1000), (300, 71, 777), (64, 64, 512)])
def test_pieces_of_the_vocabulary(kind, n, D, V, monkeypatch):
    monkeypatch.setenv("HSADMM_LOSS_HELD", "1")
    say("loss in pieces", NAMES[kind], n, D, V)
    Case(kind, n, D, V, seed=5, pad=3).run().check()


def test_no_more_logits_are_held_than_fit():
    """The workspace is bounded by the pieces, whatever the vocabulary: 2^31 bytes of logits or their gradients (a piece is 256 classes
    at least), and room for a copy and up to 64 sums of the inputs and for the slabs' numbers."""
    plan = pkg.Plan({"elem_off": [0], "c_out": [2 ** 20], "c_in": [64], "khw": [1], "mode": [0], "k": [1]})
    for n in (1, 1000, 8192, 65536):
        np_ = n + 256
        rest = 8 * np_ * (2 ** 20 // 32 + 8) + np_ * (64 * 2 + 40) + 8192
        assert pkg.hsadmm_softmax_loss_workspace(plan, 0, n, BF16, False) <= rest
        assert pkg.hsadmm_softmax_loss_workspace(plan, 0, n, BF16, True) <= 2 ** 31 + rest + 64 * 4 * 64 * np_, n
    assert pkg.hsadmm_softmax_loss_workspace(plan, 0, 0, BF16, True) > 0


@pytest.mark.parametrize("outputs", [("loss",), ("lse",), ("total",), ("dX",), ("G",), ("loss", "total"), ("dX", "total")])
@pytest.mark.parametrize("kind", [F32, BF16], ids=NAMES.get)
def test_any_output_alone(kind, outputs):
    c = Case(kind, 70, 48, 333, seed=2).run(outputs=outputs).check(outputs=outputs)
    for name, t in (("loss", c.loss), ("lse", c.lse), ("total", c.total), ("dX", c.all_dx), ("G", c.G)):
        assert name in outputs or torch.isnan(t).all()


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("D", [40, 39])
def test_accumulates(kind, D):
    c = Case(kind, 50, D, 130, seed=3)
    start = (torch.randn((130, D), generator=torch.Generator().manual_seed(9)) * 0.01).to(ref.TYPES[kind]).to(DEV)
    c.layer(c.G).copy_(start)
    c.run(accumulate=True).check(before=start)


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n", [1, 40, 600])
def test_without_any_target(kind, n):
    c = Case(kind, n, 72, 99, share=2.0)
    c.X.fill_(float("nan"))
    c.run()
    assert (c.loss[:n] == 0).all() and (c.lse[:n] == 0).all() and (c.total[:2] == 0).all()
    assert (c.dX == 0).all() and (c.layer(c.G) == 0).all()


@pytest.mark.parametrize("kind", [F32, BF16], ids=NAMES.get)
def test_rows_without_a_target_may_hold_anything(kind):
    c = Case(kind, 90, 64, 200, seed=4, share=0.5)
    none = (c.labels < 0) | (c.labels >= c.V)
    c.X[none] = torch.tensor([float("nan"), float("inf")], device=DEV).repeat(32).to(c.X.dtype)
    c.run()
    plain = Case(kind, 90, 64, 200, seed=4, share=0.5).run().check()
    for a, b in ((c.loss[:90], plain.loss[:90]), (c.dX, plain.dX), (c.G[c.off:c.off + 200 * 64], plain.G[c.off:c.off + 200 * 64])):
        assert torch.equal(a, b)
    assert (c.dX[none] == 0).all()


def test_no_rows():
    c = Case(BF16, 0, 24, 50)
    c.run()
    assert (c.total[:2] == 0).all() and (c.layer(c.G) == 0).all()
    start = torch.ones((50, 24), dtype=torch.bfloat16, device=DEV)
    c.layer(c.G).copy_(start)
    c.run(accumulate=True)
    assert torch.equal(c.layer(c.G), start)


@pytest.mark.parametrize("D", [8, 40, 64, 72])
def test_a_class_whose_logit_is_minus_infinity(D):
    """Its probability is 0; the zeros that fill a row up to a tile's end are no factors of it."""
    c = Case(F32, 40, D, 70, seed=6)
    c.X[:, 0] = c.X[:, 0].abs() + 0.1
    c.labels[c.labels == 5] = 6
    w = c.layer(c.W)
    w[5, 0] = float("-inf")
    c.run(outputs=("loss", "lse", "total"))
    x, y = c.X.double(), c.labels.long()
    at = ((y >= 0) & (y < 70)).nonzero()[:, 0]
    want = torch.nn.functional.cross_entropy(x[at] @ w.double().T, y[at], reduction="none")
    ok = c.loss[:40][at]
    assert torch.isfinite(ok).all()
    # (the bound of the same inputs without that class)
    w[5, 0] = 0.0
    bound = ref.loss_reference(F32, c.X, w, y, True, 1.0)["loss"][1][at]
    ref.close(ok, want, bound, "loss")


def test_a_row_that_is_not_finite_stays_one_rows_loss():
    c = Case(F32, 60, 32, 70, seed=7, share=0.0)
    c.X[11, 3] = float("nan")
    c.X[12, 3] = float("inf")
    c.run(outputs=("loss", "lse"))
    bad = ~torch.isfinite(c.loss[:60])
    assert bad.nonzero()[:, 0].tolist() == [11, 12]


@pytest.mark.parametrize("kind", [F32, BF16], ids=NAMES.get)
def test_large_and_small_logits(kind):
    """Logits of thousands: the largest is taken off before the exponential."""
    c = Case(kind, 64, 64, 300, seed=8, share=0.0)
    c.X.mul_(500.0)
    c.run().check()


@pytest.mark.parametrize("bits", [32, 64])
def test_labels_of_both_widths(bits):
    c = Case(F32, 80, 20, 60, seed=9, index_bits=bits)
    if bits == 64:
        c.labels[3], c.labels[4] = 2 ** 32 + 5, -2 ** 40         # (no target, whatever the lower half says)
    c.run().check()


@pytest.mark.parametrize("kind,n,D,V", [(F32, 300, 72, 1000), (BF16, 300, 71, 1000), (BF16, 1, 512, 5000)])
def test_same_bits_from_run_to_run(kind, n, D, V):
    a, b = (Case(kind, n, D, V, seed=10).run() for _ in range(2))
    for x, y in ((a.loss[:n], b.loss[:n]), (a.lse[:n], b.lse[:n]), (a.dX, b.dX), (a.layer(a.G), b.layer(b.G)), (a.total[:2], b.total[:2])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("n", [63, 64, 65, 255, 257, 2047, 2048, 2049])
@pytest.mark.parametrize("D", [24, 264])
def test_listing_rows_around_the_sizes_of_its_pieces(n, D, bits):
    """Half the rows have no target; the total's bits do not depend on what else is asked for."""
    say("listing", n, D, bits)
    case = Case(F32, n, D, 37, seed=n, share=0.5, index_bits=bits).run().check()
    total = case.total.clone()
    case.run(outputs=("total",))
    assert torch.equal(case.total[:2], total[:2])


@pytest.mark.parametrize("which", ["first", "last", "all", "none"])
@pytest.mark.parametrize("n", [1, 65, 2048, 2049])
def test_listing_one_row_or_all(n, which):
    say("listing", n, which)
    case = Case(BF16, n, 40, 9, seed=n, share=0.0)
    if which in ("first", "last"):
        keep = 0 if which == "first" else n - 1
        y = int(case.labels[keep])
        case.labels.fill_(-100)
        case.labels[keep] = y
    elif which == "none":
        case.labels.fill_(-100)
    case.run().check()


def test_gradients_against_differences():
    """The kernels' gradients in fp32 against differences of the loss in 64 bits: a step h = 1e-4 of both sides is off by h^2 / 6 times
    the third derivative, which for a softmax is at most |direction . input|^3 of its logits."""
    c = Case(F32, 24, 12, 40, seed=11).run()
    X, W, y = c.X.double(), c.layer(c.W).double(), c.labels.long()
    at = ((y >= 0) & (y < 40)).nonzero()[:, 0]
    gen = torch.Generator().manual_seed(1)
    h = 1e-4
    want = ref.loss_reference(F32, c.X, c.layer(c.W), y, True, 1.0)
    for _ in range(5):
        a, b = (torch.randn(s, generator=gen, dtype=torch.float64).to(DEV) for s in (W.shape, X.shape))

        def loss(t):
            return torch.nn.functional.cross_entropy((X + t * b)[at] @ (W + t * a).T, y[at])

        slope = (loss(h) - loss(-h)) / (2 * h)
        got = (c.layer(c.G).double() * a).sum() + (c.dX.double() * b).sum()
        moved = ((b.abs() @ W.abs().T) + X.abs() @ a.abs().T).amax() + h * (b.abs() @ a.abs().T).amax()
        # (the logits' own second derivative, b a^T, enters with the first's product)
        bound = h * h * (moved ** 3 + 3 * moved * (b.abs() @ a.abs().T).amax()) + 1e-10
        bound += (ref.rounded(F32, *want["G"]) * a.abs()).sum() + (want["dX"][1] * b.abs()).sum()
        assert abs(slope - got) <= bound


def test_captured_calls_replay_with_eager_ones_between():
    c, other = Case(BF16, 200, 64, 700, seed=12), Case(BF16, 150, 80, 400, seed=13)
    nbytes = pkg.hsadmm_softmax_loss_workspace(c.plan, 1, 200, BF16, True)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)

    def call(stream=None):
        pkg.hsadmm_softmax_loss(c.plan, 1, c.W, c.X, c.labels, workspace=ws, loss=c.loss[:200], lse=c.lse[:200], total=c.total[:2],
                                dX=c.dX, G=c.G, type=BF16, index_bits=64, stream=stream)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    inputs = [Case(BF16, 200, 64, 700, seed=s) for s in (21, 22, 23)]
    for i in inputs:
        c.X.copy_(i.X)
        c.labels.copy_(i.labels)
        c.W.copy_(i.W)
        graph.replay()
        other.run().check()
        torch.cuda.synchronize()
        i.run()
        for a, b in ((c.loss[:200], i.loss[:200]), (c.dX, i.dX), (c.layer(c.G), i.layer(i.G)), (c.total[:2], i.total[:2])):
            assert torch.equal(a, b)


def test_two_streams_with_a_workspace_each():
    cases = [Case(BF16, 500, 128, 3000, seed=30 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    spaces = [torch.zeros(pkg.hsadmm_softmax_loss_workspace(c.plan, 1, c.n, BF16, True), dtype=torch.uint8, device=DEV) for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s, ws in zip(cases, streams, spaces):
            pkg.hsadmm_softmax_loss(c.plan, 1, c.W, c.X, c.labels, workspace=ws, loss=c.loss[:c.n], lse=c.lse[:c.n], total=c.total[:2],
                                    dX=c.dX, G=c.G, type=BF16, index_bits=64, stream=s)
    torch.cuda.synchronize()
    for c in cases:
        c.check()


def test_refusals():
    c = Case(F32, 6, 20, 30)
    nbytes = pkg.hsadmm_softmax_loss_workspace(c.plan, 1, 6, F32, True)
    ws = torch.zeros(nbytes + 256, dtype=torch.uint8, device=DEV)
    good = dict(layer=1, W=c.W, X=c.X, labels=c.labels, workspace=ws, loss=c.loss[:6], dX=c.dX, G=c.G, type=F32, index_bits=64)

    def code(**change):
        a = {**good, **change}
        return pkg.hsadmm_softmax_loss(c.plan, a.pop("layer"), a.pop("W"), a.pop("X"), a.pop("labels"), check=False, **a)

    assert code() == 0
    assert code(layer=-1) == -1 and code(layer=3) == -1
    assert code(layer=2, X=8, dX=8) == -4                                          # khw != 1
    assert code(type=7) == -4 and code(index_bits=16) == -4
    assert code(W=None) == -1 and code(X=None) == -1 and code(workspace=None, workspace_bytes=nbytes) == -1
    assert code(W=c.W.data_ptr() + 8) == -1 and code(workspace=ws[8:]) == -1
    assert code(workspace_bytes=nbytes - 1) == -2
    assert code(loss=None, dX=None, G=None) == -1                                  # nothing is wanted
    assert code(scale=float("nan")) == -1 and code(scale=float("inf")) == -1
    assert code(labels=c.labels.int()) == -1 and code(X=c.X.half()) == -1 and code(X=c.X[:5]) == -1 and code(X=c.X.T) == -1
    assert code(X=c.X[:1].expand(6, 20)) == -1
    assert code(dX=c.X) == -1 and code(G=c.W) == -1 and code(loss=c.loss[:6], lse=c.loss[:6]) == -1 and code(G=c.G[:-1]) == -1
    assert code(loss=c.loss[:5]) == -1 and code(total=c.total[:1]) == -1
    assert code(labels=c.labels.data_ptr()) == -1                                  # no n
    assert code(labels=c.labels.data_ptr(), n=-1) == -1 and code(labels=8, X=16, dX=16, loss=4, n=2 ** 21 + 1) == -4
    torch.cuda.synchronize()
