"""Gradients of rows whose label already has some of the softmax, as in a model that has learnt something: the label's own term is most
of a row's gradient, and of the gradient of a class that few rows name.  Labels as of random weights have softmax - 1 = -1, which every
type holds.

Bounds.  The label's term carries fp32 steps alone into dX.  Into G it goes in two pieces of the type.  The second is at most half a step of
the first and is rounded itself, half_step^2, or it is left out where it is below a 64th of half a step: of the two the larger is
counted, half_step / 64 (half_step <= 2^-8).  The other classes' weights are small here, so that what rounding their softmax
may do (ref_tokens.py) is far below half a step of the result."""
import pytest
import torch

import paper_2512_14628_amd as pkg
from tests import ref_tokens as ref
from tests.test_gpu_loss import BF16, DEV, F16, F32, NAMES, Case, say

pytestmark = pytest.mark.gpu


def spread(kind, n, D, V, seed, named=None, few=1.0, before=16, **more):
    """A case whose labels (the first `named` classes) have softmaxes spread over (0, 1): their rows of W are orthogonal-ish and large, the
    others' a fiftieth, and a row of X is its label's row so long that the logit is about log V - 4 to log V + 4."""
    c = Case(kind, n, D, V, seed=seed, before=before, **more)
    gen = torch.Generator().manual_seed(seed + 1)
    named = V if named is None else named
    w = torch.randn((V, D), generator=gen) * (0.02 / D ** 0.5)
    w[:named] = torch.randn((named, D), generator=gen) / D ** 0.5
    y = torch.randint(0, named, (n,), generator=gen)
    if few < 1.0:
        y = torch.where(torch.rand(n, generator=gen) < few, y, -100)
    at = y.clamp(min=0)
    length = torch.log(torch.tensor(float(V))) + 8 * torch.rand(n, generator=gen) - 4
    x = w[at] / (w[at] ** 2).sum(1, keepdim=True) * length[:, None]
    dtype = ref.TYPES[kind]
    c.layer(c.W).copy_(w.to(dtype))
    c.X.copy_(x.to(dtype))
    c.labels.copy_(y.to(c.labels.dtype))
    return c


def check(c, mean=True, scale=1.0):
    half = 0.0 if c.kind == F32 else ref.half_step(c.kind)
    want = ref.loss_reference(c.kind, c.X, c.layer(c.W), c.labels.long(), mean, scale, label=(0.0, half / 64))
    p = torch.exp(-want["loss"][0][(c.labels >= 0) & (c.labels < c.V)])
    assert p.min() < 0.1 and p.max() > 0.9 and 0.3 < p.mean() < 0.7          # (the labels do have what the case is about)
    ref.close(c.dX, *want["dX"], "dX")
    value, bound = want["G"]
    ref.close(c.layer(c.G), value, ref.rounded(c.kind, value, bound), "G")


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V,named", [(300, 256, 4096, 300), (1000, 512, 8192, 4000), (64, 512, 5000, 64), (1, 256, 5000, 8), (513, 255, 1000, 400),
                                         (2500, 512, 4100, 17), (2048, 1024, 16384, 16384), (4500, 128, 2000, 3)])
def test_gradients_where_labels_have_some_of_the_softmax(kind, n, D, V, named):
    """Tiles of every size, labels that one or thousands of rows name."""
    say("spread", NAMES[kind], n, D, V, named)
    if n == 1:
        c = spread(kind, 40, D, V, 5, named)
        # (one row of them after the other)
        for i in range(40):
            one = Case(kind, 1, D, V, seed=9)
            one.layer(one.W).copy_(c.layer(c.W))
            one.X.copy_(c.X[i:i + 1])
            one.labels.copy_(c.labels[i:i + 1])
            one.run()
            want = ref.loss_reference(kind, one.X, one.layer(one.W), one.labels.long(), True, 1.0,
                                      label=(0.0, 0.0 if kind == F32 else ref.half_step(kind) / 64))
            ref.close(one.dX, *want["dX"], "dX")
            ref.close(one.layer(one.G), want["G"][0], ref.rounded(kind, *want["G"]), "G")
        return
    scale = 256.0 if kind == F16 else 1.0
    for before in (16, 12):                                  # (weights read where they lie, and copied first)
        c = spread(kind, n, D, V, n + V, named, pad=n % 7, before=before)
        check(c.run(scale=scale), scale=scale)


@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(1024, 64, 20000), (1024, 65, 20000), (24, 264, 3000), (300, 72, 1500)])
def test_pieces_of_the_vocabulary(kind, n, D, V, monkeypatch):
    """Labels in every piece, also at its ends."""
    monkeypatch.setenv("HSADMM_LOSS_HELD", "1" if n < 1000 else str(2 * 1024 * 8192))
    say("spread, pieces", NAMES[kind], n, D, V)
    for before in (16, 12):
        c = spread(kind, n, D, V, 7, few=0.8, pad=2, before=before)
        check(c.run(mean=False), mean=False)


@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
def test_accumulates(kind):
    c = spread(kind, 400, 256, 3000, 11, 300)
    gen = torch.Generator().manual_seed(3)
    start = (torch.randn((3000, 256), generator=gen) * 1e-3).to(ref.TYPES[kind]).to(DEV)
    c.layer(c.G).copy_(start)
    c.run(accumulate=True)
    half = ref.half_step(kind)
    value, bound = ref.loss_reference(kind, c.X, c.layer(c.W), c.labels.long(), True, 1.0, label=(0.0, half / 64))["G"]
    value, bound = value + start.double(), bound + ref.U * (value.abs() + start.double().abs())
    ref.close(c.layer(c.G), value, ref.rounded(kind, value, bound), "G")


@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
def test_rows_without_a_target_among_them(kind):
    c = spread(kind, 700, 128, 2000, 13, 500, few=0.4)
    c.X[c.labels < 0] = float("nan")
    check(c.run())
    assert (c.dX[c.labels < 0] == 0).all()


@pytest.mark.parametrize("outputs", [("dX",), ("G",)])
def test_either_gradient_alone(outputs):
    a, b = (spread(BF16, 600, 128, 2500, 17, 500) for _ in range(2))
    a.run()
    b.run(outputs=outputs)
    if outputs == ("dX",):
        assert torch.equal(a.dX, b.dX) and torch.isnan(b.G).all()
    else:
        assert torch.equal(a.layer(a.G), b.layer(b.G)) and torch.isnan(b.all_dx).all()


def test_captured_calls_replay_with_other_labels():
    """Which rows a tile of classes gathers follows from the labels that are there when the graph runs."""
    c = spread(BF16, 600, 128, 2500, 19, 500)
    ws = torch.zeros(pkg.hsadmm_softmax_loss_workspace(c.plan, 1, 600, BF16, True), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        pkg.hsadmm_softmax_loss(c.plan, 1, c.W, c.X, c.labels, workspace=ws, loss=c.loss[:600], dX=c.dX, G=c.G, type=BF16, index_bits=64)
    for seed, named, few in ((20, 500, 1.0), (21, 3, 0.5), (22, 2500, 0.9), (23, 1, 1.0)):
        other = spread(BF16, 600, 128, 2500, seed, named, few=few)
        for a, b in ((c.X, other.X), (c.labels, other.labels), (c.W, other.W)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        check(other.run())
        assert torch.equal(c.dX, other.dX) and torch.equal(c.layer(c.G), other.layer(other.G)) and torch.equal(c.loss[:600], other.loss[:600])
