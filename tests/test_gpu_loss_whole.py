"""16-bit layers that begin at a whole piece of 16 bytes: the weights are read where they lie, and the first pass takes all classes at once
whatever the pieces are."""
import pytest
import torch

from tests.test_gpu_loss import BF16, F16, NAMES, Case, SIZES, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(n, -(-D // 8) * 8, V) for n, D, V in SIZES])
def test_loss_and_gradients(kind, n, D, V):
    say("whole", NAMES[kind], n, D, V)
    scale = 1024.0 if kind == F16 else 1.0
    Case(kind, n, D, V, seed=n + D + V, pad=(n * 3) % 9, before=16).run(scale=scale).check(scale=scale)


@pytest.mark.parametrize("kind,n,D,V", [(BF16, 4096, 96, 4100), (BF16, 4100, 4096, 300), (F16, 300, 4096, 4096), (BF16, 4096, 4104, 4096)])
def test_large_tiles(kind, n, D, V):
    say("whole", NAMES[kind], n, D, V)
    Case(kind, n, D, V, seed=1, pad=8, share=0.05, before=16).run(mean=False).check(mean=False)


@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(20, 40, 1500), (300, 72, 1000), (300, 72, 777), (64, 64, 512), (33, 24, 257), (1, 8, 600)])
def test_pieces_of_the_vocabulary(kind, n, D, V, monkeypatch):
    monkeypatch.setenv("HSADMM_LOSS_HELD", "1")
    say("whole, pieces", NAMES[kind], n, D, V)
    Case(kind, n, D, V, seed=5, pad=3, before=16).run().check()


@pytest.mark.parametrize("outputs", [("loss",), ("dX",), ("G",), ("dX", "total")])
def test_any_output_alone(outputs):
    c = Case(BF16, 70, 48, 333, seed=2, before=16).run(outputs=outputs).check(outputs=outputs)
    for name, t in (("loss", c.loss), ("lse", c.lse), ("total", c.total), ("dX", c.all_dx), ("G", c.G)):
        assert name in outputs or torch.isnan(t).all()
