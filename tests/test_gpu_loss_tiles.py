"""hsadmm_softmax_loss where few rows meet many classes or wide rows, so that the tiles that fill the chip are larger than the rows there
are, and the largest tiles in every product and form (tests/test_loss_plan_cpu.py sweeps the arithmetic behind them)."""
import pytest

import paper_2512_14628_amd as pkg
from tests.test_gpu_loss import BF16, F16, F32, NAMES, Case, say

pytestmark = pytest.mark.gpu

LOSSES = ("loss", "lse", "total")
# Where the layer begins, in elements: 16-bit weights are read where they lie, or, not at a whole piece of 16 bytes, copied first.
BEFORE = pytest.mark.parametrize("before", [16, 12], ids=["whole", "copied"])


@BEFORE
@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(33, 64, 65536), (64, 64, 65536), (127, 64, 65536), (128, 64, 65536), (129, 64, 65536), (33, 1024, 65536),
                                   (128, 256, 70000), (100, 4096, 16384)])
def test_losses_of_a_few_dozen_rows(kind, n, D, V, before):
    say("losses", NAMES[kind], n, D, V)
    Case(kind, n, D, V, seed=n + V, pad=n % 9, before=before).run(outputs=LOSSES).check(outputs=LOSSES)


@BEFORE
@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(33, 2048, 32768), (64, 2048, 32768), (127, 2048, 32768), (128, 2048, 32768), (129, 2048, 32768),
                                   (100, 4096, 16384), (65, 1031, 65536)])
def test_gradients_of_a_few_dozen_rows(kind, n, D, V, before):
    say("gradients", NAMES[kind], n, D, V)
    scale = 1024.0 if kind == F16 else 1.0
    Case(kind, n, D, V, seed=n + D, pad=n % 9, before=before).run(scale=scale).check(scale=scale)


def test_a_few_dozen_rows_in_fp32():
    say("gradients fp32 100 1024 40000")
    Case(F32, 100, 1024, 40000, seed=3).run().check()


@BEFORE
@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(200, 4096, 16384), (256, 4096, 4096), (4096, 4096, 200)])
def test_what_the_rounding_leaves_in_large_tiles(kind, n, D, V, before):
    """Up to 256 rows or classes, and tiles of 256 in the products that take the rest as well."""
    say("rest", NAMES[kind], n, D, V)
    Case(kind, n, D, V, seed=2, share=0.05, before=before).run().check()


@BEFORE
@pytest.mark.parametrize("kind", [BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,V", [(1024, 64, 20000), (1024, 65, 20000), (1024, 4096, 20000), (120, 512, 70000)])
def test_pieces_of_the_vocabulary_in_large_tiles(kind, n, D, V, before, monkeypatch):
    monkeypatch.setenv("HSADMM_LOSS_HELD", str(2 * 1024 * 8192))
    say("pieces", NAMES[kind], n, D, V)
    c = Case(kind, n, D, V, seed=6, pad=1, before=before)
    monkeypatch.delenv("HSADMM_LOSS_HELD")
    whole = Case(kind, n, D, V, seed=6, pad=1, before=before)
    assert (pkg.hsadmm_softmax_loss_workspace(c.plan, 1, n, kind, True) <
            pkg.hsadmm_softmax_loss_workspace(whole.plan, 1, n, kind, True))            # (it does take several)
    c.run().check()
