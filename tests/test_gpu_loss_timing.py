"""The diagnostics tell the loss's launches apart: rows listed and copied by one launch, by two, and copies of the weights."""
import pytest
import torch

import paper_2512_14628_amd as pkg
from tests.test_gpu_loss import BF16, F32, NAMES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("n,D,want", [(10, 64, {"loss_few": 1}), (10, 63, {"loss_few": 1, "loss_rows": 1}), (2049, 64, {"loss_targets": 1, "loss_rows": 1}),
                                      (2049, 63, {"loss_targets": 1, "loss_rows": 2})])
def test_launches_by_their_names(kind, n, D, want):
    c = Case(kind, n, D, 30, seed=1, before=16)              # (a layer that begins at a whole piece of 16 bytes in either type)
    pkg.hsadmm_kernel_timing_enable(c.plan, True)
    c.run()
    seen = {name: launches for name, (_, launches) in pkg.hsadmm_kernel_timing_read(c.plan).items() if launches}
    listing = {k: v for k, v in seen.items() if k in ("loss_few", "loss_targets", "loss_rows")}
    assert listing == want and seen["loss_softmax"] == 1 and seen["loss_inputs"] == 1 and seen["loss_weight_gradients"] == 1
