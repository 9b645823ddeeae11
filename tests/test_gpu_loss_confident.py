"""The loss of a row whose label has nearly all of the softmax, and of logits far from zero: log(sum exp(l)) - l_label, of which the largest
logit cancels.  The logits here are exact in fp32 (32768 and 32768 minus a few units, products and sums of powers of two), so nothing
but the sum of exponentials is rounded.

Bound.  exp: the difference is exact, its product with log2 e rounds (|t| U in the exponent), the instruction adds 2 U; the sum: a term
passes at most 64 + V / 64 + 32 additions (a lane's part of a slab, a row's slabs or classes shared by 64 threads or more, the joins); the
logarithm 4 U of itself.  The step of fp32 at 32768 is 2^-8."""
import pytest
import torch

from tests import ref_tokens as ref
from tests.test_gpu_loss import BF16, DEV, F16, F32, NAMES, Case, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [F32, BF16, F16], ids=NAMES.get)
@pytest.mark.parametrize("n,V,held", [(1, 300, None), (5, 300, None), (40, 1000, None), (300, 700, None), (1, 40000, None), (100, 20000, None),
                                      (300, 20000, None), (5, 1000, "1"), (300, 1000, "1")])
def test_the_largest_logit_cancels(kind, n, V, held, monkeypatch):
    if held:
        monkeypatch.setenv("HSADMM_LOSS_HELD", held)
    say("confident", NAMES[kind], n, V, held)
    c = Case(kind, n, 8, V, seed=1, share=0.0, before=16 if n % 2 else 12)
    gap = torch.tensor([8.0, 10.0, 12.0, 14.0])[torch.arange(n) % 4].double().to(DEV)
    top = V // 3
    w, x = torch.zeros((V, 8)), torch.zeros((n, 8))
    w[:, 0], w[:, 1] = 32768.0, -2.0
    w[top, 1] = 0.0
    x[:, 0], x[:, 1] = 1.0, gap.cpu().float() / 2
    c.layer(c.W).copy_(w.to(ref.TYPES[kind]))
    c.X.copy_(x.to(ref.TYPES[kind]))
    c.labels.fill_(top)
    c.labels[n // 2:] = top if n == 1 else V - 1             # (half the rows have a label that is not the largest)
    rest = (V - 1) * torch.exp(-gap)
    value = torch.log1p(rest) + torch.where(c.labels == top, 0.0, gap)
    bound = ref.SAFE * ((64 + V / 64 + 32) * ref.U + rest / (1 + rest) * (gap + 2) * ref.U + 4 * ref.U * torch.log1p(rest) + ref.U * value)
    c.run(outputs=("loss", "lse", "total"))
    ref.close(c.loss[:n], value, bound, "loss")
    ref.close(c.lse[:n], 32768 + torch.log1p(rest), bound + 2.0 ** -9, "lse")
    ref.close(c.total[0], value.mean(), bound.max() + 2 * ref.U * value.mean(), "total")
