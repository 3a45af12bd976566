"""Waits inside the training operators' kernels that run out: what a CTA could not work on is NaN in every output that it had to write, the rest is as ever,
and the next call works.  The wait is made to run out by withholding data from one CTA; its limit is a millisecond."""
import time

import pytest
import torch

from paper_2512_15773_b200 import binding
from tests.test_gpu_train_ops import weight_case

pytestmark = pytest.mark.gpu
MS = 2_000_000                               # SM clock cycles


def lost_and_kept(call):
    """Outputs of a call whose first CTA is left waiting, and of the calls before and after it."""
    before = call()
    torch.cuda.synchronize()
    binding.arm_train_timeout(MS)
    t0 = time.perf_counter()
    lost = call()
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 5.0
    after = call()
    torch.cuda.synchronize()
    for a, b in zip(before, after):
        assert torch.equal(a, b) and torch.isfinite(a.float()).all()
    return lost, before


# dy by TMA; pairs of CTAs; rows on odd addresses; fp32.  One tap: the first CTA's tile is one that the bias gradient is taken from.
@pytest.mark.parametrize("N,L,K,O,dtype,ldy", [(1, 1001, 512, 200, "bf16", None), (1, 38011, 512, 512, "bf16", None), (64, 16, 256, 130, "bf16", 131),
                                               (300, 16, 128, 300, "fp32", None)])
def test_weight_gradient_marks_what_it_lost(N, L, K, O, dtype, ldy):
    saved, dy = weight_case(N, L, K, O, 1, dtype, 3, ldy)

    def call():
        dW, db = torch.zeros(1, K, O, device="cuda"), torch.zeros(O, device="cuda")
        ws = torch.zeros(binding.weight_grad_workspace(dy, K, 1, L), dtype=torch.uint8, device="cuda")      # (stale words would count as zeros)
        binding.weight_grad(saved, dy, dW, ws, db=db, length=L)
        return dW, db
    (dW, db), (want, want_db) = lost_and_kept(call)
    bad, bad_db = torch.isnan(dW[0]), torch.isnan(db)
    assert bad.any() and torch.equal(dW[0][~bad], want[0][~bad])
    assert bad_db.any() and torch.equal(db[~bad_db], want_db[~bad_db])
    assert bad[0].any() and (bad[0] & ~bad_db).sum() == 0          # the first CTA's tile begins at the first column: both are marked there


def test_the_limit_has_a_range():
    for n in (0, 999, 2_000_000_001):
        with pytest.raises(binding.TsdpError):
            binding.arm_train_timeout(n)
