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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
# (501 sequences of 6 x 80: the gradient of their bf16 groups takes the stream form, which has no such wait)
@pytest.mark.parametrize("N,L,C,G,films", [(301, 8, 512, 1, True), (1001, 12, 640, 2, True), (501, 6, 80, 2, False), (2003, 6, 80, 2, True)])
def test_group_norm_marks_what_it_lost(N, L, C, G, films, dtype):
    """A CTA that holds groups: the sequences that it walks (not all of them) are marked whole, in y, the statistics, dx and dfilm; dgamma and dbeta, to
    which each CTA gives a share of every channel that it has, in all of those."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dy, ga, be = rand(N, L, C).to(dtype), rand(N, L, C).to(dtype), 1 + 0.1 * rand(C), rand(C)
    film = 1 + 0.1 * rand(N, 2 * C) if films else None
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    ws = torch.zeros(binding.group_norm_grad_workspace(dy, G), dtype=torch.uint8, device="cuda")

    def norm():
        y, mean, rstd = torch.zeros_like(x), torch.zeros(N, G, device="cuda"), torch.zeros(N, G, device="cuda")
        binding.group_norm(x, ga, be, G, y, film=film, mean=mean, rstd=rstd)
        return y, mean, rstd

    def grad(copy):
        ws.zero_()
        dx, dga, dbe = torch.zeros_like(x), torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda")
        dfi = torch.zeros(N, 2 * C, device="cuda") if films else torch.zeros(N, 0, device="cuda")
        binding.group_norm_grad(dy, None if copy else x, ga, be, G, *good, dx, dga, dbe, ws, film=film, dfilm=dfi if films else None, saved_x=saved if copy else None)
        return dx, dga, dbe, dfi

    def sequences(got, want):
        bad = torch.isnan(got.float()).reshape(N, -1)
        assert torch.equal(got.reshape(N, -1)[~bad], want.reshape(N, -1)[~bad])
        return bad
    (y, mean, rstd), (wy, wm, wr) = lost_and_kept(norm)
    good = tuple(t.clone() for t in (wm, wr))
    bad = sequences(y, wy)
    seqs = bad.any(1)
    assert 0 < seqs.sum() < N and seqs[0]
    groups = bad.view(N, L, G, C // G)
    of_group = groups.all(3).all(1)
    assert torch.equal(groups.any(3).any(1), of_group)                      # a group is lost whole or not at all
    for t, w in ((mean, wm), (rstd, wr)):
        assert torch.equal(sequences(t, w), of_group)
    for copy in (False, True):
        if copy and C % 16:
            continue
        (dx, dga, dbe, dfi), (wx, wg, wb, wf) = lost_and_kept(lambda: grad(copy))
        bad = sequences(dx, wx).view(N, L, G, C // G)
        of_group = bad.all(3).all(1)
        assert (N == 501 or 0 < of_group.sum()) and of_group.sum() < N * G and torch.equal(bad.any(3).any(1), of_group)
        lost = of_group.any(0).repeat_interleave(C // G)
        for t, w in ((dga, wg), (dbe, wb)):
            assert torch.equal(torch.isnan(t), lost) and torch.equal(t[~lost], w[~lost])
        if films:
            wide = of_group.repeat_interleave(C // G, 1)
            assert torch.equal(sequences(dfi, wf), torch.cat([wide, wide], 1))
