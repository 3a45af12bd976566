"""Sums of the weight gradient over many rows, where a bound that grows with the rows would hide a lost one.

Sums of whole numbers that stay below 2^24 are exact in fp32 in any order, so dW and db have to equal them bit for bit: every row, every tap, every share of a
CTA and every part of an fp32 dy counts.  For other values the error is bounded through the kernel's own order: an accumulator takes
32 stages of 64 rows (8 with three parts), cut by at most 2 u of the terms so far after each 16 rows, and is then added, rounded (u), to a share; shares of
CTAs are added, rounded."""
import numpy as np
import pytest
import torch

from paper_2512_15773_b200 import binding
from tests.test_gpu_train_ops import TYPES, U

pytestmark = pytest.mark.gpu

# by pairs of CTAs with ragged rows, channels and columns; many tiles a unit; few tiles for all CTAs; rows that TMA cannot take; many taps
SIZES = [(240, 64, 256, 264, 5), (600, 32, 1008, 300, 1), (26, 501, 880, 520, 1), (1, 38011, 512, 512, 1), (100, 10, 1024, 2048, 5),
         (1187, 16, 77, 51, 1), (601, 32, 40, 257, 1), (130, 77, 100, 72, 3), (40, 512, 256, 256, 1), (922, 16, 141, 541, 3), (4, 100, 1000, 24, 15),
         (3, 4099, 33, 130, 7), (20481, 1, 64, 64, 3)]


def integers(g, shape, most):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").float()


def of_definition(x, dy, taps, L):
    """dW [taps, K, O] and db in 64 bits."""
    xs, d = x.double().view(-1, L, x.shape[1]), dy.double().view(-1, L, dy.shape[1])
    out = []
    for tap in range(taps):
        o = tap - taps // 2
        lo, hi = max(0, -o), max(max(0, -o), min(L, L - o))
        out.append(xs[:, lo + o:hi + o].reshape(-1, x.shape[1]).T @ d[:, lo:hi].reshape(-1, dy.shape[1]))
    return torch.stack(out), dy.double().sum(0)


def of_kernel(x, dy, taps, L, ldy=None):
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    back = torch.empty_like(x, dtype=torch.float32)
    binding.checkpoint_unpack(saved, back)
    K, O = x.shape[1], dy.shape[1]
    dW, db = torch.full((taps, K, O), float("nan"), device="cuda"), torch.full((O,), float("nan"), device="cuda")
    ws = torch.full((binding.weight_grad_workspace(dy, K, taps, L),), 255, dtype=torch.uint8, device="cuda")
    binding.weight_grad(saved, dy, dW, ws, db=db, length=L)
    return dW, db, back


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,K,O,taps", SIZES)
def test_whole_numbers_add_up_exactly(N, L, K, O, taps, dtype):
    """|x|, |dy| <= 15: sums of 41 000 products stay below 2^24."""
    g = torch.Generator(device="cuda").manual_seed(N + L + K)
    x = integers(g, (N * L, K), 15).to(TYPES[dtype])
    dy = integers(g, (N * L, O), 15).to(TYPES[dtype])
    dW, db, back = of_kernel(x, dy, taps, L)
    assert torch.equal(back, x.float())                          # (the copy of such numbers is exact)
    rW, rb = of_definition(back, dy, taps, L)
    assert float(rW.abs().max()) < 2 ** 24 and N * L * 225 < 2 ** 24
    assert torch.equal(dW.double(), rW) and torch.equal(db.double(), rb)


@pytest.mark.parametrize("ldy", [520, 513, 527])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_whole_numbers_of_strided_rows_add_up_exactly(dtype, ldy):
    g = torch.Generator(device="cuda").manual_seed(ldy)
    x, wide = integers(g, (9001, 144), 15).to(TYPES[dtype]), integers(g, (9001, ldy), 15).to(TYPES[dtype])
    dy = wide[:, 1:513] if ldy == 527 else wide[:, :512]
    dW, db, back = of_kernel(x, dy, 3, 9001)
    rW, rb = of_definition(back, dy, 3, 9001)
    assert torch.equal(dW.double(), rW) and torch.equal(db.double(), rb)


@pytest.mark.parametrize("N,L,K,O,taps", [(1, 38011, 512, 512, 1), (922, 16, 141, 541, 3), (240, 64, 256, 264, 5), (601, 32, 40, 257, 1)])
def test_every_part_of_an_fp32_row_counts(N, L, K, O, taps):
    """dy of 20 significant bits, three bf16 parts: whole numbers below 2^20, odd ones, against an x with at most 15 ones in a column."""
    g = torch.Generator(device="cuda").manual_seed(K)
    rows = N * L
    x = torch.zeros(rows, K, device="cuda")
    at = torch.randint(0, rows, (15, K), generator=g, device="cuda")
    x.scatter_(0, at, torch.ones(15, K, device="cuda"))
    x[rows - 1] = 1.0
    x[0] = 1.0                                                   # (17 in all; that their terms stay below 2^24 is asserted)
    dy = 2 * torch.randint(-2 ** 18, 2 ** 18, (rows, O), generator=g, device="cuda").float() + 1
    dW, _, back = of_kernel(x, dy, taps, L)
    rW, _ = of_definition(back, dy, taps, L)
    terms, _ = of_definition(back, dy.abs(), taps, L)
    assert float(terms.max()) < 2 ** 24
    assert torch.equal(dW.double(), rW)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,K,O,taps", SIZES)
def test_sums_of_many_rows_keep_their_digits(N, L, K, O, taps, dtype):
    g = torch.Generator(device="cuda").manual_seed(N * L + O)
    x = torch.randn(N * L, K, generator=g, device="cuda").add_(0.3).to(TYPES["bf16"])
    dy = torch.randn(N * L, O, generator=g, device="cuda").add_(0.1).to(TYPES[dtype])
    dW, db, back = of_kernel(x, dy, taps, L)
    rW, rb = of_definition(back, dy, taps, L)
    aW, ab = of_definition(back.abs(), dy.abs(), taps, L)
    stages, chunk, parts = -(-N * L // 64), 32 if dtype == "bf16" else 8, 1 if dtype == "bf16" else 3
    in_one = 4 * parts * min(chunk, stages)                      # cuts of an accumulator, each of at most 2 u of the terms in it
    roundings = -(-stages // chunk) + 148 + 8                    # of a share, of the joining of shares
    assert ((dW.double() - rW).abs() <= (2 * in_one + roundings) * U * aW + 1e-30).all()
    # db: 64 rows of a stage (of three parts) in up to 16 rows a thread, its stages one after the other, then 128 threads' shares and those of CTAs
    assert ((db.double() - rb).abs() <= (16 * parts + stages + 148 + 256) * U * ab + 1e-30).all()


def test_an_accumulator_does_not_take_all_rows():
    """Values of one sign: what the tensor core cuts off goes all to one side, 4e-9 of the sum a step of 16 rows.  Within 32 stages that adds up to 128 / 2 of
    it on average, 2.6e-7, and the additions of the 19 accumulators to their shares are off by 19 u = 1.1e-6 at most, of the shares by 16 u more;
    over all 2376 steps it would be 4.7e-6 and more."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.rand(38011, 512, generator=g, device="cuda").add_(0.5).to(torch.bfloat16)
    dy = torch.rand(38011, 512, generator=g, device="cuda").add_(0.5).to(torch.bfloat16)
    dW, _, back = of_kernel(x, dy, 1, 38011)
    rW, _ = of_definition(back, dy, 1, 38011)
    assert float((dW.double() / rW - 1).abs().max()) < 2.6e-7 * 2 + 35 * U
