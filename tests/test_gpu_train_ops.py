"""The operators of a training step against their 64-bit definitions (oracle/train.py).

Tolerances.  u = 2^-24 is the largest relative error of one fp32 operation, half = finfo(type).eps / 2 that of rounding a result to its
type.  A sum of n fp32 terms taken in an order of depth k is off by at most k u sum |terms|; no sum here is deeper than DEPTH: a lane
adds every (rows / lanes)-th value one after the other (at most 64 in these tests, asserted through the sizes below), then lanes, warps, CTAs.
The exponential is off by 2 units and by the rounding of z log2(e): (2 + 2 |z|) u, 1.4 |z| of it through the rounded product."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2512_15773_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEPTH = 160
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def half(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def rng_tensor(rng, shape, dtype, offset=0.5, scale=1.0):
    t = torch.tensor(rng.normal(size=shape) * scale + offset, dtype=torch.float32).to(TYPES[dtype])
    return t.cuda()


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def strided(shape, dtype, layout):
    """A tensor [N, L, C] of this layout and the buffer it lies in."""
    N, L, C = shape
    if layout == "dense":
        buf = torch.zeros(N, L, C, dtype=TYPES[dtype], device="cuda")
        return buf, buf
    if layout == "padded":                     # two zero rows before and after the sequence
        buf = torch.zeros(N, L + 4, C, dtype=TYPES[dtype], device="cuda")
        return buf[:, 2:2 + L], buf
    if layout == "slice":                      # channels of a wider row, 16-byte pieces
        buf = torch.zeros(N, L, C + 16, dtype=TYPES[dtype], device="cuda")
        return buf[:, :, 8:8 + C], buf
    if layout == "odd":                        # rows on odd addresses
        buf = torch.zeros(N, L, C + 3, dtype=TYPES[dtype], device="cuda")
        return buf[:, :, 1:1 + C], buf
    buf = torch.zeros(L, N, C, dtype=TYPES[dtype], device="cuda")             # positions first
    return buf.transpose(0, 1), buf


# ------------------------------------------------------------------------------------------------ 8-bit copies
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,C", [(1, 1), (3, 31), (2, 32), (5, 33), (37, 100), (7, 256), (129, 40), (4, 2048), (3, 2056), (300, 8)])
def test_copies_are_exact(rows, C, dtype):
    rng = np.random.default_rng(rows * 1000 + C)
    x = torch.tensor(rng.normal(size=(rows, C)) * np.exp(3 * rng.normal(size=(rows, 1))), dtype=torch.float32)
    special = [0.0, -0.0, 127.5, -127.5, 127.4, 126.5, 2.0 ** -130, -2.0 ** -149, 3.38e38, -3.38e38, 1e-30]
    for i, v in enumerate(special):
        if i < rows and rows > 4:
            x[i, rng.integers(C)] = v
    if rows > 20:
        x[11] = 0.0
        x[12] *= 2.0 ** -126
        x[13, C // 2], x[14, 0], x[15, C - 1] = float("inf"), float("nan"), float("-inf")
        x[16, :] = 3.4e38 if dtype == "fp32" else 3.38e38
    x = x.to(TYPES[dtype]).cuda()
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    q, s = train.pack(host(x))
    assert np.array_equal(saved[1].cpu().numpy(), s)
    assert np.array_equal(saved[0].cpu().numpy(), q)
    for t in TYPES:
        back = torch.empty_like(x, dtype=TYPES[t])
        binding.checkpoint_unpack(saved, back)
        assert np.array_equal(host(back), train.unpack(q, s), equal_nan=True)


@pytest.mark.parametrize("layout", ["padded", "slice", "odd", "positions first"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_copies_of_strided_tensors(layout, dtype):
    rng = np.random.default_rng(7)
    x, buf = strided((3, 5, 48), dtype, layout)
    buf.fill_(7.0)
    x.copy_(rng_tensor(rng, (3, 5, 48), dtype))
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    q, s = train.pack(host(x).reshape(15, 48))
    assert np.array_equal(saved[0].cpu().numpy().reshape(15, 48), q) and np.array_equal(saved[1].cpu().numpy().reshape(15, 2), s)
    before = buf.clone()
    keep = x.clone()
    x.zero_()
    binding.checkpoint_unpack(saved, x)
    assert np.array_equal(host(x).reshape(15, 48), train.unpack(q, s))
    x.copy_(keep)
    assert torch.equal(buf, before)            # nothing between the rows was written


# ------------------------------------------------------------------------------------------------ GroupNorm
def norm_inputs(N, L, C, G, dtype, film, seed, layout="dense", offset=0.5):
    rng = np.random.default_rng(seed)
    x, _ = strided((N, L, C), dtype, layout)
    x.copy_(rng_tensor(rng, (N, L, C), dtype, offset) * torch.exp(0.3 * rng_tensor(rng, (C,), "fp32", 0)).to(TYPES[dtype]))
    ga, be = rng_tensor(rng, (C,), "fp32", 1, 0.2), rng_tensor(rng, (C,), "fp32", 0, 0.2)
    fi = None
    if film:
        fi = rng_tensor(rng, (N, 2 * C), "fp32", 0, 0.3)
        fi[:, :C] += 1
    return rng, x, ga, be, fi


# sizes: single values, one position, UNet levels, odd widths, groups wider than a CTA's threads, long sequences over several CTAs
NORM_SIZES = [(1, 1, 8, 1), (2, 1, 5, 5), (3, 7, 6, 3), (1, 16, 256, 8), (5, 16, 512, 8), (2, 4, 1024, 8), (3, 33, 40, 4), (2, 50, 1024, 1),
              (2, 700, 320, 32), (1, 1500, 64, 8), (1, 2500, 77, 7), (2, 9, 2048, 1), (3, 5, 2049, 3), (1, 3, 2000, 2), (40, 8, 96, 32), (700, 16, 64, 8),
              (3, 50, 256, 2), (2, 100, 64, 2), (2, 33, 128, 2), (1, 17, 1024, 16)]


def norm_bound(dtype, x, y, mean, rstd, ga, fi, N, C, G):
    """|h| <= hmax.  mean: off by DEPTH u max|x - pivot| + u |mean|, rstd by a relative DEPTH u; h by their sum; z by gamma times that and
    two roundings; act has a slope of at most 1.1 and an error of (2 + 2 |z|) u |a| + 4 u |a| of its own; FiLM two more roundings."""
    w = C // G
    xg = np.abs(host(x)).reshape(N, -1, G, w).max(axis=(1, 3))
    hmax = np.abs((host(x).reshape(N, -1, G, w) - mean[:, None, :, None]) * rstd[:, None, :, None]).max(axis=(1, 3))
    dh = (DEPTH * U * 2 * xg) * rstd + hmax * (DEPTH + 3) * U                     # [N, G]
    dz = np.repeat(dh, w, axis=1)[:, None, :] * np.abs(host(ga)) + 2 * U * (np.repeat(hmax, w, axis=1)[:, None, :] * np.abs(host(ga)) + 1)
    zmax = np.repeat(hmax, w, axis=1)[:, None, :] * np.abs(host(ga)) + 1
    da = 1.2 * dz + (8 + 3 * np.minimum(zmax, 24)) * U * zmax
    scale = 1.0 if fi is None else np.abs(host(fi))[:, None, :C]
    return da * scale + 3 * U * np.abs(y) + (half(dtype) * np.abs(y) * (1 + 4 * U) if dtype != "fp32" else 0) + 3 * U


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act,film", [("mish", True), ("silu", False), ("gelu", True), ("none", False)])
@pytest.mark.parametrize("N,L,C,G", NORM_SIZES)
def test_norm(N, L, C, G, act, film, dtype):
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, dtype, film, L * C + N)
    y = torch.full_like(x, float("nan"))
    mean, rstd = torch.full((N, G), float("nan"), device="cuda"), torch.full((N, G), float("nan"), device="cuda")
    binding.group_norm(x, ga, be, G, y, act=act, film=fi, mean=mean, rstd=rstd)
    ry, rm, rr = train.group_norm(host(x), host(ga), host(be), G, act, None if fi is None else host(fi))
    xmax = np.abs(host(x)).max()
    assert np.max(np.abs(host(mean) - rm)) <= DEPTH * U * 2 * xmax
    # the variance is off by DEPTH u of itself and by the square of the mean's error; eps keeps rstd below 1 / sqrt(eps)
    assert np.max(np.abs(host(rstd) / rr - 1)) <= (DEPTH + 4) * U + 0.5 * (DEPTH * U * 2 * xmax) ** 2 * np.max(rr) ** 2
    assert (np.abs(host(y) - ry) <= norm_bound(dtype, x, ry, rm, rr, ga, fi, N, C, G)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,C,G", [(2, 16, 256, 8), (3, 5, 40, 4), (2, 7, 77, 7), (1, 900, 96, 3), (2, 3, 2000, 2), (30, 16, 64, 8),
                                     (3, 41, 128, 2)])
def test_norm_saves_copies_of_its_input_and_output(N, L, C, G, dtype):
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, dtype, True, 11 * C)
    y, plain = torch.empty_like(x), torch.empty_like(x)
    sx, sy = binding.saved_like(x), binding.saved_like(x)
    binding.group_norm(x, ga, be, G, y, film=fi, saved_x=sx, saved_y=sy)
    binding.group_norm(x, ga, be, G, plain, film=fi)
    for t, saved in ((x, sx), (y, sy)):
        want = binding.saved_like(t)
        binding.checkpoint_pack(t, want)
        assert torch.equal(saved[0], want[0]) and torch.equal(saved[1], want[1])
    only = binding.saved_like(x)
    binding.group_norm(x, ga, be, G, x, film=fi, saved_x=only)           # in place: the copy is still that of the input
    assert torch.equal(only[0], sx[0]) and torch.equal(only[1], sx[1]) and torch.equal(x, y)
    assert np.max(np.abs(host(plain) - host(y))) <= 2 * half(dtype) * np.max(np.abs(host(y))) + 1e-5


@pytest.mark.parametrize("layout", ["padded", "slice", "odd", "positions first"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norm_and_gradient_on_strided_tensors(layout, dtype):
    N, L, C, G = 3, 16, 64, 8
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, dtype, True, 5, layout)
    dense = x.contiguous()
    y, buf = strided((N, L, C), dtype, layout)
    buf.fill_(7.0)
    outside = buf.clone()
    mean, rstd = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    binding.group_norm(x, ga, be, G, y, film=fi, mean=mean, rstd=rstd)
    ry, rm, rr = train.group_norm(host(dense), host(ga), host(be), G, "mish", host(fi))
    assert (np.abs(host(y) - ry) <= norm_bound(dtype, dense, ry, rm, rr, ga, fi, N, C, G)).all()
    dy, _ = strided((N, L, C), dtype, layout)
    dy.copy_(rng_tensor(rng, (N, L, C), dtype, 0))
    dx, dbuf = strided((N, L, C), dtype, layout)
    dbuf.fill_(7.0)
    check_gradient(dy, x, None, ga, be, G, mean, rstd, "mish", fi, dtype, dx)
    for t, b in ((y, buf), (dx, dbuf)):
        t.fill_(7.0)
        assert torch.equal(b, outside)


def check_gradient(dy, x, saved, ga, be, G, mean, rstd, act, fi, dtype, dx=None):
    N, L, C = dy.shape
    w = C // G
    dx = torch.full_like(dy, float("nan")) if dx is None else dx
    assert L <= 4096 and N <= 4096                    # (what DEPTH stands for)
    dga, dbe = torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    dfi = None if fi is None else torch.full((N, 2 * C), float("nan"), device="cuda")
    ws = torch.empty(binding.group_norm_grad_workspace(dy, G), dtype=torch.uint8, device="cuda")
    binding.group_norm_grad(dy, x, ga, be, G, mean, rstd, dx, dga, dbe, ws, act=act, film=fi, dfilm=dfi, saved_x=saved)
    xs = host(x) if x is not None else train.unpack(saved[0].cpu().numpy().reshape(N * L, C), saved[1].cpu().numpy().reshape(N * L, -1)).reshape(N, L, C)
    m, r = host(mean), host(rstd)
    rdx, rga, rbe, rfi = train.group_norm_grad(host(dy), xs, host(ga), host(be), G, m, r, act, None if fi is None else host(fi))
    # Bounds.  h is off by 3 u |h| + u |x| rstd (the subtraction is exact in relative terms but for its own rounding), z by gamma times that
    # and 2 u |z|; act' has a slope of at most 1.2 in z and an error of its own of (10 + 3 |z|) u; so dz is off by e_dz |dy scale|.
    wide = lambda t: np.repeat(t, w, axis=1)[:, None, :]  # noqa: E731
    h = (xs - wide(m)) * wide(r)
    e_h = 4 * U * (np.abs(h) + np.abs(xs) * wide(r) * 0.5)
    z = np.abs(h * host(ga)) + np.abs(host(be))
    e_z = e_h * np.abs(host(ga)) + 3 * U * z
    sc = 1.0 if fi is None else np.abs(host(fi))[:, None, :C]
    a, da = train.act(act, h * host(ga) + host(be))
    g = np.abs(host(dy)) * sc
    e_dz = g * (1.2 * e_z + (12 + 3 * np.minimum(z, 24)) * U * (1 + z * 0.3))
    dz = g * np.abs(da)
    depth = (DEPTH + 16) * U                                                     # of a sum over positions, lanes, CTAs, sequences
    assert (np.abs(host(dbe) - rbe) <= (e_dz + depth * dz).sum((0, 1)) + 1e-30).all()
    assert (np.abs(host(dga) - rga) <= (e_dz * np.abs(h) + dz * e_h + depth * dz * np.abs(h)).sum((0, 1)) + 1e-30).all()
    if fi is not None:
        ady = np.abs(host(dy))
        e_a = 1.2 * e_z + (12 + 3 * np.minimum(z, 24)) * U * z
        assert (np.abs(host(dfi)[:, :C] - rfi[:, :C]) <= (ady * e_a + depth * ady * np.abs(a)).sum(1) + 1e-30).all()
        assert (np.abs(host(dfi)[:, C:] - rfi[:, C:]) <= (depth * ady).sum(1) + 1e-30).all()
    gam = np.abs(host(ga))
    of_group = lambda t: wide(t.reshape(N, L, G, w).mean(axis=(1, 3)))  # noqa: E731
    e_m1 = of_group((e_dz + (depth + 40 * U) * dz) * gam)
    e_m2 = of_group((e_dz * np.abs(h) + dz * e_h + (depth + 40 * U) * dz * np.abs(h)) * gam)
    m1, m2 = of_group(dz * gam), of_group(dz * np.abs(h) * gam)
    e_dx = wide(r) * (e_dz * gam + e_m1 + np.abs(h) * e_m2 + e_h * m2 + 6 * U * (dz * gam + m1 + np.abs(h) * m2))
    assert (np.abs(host(dx) - rdx) <= e_dx + (half(dtype) * np.abs(rdx) * 1.01 if dtype != "fp32" else 0) + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("act,film", [("mish", True), ("silu", False), ("gelu", True), ("none", False)])
@pytest.mark.parametrize("N,L,C,G", NORM_SIZES)
def test_norm_gradient(N, L, C, G, act, film, saved, dtype):
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, dtype, film, L * C + N + 1)
    dy = rng_tensor(rng, (N, L, C), dtype, 0.1)
    _, m, r = train.group_norm(host(x), host(ga), host(be), G, act)
    mean, rstd = (torch.tensor(t, dtype=torch.float32, device="cuda") for t in (m, r))
    s = None
    if saved:
        s = binding.saved_like(x)
        binding.checkpoint_pack(x, s)
    check_gradient(dy, None if saved else x, s, ga, be, G, mean, rstd, act, fi, dtype)


# More sequences than a CTA, a warp or a cluster takes at once: each walks over several (a warp per group; a CTA per set of groups; clusters over
# long sequences), an uneven number of them.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,C,G", [(3001, 4, 256, 8), (901, 50, 128, 2), (2001, 16, 96, 4), (701, 600, 16, 2)])
def test_walks_over_many_sequences(N, L, C, G, dtype):
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, dtype, True, N)
    y, mean, rstd = torch.full_like(x, float("nan")), torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    sx, sy = binding.saved_like(x), binding.saved_like(x)
    binding.group_norm(x, ga, be, G, y, film=fi, mean=mean, rstd=rstd, saved_x=sx, saved_y=sy)
    ry, rm, rr = train.group_norm(host(x), host(ga), host(be), G, "mish", host(fi))
    assert (np.abs(host(y) - ry) <= norm_bound(dtype, x, ry, rm, rr, ga, fi, N, C, G)).all()
    for t, s in ((x, sx), (y, sy)):
        want = binding.saved_like(t)
        binding.checkpoint_pack(t, want)
        assert torch.equal(s[0], want[0]) and torch.equal(s[1], want[1])
    dy = rng_tensor(rng, (N, L, C), dtype, 0.1)
    check_gradient(dy, x, None, ga, be, G, mean, rstd, "mish", fi, dtype)
    check_gradient(dy, None, sx, ga, be, G, mean, rstd, "mish", fi, dtype)


# Sets of groups in a CTA: whole dense rows of many short sequences, sets of 512 bytes and more of a row, groups wider than a warp takes.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,C,G", [(1901, 2, 128, 16), (1803, 16, 512, 32), (7, 8, 512, 1), (33, 12, 640, 2), (1301, 5, 640, 8), (37, 3, 1024, 1),
                                     (2003, 1, 96, 6)])
def test_sets_of_groups(N, L, C, G, dtype):
    test_walks_over_many_sequences(N, L, C, G, dtype)


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_sets_of_groups_on_strided_rows(saved, dtype):
    N, L, C, G = 31, 6, 640, 2
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, dtype, True, 77)
    dy = rng_tensor(rng, (N, L, C), dtype, 0.1)
    out = []
    for pad, shift in ((0, 0), (64, 32)):
        apart = [torch.full((N, L + 2 * (pad > 0), C + pad), 7.0, dtype=x.dtype, device="cuda") for _ in range(4)]
        rows = [t[:, :L, shift:shift + C] for t in apart]
        rows[0].copy_(x)
        rows[2].copy_(dy)
        mean, rstd = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
        keep = binding.saved_like(x) if saved else None
        binding.group_norm(rows[0], ga, be, G, rows[1], film=fi, mean=mean, rstd=rstd, saved_x=keep)
        dga, dbe, dfi = torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(N, 2 * C, device="cuda")
        ws = torch.empty(binding.group_norm_grad_workspace(rows[2], G), dtype=torch.uint8, device="cuda")
        binding.group_norm_grad(rows[2], None if saved else rows[0], ga, be, G, mean, rstd, rows[3], dga, dbe, ws, film=fi, dfilm=dfi, saved_x=keep)
        out.append([rows[1].clone(), rows[3].clone(), mean, rstd, dga, dbe, dfi])
        if pad:
            for t in (apart[1], apart[3]):
                t[:, :L, shift:shift + C] = 7.0
                assert (t == 7.0).all()                       # what lies between rows stays
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_offsets_past_32_bits():
    """Sequences and rows more than 2^32 bytes apart, in one buffer of 11 GB."""
    far, N, L, C, G = (1 << 31) + 24, 3, 16, 64, 2
    buf = torch.empty(2 * far + L * C + 64, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (N, L, C), (far, C, 1))
    rng = np.random.default_rng(2)
    x.copy_(rng_tensor(rng, (N, L, C), "bf16"))
    near = x.contiguous()
    ga, be = rng_tensor(rng, (C,), "fp32", 1, 0.2), rng_tensor(rng, (C,), "fp32", 0, 0.2)
    mean, rstd = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    sx, want = binding.saved_like(near), torch.empty_like(near)
    binding.group_norm(near, ga, be, G, want, mean=mean, rstd=rstd)
    y = torch.empty_like(near)
    binding.group_norm(x, ga, be, G, y, saved_x=sx)
    assert torch.equal(y, want)
    dx = [torch.empty_like(near) for _ in range(2)]
    dga, dbe = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(binding.group_norm_grad_workspace(near, G), dtype=torch.uint8, device="cuda")
    for t, o in ((near, dx[0]), (x, dx[1])):
        binding.group_norm_grad(t, t, ga, be, G, mean, rstd, o, dga, dbe, ws)
    assert torch.equal(*dx)
    x.zero_()
    binding.checkpoint_unpack(sx, x)
    back = torch.empty_like(near)
    binding.checkpoint_unpack(sx, back)
    assert torch.equal(x, back)
    rows = torch.as_strided(buf, (3, C), (far, 1))                  # rows of a weight gradient's dy
    rows.copy_(near[0, :3])
    saved = (sx[0].view(-1, C)[:3].contiguous(), sx[1].view(-1, 2)[:3].contiguous())
    check_weight(saved, rows, 1, 3)
    # long sequences (clusters), one value at a time
    wide = torch.as_strided(buf, (2, 300, 7), (far, 11, 1))
    wide.copy_(rng_tensor(rng, (2, 300, 7), "bf16"))
    tight = wide.contiguous()
    m, r = torch.empty(2, 7, device="cuda"), torch.empty(2, 7, device="cuda")
    a, b = torch.empty_like(tight), torch.empty_like(tight)
    binding.group_norm(tight, ga[:7], be[:7], 7, a, mean=m, rstd=r)
    binding.group_norm(wide, ga[:7], be[:7], 7, b)
    assert torch.equal(a, b)
    d1, d2, d3 = torch.empty(7, device="cuda"), torch.empty(7, device="cuda"), torch.empty_like(tight)
    ws = torch.empty(binding.group_norm_grad_workspace(tight, 7), dtype=torch.uint8, device="cuda")
    binding.group_norm_grad(tight, tight, ga[:7], be[:7], 7, m, r, a, d1, d2, ws)
    binding.group_norm_grad(wide, wide, ga[:7], be[:7], 7, m, r, d3, d1, d2, ws)
    assert torch.equal(a, d3)


def test_broadcast_inputs():
    """A dy of one position for all, an x of one sequence for all: strides of zero."""
    N, L, C, G = 4, 16, 64, 2
    rng, x, ga, be, _ = norm_inputs(N, L, C, G, "bf16", False, 6)
    one, dy = x[:1].expand(N, L, C), rng_tensor(rng, (1, 1, C), "bf16", 0).expand(N, L, C)
    mean, rstd = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    y, want = torch.empty(N, L, C, dtype=x.dtype, device="cuda"), torch.empty(N, L, C, dtype=x.dtype, device="cuda")
    binding.group_norm(one, ga, be, G, y, mean=mean, rstd=rstd)
    binding.group_norm(one.contiguous(), ga, be, G, want)
    assert torch.equal(y, want)
    check_gradient(dy, one, None, ga, be, G, mean, rstd, "mish", None, "bf16", torch.empty_like(y))
    saved = binding.saved_like(x.view(N * L, C))
    binding.checkpoint_pack(x.view(N * L, C), saved)
    check_weight(saved, dy[0, :1].expand(N * L, C), 3, L)


def test_gradients_in_place():
    for L, C, G in ((16, 256, 8), (16, 96, 4), (700, 20, 2)):        # a warp per group, a CTA per set, clusters
        rng, x, ga, be, fi = norm_inputs(3, L, C, G, "bf16", True, L)
        mean, rstd = torch.empty(3, G, device="cuda"), torch.empty(3, G, device="cuda")
        y = torch.empty_like(x)
        binding.group_norm(x, ga, be, G, y, film=fi, mean=mean, rstd=rstd)
        dy, dga, dbe = rng_tensor(rng, (3, L, C), "bf16", 0), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ws = torch.empty(binding.group_norm_grad_workspace(dy, G), dtype=torch.uint8, device="cuda")
        dx = torch.empty_like(dy)
        binding.group_norm_grad(dy, x, ga, be, G, mean, rstd, dx, dga, dbe, ws, film=fi)
        binding.group_norm_grad(dy, x, ga, be, G, mean, rstd, dy, dga, dbe, ws, film=fi)
        assert torch.equal(dx, dy)
        binding.group_norm(x, ga, be, G, x, film=fi)
        assert torch.equal(x, y)


def test_gradient_against_differences_of_the_kernel_itself():
    """fp32: (loss(x + d v) - loss(x - d v)) / 2 d against <dx, v>, the loss summed in 64 bits.  With d = 2^-7 the difference's own
    error is d^2 / 6 of a third derivative (of the order of |v|^3, here a few) and 2^-24 |y| sqrt(values) / d of rounding: 1e-3 of the sums."""
    N, L, C, G = 2, 16, 64, 8
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, "fp32", True, 21)
    dy, v = rng_tensor(rng, (N, L, C), "fp32", 0), rng_tensor(rng, (N, L, C), "fp32", 0)
    mean, rstd = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dga, dbe = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")

    def loss(t):
        binding.group_norm(t, ga, be, G, y, film=fi)
        return float((y.double() * dy.double()).sum())
    binding.group_norm(x, ga, be, G, y, film=fi, mean=mean, rstd=rstd)
    ws = torch.empty(binding.group_norm_grad_workspace(dy, G), dtype=torch.uint8, device="cuda")
    binding.group_norm_grad(dy, x, ga, be, G, mean, rstd, dx, dga, dbe, ws, film=fi)
    d = 2.0 ** -7
    num = (loss(x + d * v) - loss(x - d * v)) / (2 * d)
    size = float((dx.double().abs() * v.double().abs()).sum())
    assert abs(num - float((dx.double() * v.double()).sum())) <= 1e-3 * size


def test_values_that_are_not_finite_stay_in_their_group():
    N, L, C, G = 2, 16, 64, 8
    rng, x, ga, be, _ = norm_inputs(N, L, C, G, "fp32", False, 8)
    good = torch.empty_like(x)
    binding.group_norm(x, ga, be, G, good)
    x[1, 3, 17] = float("inf")
    x[0, 5, 63] = float("nan")
    y, saved = torch.empty_like(x), binding.saved_like(x)
    binding.group_norm(x, ga, be, G, y, saved_x=saved)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, :, 16:24] = True
    bad[0, :, 56:64] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], good[~bad])
    assert (saved[1][1, 3] == torch.tensor([255, saved[1][1, 3, 1]], device="cuda", dtype=torch.uint8)).all() and saved[1][0, 5, 1] == 255


def test_large_mean_costs_no_digits():
    """Values 1000 + small: the variance is that of the small part.  x itself is exact; its spread of 1 is held to u |x| = 6e-5."""
    N, L, C, G = 2, 600, 32, 4
    rng, x, ga, be, _ = norm_inputs(N, L, C, G, "fp32", False, 9, offset=1000.0)
    y, mean, rstd = torch.empty_like(x), torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    binding.group_norm(x, ga, be, G, y, act="none", mean=mean, rstd=rstd)
    ry, rm, rr = train.group_norm(host(x), host(ga), host(be), G, "none")
    # pivots are values of the channel: sums are of deviations, at most 8 of them wide; the mean itself is rounded to u 1000
    assert np.max(np.abs(host(rstd) / rr - 1)) <= 8 * DEPTH * U
    assert np.max(np.abs(host(y) - ry)) <= 2 * (2 * 1000 * U + 8 * DEPTH * U) * np.max(rr)


def test_empty_batches_and_refusals():
    e = torch.empty(0, 16, 64, device="cuda")
    ga = torch.ones(64, device="cuda")
    binding.group_norm(e, ga, ga, 8, e)
    dga, dbe = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    ws = torch.empty(binding.group_norm_grad_workspace(e, 8), dtype=torch.uint8, device="cuda")
    z = torch.empty(0, 8, device="cuda")
    binding.group_norm_grad(e, e, ga, ga, 8, z, z, e, dga, dbe, ws)
    assert not dga.any() and not dbe.any()
    r = torch.empty(0, 64, device="cuda")
    dW, db = torch.ones(64, 64, device="cuda"), torch.ones(64, device="cuda")
    wws = torch.empty(binding.weight_grad_workspace(r, 64), dtype=torch.uint8, device="cuda")
    binding.weight_grad(binding.saved_like(r), r, dW, wws, db=db)
    assert not dW.any() and not db.any()
    x = torch.zeros(2, 16, 64, device="cuda")
    with pytest.raises(ValueError):
        binding.group_norm(x, ga, ga, 8, x.bfloat16())
    with pytest.raises(ValueError):
        binding.group_norm(x, ga.bfloat16(), ga, 8, x)
    with pytest.raises(ValueError):
        binding.group_norm(x.transpose(1, 2), ga, ga, 8, x.transpose(1, 2))
    with pytest.raises(ValueError):
        binding.group_norm(x.half(), ga, ga, 8, x.half())
    with pytest.raises(ValueError):
        binding.group_norm_grad(x, None, ga, ga, 8, z, z, x, dga, dbe, ws)
    with pytest.raises(binding.TsdpError):
        binding.group_norm(x, ga, ga, 7, x)
    with pytest.raises(binding.TsdpError):            # workspace too small
        st = torch.zeros(2, 8, device="cuda")
        binding.group_norm_grad(x, x, ga, ga, 8, st, st, x, dga, dbe, ws[:16])
    with pytest.raises(binding.TsdpError):            # rows written over each other
        binding.group_norm(x, ga, ga, 8, x[:1].expand(2, 16, 64))


# ------------------------------------------------------------------------------------------------ weight gradient
def weight_case(N, L, K, O, taps, dtype, seed, ldy=None):
    rng = np.random.default_rng(seed)
    x = rng_tensor(rng, (N * L, K), "bf16", 0.3)
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    wide = torch.full((N * L, ldy or O), 3.0, dtype=TYPES[dtype], device="cuda")
    dy = wide[:, :O]
    dy.copy_(rng_tensor(rng, (N * L, O), dtype, 0.1))
    return saved, dy


def check_weight(saved, dy, taps, L, with_db=True, stream=0):
    rows, O = dy.shape
    K = saved[0].shape[1]
    dW = torch.full((taps, K, O), float("nan"), device="cuda")
    db = torch.full((O,), float("nan"), device="cuda") if with_db else None
    ws = torch.full((binding.weight_grad_workspace(dy, K, taps, L),), 255, dtype=torch.uint8, device="cuda")
    binding.weight_grad(saved, dy, dW, ws, db=db, length=L, stream=stream)
    x = train.unpack(saved[0].cpu().numpy(), saved[1].cpu().numpy())
    rW, rb = train.weight_grad(x, host(dy), taps, L)
    aW, ab = train.weight_grad(np.abs(x), np.abs(host(dy)), taps, L)
    # products are exact; an accumulator takes 16 rows (three times where dy comes in three parts) per step and may cut a result where the
    # definition rounds it, 2 u of the running sum each; shares of CTAs are added in at most 148 steps, each half of that
    steps = 3 * (rows / 16 + 4) + 148
    assert (np.abs(host(dW) - rW) <= 2 * U * steps * aW + 1e-30).all()
    if with_db:
        assert (np.abs(host(db) - rb) <= U * (rows / 512 + 80) * ab + 1e-30).all()
    return dW, db


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,K,O,taps", [(1, 64, 128, 64, 1), (1, 64, 128, 128, 1), (1, 128, 128, 256, 1), (1, 1, 1, 1, 1), (1, 17, 32, 8, 1),
                                          (3, 16, 128, 512, 1), (7, 143, 77, 130, 3), (5, 4, 48, 72, 5), (9, 16, 256, 264, 5), (2, 3, 130, 100, 7),
                                          (1, 1001, 512, 200, 1), (33, 16, 300, 65, 3), (300, 1, 64, 64, 3), (4, 100, 1000, 24, 15)])
def test_weight_gradient(N, L, K, O, taps, dtype):
    saved, dy = weight_case(N, L, K, O, taps, dtype, N * L + K)
    check_weight(saved, dy, taps, L)


# Large enough for pairs of CTAs (148 SMs: 2368 steps of 64 rows over 256 x 256 tiles), with ragged rows, channels and columns; many
# tiles a unit; several roundings of one accumulator.
@pytest.mark.parametrize("N,L,K,O,taps", [(240, 64, 256, 264, 5), (600, 32, 1008, 300, 1), (26, 501, 880, 520, 1), (1, 38011, 512, 512, 1),
                                          (100, 10, 1024, 2048, 5)])
def test_weight_gradient_by_pairs(N, L, K, O, taps):
    saved, dy = weight_case(N, L, K, O, taps, "bf16", N * L + K)
    check_weight(saved, dy, taps, L)


# Many rows over few tiles: 8 to 148 CTAs (or pairs) share a tile, whose sums groups of the joining threads take side by side.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,L,K,O,taps", [(400, 16, 200, 130, 1), (1187, 16, 77, 51, 1), (601, 32, 40, 257, 1), (130, 77, 100, 72, 3),
                                          (64, 16, 256, 256, 5), (40, 512, 256, 256, 1)])
def test_weight_gradient_of_few_tiles(N, L, K, O, taps, dtype):
    saved, dy = weight_case(N, L, K, O, taps, dtype, N * L + K)
    check_weight(saved, dy, taps, L)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("O,ldy", [(128, 136), (128, 131), (100, 104), (256, 1024)])
def test_weight_gradient_of_strided_rows(O, ldy, dtype):
    saved, dy = weight_case(6, 16, 96, O, 3, dtype, ldy, ldy)
    check_weight(saved, dy, 3, 16)
    check_weight(saved, dy, 3, 16, with_db=False)


def test_weight_gradient_takes_the_order_of_its_sums_from_the_sizes_alone():
    saved, dy = weight_case(64, 16, 256, 512, 1, "bf16", 1)
    a, da = check_weight(saved, dy, 1, 16)
    for _ in range(3):
        b, db = check_weight(saved, dy, 1, 16)
        assert torch.equal(a, b) and torch.equal(da, db)


def test_weight_gradient_of_fp32_rows_is_that_of_fp32():
    """dy with 24 significant bits, one row: each entry is one product, exact but for its rounding to fp32."""
    x = torch.arange(-100, 101, dtype=torch.float32, device="cuda")[None, :]
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    dy = (1 + torch.arange(64, device="cuda") * 2.0 ** -23).float()[None, :] * 1.2345678
    dW = torch.empty(201, 64, device="cuda")
    ws = torch.empty(binding.weight_grad_workspace(dy, 201), dtype=torch.uint8, device="cuda")
    binding.weight_grad(saved, dy, dW, ws)
    want = train.unpack(saved[0].cpu().numpy(), saved[1].cpu().numpy()).T @ host(dy)
    assert (np.abs(host(dW) - want) <= 3 * 2 * U * np.abs(want)).all()       # three additions, cut or rounded


def test_blocks_that_are_not_finite_reach_their_own_rows_of_the_gradient():
    saved, dy = weight_case(2, 32, 96, 64, 1, "bf16", 4)
    dW, _ = check_weight(saved, dy, 1, 64)
    saved[1][5, 1] = 255
    got = torch.empty_like(dW)
    ws = torch.empty(binding.weight_grad_workspace(dy, 96, 1, 64), dtype=torch.uint8, device="cuda")
    binding.weight_grad(saved, dy, got, ws, length=64)
    assert torch.isnan(got[:, 32:64]).all() and torch.equal(got[:, :32], dW[:, :32]) and torch.equal(got[:, 64:], dW[:, 64:])


# ------------------------------------------------------------------------------------------------ together
def _block(rows_x, W, b, ga, be, G, N, L, smp, ws, state):
    """projection -> GroupNorm + Mish, what the backward pass needs kept in eight bits; mean-square loss against state['goal']."""
    C = W.shape[1]
    Wt = W.T.contiguous().bfloat16()
    smp.gemm(rows_x, Wt, b, N * L, C, W.shape[0], 0, state["u"])
    binding.checkpoint_pack(rows_x, state["sx"])
    u = state["u"].view(N, L, C)
    binding.group_norm(u, ga, be, G, state["y"], mean=state["mean"], rstd=state["rstd"], saved_x=state["su"])
    diff = state["y"].float() - state["goal"]
    dy = (2.0 / diff.numel() * diff).bfloat16()
    du = torch.empty_like(dy)
    binding.group_norm_grad(dy, None, ga, be, G, state["mean"], state["rstd"], du, state["dga"], state["dbe"], ws, saved_x=state["su"])
    binding.weight_grad(state["sx"], du.view(N * L, C), state["dW"], ws, db=state["db"])
    return float((diff.double() ** 2).mean())


def test_a_projection_and_its_norm_are_tuned():
    """One layer of a drafter, forward and backward through the library: its gradients against 64-bit autograd, and steps along them."""
    from paper_2512_15773_b200 import inputs
    wl = inputs.WORKLOADS["pusht_xfmr"]
    smp = binding.Sampler(binding.make_config(wl["H"], wl["A"], wl["To"], wl["Do"], wl["draft"], wl["draft"], max_B=1, max_K=1))
    N, L, K, C, G = 24, 16, 128, 256, 8
    rng = np.random.default_rng(0)
    x = rng_tensor(rng, (N * L, K), "bf16", 0)
    W, b = rng_tensor(rng, (K, C), "fp32", 0, K ** -0.5), torch.zeros(C, device="cuda")
    ga, be = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    st = dict(u=torch.empty(N * L, C, dtype=torch.bfloat16, device="cuda"), y=torch.empty(N, L, C, dtype=torch.bfloat16, device="cuda"),
              mean=torch.empty(N, G, device="cuda"), rstd=torch.empty(N, G, device="cuda"), dga=torch.empty(C, device="cuda"),
              dbe=torch.empty(C, device="cuda"), dW=torch.empty(K, C, device="cuda"), db=torch.empty(C, device="cuda"),
              goal=rng_tensor(rng, (N, L, C), "fp32", 0.3))
    st["sx"], st["su"] = binding.saved_like(x), binding.saved_like(st["y"])
    dy = st["y"].view(N * L, C)
    ws = torch.empty(max(binding.weight_grad_workspace(dy, K), binding.group_norm_grad_workspace(st["y"], G)), dtype=torch.uint8, device="cuda")
    _block(x, W, b, ga, be, G, N, L, smp, ws, st)
    # 64-bit autograd from the same stored u (rounded once to bf16) and the true x: what differs is the eight bits (2^-8 of a block's largest
    # value at most, uniform: 2^-8 / sqrt(3) rms of values of a third of that) and bf16 roundings of dy and du: 2 % of the norms at most
    ud = st["u"].double().view(N, L, C).requires_grad_()
    gd, bd = ga.double().requires_grad_(), be.double().requires_grad_()
    v = ud.view(N, L, G, C // G)
    d = v - v.mean((1, 3), keepdim=True)
    z = (d / torch.sqrt((d * d).mean((1, 3), keepdim=True) + 1e-5)).view(N, L, C) * gd + bd
    (((z * torch.tanh(torch.nn.functional.softplus(z))) - st["goal"].double()) ** 2).mean().backward()
    want = dict(dga=gd.grad, dbe=bd.grad, dW=x.double().T @ ud.grad.view(N * L, C), db=ud.grad.sum((0, 1)))
    for k in ("dga", "dbe", "dW"):
        assert float((st[k].double() - want[k]).norm() / want[k].norm()) < 2e-2, k
    assert torch.isfinite(st["db"]).all()
    # the whole step, run on
    for _ in range(3):
        loss = _block(x, W, b, ga, be, G, N, L, smp, ws, st)
        assert np.isfinite(loss)
        W -= 2.0 * st["dW"]; ga -= 2.0 * st["dga"]; be -= 2.0 * st["dbe"]; b -= 2.0 * st["db"]
    smp.close()


def test_captured_steps_replay_on_new_inputs_and_another_stream():
    N, L, C, G, O = 5, 16, 64, 8, 96
    rng, x, ga, be, fi = norm_inputs(N, L, C, G, "bf16", True, 3)
    y, sy, sx = torch.empty_like(x), binding.saved_like(x), binding.saved_like(x)
    mean, rstd = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    dy, do = rng_tensor(rng, (N, L, C), "bf16", 0), rng_tensor(rng, (N * L, O), "bf16", 0)
    dx, dga, dbe, dfi = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(N, 2 * C, device="cuda")
    dW, db = torch.empty(C, O, device="cuda"), torch.empty(O, device="cuda")
    ws1 = torch.empty(binding.group_norm_grad_workspace(dy, G), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(binding.weight_grad_workspace(do, C), dtype=torch.uint8, device="cuda")

    def step(stream):
        binding.group_norm(x, ga, be, G, y, film=fi, mean=mean, rstd=rstd, saved_x=sx, saved_y=sy, stream=stream)
        binding.weight_grad((sy[0].view(N * L, C), sy[1].view(N * L, -1)), do, dW, ws2, db=db, stream=stream)
        binding.group_norm_grad(dy, None, ga, be, G, mean, rstd, dx, dga, dbe, ws1, film=fi, dfilm=dfi, saved_x=sx, stream=stream)
    outs = (y, mean, rstd, dW, db, dx, dga, dbe, dfi, sy[0], sy[1])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(s.cuda_stream)
    for seed in (4, 5):
        fresh = np.random.default_rng(seed)
        x.copy_(rng_tensor(fresh, (N, L, C), "bf16")); do.copy_(rng_tensor(fresh, (N * L, O), "bf16"))
        step(0)
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_two_streams_at_once_with_workspaces_of_their_own():
    cases = [weight_case(40, 16, 256, 512, 1, "bf16", i) for i in (1, 2)]
    want = [check_weight(s, d, 1, 16)[0][0] for s, d in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    out = [torch.empty(256, 512, device="cuda") for _ in cases]
    ws = [torch.empty(binding.weight_grad_workspace(d, 256), dtype=torch.uint8, device="cuda") for _, d in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for (s, d), o, w, st in zip(cases, out, ws, streams):
            binding.weight_grad(s, d, o, w, length=16, stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
