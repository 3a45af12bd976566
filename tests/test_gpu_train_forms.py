"""GroupNorm and its gradients in each of their forms, where a form can go wrong alone: values far from zero, groups of one value, strided rows,
values that are not finite.

The forms (paper_2512_15773_b200/csrc/group_norm_plan.cuh): one warp a group, a team of warps, slabs, the stream form.  u = 2^-24."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2512_15773_b200 import binding
from tests.test_gpu_train_ops import DEPTH, TYPES, U, half, host, rng_tensor

pytestmark = pytest.mark.gpu

# (N, L, C, groups) of dense rows
FORMS = {"warp": (3, 16, 128, 2), "warps of 32": (3, 16, 256, 8), "team": (3, 64, 256, 2), "slab": (3, 8, 512, 1), "slab of 320": (3, 16, 640, 2),
         "stream": (2, 256, 64, 8), "cluster": (1, 2048, 64, 4)}


def empty(*shape):
    return torch.full(shape, float("nan"), device="cuda")


def forward(x, ga, be, G, act="none", film=None, **kw):
    y, mean, rstd = torch.full_like(x, float("nan")), empty(x.shape[0], G), empty(x.shape[0], G)
    binding.group_norm(x, ga, be, G, y, act=act, film=film, mean=mean, rstd=rstd, **kw)
    return y, mean, rstd


def backward(dy, x, saved, ga, be, G, mean, rstd, act="none", film=None, dx=None):
    N, _, C = dy.shape
    dx, dga, dbe = torch.full_like(dy, float("nan")) if dx is None else dx, empty(C), empty(C)
    dfi = None if film is None else empty(N, 2 * C)
    ws = torch.empty(binding.group_norm_grad_workspace(dy, G), dtype=torch.uint8, device="cuda")
    binding.group_norm_grad(dy, x, ga, be, G, mean, rstd, dx, dga, dbe, ws, act=act, film=film, dfilm=dfi, saved_x=saved)
    return dx, dga, dbe, dfi


def packed(x):
    saved = binding.saved_like(x)
    binding.checkpoint_pack(x, saved)
    return saved


def affine(rng, C):
    return rng_tensor(rng, (C,), "fp32", 1, 0.2), rng_tensor(rng, (C,), "fp32", 0, 0.2)


# ------------------------------------------------------------------------------------------------ far from zero
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", [f for f, (_, L, C, G) in FORMS.items() if not (L * C // G) & (L * C // G - 1)])      # (other counts' means: below)
def test_groups_of_one_value_are_normalised_to_nothing(form, dtype):
    """A group that is 1000 everywhere (its sums are exact: 1000 2^k): y is beta, but for one rounding, and h is zero."""
    N, L, C, G = FORMS[form]
    rng = np.random.default_rng(1)
    ga, be = affine(rng, C)
    x = torch.full((N, L, C), 1000.0, dtype=TYPES[dtype], device="cuda")
    y, mean, rstd = forward(x, ga, be, G)
    assert (mean == 1000).all() and (host(y) == be.to(TYPES[dtype]).double().cpu().numpy()).all()
    dy = rng_tensor(rng, (N, L, C), dtype, 0.1)
    for s in (None, packed(x)):
        _, dga, _, _ = backward(dy, None if s else x, s, ga, be, G, mean, rstd)
        assert (dga == 0).all()


def check_far(dy, x, saved, ga, be, G, mean, rstd, dtype):
    """dx and dgamma of the identity.  x - mean is one rounding, its product with rstd another: h is off by 2 u |h| (and a second order), whatever the size
    of x.  Sums have a depth of DEPTH at most."""
    N, L, C = dy.shape
    dx, dga, dbe, _ = backward(dy, x, saved, ga, be, G, mean, rstd)
    xs = host(x) if x is not None else train.unpack(saved[0].cpu().numpy().reshape(N * L, C), saved[1].cpu().numpy().reshape(N * L, -1)).reshape(N, L, C)
    wide = lambda t: np.repeat(t, C // G, axis=1)[:, None, :]  # noqa: E731
    m, r, d, gam = wide(host(mean)), wide(host(rstd)), np.abs(host(dy)), np.abs(host(ga))
    h = np.abs((xs - m) * r)
    rdx, rga, rbe, _ = train.group_norm_grad(host(dy), xs, host(ga), host(be), G, host(mean), host(rstd), "none")
    depth = (DEPTH + 16) * U
    assert (np.abs(host(dbe) - rbe) <= depth * d.sum((0, 1))).all()
    assert (np.abs(host(dga) - rga) <= (depth + 3 * U) * (d * h).sum((0, 1))).all()
    of_group = lambda t: wide(t.reshape(N, L, G, C // G).mean(axis=(1, 3)))  # noqa: E731
    m1, m2 = of_group(d * gam), of_group(d * gam * h)
    e = r * ((depth + 3 * U) * (m1 + h * m2) + 3 * U * h * m2 + 6 * U * (d * gam + m1 + h * m2))
    assert (np.abs(host(dx) - rdx) <= e + (half(dtype) * np.abs(rdx) * 1.01 if dtype != "fp32" else 0) + 1e-30).all()


@pytest.mark.parametrize("offset", [0.0, 100.0, 4000.0])
@pytest.mark.parametrize("form", FORMS)
def test_gradients_far_from_zero_keep_their_digits(form, offset):
    N, L, C, G = FORMS[form]
    rng = np.random.default_rng(int(offset) + L)
    ga, be = affine(rng, C)
    x, dy = rng_tensor(rng, (N, L, C), "fp32", offset), rng_tensor(rng, (N, L, C), "fp32", 0.1)
    for s in (None, packed(x)):
        v = host(x) if s is None else train.unpack(s[0].cpu().numpy().reshape(N * L, C), s[1].cpu().numpy().reshape(N * L, -1)).reshape(N, L, C)
        _, m, r = train.group_norm(v, host(ga), host(be), G, "none")
        mean, rstd = (torch.tensor(t, dtype=torch.float32, device="cuda") for t in (m, r))
        check_far(dy, None if s else x, s, ga, be, G, mean, rstd, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [0.1, -1000.1, 77777.0])
@pytest.mark.parametrize("N,L,C,G", [*FORMS.values(), (3, 3, 128, 2), (2, 11, 256, 4), (2, 50, 128, 2), (3, 7, 160, 2), (5, 3, 640, 1), (2, 77, 15, 3),
                                     (1, 1500, 96, 3), (1, 40, 3000, 2)])
def test_a_group_of_one_value_has_that_mean(N, L, C, G, value, dtype):
    """Whatever the number of values and however their sum is rounded: the mean is the value, y beta, rstd that of no variance."""
    rng = np.random.default_rng(L)
    ga, be = affine(rng, C)
    x = torch.full((N, L, C), value, dtype=TYPES[dtype], device="cuda")
    y, mean, rstd = forward(x, ga, be, G)
    assert (mean == float(x[0, 0, 0])).all()
    assert (host(y) == be.to(TYPES[dtype]).double().cpu().numpy()).all()
    assert (np.abs(host(rstd) * np.float32(1e-5) ** 0.5 - 1) <= 8 * U).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", ["warp", "warps of 32", "team", "slab"])
def test_near_zero_the_mean_is_that_of_the_sum(form, dtype):
    """Values of few bits down to 2^-12: sums of 4096 of them are exact (below 2^12), and over 2^k values so is the mean; what corrects a large mean must not
    spoil it."""
    N, L, C, G = FORMS[form]
    g = torch.Generator(device="cuda").manual_seed(C)
    x = (torch.round(torch.randn(N, L, C, generator=g, device="cuda").bfloat16().float() * 4096) / 4096).to(TYPES[dtype])
    ga, be = affine(np.random.default_rng(2), C)
    _, mean, _ = forward(x, ga, be, G)
    want = x.double().view(N, L, G, C // G).mean((1, 3))
    assert (want.abs() < 0.5).all() and torch.equal(mean.double(), want)


@pytest.mark.parametrize("offset", [0.0, 100.0, 4000.0])
@pytest.mark.parametrize("form", FORMS)
def test_far_from_zero_the_mean_is_off_by_its_own_rounding(form, offset):
    """fp32: the mean is rounded to u |mean| and off by DEPTH u of the widest deviation; so are x - mean; rstd is off by a relative DEPTH u."""
    N, L, C, G = FORMS[form]
    rng = np.random.default_rng(int(offset) + L + 1)
    ga, be = affine(rng, C)
    x = rng_tensor(rng, (N, L, C), "fp32", offset)
    y, mean, rstd = forward(x, ga, be, G)
    ry, rm, rr = train.group_norm(host(x), host(ga), host(be), G, "none")
    wide = lambda t: np.repeat(t, C // G, axis=1)[:, None, :]  # noqa: E731
    d = np.abs(host(x) - wide(rm)).reshape(N, L, G, C // G).max(axis=(1, 3))
    e_m = 1.01 * U * np.abs(rm) + DEPTH * U * d
    assert (np.abs(host(mean) - rm) <= e_m).all()
    # (the variance about a mean that is off by e_m is larger by e_m^2; only its own rounding counts beside DEPTH u)
    assert (np.abs(host(rstd) / rr - 1) <= (DEPTH + 4) * U + 0.5 * (e_m * rr) ** 2).all()
    h = np.abs((host(x) - wide(rm)) * wide(rr))
    e = np.abs(host(ga)) * (wide(rr) * wide(e_m) + h * (DEPTH + 8) * U + h * wide(0.5 * (e_m * rr) ** 2)) + 3 * U * (np.abs(ry) + np.abs(host(be)))
    assert (np.abs(host(y) - ry) <= e).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("first,rest,spread", [(1000.0, 0.1, 0.0), (1000.0, 0.0, 1.0), (0.0, 500.0, 1.0), (-3e4, 3e4, 0.25)])
@pytest.mark.parametrize("L,C,G", [(16384, 1024, 1), (9001, 64, 4), (5003, 30, 3)])
def test_a_first_position_unlike_the_rest_costs_no_digits(L, C, G, first, rest, spread, dtype):
    """A thread merges eight positions at a time, L / 64 times at most (8 CTAs share a sequence): the sum of squares, whose terms are all positive, is off by
    as many u and those of the merging of threads (DEPTH)."""
    rng = np.random.default_rng(L)
    ga, be = affine(rng, C)
    x = rng_tensor(rng, (1, L, C), dtype, rest, spread)
    x[:, 0] = first
    y, mean, rstd = forward(x, ga, be, G)
    ry, rm, rr = train.group_norm(host(x), host(ga), host(be), G, "none")
    w = C // G
    wide = lambda t: np.repeat(t, w, axis=1)[:, None, :]  # noqa: E731
    apart = np.abs(host(x) - wide(rm)).reshape(1, L, G, w).mean(axis=(1, 3))
    e_m = 1.01 * U * np.abs(rm) + 8 * DEPTH * U * apart              # (sums about a mean that is still on its way: at most 8 times those about the last one)
    assert (np.abs(host(mean) - rm) <= e_m).all()
    e_r = (L / 64 + DEPTH) * U + 0.5 * (e_m * rr) ** 2
    assert (np.abs(host(rstd) / rr - 1) <= e_r).all()
    h = np.abs((host(x) - wide(rm)) * wide(rr))
    e = np.abs(host(ga)) * (wide(rr * e_m) + h * (wide(e_r) + 6 * U)) + 3 * U * (np.abs(ry) + np.abs(host(be)))
    assert (np.abs(host(y) - ry) <= e + (half(dtype) * np.abs(ry) * 1.01 if dtype != "fp32" else 0)).all()


# ------------------------------------------------------------------------------------------------ streams
def test_calls_without_a_stream_join_a_capture():
    """Under torch.cuda.graph the current stream is the captured one; the replay works on what the inputs hold by then."""
    N, L, C, G = 3, 16, 128, 2
    rng = np.random.default_rng(4)
    ga, be = affine(rng, C)
    x, dy = rng_tensor(rng, (N, L, C), "bf16"), rng_tensor(rng, (N, L, C), "bf16", 0)
    y, dx, saved = torch.empty_like(x), torch.empty_like(x), binding.saved_like(x)
    mean, rstd, dga, dbe = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    dW, db = torch.empty(C, C, device="cuda"), torch.empty(C, device="cuda")
    flat = saved[0].view(N * L, C), saved[1].view(N * L, -1)
    ws = torch.empty(max(binding.group_norm_grad_workspace(dy, G), binding.weight_grad_workspace(dy.view(N * L, C), C)), dtype=torch.uint8, device="cuda")

    def step():
        binding.group_norm(x, ga, be, G, y, mean=mean, rstd=rstd)
        binding.checkpoint_pack(x, saved)
        binding.group_norm_grad(dy, None, ga, be, G, mean, rstd, dx, dga, dbe, ws, saved_x=saved)
        binding.weight_grad(flat, dx.view(N * L, C), dW, ws, db=db)
        binding.checkpoint_unpack(saved, x)
    outs = (y, mean, rstd, dx, dga, dbe, dW, db, x)
    step()                                               # (kernels are set up outside the capture or within: either will do)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    fresh = rng_tensor(rng, (N, L, C), "bf16")
    x.copy_(fresh)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    x.copy_(fresh)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_calls_under_a_stream_of_torch_follow_its_work():
    N, L, C, G = 64, 16, 512, 8
    rng = np.random.default_rng(5)
    ga, be = affine(rng, C)
    x = rng_tensor(rng, (N, L, C), "fp32")
    want = forward(x, ga, be, G)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        late, y = torch.zeros_like(x), torch.empty_like(x)
        a = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            a = a @ a.clamp(-1e-3, 1e-3)                 # some milliseconds before x is there
        late.add_(x).add_(0.0 * a[0, 0].clamp(-1, 1))
        binding.group_norm(late, ga, be, G, y, act="none")
        got = y.clone()
    s.synchronize()
    assert torch.equal(got, want)


# ------------------------------------------------------------------------------------------------ layouts
def laid_out(shape, dtype, layout):
    """An empty tensor [N, L, C] of this layout and the buffer around it, full of sevens.  All but the last keep rows in 16-byte pieces, and so the form that
    dense rows take."""
    N, L, C = shape
    full = lambda *s: torch.full(s, 7.0, dtype=TYPES[dtype], device="cuda")  # noqa: E731
    if layout == "padded":                                  # two rows before and after the sequence, the UNet's own layout
        buf = full(N, L + 4, C)
        return buf[:, 2:2 + L], buf
    if layout == "slice":                                   # channels of a wider row
        buf = full(N, L, C + 64)
        return buf[:, :, 32:32 + C], buf
    if layout == "positions first":
        buf = full(L, N, C)
        return buf.transpose(0, 1), buf
    if layout == "every other":                             # sequences and rows of a larger tensor
        buf = full(2 * N, 2 * L, C)
        return buf[::2, ::2], buf
    buf = full(N, L, C + 3)                                 # odd addresses: the stream form, whatever dense rows take
    return buf[:, :, 1:1 + C], buf


LAYOUTS = ["padded", "slice", "positions first", "every other"]


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("form", FORMS)
def test_strided_rows_give_the_bits_of_dense_ones(form, layout, dtype, saved):
    N, L, C, G = FORMS[form]
    rng = np.random.default_rng(L + C)
    ga, be = affine(rng, C)
    film = rng_tensor(rng, (N, 2 * C), "fp32", 0.5, 0.3)
    dense = [rng_tensor(rng, (N, L, C), dtype, 0.4), rng_tensor(rng, (N, L, C), dtype, 0.1)]
    def both(x, dy, y, dx):
        sx, sy = (binding.saved_like(dense[0]), binding.saved_like(dense[0])) if saved else (None, None)
        mean, rstd = empty(N, G), empty(N, G)
        binding.group_norm(x, ga, be, G, y, film=film, mean=mean, rstd=rstd, saved_x=sx, saved_y=sy)
        grads = backward(dy, None if saved else x, sx, ga, be, G, mean, rstd, "mish", film, dx)
        return [y, mean, rstd, *grads, *(sx + sy if saved else ())]
    want = both(*dense, *[torch.full_like(dense[0], float("nan")) for _ in range(2)])
    apart = [laid_out((N, L, C), dtype, layout) for _ in range(4)]
    for (t, _), v in zip(apart, dense):
        t.copy_(v)
    got = both(*[t for t, _ in apart])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for t, buf in apart[2:]:
        t.fill_(7.0)
        assert (buf == 7.0).all()                            # nothing between the rows was written


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", FORMS)
def test_inputs_of_one_row_for_all(form, dtype):
    """Strides of zero: an x of one sequence for all, of one position for all; a dy of one row for all."""
    N, L, C, G = FORMS[form]
    rng = np.random.default_rng(C)
    ga, be = affine(rng, C)
    x, row = rng_tensor(rng, (1, L, C), dtype).expand(N, L, C), rng_tensor(rng, (1, 1, C), dtype).expand(N, L, C)
    out = lambda: torch.full((N, L, C), float("nan"), dtype=TYPES[dtype], device="cuda")  # noqa: E731
    for t in (x, row):
        y, want, stats, dense = out(), out(), (empty(N, G), empty(N, G)), (empty(N, G), empty(N, G))
        binding.group_norm(t, ga, be, G, y, mean=stats[0], rstd=stats[1])
        binding.group_norm(t.contiguous(), ga, be, G, want, mean=dense[0], rstd=dense[1])
        assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(stats, dense))
        got = backward(row, t, None, ga, be, G, *stats, "mish", None, out())
        ref = backward(row.contiguous(), t.contiguous(), None, ga, be, G, *stats, "mish", None, out())
        assert all(torch.equal(a, b) for a, b in zip(got[:3], ref[:3]))


# ------------------------------------------------------------------------------------------------ what is not finite
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("form", FORMS)
def test_what_is_not_finite_stays_in_its_group(form, bad, dtype):
    """In x: its group's y, dx and dfilm are NaN and the statistics not finite, its block's copy stands for NaN, its channels' dgamma are NaN; all else keeps its
    bits.  (A gradient that reads x from its copy meets NaN in all groups of that block.)  In dy: no dx of its group is finite, which subtracts an
    infinite mean; nor are dgamma and dbeta of its channel."""
    N, L, C, G = FORMS[form]
    w = C // G
    rng = np.random.default_rng(C + 1)
    ga, be = affine(rng, C)
    film = rng_tensor(rng, (N, 2 * C), "fp32", 0.5, 0.3)
    x, dy = rng_tensor(rng, (N, L, C), dtype), rng_tensor(rng, (N, L, C), dtype, 0.1)

    def run(x, dy):
        sx, sy, y, mean, rstd = binding.saved_like(x), binding.saved_like(x), torch.full_like(x, 7.0), empty(N, G), empty(N, G)
        binding.group_norm(x, ga, be, G, y, film=film, mean=mean, rstd=rstd, saved_x=sx, saved_y=sy)
        return [y, mean, rstd, sx, sy] + [backward(dy, None if s else x, s, ga, be, G, mean, rstd, "mish", film) for s in (None, sx)]
    good = run(x, dy)
    n, l, c = N - 1, L // 2, C - 1
    grp = c // w
    xb, dyb = x.clone(), dy.clone()
    xb[n, l, c] = bad
    dyb[n, l, c] = bad
    here = torch.zeros(N, L, C, dtype=torch.bool, device="cuda")
    here[n, :, grp * w:grp * w + w] = True
    per_group = torch.zeros(N, G, dtype=torch.bool, device="cuda")
    per_group[n, grp] = True
    channels = here.any(0).any(0)
    films = torch.cat([here.any(1), torch.zeros(N, C, dtype=torch.bool, device="cuda")], 1)      # (of the scale; that of the bias is a sum of dy)

    def nan_there(a, b, where):
        assert torch.isnan(a[where]).all() and torch.equal(a[~where], b[~where])
    got = run(xb, dy)
    nan_there(got[0], good[0], here)
    for i in (1, 2):
        assert not torch.isfinite(got[i][n, grp]) and torch.equal(got[i][~per_group], good[i][~per_group])
    blocks = torch.zeros(N, L, -(-C // 32), dtype=torch.bool, device="cuda")
    blocks[n, l, c // 32] = True
    assert (got[3][1][blocks] == 255).all() and torch.equal(got[3][1][~blocks], good[3][1][~blocks])
    inside = torch.zeros_like(blocks)
    inside[n, :, grp * w // 32:(grp * w + w - 1) // 32 + 1] = True
    assert (got[4][1][inside] == 255).all() and torch.equal(got[4][1][~inside], good[4][1][~inside])
    for copy, g, want in zip((False, True), got[5:], good[5:]):
        if copy:
            c0, c1 = min(c // 32 * 32 // w, grp) * w, C                    # (c is the last channel: its block and its group end together)
            here[n, :, c0:c1] = True
            channels[c0:c1] = True
            films[n, c0:c1] = True
        nan_there(g[0], want[0], here)
        nan_there(g[1], want[1], channels)
        nan_there(g[2], want[2], channels)
        nan_there(g[3], want[3], films)
    here[:] = False
    here[n, :, grp * w:] = True
    got = run(x, dyb)
    for a, b in zip(got[:3], good[:3]):
        assert torch.equal(a, b)
    for g, want in zip(got[5:], good[5:]):
        assert not torch.isfinite(g[0][n, l, c]) and not torch.isfinite(g[0][here]).any() and torch.equal(g[0][~here], want[0][~here])
        for i in (1, 2):
            keep = torch.arange(C, device="cuda") != c
            assert not torch.isfinite(g[i][c]) and torch.equal(g[i][keep], want[i][keep])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["mish", "silu", "gelu", "none"])
@pytest.mark.parametrize("N,L,C,G", [(3, 3, 128, 2), (3, 15, 256, 8), (2, 61, 256, 2), (3, 7, 640, 2), (2, 255, 64, 8), (1, 2045, 60, 4)])
def test_rows_that_are_not_there_count_nothing(N, L, C, G, act, dtype):
    """Lengths that leave places of a tile without a row, and a mean times rstd past the largest fp32 (2^120 everywhere, rstd of an eps of 2^-40): h is zero where
    there are rows, so dgamma is zero, and dbeta the sum of dy act'(beta), a sum of L N terms."""
    rng = np.random.default_rng(L)
    ga, be = affine(rng, C)
    x, dy = torch.full((N, L, C), 2.0 ** 120, dtype=TYPES[dtype], device="cuda"), rng_tensor(rng, (N, L, C), dtype, 0.1)
    mean, rstd = torch.full((N, G), 2.0 ** 120, device="cuda"), torch.full((N, G), 2.0 ** 20, device="cuda")
    film = rng_tensor(rng, (N, 2 * C), "fp32", 0.5, 0.3)
    want = host(dy) * host(film)[:, None, :C] * train.act(act, host(be))[1]
    for s in (None, packed(x)):
        dx, dga, dbe, dfi = backward(dy, None if s else x, s, ga, be, G, mean, rstd, act, film)
        assert (dga == 0).all() and torch.isfinite(dx).all() and torch.isfinite(dfi).all()
        assert (np.abs(host(dbe) - want.sum((0, 1))) <= (DEPTH + 32) * U * (np.abs(host(dy)) * np.abs(host(film))[:, None, :C] * 1.2).sum((0, 1))).all()
