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
