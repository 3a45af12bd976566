"""The 64-bit definitions of the training operators: copies on chosen values, gradients against central differences."""
import numpy as np
import pytest

from oracle import nets, train


def test_copy_of_chosen_blocks():
    x = np.zeros((5, 40))
    x[0, :4] = [1.0, 127.4, 0.5, -3.0]             # steps of one; halves go to the even number
    x[1, :3] = [127.5, 1.0, 3.0]                   # 127.5 would round to 128: steps of two
    x[2, 0] = np.inf
    x[3, :2] = [2.0 ** -140, -1e-3]
    x[4, 39] = 3.4028234663852886e38               # the largest fp32 stands at 127 steps of 2^121
    q, s = train.pack(x)
    assert q[0, :4].tolist() == [1, 127, 0, -3] and s[0, 0] == 127
    assert q[1, :3].tolist() == [64, 0, 2] and s[1, 0] == 128
    assert s[2, 0] == 255 and s[2, 1] == 1
    assert abs(int(q[3, 1])) >= 64 and q[3, 0] == 0
    assert q[4, 39] == 127 and s[4, 1] == 248
    back = train.unpack(q, s)
    assert np.isnan(back[2, :32]).all() and not back[2, 32:].any()
    step = 2.0 ** (np.repeat(s.astype(float), 32, axis=1)[:, :40] - 127)
    ok = np.ones_like(x, dtype=bool); ok[2, :32] = False; ok[4, 39] = False
    assert (np.abs(back - x)[ok] <= step[ok] / 2).all()


@pytest.mark.parametrize("name", ["none", "mish", "silu", "gelu"])
def test_activation_derivatives(name):
    z = np.linspace(-12, 12, 241)
    d = 1e-5
    num = (train.act(name, z + d)[0] - train.act(name, z - d)[0]) / (2 * d)
    assert np.max(np.abs(train.act(name, z)[1] - num)) < 1e-8
    if name == "mish":
        assert np.max(np.abs(train.act(name, z)[0] - nets.mish(z))) < 1e-15


@pytest.mark.parametrize("name,film", [("mish", True), ("silu", False), ("gelu", True), ("none", False)])
def test_norm_gradients_against_central_differences(name, film):
    rng = np.random.default_rng(3)
    N, L, C, G = 2, 5, 6, 3
    x, dy = rng.normal(size=(N, L, C)) + 0.5, rng.normal(size=(N, L, C))
    ga, be = 1 + 0.2 * rng.normal(size=C), 0.2 * rng.normal(size=C)
    fi = 1 + 0.3 * rng.normal(size=(N, 2 * C)) if film else None
    y, mean, rstd = train.group_norm(x, ga, be, G, name, fi)
    got = train.group_norm_grad(dy, x, ga, be, G, mean, rstd, name, fi)
    for which, arr in enumerate((x, ga, be) + ((fi,) if film else ())):
        num = np.zeros_like(arr)
        for i in np.ndindex(arr.shape):
            keep, d = arr[i], 1e-6
            arr[i] = keep + d; up = (train.group_norm(x, ga, be, G, name, fi)[0] * dy).sum()
            arr[i] = keep - d; dn = (train.group_norm(x, ga, be, G, name, fi)[0] * dy).sum()
            arr[i] = keep
            num[i] = (up - dn) / (2 * d)
        assert np.max(np.abs(got[which] - num)) < 1e-7 * max(1, np.max(np.abs(num))), which


def test_norm_is_that_of_the_network():
    rng = np.random.default_rng(4)
    x, ga, be = rng.normal(size=(7, 12)), rng.normal(size=12), rng.normal(size=12)
    y = train.group_norm(x[None], ga, be, 4)[0][0]
    assert np.max(np.abs(y - nets.mish(nets.group_norm(x, ga, be, 4)))) < 1e-14


def test_weight_gradient_against_central_differences():
    rng = np.random.default_rng(5)
    N, L, K, O = 2, 6, 3, 2
    x, W, b, dy = rng.normal(size=(N, L, K)), rng.normal(size=(5, K, O)), rng.normal(size=O), rng.normal(size=(N, L, O))
    dW, db = train.weight_grad(x.reshape(N * L, K), dy.reshape(N * L, O), 5, L)
    loss = lambda: sum((nets.conv1d_k5(x[n], W, b) * dy[n]).sum() for n in range(N))  # noqa: E731
    for arr, got in ((W, dW), (b, db)):
        for i in np.ndindex(arr.shape):
            keep = arr[i]
            arr[i] = keep + 0.5; up = loss()
            arr[i] = keep - 0.5; dn = loss()
            arr[i] = keep
            assert abs(up - dn - got[i]) < 1e-11                      # the loss is linear in W and b


def test_copies_at_the_ends_of_the_range():
    """Off by half a step, 1 / 127.5 of the block's largest magnitude; but by up to a step where q is held at 127, and by 2^-127 for the smallest blocks."""
    x = np.zeros((6, 32))
    x[:, 0] = [3.4e38, 127.5 * 2.0 ** 121, 127.49 * 2.0 ** 121, 2.0 ** -127, 1.01 * 2.0 ** -127, 127.5 * 2.0 ** -60]
    q, s = train.pack(x)
    off, step = np.abs(train.unpack(q, s) - x)[:, 0], 2.0 ** (s[:, 0].astype(float) - 127)
    assert list(s[:4, 0]) == [248, 248, 248, 1] and list(q[:4, 0]) == [127, 127, 127, 0]
    assert 0.5 * step[0] < off[0] < step[0] and off[1] == 0.5 * step[1] and (off[2:] <= 0.5 * step[2:]).all()
    assert s[5, 0] == 68 and q[5, 0] == 64 and off[5] <= x[5, 0] / 127.5
