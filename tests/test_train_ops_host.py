"""Refusals of the training operators: everything here is answered before a device is touched."""
import ctypes

import pytest

from paper_2512_15773_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


SAVED = binding.SavedT(4096, 4096)           # addresses that are never followed
P = 1 << 16


def norm(N=2, L=4, C=64, groups=8, dtype=1, act=1, eps=1e-5):
    return binding.NormT(dtype, N, L, C, groups, act, eps)


BAD_SHAPES = [dict(C=60), dict(groups=0), dict(L=0), dict(N=-1), dict(dtype=2), dict(act=4), dict(act=-1), dict(eps=0.0), dict(eps=float("nan")),
              dict(C=4096, groups=1), dict(C=0), dict(N=(1 << 30) + 1), dict(L=(1 << 30) + 1), dict(C=1 << 25, groups=1 << 22)]


@pytest.mark.parametrize("bad", BAD_SHAPES)
def test_norm_shapes(lib, bad):
    n = norm(**bad)
    assert lib.tsdp_group_norm(0, n, P, 256, 64, P, P, None, P, 256, 64, None, None, None, None, None) == 1
    assert lib.tsdp_group_norm_grad(0, n, P, 256, 64, P, 256, 64, None, P, P, None, P, P, P, 256, 64, P, P, None, P, 1 << 30, None) == 1
    assert lib.tsdp_group_norm_grad_workspace(0, n) == 0


def test_norm_pointers_and_strides(lib):
    ok = [0, norm(), P, 256, 64, P, P, None, P, 256, 64, None, None, None, None, None]
    for i, v in ((0, -1), (0, 64), (1, None), (2, None), (3, -1), (5, None), (6, None), (8, None), (9, 255), (10, 63), (13, binding.SavedT(0, 4096)),
                 (14, binding.SavedT(4096, 0))):
        args = list(ok); args[i] = v
        assert lib.tsdp_group_norm(*args) == 1, i
    assert lib.tsdp_group_norm(0, norm(N=0), None, 0, 0, None, None, None, None, 0, 0, None, None, None, None, None) == 0


def test_copy_arguments(lib):
    for name in ("tsdp_checkpoint_pack", "tsdp_checkpoint_unpack"):
        f = getattr(lib, name)
        order = (lambda x, c: (x, 256, 64, 2, 4, 64, c)) if name.endswith("_pack") and "un" not in name else (lambda x, c: (c, x, 256, 64, 2, 4, 64))
        assert f(0, 1, *order(None, SAVED), None) == 1
        assert f(0, 1, *order(P, None), None) == 1
        assert f(0, 2, *order(P, SAVED), None) == 1
        assert f(-1, 1, *order(P, SAVED), None) == 1
    assert lib.tsdp_checkpoint_pack(0, 1, None, 0, 0, 0, 4, 64, None, None) == 0
    assert lib.tsdp_checkpoint_unpack(0, 1, SAVED, P, 256, 63, 2, 4, 64, None) == 1          # rows that overlap
    assert lib.tsdp_checkpoint_pack(0, 1, P, 256, 64, 2, 4, 0, SAVED, None) == 1


def test_weight_arguments(lib):
    ok = [0, 1, SAVED, P, 128, 2, 16, 64, 128, 1, P, P, P, 1 << 40, None]
    for i, v in ((0, -1), (1, 2), (4, -1), (5, -1), (6, 0), (7, 0), (8, 0), (9, 0), (9, 2), (9, 17), (10, None), (5, 1 << 28)):
        args = list(ok); args[i] = v
        assert lib.tsdp_weight_grad(*args) == 1, i
    assert lib.tsdp_weight_grad_workspace(0, 1, 2, 16, 64, 128, 2) == 0
    assert lib.tsdp_weight_grad_workspace(0, 1, 2, 0, 64, 128, 1) == 0


def test_every_plan_of_the_listed_ranges_fits_a_fixed_workspace(lib):
    for K in (8, 77, 512, 1024):
        for out in (8, 130, 512, 2048):
            for taps in (1, 3, 5):
                for rows in (16, 1001, 45056):
                    for dtype in (0, 1):
                        assert 0 < lib.tsdp_weight_grad_workspace(0, dtype, 1, rows, K, out, taps) <= 64 << 20
    for N, C, G in ((1, 256, 8), (4096, 512, 8), (4096, 2048, 32), (1 << 20, 8, 8), (3, 320, 32)):
        assert 0 < lib.tsdp_group_norm_grad_workspace(0, norm(N=N, C=C, groups=G)) <= 64 << 20


def test_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 64)
    with pytest.raises(ValueError, match="CUDA"):
        binding.checkpoint_pack(x, binding.saved_like(x))
    q, s = binding.saved_like(torch.zeros(3, 70))
    assert q.shape == (3, 70) and s.shape == (3, 3) and q.dtype == torch.int8 and s.dtype == torch.uint8
    with pytest.raises(ValueError, match="act"):
        binding._act("relu")
    cpu = x.get_device()
    with pytest.raises(ValueError, match="scale"):
        binding._saved((q, s[:, :2].contiguous()), "saved", 3, 70, cpu)
    with pytest.raises(ValueError, match="channels"):
        binding._saved((q, s), "saved", 7, 30, cpu)
    with pytest.raises(ValueError, match="without gaps"):
        binding._dense(x.transpose(0, 1), "x", x.numel(), torch.float32, cpu)
    with pytest.raises(ValueError, match="x: 512 values"):
        binding._dense(x, "x", 512, torch.bfloat16, cpu)


class Rows:
    """Stands for a tensor on a GPU: the sizes of one, no memory."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, *shape):
        import torch
        self.shape, self.dtype = shape, torch.bfloat16

    def stride(self):
        return tuple(0 if i + 1 < len(self.shape) else 1 for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def data_ptr(self):
        return P

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def is_contiguous(self):
        return True


@pytest.mark.parametrize("shape", [(2**32 + 5, 1), (2**32 + 1, 4, 64), (2, 2**32 + 4, 64)])
def test_sizes_past_an_int_are_not_cut(lib, shape):
    """2^32 + 5 rows are not five."""
    import torch
    x, f32 = Rows(*shape), torch.zeros(shape[-1])
    q, b = Rows(*shape), Rows(*shape[:-1], -(-shape[-1] // 32))
    q.dtype, b.dtype = torch.int8, torch.uint8
    with pytest.raises(ValueError):
        binding.checkpoint_pack(x, (q, b))
    with pytest.raises(ValueError):
        binding.checkpoint_unpack((q, b), x)
    with pytest.raises(ValueError):
        binding.group_norm(x, f32, f32, 1, x)
    with pytest.raises(ValueError):
        binding.group_norm_grad_workspace(x, 1)
    if len(shape) == 2:
        with pytest.raises(ValueError):
            binding.weight_grad_workspace(x, 32, length=5)
