"""A call of the training operators that CUDA refuses leaves nothing behind: the sampler's and torch's next calls work."""
import numpy as np
import pytest
import torch

from paper_2512_15773_b200 import binding
from tests import helpers as hp
from tests.test_gpu_kernels import _gemm_case

pytestmark = pytest.mark.gpu


def test_a_refused_call_is_not_taken_for_the_next_one():
    lib, nowhere = binding.load_library(), torch.cuda.device_count()
    smp, *_ = hp.setup(hp.small_xfmr_workload(1), max_B=1, max_K=1)
    x = torch.ones(2, 16, 64, device="cuda")
    ga, saved = torch.ones(64, device="cuda"), binding.saved_like(x)
    p, g, s = x.data_ptr(), ga.data_ptr(), binding.SavedT(saved[0].data_ptr(), saved[1].data_ptr())
    n, room = binding.NormT(0, 2, 16, 64, 8, 1, 1e-5), torch.empty(1 << 20, device="cuda")
    w = room.data_ptr()
    calls = [lambda: lib.tsdp_checkpoint_pack(nowhere, 0, p, 1024, 64, 2, 16, 64, s, None),
             lambda: lib.tsdp_checkpoint_unpack(nowhere, 0, s, p, 1024, 64, 2, 16, 64, None),
             lambda: lib.tsdp_group_norm(nowhere, n, p, 1024, 64, g, g, None, p, 1024, 64, None, None, None, None, None),
             lambda: lib.tsdp_group_norm_grad(nowhere, n, p, 1024, 64, p, 1024, 64, None, g, g, None, g, g, p, 1024, 64, g, g, None, w, 1 << 22, None),
             lambda: lib.tsdp_weight_grad(nowhere, 0, s, p, 64, 2, 16, 64, 64, 1, w, None, w, 1 << 22, None)]
    rng = np.random.default_rng(0)
    assert lib.tsdp_group_norm_grad_workspace(nowhere, n) > 0
    _gemm_case(smp, 256, 128, 128, 0, rng)
    for call in calls:
        assert call() == 4                                   # TSDP_ERR_CUDA: the device does not exist
        _gemm_case(smp, 256, 128, 128, 0, rng)
        assert float(x.sum()) == 2 * 16 * 64
    smp.close()
