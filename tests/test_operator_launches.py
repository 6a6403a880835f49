"""How the operators launch their kernels, seen on the host (tests/standin.py)."""
import re

import pytest

import linear_pool
import standin

DEFAULT_LDS = 64 * 1024          # what a launch may ask for without raising the kernel's limit


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return standin.build(str(tmp_path_factory.mktemp("standin")))


def linear(op, M, K, N, nk=0, activation=0, **k):
    return dict(op=op, fields=dict(M=M, K=K, N=N, weight_layout=nk, activation=activation), **k)


def test_lds_limits_are_raised_on_every_device(lib):
    """A launch with more LDS than a kernel may have by default needs the kernel's limit raised on the device that it goes to; on the second device in
    turn as on the first."""
    calls = []
    for device in (0, 1, 3, 0):
        for M, K, N in ((1, 256, 512), (40, 4096, 768), (700, 512, 512), (4096, 2048, 4096), (1187, 2880, 1160), (960, 4480, 2936), (166, 13184, 264), (4306, 64, 16), (12096, 64, 8)):
            for nk in (0, 1):
                calls += [linear(op, M, K, N, nk, device=device) for op in ("linear", "linear_backward")]
        for width in (64, 8192, 8200, 16384):
            for stream in (0, 1):
                calls += [dict(op=op, fields=dict(rows=40, width=width, stream_type=stream, eps=1e-6, residual_scale=1.0), device=device) for op in ("norm", "norm_backward")]
    out, _ = standin.run(lib, calls)
    assert all(c["status"] == 0 and c["launches"] for c in out)
    large = [l for c in out for l in c["launches"] if l.lds > DEFAULT_LDS]
    for what in ("gemm_direct_kernel", "linear_rows_kernel", "linear_tiles_kernel", "gemm_blocks_kernel", "residual_norm_backward_kernel"):
        assert {l.device for l in large if l.kernel.startswith(what)} == {0, 1, 3}, what
    assert not sorted({(l.kernel, l.device) for l in large if l.limit < l.lds})


def test_every_kernel_of_the_linear_operator_is_reached(lib):
    """... by a call of the pool that tests/test_gpu_linear_kernels.py draws its calls from; a kernel that no size takes has no place in the library."""
    by = linear_pool.reached(lib)
    assert len(by) > 40
    assert not [k for k, calls in by.items() if not calls and linear_pool.of_the_operator(k)]
    for kernel, calls in by.items():
        if kernel.startswith("linear_tiles_kernel"):
            columns = int(re.search(r"TileCfg<\d+, (\d+)", kernel).group(1))
            assert any(c["fields"]["N"] % columns for c in calls), kernel
