"""Refusals and sizes of the operators around the pair that need no GPU: what breaks a rule is refused before any pointer is
looked at, and a workspace's size follows from the struct alone."""
import pytest

import paper_2512_10236_amd as F

P = 1 << 20          # an address that is aligned and never read: every call here is refused for another reason
ALIGNED = [P] * 8


def status(fn, *args):
    with pytest.raises(F.FiccoError) as e:
        fn(*args)
    return e.value.status


def linear(backward=False, **k):
    op = F.ficco_linear_t(**{**dict(M=8, K=64, N=64), **k})
    if backward:
        return status(F.ficco_linear_backward, op, P, P, P, P, P, P, P, P, 1 << 30, None)
    return status(F.ficco_linear, op, P, P, P, P, P, P, P, 1 << 30, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(M=-1), dict(M=1 << 31), dict(K=0), dict(K=96), dict(K=(1 << 22) + 64), dict(N=0), dict(N=12), dict(N=(1 << 22) + 8), dict(lda=56),
                                 dict(lda=68), dict(lda=(1 << 22) + 8), dict(ldc=56), dict(ldc=68), dict(ld_residual=60), dict(ld_residual=56), dict(ld_pre=60), dict(ld_pre=56),
                                 dict(ld_pre=(1 << 22) + 8), dict(ld_residual=(1 << 22) + 8)])
def test_linear_shapes(backward, bad):
    assert linear(backward, **bad) == F.FICCO_ERR_SHAPE
    op = F.ficco_linear_t(**{**dict(M=8, K=64, N=64), **bad})
    assert status(F.ficco_linear_workspace, op, backward) == F.FICCO_ERR_SHAPE


def test_linear_backward_has_its_own_row_limit():
    assert linear(True, M=(1 << 22) + 1) == F.FICCO_ERR_SHAPE
    assert F.ficco_linear_workspace(F.ficco_linear_t(M=(1 << 22) + 1, K=64, N=64, weight_layout=F.FICCO_WEIGHT_NK)) == 0


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(weight_layout=2), dict(weight_layout=-1), dict(activation=5), dict(activation=-1), dict(bias_type=2), dict(bias_type=-1), dict(reserved=1)])
def test_linear_values(backward, bad):
    assert linear(backward, **bad) == F.FICCO_ERR_ARG


def test_linear_pointers():
    op = F.ficco_linear_t(M=8, K=64, N=64, activation=F.FICCO_ACT_SILU)
    for missing in (1, 2, 6):
        args = [op, P, P, P, P, P, P, P, 1 << 30, None]
        args[missing] = None
        assert status(F.ficco_linear, *args) == F.FICCO_ERR_ARG
        args[missing] = P + 8
        assert status(F.ficco_linear, *args) == F.FICCO_ERR_ARG
    for missing in (1, 2, 3, 4, 8):
        args = [op, P, P, P, P, P, P, P, P, 1 << 30, None]
        args[missing] = None
        assert status(F.ficco_linear_backward, *args) == F.FICCO_ERR_ARG
    assert status(F.ficco_linear, None, P, P, P, P, P, P, P, 1 << 30, None) == F.FICCO_ERR_ARG
    assert F.load().ficco_linear_workspace(op, 0, None) == F.FICCO_ERR_ARG


def test_linear_workspace_holds_what_is_laid_out():
    t = F.ficco_linear_t
    # a [K,N] weight is re-laid out where parts of tiles are the fastest, and read in place elsewhere, as an [N,K] one is
    assert F.ficco_linear_workspace(t(M=198, K=13440, N=2392)) == 2 * 13440 * 2392
    assert F.ficco_linear_workspace(t(M=198, K=13440, N=2392, weight_layout=F.FICCO_WEIGHT_NK)) == 0
    assert F.ficco_linear_workspace(t(M=4096, K=4096, N=4096)) == 0 == F.ficco_linear_workspace(t(M=16, K=1024, N=512))
    assert F.ficco_linear_workspace(t(M=0, K=4096, N=4096)) == 0 == F.ficco_linear_workspace(t(M=0, K=4096, N=4096), True)
    # dZ in both orders, A turned and the column sums; M and N to whole k-tiles. With whole k-tiles of rows A stays as it is
    least = 2 * (100 * 128 + 72 * 128 + 64 * 128 + 64 * 128)
    assert least <= F.ficco_linear_workspace(t(M=100, K=64, N=72, activation=F.FICCO_ACT_SILU), True) <= least + 8192
    z = 2 * 8192 * 4096
    assert 2 * z <= F.ficco_linear_workspace(t(M=8192, K=8192, N=4096, activation=F.FICCO_ACT_SILU), True) <= 2 * z + 128 * 4096 * 4 + 8192
    assert z <= F.ficco_linear_workspace(t(M=8192, K=8192, N=4096), True) <= z + 128 * 4096 * 4 + 8192


def norm(backward=False, **k):
    op = F.ficco_residual_norm_t(**{**dict(rows=8, width=64, residual_scale=1.0, eps=1e-6), **k})
    if backward:
        return status(F.ficco_residual_norm_backward, op, P, P, P, P, P, P, P, P, P, P, P, P, P, 1 << 30, None)
    return status(F.ficco_residual_norm, op, P, P, P, P, P, P, P, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=12), dict(width=16392), dict(gate_rows=-1)])
def test_norm_shapes(backward, bad):
    assert norm(backward, **bad) == F.FICCO_ERR_SHAPE


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(stream_type=2), dict(param_type=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(residual_scale=float("inf"))])
def test_norm_values(backward, bad):
    assert norm(backward, **bad) == F.FICCO_ERR_ARG


def test_norm_pointers():
    op = F.ficco_residual_norm_t(rows=8, width=64, residual_scale=1.0, eps=1e-6)
    for missing in (1, 2, 5, 6, 7):          # x, block, y, and the two that go together
        args = [op, P, P, P, P, P, P, P, None]
        args[missing] = None
        assert status(F.ficco_residual_norm, *args) == F.FICCO_ERR_ARG
    names = ["op", "y", "block", "post", "gate", "pre", "dy", "dh", "dx", "dblock", "dpost", "dgate", "dpre", "workspace"]
    # a sum for a parameter that is not there; a norm whose gradient is not; y and block where a norm needs them; the workspace
    for missing in ("post", "gate", "pre", "dh", "y", "block", "workspace"):
        args = [op] + [P] * 13 + [1 << 30, None]
        args[names.index(missing)] = None
        assert status(F.ficco_residual_norm_backward, *args) == F.FICCO_ERR_ARG


def test_norm_workspace_is_three_sums_a_chunk():
    for rows, width, gate_rows in [(1, 8, 0), (1000, 64, 0), (16384, 4096, 2048), (16384, 4096, 3), (3000, 16384, 7), (5, 512, 2)]:
        n = F.ficco_residual_norm_workspace(F.ficco_residual_norm_t(rows=rows, width=width, gate_rows=gate_rows, eps=1e-6))
        assert n > 0 and n % (12 * width) == 0 and n // (12 * width) <= max(2 * 2048, 2)
    assert F.ficco_residual_norm_workspace(F.ficco_residual_norm_t(rows=0, width=64)) == 0


def balance(**k):
    op = F.ficco_expert_balance_t(**{**dict(tokens=8, experts=4, top_k=2, coefficient=1.0), **k})
    return (status(F.ficco_expert_balance, op, P, P, P, P, P, P, P, 1 << 30, None), status(F.ficco_expert_balance_backward, op, P, P, P, P, P, P, None),
            status(F.ficco_expert_balance_workspace, op))


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=1 << 31), dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=65), dict(group_tokens=-1), dict(ld_logits=3),
                                 dict(tokens=(1 << 20) + 1, group_tokens=1), dict(tokens=(1 << 31) - 1, top_k=2), dict(tokens=1 << 30, group_tokens=1 << 28, top_k=8)])
def test_balance_shapes(bad):
    assert set(balance(**bad)) == {F.FICCO_ERR_SHAPE}


@pytest.mark.parametrize("bad", [dict(logits_type=2), dict(logits_type=-1), dict(coefficient=float("nan")), dict(coefficient=float("inf"))])
def test_balance_values(bad):
    assert set(balance(**bad)) == {F.FICCO_ERR_ARG}


def test_balance_pointers():
    op = F.ficco_expert_balance_t(tokens=8, experts=4, top_k=2, coefficient=1.0)
    for missing in (1, 2, 4, 5):
        args = [op, P, P, P, P, P, P, P, 1 << 30, None]
        args[missing] = None
        assert status(F.ficco_expert_balance, *args) == F.FICCO_ERR_ARG
        args[missing] = P + 1
        assert status(F.ficco_expert_balance, *args) == F.FICCO_ERR_ARG
    for missing in (1, 3, 4, 6):
        args = [op, P, P, P, P, P, P, None]
        args[missing] = None
        assert status(F.ficco_expert_balance_backward, *args) == F.FICCO_ERR_ARG
    assert F.ficco_expert_balance_workspace(op) == 0
    assert F.ficco_expert_balance_workspace(F.ficco_expert_balance_t(tokens=0, experts=4, top_k=2)) == 0


def test_a_tensor_whose_rows_are_strided_inside_is_refused():
    torch = pytest.importorskip("torch")
    t = torch.zeros(64, 64, dtype=torch.int16)
    op = F.ficco_linear_t(M=64, K=64, N=64)
    assert status(F.ficco_linear, op, t.t(), P, None, None, None, P, P, 1 << 30, None) == F.FICCO_ERR_ARG
