"""Every kernel of the linear operator, whole products and their gradients, against the definition in 64 bits with the tolerances of
test_gpu_linear.py; the sizes are those that the library launches each kernel for (linear_pool.py), rows and columns that fill no tile among them."""
import pytest

import linear_pool
import paper_2512_10236_amd as F
import standin
from test_gpu_linear import E, U, act64, backward, forward, seeded, slope64, weight, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PARTS = 8


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    return linear_pool.picked(linear_pool.reached(standin.build(str(tmp_path_factory.mktemp("standin")))))


def check_forward(gpu, M, K, N, nk):
    normal = seeded(gpu, M + K + N)
    A, W, R, bias = normal(M, K), weight(normal, K, N, not nk), normal(M, N), normal(N, std=0.5, dtype=torch.float32)
    op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=nk, activation=F.FICCO_ACT_SILU, bias_type=F.FICCO_F32)
    C, pre = (torch.full((M + 1, N), fill, dtype=torch.bfloat16, device=gpu["dev"]) for fill in (99.0, 98.0))
    forward(gpu, op, A, W, bias, R, pre, C)
    Wk = (W.t() if nk else W).double()
    z = A.double() @ Wk + bias.double()
    dz = 2 * (K + 2) * E * (A.double().abs() @ Wk.abs() + bias.double().abs())
    ref = act64(z, "silu") + R.double()
    within(C[:M], ref, U * ref.abs() + 1.13 * dz + 4e-6 * z.abs() + 2 * E * ref.abs(), "C")
    within(pre[:M], z, U * z.abs() + dz, "pre")
    assert (C[M] == 99).all() and (pre[M] == 98).all()


def check_backward(gpu, M, K, N, nk):
    normal = seeded(gpu, M + K + N + 1)
    A, W, dC, z = normal(M, K), weight(normal, K, N, not nk), normal(M, N), normal(M, N, std=1.5)
    op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=nk, activation=F.FICCO_ACT_SILU)
    dA, dW = (torch.full((t.shape[0] + 1, t.shape[1]), 99.0, dtype=torch.bfloat16, device=gpu["dev"]) for t in (A, W))
    db = torch.full((N + 1,), 99.0, device=gpu["dev"])
    backward(gpu, op, A, W, z, dC, dA, dW, db)
    Wk = (W.t() if nk else W).double()
    dz = dC.double() * slope64(z.double(), "silu")
    wref, wsize = A.double().t() @ dz, A.double().t().abs() @ dz.abs()
    if nk:
        wref, wsize = wref.t(), wsize.t()
    for name, got, ref, size, terms in [("dA", dA[:M], dz @ Wk.t(), dz.abs() @ Wk.t().abs(), N), ("dW", dW[:-1], wref, wsize, M)]:
        within(got, ref, U * ref.abs() + (U * 1.01 + 2 * (terms + 64) * E + 4e-6) * size, name)
        assert (got.double() - ref).norm() <= 3.4e-3 * ref.norm(), name
    within(db[:N], dz.sum(0), (M + 2) * E * dz.abs().sum(0) + 4e-6 * dC.double().abs().sum(0), "dbias")
    assert (dA[M] == 99).all() and (dW[-1] == 99).all() and db[N] == 99


@pytest.mark.parametrize("part", range(PARTS))
def test_every_kernel(gpu, calls, part):
    for op, M, K, N, nk in calls[part::PARTS]:
        print("ficco_" + op, M, K, N, "nk" if nk else "kn", flush=True)
        (check_forward if op == "linear" else check_backward)(gpu, M, K, N, nk)
