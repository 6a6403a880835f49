"""ficco_linear and ficco_linear_backward against the definition in 64 bits.

Tolerances, from the arithmetic. u = 2^-8 is half a step of bf16 relative to a value, e = 2^-24 that of fp32.
  z      a sum of K products in fp32 in any order and a bias: off by at most (K + 2) e (|A||W| + |bias|); twice that, since a matrix
         instruction's own sums may be cut instead of rounded
  act    its slope is below 1.13, so the same again times that, and its own evaluation 4e-6 of |z|
  C      one rounding u of the value, and the sum with the residual in fp32
  dA, dW one rounding u of the result, and each dZ's rounding u: u |dZ||W|; in the 2-norm a rounding is off by u / sqrt(3) of
         the norm at most, two independent ones by sqrt(2) times that: 3.2e-3, 3.4e-3 with the sums
  dbias  M e sum |dZ|, and the slope's evaluation 4e-6 sum |dC|
"""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, E = 2.0 ** -8, 2.0 ** -24
ACTS = {"none": F.FICCO_ACT_NONE, "relu": F.FICCO_ACT_RELU, "gelu": F.FICCO_ACT_GELU, "gelu_tanh": F.FICCO_ACT_GELU_TANH, "silu": F.FICCO_ACT_SILU}


def act64(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return torch.relu(z)
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z)


def slope64(z, kind):
    z = z.clone().requires_grad_()
    return torch.autograd.grad(act64(z, kind).sum(), z)[0]


def seeded(gpu, seed):
    g = torch.Generator(device=gpu["dev"])
    g.manual_seed(seed)
    return lambda *shape, std=1.0, dtype=torch.bfloat16: (torch.randn(*shape, generator=g, device=gpu["dev"]) * std).to(dtype)


def strided(t, ld, fill=7.0):
    """The same values in rows `ld` apart, something else between them."""
    out = torch.full((t.shape[0] + 1, ld), fill, dtype=t.dtype, device=t.device)
    out[:t.shape[0], :t.shape[1]] = t
    return out


def workspace(gpu, op, backward):
    n = F.ficco_linear_workspace(op, backward)
    return (torch.full((n,), 0xFF, dtype=torch.uint8, device=gpu["dev"]), n) if n else (None, 0)     # NaNs, whatever is read of it as bf16


def forward(gpu, op, A, W, bias, residual, pre, C):
    ws, n = workspace(gpu, op, False)
    torch.cuda.synchronize()
    F.ficco_linear(op, A, W, bias, residual, pre, C, ws, n, gpu["cs"])
    torch.cuda.synchronize()


def backward(gpu, op, A, W, z, dC, dA, dW, dbias):
    ws, n = workspace(gpu, op, True)
    torch.cuda.synchronize()
    F.ficco_linear_backward(op, A, W, z, dC, dA, dW, dbias, ws, n, gpu["cs"])
    torch.cuda.synchronize()


def weight(normal, K, N, kn):
    return normal(K, N, std=K ** -0.5) if kn else normal(N, K, std=K ** -0.5)


def within(got, ref, tol, what):
    assert torch.isfinite(got).all(), what
    over = (got.double() - ref).abs() - tol
    assert (over <= 0).all(), f"{what}: {over.max().item()} over"


# one row to more than a tile of each kind, odd ones; k of one k-tile to many; columns that fill no tile and no lane's eight
SIZES = [(1, 64, 8), (1, 4096, 768), (3, 128, 40), (16, 2112, 264), (17, 64, 520), (33, 512, 72), (64, 4096, 768), (65, 1024, 200), (127, 192, 1032), (300, 576, 1160), (1000, 320, 328),
         (2311, 128, 2056), (4100, 64, 1544), (530, 8192, 136), (198, 13440, 2392), (1404, 13888, 464), (9, 8192, 1032), (1, 5120, 1160), (40, 16384, 520), (300, 10624, 456), (16, 2112, 2056)]


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward(gpu, M, K, N, kn):
    normal = seeded(gpu, M * 7 + K + N)
    A, W, R = normal(M, K), weight(normal, K, N, kn), normal(M, N)
    Wk = (W if kn else W.t()).double()
    z0, size = A.double() @ Wk, A.double().abs() @ Wk.abs()
    for n, (kind, bias_type) in enumerate([("none", None), ("relu", "bf16"), ("gelu", "f32"), ("gelu_tanh", "bf16"), ("silu", "f32")]):
        bias = None if bias_type is None else normal(N, std=0.5, dtype=torch.bfloat16 if bias_type == "bf16" else torch.float32)
        with_residual, with_pre = n % 2 == 1, n in (2, 3, 4)
        op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=F.FICCO_WEIGHT_KN if kn else F.FICCO_WEIGHT_NK, activation=ACTS[kind],
                              bias_type=F.FICCO_F32 if bias_type == "f32" else F.FICCO_BF16)
        C = torch.full((M + 1, N), 99.0, dtype=torch.bfloat16, device=gpu["dev"])
        pre = torch.full_like(C, 98.0) if with_pre else None
        print("ficco_linear", M, K, N, "kn" if kn else "nk", kind, flush=True)
        forward(gpu, op, A, W, bias, R if with_residual else None, pre, C)
        z = z0 if bias is None else z0 + bias.double()
        dz = 2 * (K + 2) * E * (size + (0 if bias is None else bias.double().abs()))
        ref = act64(z, kind) + (R.double() if with_residual else 0)
        within(C[:M], ref, U * ref.abs() + 1.13 * dz + 4e-6 * z.abs() + 2 * E * ref.abs(), f"C {kind}")
        assert (C[M] == 99.0).all()
        if with_pre:
            within(pre[:M], z, U * z.abs() + dz, f"pre {kind}")
            assert (pre[M] == 98.0).all()


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("M", [5, 200, 1500])
def test_rows_at_strides_of_their_own(gpu, M, kn):
    """Row strides of every operand, and a result over the residual; what lies between the rows stays."""
    K, N = 256, 392
    normal = seeded(gpu, M)
    A, W, R = normal(M, K), weight(normal, K, N, kn), normal(M, N)
    dense = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=F.FICCO_ACT_GELU)
    C0, pre0 = torch.empty(M, N, dtype=torch.bfloat16, device=gpu["dev"]), torch.empty(M, N, dtype=torch.bfloat16, device=gpu["dev"])
    forward(gpu, dense, A, W, None, R, pre0, C0)
    op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=F.FICCO_ACT_GELU, lda=K + 40, ldc=N + 8, ld_residual=N + 8, ld_pre=N + 16)
    RC, pre = strided(R, N + 8), strided(torch.zeros_like(R), N + 16, 5.0)
    forward(gpu, op, strided(A, K + 40, float("nan")), W, None, RC, pre, RC)
    assert torch.equal(RC[:M, :N], C0) and (RC[:M, N:] == 7).all() and (RC[M] == 7).all()
    assert torch.equal(pre[:M, :N], pre0) and (pre[:M, N:] == 5).all() and (pre[M] == 5).all()
    # ... and of the backward's inputs
    dC = normal(M, N)
    outs = []
    for o, a, z, d in [(dense, A, pre0, dC), (op, strided(A, K + 40, float("nan")), pre, strided(dC, N + 8, float("nan")))]:
        dA, dW, db = torch.empty_like(A), torch.empty_like(W), torch.empty(N, device=gpu["dev"])
        backward(gpu, o, a, W, z, d, dA, dW, db)
        outs.append((dA, dW, db))
    for x, y in zip(*outs):
        assert torch.equal(x, y)


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("M,K,N", [(512, 4096, 8), (640, 128, 72), (640, 512, 2048), (530, 256, 136)])
def test_rows_whose_offsets_pass_32_bits(gpu, M, K, N, kn):
    """All matrices with rows side by side in one buffer whose rows are as far apart as they may be: 4 GiB and more in all."""
    far = 1 << 22
    normal = seeded(gpu, M + K)
    A, W, R, dC = normal(M, K), weight(normal, K, N, kn), normal(M, N), normal(M, N)
    store = torch.full((M, far), 7.0, dtype=torch.bfloat16, device=gpu["dev"])
    fA, fC, fpre, fdC = (store[:, at:at + n] for at, n in ((0, K), (8192, N), (16384, N), (24576, N)))
    fA.copy_(A), fC.copy_(R), fdC.copy_(dC)
    outs = []
    for ld, a, c, pre, d in [(0, A, R, torch.empty_like(R), dC), (far, fA, fC, fpre, fdC)]:
        op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=F.FICCO_ACT_SILU, lda=ld, ldc=ld, ld_residual=ld, ld_pre=ld)
        dA, dW, db = torch.empty_like(A), torch.empty_like(W), torch.empty(N, device=gpu["dev"])
        forward(gpu, op, a, W, None, c, pre, c)
        backward(gpu, op, a, W, pre, d, dA, dW, db)
        outs.append((c, pre, dA, dW, db))
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    assert (store[:, 8192 + N:16384] == 7).all() and (store[:, 16384 + N:24576] == 7).all()


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 8), (3, 128, 40), (64, 256, 64), (100, 64, 72), (257, 576, 264), (1187, 320, 1160), (70, 2048, 136), (2100, 192, 128), (1, 768, 4096), (3, 512, 8192), (48, 1280, 10624),
                                   (40, 2048, 520), (600, 192, 8896), (2, 7168, 640), (9, 576, 16384)])
def test_backward(gpu, M, K, N, kn):
    normal = seeded(gpu, M * 5 + K + N)
    A, W, dC, z = normal(M, K), weight(normal, K, N, kn), normal(M, N), normal(M, N, std=1.5)
    Wk = (W if kn else W.t()).double()
    for kind in ("none", "relu", "gelu", "gelu_tanh", "silu"):
        op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=ACTS[kind])
        dA = torch.full((M + 1, K), 99.0, dtype=torch.bfloat16, device=gpu["dev"])
        dW = torch.full((W.shape[0] + 1, W.shape[1]), 99.0, dtype=torch.bfloat16, device=gpu["dev"])
        db = torch.full((N + 1,), 99.0, device=gpu["dev"])
        print("ficco_linear_backward", M, K, N, "kn" if kn else "nk", kind, flush=True)
        backward(gpu, op, A, W, None if kind == "none" else z, dC, dA, dW, db)
        dz = dC.double() if kind == "none" else dC.double() * slope64(z.double(), kind)
        rounded = 0 if kind in ("none", "relu") else U
        refs = {"dA": (dA[:M], dz @ Wk.t(), dz.abs() @ Wk.t().abs(), N), "dW": (dW[:-1], A.double().t() @ dz, A.double().t().abs() @ dz.abs(), M)}
        if not kn:
            refs["dW"] = (refs["dW"][0], refs["dW"][1].t(), refs["dW"][2].t(), M)
        for name, (got, ref, size, terms) in refs.items():
            within(got, ref, U * ref.abs() + (rounded * 1.01 + 2 * (terms + 64) * E) * size + 4e-6 * size, f"{name} {kind}")
            norm = ref.norm()
            assert (got.double() - ref).norm() <= 3.4e-3 * norm, (name, kind)
        within(db[:N], dz.sum(0), (M + 2) * E * dz.abs().sum(0) + 4e-6 * dC.double().abs().sum(0), f"dbias {kind}")
        assert (dA[M] == 99).all() and (dW[-1] == 99).all() and db[N] == 99


def test_each_gradient_alone_is_the_same(gpu):
    M, K, N = 150, 128, 200
    normal = seeded(gpu, 3)
    A, W, dC, z = normal(M, K), normal(K, N, std=K ** -0.5), normal(M, N), normal(M, N)
    op = F.ficco_linear_t(M=M, K=K, N=N, activation=F.FICCO_ACT_SILU)

    def outs():
        return [torch.zeros_like(A), torch.zeros_like(W), torch.zeros(N, device=gpu["dev"])]
    whole = outs()
    backward(gpu, op, A, W, z, dC, *whole)
    for k in range(3):
        one = outs()
        backward(gpu, op, A, W, z, dC, *[t if i == k else None for i, t in enumerate(one)])
        assert torch.equal(one[k], whole[k])
    backward(gpu, op, None, None, z, dC, None, None, one[2])
    assert torch.equal(one[2], whole[2])
    backward(gpu, op, A, W, z, dC, None, None, None)


@pytest.mark.parametrize("kind", ["relu", "gelu", "gelu_tanh", "silu"])
def test_gradients_are_those_of_differences(gpu, kind):
    """Along the gradient itself the loss sum(dC C) grows by its squared norm: central differences of the definition in 64 bits,
    at the stored value of z. The stored z and the gradients are rounded to bf16: 2-norms as above, and u of z times the
    activations' curvature (below 1.2) on dZ, of independent signs."""
    M, K, N = 96, 128, 104
    normal = seeded(gpu, 11)
    A, W, dC, bias = normal(M, K), normal(K, N, std=K ** -0.5), normal(M, N), normal(N, dtype=torch.float32)
    op = F.ficco_linear_t(M=M, K=K, N=N, activation=ACTS[kind], bias_type=F.FICCO_F32)
    pre, C = torch.empty(M, N, dtype=torch.bfloat16, device=gpu["dev"]), torch.empty(M, N, dtype=torch.bfloat16, device=gpu["dev"])
    forward(gpu, op, A, W, bias, None, pre, C)
    dA, dW, db = torch.empty_like(A), torch.empty_like(W), torch.empty(N, device=gpu["dev"])
    backward(gpu, op, A, W, pre, dC, dA, dW, db)

    def loss(a, w, b):
        return (dC.double() * act64(a @ w + b, kind)).sum()
    a, w, b = A.double(), W.double(), bias.double()
    for got, at in [(dA, lambda t, g: (a + t * g, w, b)), (dW, lambda t, g: (a, w + t * g, b)), (db, lambda t, g: (a, w, b + t * g))]:
        g = got.double()
        t = 1e-5 / g.abs().max()
        want = (loss(*at(t, g)) - loss(*at(-t, g))) / (2 * t)
        assert abs(want / g.norm() ** 2 - 1) <= 0.02, kind


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
def test_no_rows(gpu, kn):
    K, N = 128, 72
    op = F.ficco_linear_t(M=0, K=K, N=N, weight_layout=int(not kn), activation=F.FICCO_ACT_SILU)
    dW, db = torch.full((K, N) if kn else (N, K), 9.0, dtype=torch.bfloat16, device=gpu["dev"]), torch.full((N,), 9.0, device=gpu["dev"])
    F.ficco_linear(op, None, None, None, None, None, None, None, 0, gpu["cs"])
    torch.cuda.synchronize()
    F.ficco_linear_backward(op, None, None, None, None, None, dW, db, None, 0, gpu["cs"])
    torch.cuda.synchronize()
    assert (dW == 0).all() and (db == 0).all()


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("M", [2, 40, 700])
def test_what_is_not_finite_stays_in_its_row_and_column(gpu, M, kn):
    K, N = 192, 136
    normal = seeded(gpu, 17)
    A, W = normal(M, K), weight(normal, K, N, kn)
    A[0, 5] = float("nan")
    A[1, 70] = float("inf")
    bias = normal(N)
    bias[9] = float("-inf")
    op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=F.FICCO_ACT_RELU)
    C = torch.empty(M, N, dtype=torch.bfloat16, device=gpu["dev"])
    forward(gpu, op, A, W, bias, None, None, C)
    Wk = (W if kn else W.t()).double()
    ref = torch.relu(A.double() @ Wk + bias.double())
    assert torch.equal(torch.isnan(C), torch.isnan(ref)) and torch.equal(torch.isinf(C), torch.isinf(ref))
    assert torch.isnan(C[0]).all() and torch.isfinite(C[2:]).all()


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_slopes_of_large_values_are_0_and_1(gpu, kind):
    z = torch.tensor([[1e30, -1e30, 60.0, -60.0, 3e4, -3e4, 0.0, -0.0]], dtype=torch.bfloat16, device=gpu["dev"])
    A, W, dC = torch.ones(1, 64, dtype=torch.bfloat16, device=gpu["dev"]), torch.zeros(64, 8, dtype=torch.bfloat16, device=gpu["dev"]), torch.ones_like(z)
    db = torch.empty(8, device=gpu["dev"])
    backward(gpu, F.ficco_linear_t(M=1, K=64, N=8, activation=ACTS[kind]), A, W, z, dC, None, None, db)
    assert (db - torch.tensor([1, 0, 1, 0, 1, 0, 0.5, 0.5], device=gpu["dev"])).abs().max() <= 1e-6


def test_captured_calls_replay(gpu):
    """Forward and backward in one graph, replayed with new inputs and eager work between the replays."""
    M, K, N = 300, 256, 264
    normal = seeded(gpu, 23)
    A, W, bias, dC = normal(M, K), normal(K, N, std=K ** -0.5), normal(N), normal(M, N)
    op = F.ficco_linear_t(M=M, K=K, N=N, activation=F.FICCO_ACT_GELU_TANH)
    new = lambda: [torch.zeros(M, N, dtype=torch.bfloat16, device=gpu["dev"]), torch.zeros(M, N, dtype=torch.bfloat16, device=gpu["dev"]),  # noqa: E731
                   torch.zeros_like(A), torch.zeros_like(W), torch.zeros(N, device=gpu["dev"])]
    (ws, n), (wb, nb) = workspace(gpu, op, False), workspace(gpu, op, True)

    def step(out, stream):
        F.ficco_linear(op, A, W, bias, None, out[0], out[1], ws, n, stream)
        F.ficco_linear_backward(op, A, W, out[0], dC, out[2], out[3], out[4], wb, nb, stream)
    eager, replayed = new(), new()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(eager, stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(replayed, stream)
    for turn in range(4):
        A.copy_(normal(M, K))
        dC.copy_(normal(M, N))
        torch.cuda.synchronize()
        step(eager, stream)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager, replayed):
            assert torch.equal(x, y), turn


def test_refusals_on_the_device(gpu):
    t = torch.zeros(64 * 4096, dtype=torch.bfloat16, device=gpu["dev"])
    host = torch.zeros(64 * 64, dtype=torch.bfloat16)
    op = F.ficco_linear_t(M=64, K=64, N=64, weight_layout=F.FICCO_WEIGHT_NK)

    def refused(fn, *args):
        with pytest.raises(F.FiccoError) as e:
            fn(*args)
        assert e.value.status == F.FICCO_ERR_ARG
    for k in (1, 2, 6):
        args = [op, t, t, None, None, None, t, None, 0, gpu["cs"]]
        args[k] = host
        refused(F.ficco_linear, *args)
        args[k] = host.pin_memory()
        refused(F.ficco_linear, *args)
    # (buffers as large as the call says, should it be taken)
    big = F.ficco_linear_t(M=198, K=13440, N=2392)
    n = F.ficco_linear_workspace(big)
    assert n == 2 * 13440 * 2392
    A, W, C, ws = [torch.zeros(k, dtype=torch.bfloat16, device=gpu["dev"]) for k in (198 * 13440, 13440 * 2392, 198 * 2392, 13440 * 2392)]
    refused(F.ficco_linear, big, A, W, None, None, None, C, None, 0, gpu["cs"])
    refused(F.ficco_linear, big, A, W, None, None, None, C, ws, n - 1, gpu["cs"])
    refused(F.ficco_linear_backward, op, t, t, None, t, t, t, None, t, F.ficco_linear_workspace(op, True) - 1, gpu["cs"])


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("M,K,N", [(256, 256, 512), (512, 2048, 1024), (1024, 1152, 1544), (2048, 832, 2112), (4096, 512, 384), (8192, 64, 72), (128, 4096, 4096)])
def test_products_that_read_their_operands_as_they_are(gpu, M, K, N, kn):
    """Row counts that are whole k-tiles, at which dW reads A and dZ in place, and [K,N] weights large enough for the tiles that read
    them in place: forward, and backward with and without an activation."""
    normal = seeded(gpu, M + K * 3 + N)
    A, W, dC, z, bias = normal(M, K), weight(normal, K, N, kn), normal(M, N), normal(M, N, std=1.5), normal(N)
    Wk = (W if kn else W.t()).double()
    for kind in ("none", "gelu_tanh"):
        op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=ACTS[kind])
        C = torch.full((M + 1, N), 99.0, dtype=torch.bfloat16, device=gpu["dev"])
        print("ficco_linear", M, K, N, "kn" if kn else "nk", kind, flush=True)
        forward(gpu, op, A, W, bias, None, None, C)
        v = A.double() @ Wk + bias.double()
        ref = act64(v, kind)
        within(C[:M], ref, (U + 2 * E) * ref.abs() + 2.26 * (K + 2) * E * (A.double().abs() @ Wk.abs() + bias.double().abs()) + 4e-6 * v.abs(), f"C {kind}")
        assert (C[M] == 99).all()
        dA = torch.full((M + 1, K), 99.0, dtype=torch.bfloat16, device=gpu["dev"])
        dW = torch.full((W.shape[0] + 1, W.shape[1]), 99.0, dtype=torch.bfloat16, device=gpu["dev"])
        db = torch.empty(N, device=gpu["dev"])
        backward(gpu, op, A, W, None if kind == "none" else z, dC, dA, dW, db)
        dz = dC.double() if kind == "none" else dC.double() * slope64(z.double(), kind)
        rounded = 0 if kind == "none" else U
        wref, wsize = A.double().t() @ dz, A.double().t().abs() @ dz.abs()
        if not kn:
            wref, wsize = wref.t(), wsize.t()
        for name, got, ref, size, terms in [("dA", dA[:M], dz @ Wk.t(), dz.abs() @ Wk.t().abs(), N), ("dW", dW[:-1], wref, wsize, M)]:
            within(got, ref, U * ref.abs() + (rounded * 1.01 + 2 * (terms + 64) * E + 4e-6) * size, f"{name} {kind}")
            assert (got.double() - ref).norm() <= 3.4e-3 * ref.norm(), (name, kind)
        within(db, dz.sum(0), (M + 2) * E * dz.abs().sum(0) + 4e-6 * dC.double().abs().sum(0), f"dbias {kind}")
        assert (dA[M] == 99).all() and (dW[-1] == 99).all()
