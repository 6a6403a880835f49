"""Operands at addresses that have the alignment the interface asks for and no more give the bits that aligned ones give."""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def moved(x, elements):
    """The same values `elements` of theirs behind an aligned address."""
    out = torch.empty(x.numel() + 32, dtype=x.dtype, device=x.device)[elements:elements + x.numel()].view(x.shape)
    return out.copy_(x)


@pytest.mark.parametrize("kn", [True, False], ids=["kn", "nk"])
@pytest.mark.parametrize("bias_type", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(3, 128, 136), (700, 256, 520)])
def test_linear(gpu, M, K, N, bias_type, kn):
    dev = gpu["dev"]
    g = torch.Generator(device=dev)
    g.manual_seed(M)
    n = lambda *s, t=torch.bfloat16: torch.randn(*s, generator=g, device=dev).to(t)  # noqa: E731
    A, W, dC, bias = n(M, K), n(K, N) if kn else n(N, K), n(M, N), n(N, t=bias_type)
    op = F.ficco_linear_t(M=M, K=K, N=N, weight_layout=int(not kn), activation=F.FICCO_ACT_SILU, bias_type=int(bias_type == torch.float32))
    nf, nb = F.ficco_linear_workspace(op), F.ficco_linear_workspace(op, True)
    ws = torch.empty(max(nf, nb, 16), dtype=torch.uint8, device=dev)
    results = []
    for off in (0, 1, 3):
        # matrices stay at 16 bytes, 8 elements further
        a, w, d, b = moved(A, 8 * off), moved(W, 8 * off), moved(dC, 8 * off), moved(bias, off)
        C, pre, dA, dW, db = moved(torch.zeros_like(dC), 8 * off), moved(torch.zeros_like(dC), 0), moved(torch.zeros_like(A), 0), moved(torch.zeros_like(W), 8), moved(torch.zeros(N, device=dev), off)
        torch.cuda.synchronize()
        F.ficco_linear(op, a, w, b, None, pre, C, ws, nf, gpu["cs"])
        F.ficco_linear_backward(op, a, w, pre, d, dA, dW, db, ws, nb, gpu["cs"])
        torch.cuda.synchronize()
        results.append([C, pre, dA, dW, db])
    assert all(torch.equal(x, y) for r in results[1:] for x, y in zip(r, results[0]))


@pytest.mark.parametrize("experts", [6, 256])
def test_balance(gpu, experts):
    dev, T = gpu["dev"], 5000
    g = torch.Generator(device=dev)
    g.manual_seed(experts)
    logits = torch.randn(T, experts, generator=g, device=dev)
    ids = torch.randint(0, experts, (T, 3), generator=g, device=dev, dtype=torch.int32)
    valid = (torch.rand(T, generator=g, device=dev) < 0.7).to(torch.uint8)
    op = F.ficco_expert_balance_t(tokens=T, group_tokens=1700, experts=experts, top_k=3, logits_type=F.FICCO_F32, coefficient=0.5)
    n = F.ficco_expert_balance_workspace(op)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    results = []
    for off in (0, 1, 3):
        x, i, v, up = moved(logits, off), moved(ids, off), moved(valid, off), moved(torch.full((1,), 2.0, device=dev), off)
        counts, group_valid, loss = moved(torch.zeros(3, experts, dtype=torch.int32, device=dev), off), moved(torch.zeros(3, dtype=torch.int32, device=dev), off), moved(torch.zeros(1, device=dev), off)
        out = moved(torch.zeros_like(logits), off)
        torch.cuda.synchronize()
        F.ficco_expert_balance(op, x, i, v, counts, group_valid, loss, ws, n, gpu["cs"])
        F.ficco_expert_balance_backward(op, x, v, counts, group_valid, up, out, gpu["cs"])
        torch.cuda.synchronize()
        results.append([counts, group_valid, loss, out])
    assert all(torch.equal(x, y) for r in results[1:] for x, y in zip(r, results[0]))
