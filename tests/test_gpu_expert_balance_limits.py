"""ficco_expert_balance at the largest number of tokens that its shape rule allows."""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

T = (1 << 31) - 1


@pytest.mark.parametrize("group", [0, 3 << 29], ids=["one", "short_last"])
def test_all_tokens_that_there_may_be(gpu, group):
    """2^31 - 1 tokens and two experts, a third of the tokens padding, in one group or in two, the second shorter and its last chunks
    empty. All logits are zero, so that a probability is 1/2 and sums of them are exact up to 2^23: the loss is coefficient * E / (2 k)
    to the 100 additions of each group's chunks, 100 e = 2^-17 of it. The gradient is s (c_e - n / 2) / 2 for every valid token, off by
    2^-16 of the counts' distance and one rounding to bf16; the counts themselves are whole numbers and equal."""
    dev = gpu["dev"]
    g = torch.Generator(device=dev)
    g.manual_seed(21)
    logits = torch.zeros(T, 2, dtype=torch.bfloat16, device=dev)
    valid, ids = torch.empty(T, dtype=torch.uint8, device=dev), torch.empty(T, 1, dtype=torch.int32, device=dev)
    step = 1 << 28
    for at in range(0, T, step):
        n = min(step, T - at)
        valid[at:at + n] = torch.rand(n, generator=g, device=dev) < 0.66
        ids[at:at + n, 0] = torch.rand(n, generator=g, device=dev) < 0.3
    valid[-1], ids[-1] = 1, 1
    size = group or T
    groups = -(-T // size)
    counts, n_valid = [[0, 0] for _ in range(groups)], [0] * groups
    for k in range(groups):
        for at in range(k * size, min((k + 1) * size, T), step):
            end = min(at + step, (k + 1) * size, T)
            v, one = valid[at:end] != 0, ids[at:end, 0] == 1
            n, ones = v.sum().item(), (v & one).sum().item()
            n_valid[k] += n
            counts[k][0] += n - ones
            counts[k][1] += ones
    op = F.ficco_expert_balance_t(tokens=T, group_tokens=group, experts=2, top_k=1, logits_type=F.FICCO_BF16, coefficient=0.5)
    got, got_n, loss = torch.full((groups + 1, 2), -7, dtype=torch.int32, device=dev), torch.full((groups + 1,), -7, dtype=torch.int32, device=dev), torch.full((1,), 9.0, device=dev)
    n = F.ficco_expert_balance_workspace(op)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    print("ficco_expert_balance", T, group, flush=True)
    F.ficco_expert_balance(op, logits, ids, valid, got, got_n, loss, ws, n, gpu["cs"])
    torch.cuda.synchronize()
    assert got.tolist() == counts + [[-7, -7]] and got_n.tolist() == n_valid + [-7]
    assert abs(loss.item() - 0.5) <= 2.0 ** -16 * 0.5
    print("ficco_expert_balance_backward", T, group, flush=True)
    F.ficco_expert_balance_backward(op, logits, valid, got, got_n, None, logits, gpu["cs"])
    torch.cuda.synchronize()
    for k in range(groups):
        s = 0.5 * 2 / (groups * n_valid[k] ** 2)
        for e in (0, 1):
            want = s * 0.5 * (counts[k][e] - n_valid[k] / 2)
            for at in range(k * size, min((k + 1) * size, T), step):
                end = min(at + step, (k + 1) * size, T)
                v, d = valid[at:end] != 0, logits[at:end, e].float()
                assert (d[~v] == 0).all()
                assert ((d[v] - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * abs(want)).all()
