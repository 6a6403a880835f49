"""Equal calls of ficco_expert_balance and its backward give equal bits, wherever their buffers lie."""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def at(values, offset):
    """The same values, `offset` elements behind an aligned address, the rows as far apart as they were."""
    T, ld = values.shape
    out = torch.empty(T * ld + 8, dtype=values.dtype, device=values.device)[offset:offset + T * ld].view(T, ld)
    out.copy_(values)
    return out


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("experts,ld,group", [(5, 0, 0), (64, 0, 90), (128, 0, 0), (130, 0, 0), (132, 0, 500), (256, 0, 0), (256, 258, 0), (260, 300, 700), (512, 0, 0), (515, 0, 0), (1000, 0, 333), (1024, 0, 0)])
def test_bits_do_not_depend_on_where_a_buffer_lies(gpu, experts, ld, group, kind):
    T, dev = 1500, gpu["dev"]
    dtype, code = {"f32": (torch.float32, F.FICCO_F32), "bf16": (torch.bfloat16, F.FICCO_BF16)}[kind]
    g = torch.Generator(device=dev)
    g.manual_seed(experts + ld)
    logits = (torch.randn(T, ld or experts, generator=g, device=dev) * 2).to(dtype)
    ids = torch.randint(0, experts, (T, 4), generator=g, device=dev, dtype=torch.int32)
    valid = (torch.rand(T, generator=g, device=dev) < 0.8).to(torch.uint8)
    op = F.ficco_expert_balance_t(tokens=T, group_tokens=group, ld_logits=ld, experts=experts, top_k=4, logits_type=code, coefficient=0.25)
    n = F.ficco_expert_balance_workspace(op)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    groups = -(-T // (group or T))
    first = None
    for where, dwhere in ((0, 0), (1, 1), (2, 0), (0, 3), (4, 4)):
        x, out = at(logits, where), at(torch.zeros_like(logits), dwhere)
        counts, n_valid, loss = torch.empty(groups, experts, dtype=torch.int32, device=dev), torch.empty(groups, dtype=torch.int32, device=dev), torch.empty(1, device=dev)
        torch.cuda.synchronize()
        F.ficco_expert_balance(op, x, ids, valid, counts, n_valid, loss, ws, n, gpu["cs"])
        F.ficco_expert_balance_backward(op, x, valid, counts, n_valid, None, out, gpu["cs"])
        torch.cuda.synchronize()
        got = [counts, n_valid, loss, out[:, :experts].contiguous()]
        if first is None:
            first = got
            assert torch.isfinite(got[3]).all() and got[3].any()
        assert all(torch.equal(a, b) for a, b in zip(got, first)), (where, dwhere)
