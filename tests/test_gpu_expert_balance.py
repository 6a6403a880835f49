"""ficco_expert_balance and its backward against the definition in 64 bits. Counts are whole numbers and equal. With e = 2^-24: a
probability is off by (|x - max| + 6) e at most, from its exponent, its sum and a division, which for these logits is below
64 e; the loss is a sum of positive terms and off by that and the additions of up to 2000 in a row, 2^-12 in all. The gradient
is scale p (c - sum c p): off by 2^-16 of scale p (|c - mean| + sum |c - mean| p), and rounded once."""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, F.FICCO_F32, 2.0 ** -24), "bf16": (torch.bfloat16, F.FICCO_BF16, 2.0 ** -8)}


class Case:
    def __init__(self, gpu, tokens, experts, top_k, group=0, logits="f32", padded=False, ld=0, seed=0):
        g = torch.Generator(device=gpu["dev"])
        g.manual_seed(seed + tokens + experts)
        self.gpu, self.T, self.E, self.k, self.group, dev = gpu, tokens, experts, top_k, group or tokens, gpu["dev"]
        self.groups, self.type = -(-tokens // self.group), TYPES[logits]
        self.store = torch.full((tokens, ld or experts), 55.0, dtype=self.type[0], device=dev)
        self.logits = self.store[:, :experts]
        self.logits.copy_(torch.randn(tokens, experts, generator=g, device=dev) * 2)
        self.ids = torch.randint(0, experts, (tokens, top_k), generator=g, device=dev, dtype=torch.int32)
        self.valid = (torch.rand(tokens, generator=g, device=dev) < 0.7).to(torch.uint8) if padded else None
        self.op = F.ficco_expert_balance_t(tokens=tokens, group_tokens=group, ld_logits=ld, experts=experts, top_k=top_k, logits_type=self.type[1], coefficient=0.25)
        self.counts = torch.full((self.groups + 1, experts), -7, dtype=torch.int32, device=dev)
        self.group_valid = torch.full((self.groups + 1,), -7, dtype=torch.int32, device=dev)
        self.loss = torch.full((2,), 9.0, device=dev)

    def forward(self, loss=True):
        n = F.ficco_expert_balance_workspace(self.op)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=self.gpu["dev"]) if n else None
        torch.cuda.synchronize()
        F.ficco_expert_balance(self.op, self.logits if loss else None, self.ids, self.valid, self.counts, self.group_valid, self.loss if loss else None, ws, n, self.gpu["cs"])
        torch.cuda.synchronize()

    def backward(self, dloss=None, in_place=False):
        out = self.store if in_place else torch.full_like(self.store, 44.0)
        torch.cuda.synchronize()
        F.ficco_expert_balance_backward(self.op, self.logits, self.valid, self.counts, self.group_valid, dloss, out, self.gpu["cs"])
        torch.cuda.synchronize()
        return out

    def reference(self):
        """counts, valid tokens, loss, gradient, and the gradient's size of what is added, on the CPU."""
        T, E = self.T, self.E
        ids, valid = self.ids.cpu().long(), torch.ones(T, dtype=torch.bool) if self.valid is None else self.valid.cpu() != 0
        x = self.logits.cpu().double()
        p = torch.zeros(T, E, dtype=torch.float64)
        some = valid & (x > -torch.inf).any(1)
        p[some] = torch.softmax(x[some], 1)
        at = torch.arange(T) // self.group
        use = valid[:, None] & (ids >= 0) & (ids < E)
        flat = (at[:, None] * E + ids)[use]
        counts = torch.bincount(flat, minlength=self.groups * E).view(self.groups, E)
        n = torch.bincount(at[valid], minlength=self.groups)
        scale = 0.25 * E / (self.groups * self.k) / n.clamp(min=1).double() ** 2 * (n > 0)
        c = counts.double()[at]
        loss = ((p * c).sum(1) * scale[at]).sum()
        d = c - c.mean(1, keepdim=True)
        grad = scale[at][:, None] * p * (c - (p * c).sum(1, keepdim=True))
        size = scale[at][:, None] * p * (d.abs() + (p * d.abs()).sum(1, keepdim=True))
        return counts, n, loss, grad, size


def check(c, dloss=None):
    c.forward()
    counts, n, loss, grad, size = c.reference()
    assert torch.equal(c.counts[:-1].cpu().long(), counts) and (c.counts[-1] == -7).all()
    assert torch.equal(c.group_valid[:-1].cpu().long(), n) and c.group_valid[-1] == -7
    assert abs(c.loss[0].item() - loss.item()) <= 2.0 ** -12 * loss.item() and c.loss[1] == 9
    out = c.backward(dloss)
    up = 1.0 if dloss is None else dloss.item()
    got = out[:, :c.E].cpu().double()
    assert torch.isfinite(got).all()
    over = (got - up * grad).abs() - abs(up) * (c.type[2] * grad.abs() + 2.0 ** -16 * size) - 1e-38
    assert (over <= 0).all(), over.max().item()
    assert (out[:, c.E:] == 44).all()


@pytest.mark.parametrize("kind", [dict(tokens=1, experts=1, top_k=1), dict(tokens=64, experts=8, top_k=2), dict(tokens=63, experts=5, top_k=3, logits="bf16", padded=True),
                                  dict(tokens=1000, experts=16, top_k=1, group=7, padded=True), dict(tokens=777, experts=17, top_k=4, group=100, ld=24, logits="bf16"),
                                  dict(tokens=5000, experts=33, top_k=2, padded=True), dict(tokens=4096, experts=64, top_k=6, group=1024), dict(tokens=300, experts=65, top_k=8, group=1),
                                  dict(tokens=9001, experts=128, top_k=8, group=4000, padded=True, logits="bf16"), dict(tokens=20000, experts=256, top_k=8, group=5000, padded=True),
                                  dict(tokens=3001, experts=257, top_k=2, ld=300), dict(tokens=2500, experts=1000, top_k=64, padded=True), dict(tokens=40, experts=1024, top_k=1, group=3),
                                  dict(tokens=70000, experts=8, top_k=2), dict(tokens=5, experts=8, top_k=2, group=100)], ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_against_the_definition(gpu, kind):
    check(Case(gpu, **kind))


@pytest.mark.parametrize("experts", [6, 64, 200])
def test_masks_and_dropped_slots(gpu, experts):
    """Experts a token may not use, tokens with none left, groups without a valid token, ids outside the range, the same id in
    every slot, and logits of padding that are not numbers."""
    c = Case(gpu, 1200, experts, 3, group=100, padded=True, seed=5)
    c.logits[::3, 1:3] = float("-inf")
    c.logits[7] = float("-inf")
    c.valid[7] = 1
    c.logits[8] = torch.finfo(torch.float32).min
    c.valid[8] = 1
    c.valid[300:400] = 0
    c.logits[c.valid == 0] = float("nan")
    c.ids[::5, 1] = -1
    c.ids[1::5, 0] = experts
    c.ids[2::5, 2] = 2 ** 31 - 1
    c.ids[3::5] = c.ids[3::5, :1].clone()
    check(c, torch.tensor([-3.5], device=gpu["dev"]))
    out = c.backward()
    assert (out[c.valid == 0] == 0).all() and (out[7] == 0).all()


def test_what_is_not_a_number_shows(gpu):
    c = Case(gpu, 50, 12, 2)
    c.logits[4, 3] = float("nan")
    c.logits[9] = float("nan")
    c.forward()
    assert torch.isnan(c.loss[0])
    out = c.backward()
    rows = torch.isnan(out).all(1)
    assert rows[4] and rows[9] and not torch.isnan(out[[r for r in range(50) if r not in (4, 9)]]).any()


def test_even_routing_gives_the_coefficient(gpu):
    for experts, logits in [(8, "f32"), (96, "bf16")]:
        c = Case(gpu, experts * 20, experts, 1, logits=logits)
        c.logits.zero_()
        c.ids.copy_((torch.arange(c.T, device=gpu["dev"]) % experts).to(torch.int32)[:, None])
        c.forward()
        assert abs(c.loss[0].item() / 0.25 - 1) <= 1e-5
        assert (c.backward() == 0).all()


def test_counts_alone_and_gradient_in_place(gpu):
    c = Case(gpu, 3000, 40, 4, group=700, padded=True, ld=48)
    c.forward(loss=False)
    counts, n = c.counts.clone(), c.group_valid.clone()
    assert c.loss[0] == 9
    c.forward()
    assert torch.equal(c.counts, counts) and torch.equal(c.group_valid, n)
    out = c.backward()
    kept = c.store[:, 40:].clone()
    assert torch.equal(c.backward(in_place=True)[:, :40], out[:, :40]) and torch.equal(c.store[:, 40:], kept)


def test_no_tokens(gpu):
    op = F.ficco_expert_balance_t(tokens=0, experts=8, top_k=2, coefficient=1.0)
    loss = torch.full((1,), 9.0, device=gpu["dev"])
    F.ficco_expert_balance(op, None, None, None, None, None, loss, None, 0, gpu["cs"])
    F.ficco_expert_balance_backward(op, None, None, None, None, None, None, gpu["cs"])
    torch.cuda.synchronize()
    assert loss[0] == 0


def test_captured_calls_replay(gpu):
    for kind in (dict(tokens=100, experts=8, top_k=2), dict(tokens=6000, experts=64, top_k=4, group=1500)):
        c = Case(gpu, **kind)
        n, stream = F.ficco_expert_balance_workspace(c.op), torch.cuda.Stream()
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device=gpu["dev"])
        outs = lambda: [torch.empty_like(c.counts), torch.empty_like(c.group_valid), torch.zeros(1, device=gpu["dev"]), torch.empty_like(c.store)]  # noqa: E731

        def step(o):
            F.ficco_expert_balance(c.op, c.logits, c.ids, None, o[0], o[1], o[2], ws, n, stream)
            F.ficco_expert_balance_backward(c.op, c.logits, None, o[0], o[1], o[2], o[3], stream)
        eager, replayed = outs(), outs()
        for o in (eager, replayed):
            o[0].zero_(), o[1].zero_()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(replayed)
        for turn in range(4):
            c.store.normal_()
            c.ids.random_(0, c.E)
            torch.cuda.synchronize()
            step(eager)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, replayed)), turn


def test_refusals_on_the_device(gpu):
    c = Case(gpu, 6000, 64, 2)
    n = F.ficco_expert_balance_workspace(c.op)
    assert n > 0
    ws, host = torch.empty(n, dtype=torch.uint8, device=gpu["dev"]), torch.zeros(8)
    for args in [(c.logits, c.ids, None, c.counts, c.group_valid, c.loss, None, n), (c.logits, c.ids, None, c.counts, c.group_valid, c.loss, ws, n - 1),
                 (c.logits, c.ids, None, c.counts, c.group_valid, host, ws, n), (c.logits, c.ids, host, c.counts, c.group_valid, c.loss, ws, n)]:
        with pytest.raises(F.FiccoError) as e:
            F.ficco_expert_balance(c.op, *args, gpu["cs"])
        assert e.value.status == F.FICCO_ERR_ARG


def test_rows_whose_offsets_pass_32_bits(gpu):
    """2^32 values from the first row to the last; the last group's results are those of the group by itself, but for the share that
    a group has in the loss, a power of two here."""
    groups, size = 1024, 4096
    c = Case(gpu, groups * size, 64, 4, group=size, logits="bf16", ld=1024)
    c.forward()
    one = Case(gpu, size, 64, 4, logits="bf16")
    one.logits.copy_(c.logits[-size:])
    one.ids = c.ids[-size:].clone()
    one.op.coefficient /= groups
    one.forward()
    assert torch.equal(c.counts[groups - 1], one.counts[0]) and c.group_valid[groups - 1] == size
    assert torch.equal(c.backward(in_place=True)[-size:, :64], one.backward())
