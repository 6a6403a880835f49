"""ficco_residual_norm and ficco_residual_norm_backward against the definition in 64 bits.

Tolerances, with u = 2^-8 and e = 2^-24 as half a step of bf16 and fp32 relative to a value. A row's sum of D squares in fp32 is
off by at most (D / threads + 12) e of itself, its root's reciprocal by half of that and a few e: below 100 e for a row of 16384
over 64 threads or more. So n, y, h are off by 2^-16 of their largest part each (|s x| + |g n| for y, and h's own size, which
those change by the same share of y's parts), before the one rounding. Gradients likewise, of the sizes of the parts that are
added; sums over T rows add T e of the sum of sizes."""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, E, P = 2.0 ** -8, 2.0 ** -24, 2.0 ** -16
EPS = 1e-5


def rms(v):
    return torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)


class Case:
    def __init__(self, gpu, rows, width, gate_rows=0, gate=True, post=True, pre=True, stream="bf16", param="bf16", scale=0.75, seed=0):
        g = torch.Generator(device=gpu["dev"])
        g.manual_seed(seed + rows + width)
        types = {"bf16": torch.bfloat16, "f32": torch.float32}
        normal = lambda *s, std=1.0, mean=0.0, t=torch.bfloat16: (torch.randn(*s, generator=g, device=gpu["dev"]) * std + mean).to(t)  # noqa: E731
        self.gpu, self.rows, self.width, self.gate_rows, self.scale = gpu, rows, width, gate_rows, scale
        self.x, self.block = normal(rows, width, std=2.0, t=types[stream]), normal(rows, width)
        self.post = normal(width, std=0.2, mean=1.0, t=types[param]) if post else None
        self.pre = normal(width, std=0.2, mean=1.0, t=types[param]) if pre else None
        self.gate = normal(*((-(-rows // gate_rows), width) if gate_rows else (width,)), std=0.5, mean=0.5, t=types[param]) if gate else None
        self.dy, self.dh = normal(rows, width, t=types[stream]), normal(rows, width) if pre else None
        self.stream = types[stream]
        self.op = F.ficco_residual_norm_t(rows=rows, width=width, gate_rows=gate_rows, stream_type=int(stream == "f32"), param_type=int(param == "f32"), residual_scale=scale, eps=EPS)

    def half_step(self):
        return U if self.stream == torch.bfloat16 else E

    def row_gate(self):
        if self.gate is None:
            return torch.ones(1, 1, dtype=torch.float64, device=self.x.device)
        g = self.gate.double()
        return g[torch.arange(self.rows, device=g.device) // self.gate_rows] if self.gate_rows else g[None]

    def branch(self):
        b = self.block.double()
        return b if self.post is None else b * rms(b) * self.post.double()

    def forward(self, y=None, h=None):
        y = torch.full((self.rows + 1, self.width), 99.0, dtype=self.stream, device=self.x.device) if y is None else y
        h = torch.full((self.rows + 1, self.width), 98.0, dtype=torch.bfloat16, device=self.x.device) if h is None and self.pre is not None else h
        torch.cuda.synchronize()
        F.ficco_residual_norm(self.op, self.x, self.block, self.post, self.gate, self.pre, y, h, self.gpu["cs"])
        torch.cuda.synchronize()
        return y, h

    def backward(self, y, want="dx dblock dpost dgate dpre", dx=None):
        dev, out = self.x.device, {}
        shapes = {"dx": (self.rows + 1, self.width), "dblock": (self.rows + 1, self.width), "dpost": (self.width,), "dgate": self.gate.shape if self.gate is not None else None, "dpre": (self.width,)}
        has = {"dpost": self.post, "dgate": self.gate, "dpre": self.pre}
        for k in want.split():
            if k in has and has[k] is None:
                continue
            out[k] = torch.full(shapes[k], 97.0, dtype=self.stream if k == "dx" else torch.bfloat16 if k == "dblock" else torch.float32, device=dev)
        if dx is not None:
            out["dx"] = dx
        n = F.ficco_residual_norm_workspace(self.op)
        ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=dev)
        torch.cuda.synchronize()
        F.ficco_residual_norm_backward(self.op, y, self.block, self.post, self.gate, self.pre, self.dy, self.dh, *[out.get(k) for k in ("dx", "dblock", "dpost", "dgate", "dpre")], ws, n, self.gpu["cs"])
        torch.cuda.synchronize()
        return out


def within(got, ref, tol, what):
    assert torch.isfinite(got).all(), what
    over = (got.double() - ref).abs() - tol
    assert (over <= 0).all(), f"{what}: {over.max().item()} over"


CASES = [dict(rows=1, width=8), dict(rows=1, width=16384), dict(rows=3, width=264, stream="f32", param="f32"), dict(rows=7, width=512, gate_rows=1), dict(rows=130, width=520, gate_rows=64),
         dict(rows=33, width=1024, gate_rows=2, stream="f32"), dict(rows=371, width=1160, post=False, gate=False), dict(rows=50, width=2048, gate=False, param="f32"),
         dict(rows=1100, width=2056, pre=False, stream="f32"), dict(rows=77, width=4096, post=False, gate_rows=10, param="f32"), dict(rows=600, width=4104, stream="f32", param="f32", gate_rows=599),
         dict(rows=520, width=8192, gate_rows=130), dict(rows=9, width=8200, stream="f32"), dict(rows=300, width=16376, gate_rows=7, param="f32"), dict(rows=5000, width=64, gate_rows=3),
         dict(rows=9001, width=72, gate_rows=2000, stream="f32", param="f32"), dict(rows=700, width=512, post=False, gate=False, pre=False), dict(rows=4099, width=128, gate_rows=0, scale=-1.5),
         dict(rows=5, width=512, gate_rows=9), dict(rows=2500, width=1024, gate_rows=2500), dict(rows=2, width=520, gate_rows=1), dict(rows=3, width=2048, gate_rows=2),
         dict(rows=3, width=4096, stream="f32"), dict(rows=3, width=4104), dict(rows=2, width=64, gate=False, param="f32")]


@pytest.mark.parametrize("kind", CASES, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_forward(gpu, kind):
    c = Case(gpu, **kind)
    y, h = c.forward()
    n = c.row_gate() * c.branch()
    ref = c.scale * c.x.double() + n
    parts = (c.scale * c.x.double()).abs() + n.abs()
    within(y[:-1], ref, c.half_step() * ref.abs() + P * parts, "y")
    assert (y[-1] == 99).all()
    if h is not None:
        w, r = c.pre.double(), rms(ref)
        href = ref * r * w
        within(h[:-1], href, U * href.abs() + 2 * P * (parts * r * w.abs()), "h")
        assert (h[-1] == 98).all()


def gradients(c, y):
    """(value, size of what is added) of every gradient, in 64 bits."""
    dy, b, y, g = c.dy.double(), c.block.double(), y.double(), c.row_gate()
    size, out = dy.abs(), {}
    if c.dh is not None:
        r, dh = rms(y), c.dh.double()
        u, yh = c.pre.double() * dh, y * r
        m = (u * yh).mean(1, keepdim=True)
        out["dpre"] = ((dh * yh).sum(0), (dh * yh).abs().sum(0))
        dy = dy + r * (u - yh * m)
        size = size + r * (u.abs() + yh.abs() * (u * yh).abs().mean(1, keepdim=True))
    out["dx"] = (c.scale * dy, abs(c.scale) * size)
    n = c.branch()
    if c.gate is not None:
        each, sizes = dy * n, size * n.abs()
        if c.gate_rows:
            at = torch.arange(c.rows, device=y.device) // c.gate_rows
            zero = torch.zeros(c.gate.shape, dtype=torch.float64, device=y.device)
            out["dgate"] = (zero.index_add(0, at, each), zero.index_add(0, at, sizes))
        else:
            out["dgate"] = (each.sum(0), sizes.sum(0))
    d, size = dy * g, size * g.abs()
    if c.post is not None:
        r, w = rms(b), c.post.double()
        bh = b * r
        out["dpost"] = ((d * bh).sum(0), (size * bh.abs()).sum(0))
        d, size = r * (d * w - bh * (d * w * bh).mean(1, keepdim=True)), r * (size * w.abs() + bh.abs() * (size * w.abs() * bh.abs()).mean(1, keepdim=True))
    out["dblock"] = (d, size)
    return out


@pytest.mark.parametrize("kind", CASES, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_backward(gpu, kind):
    c = Case(gpu, **kind)
    y = c.x
    out = c.backward(y)
    for name, (ref, size) in gradients(c, y).items():
        got = out[name][:-1] if name in ("dx", "dblock") else out[name]
        half = c.half_step() if name == "dx" else U if name == "dblock" else E
        sums = 0 if name in ("dx", "dblock") else (c.rows + 2) * E
        within(got, ref, half * ref.abs() + (2 * P + sums) * size, name)
    assert (out["dx"][-1] == 97).all() and (out["dblock"][-1] == 97).all()


def test_gradients_are_those_of_differences(gpu):
    """Along each gradient the loss sum(y dy) + sum(h dh) of the forward's definition in 64 bits grows by its squared norm; y is
    given to the backward rounded to fp32, and dblock rounded to bf16."""
    c = Case(gpu, 40, 264, gate_rows=9, stream="f32", param="f32")
    leaves = {k: v.double() for k, v in (("dx", c.x), ("dblock", c.block), ("dpost", c.post), ("dgate", c.gate), ("dpre", c.pre))}
    at = torch.arange(c.rows, device=c.x.device) // c.gate_rows

    def loss(v):
        b = v["dblock"]
        y = c.scale * v["dx"] + v["dgate"][at] * b * rms(b) * v["dpost"]
        return (y * c.dy.double()).sum() + (y * rms(y) * v["dpre"] * c.dh.double()).sum()
    y, _ = c.forward()
    out = c.backward(y)
    for name in leaves:
        g = (out[name][:-1] if name in ("dx", "dblock") else out[name]).double()
        t = 1e-4 / g.abs().max()
        want = (loss({**leaves, name: leaves[name] + t * g}) - loss({**leaves, name: leaves[name] - t * g})) / (2 * t)
        assert abs(want / g.norm() ** 2 - 1) <= (U if name == "dblock" else 1e-4), name


def test_in_place_and_parts(gpu):
    c = Case(gpu, 90, 1032, gate_rows=20)
    y0, h0 = c.forward()
    whole = c.backward(y0)
    for name in whole:
        one = c.backward(y0, name)
        assert torch.equal(one[name], whole[name]), name
    dy = c.dy.clone()
    c.dy = dy
    assert torch.equal(c.backward(y0, "dblock dpost dgate dpre", dx=dy)["dx"], whole["dx"][:-1])
    x = c.x.clone()
    c.x = x
    assert torch.equal(c.forward(y=x)[0], y0[:-1])


def test_gradients_that_do_not_come(gpu):
    """No dy, or no dh with the norm in front of the next block there: the same as zeros."""
    c = Case(gpu, 60, 520, gate_rows=7)
    y, _ = c.forward()
    dy, dh = c.dy, c.dh
    c.dy = torch.zeros_like(dy)
    zeros = c.backward(y)
    c.dy = None
    none = c.backward(y)
    for k in zeros:
        assert torch.equal(zeros[k], none[k]), k
    c.dy, c.dh = dy, torch.zeros_like(dh)
    zeros = c.backward(y, "dx dblock dpost dgate")
    c.dh = None
    none = c.backward(None, "dx dblock dpost dgate")
    for k in zeros:
        assert torch.equal(zeros[k], none[k]), k


def test_rows_of_zeros_and_of_nothing_finite(gpu):
    """A row of zeros has a norm of zeros and finite gradients; what is not finite in one row stays in it, but for the sums over rows."""
    c = Case(gpu, 12, 520, gate=False)
    c.x[3] = 0
    c.block[3] = 0
    c.block[5, 7] = float("nan")
    c.x[6, 9] = float("inf")
    y, h = c.forward()
    assert (h[3] == 0).all() and (y[3] == 0).all()
    out = c.backward(y)
    for t in (y[:-1], h[:-1], out["dx"][:-1], out["dblock"][:-1]):
        rest = [r for r in range(12) if r not in (5, 6)]
        assert torch.isfinite(t[rest]).all()
    assert torch.isnan(h[5]).all() and torch.isnan(h[6, 9])


@pytest.mark.parametrize("width", [520, 8200])
def test_rows_of_zeros_with_a_tiny_eps(gpu, width):
    """1 / sqrt(eps) = 1e15 there, whose cube is past fp32's range; the gradients are dY = dy + r w dh and db = r p g dY."""
    c = Case(gpu, 6, width, stream="f32", param="f32")
    c.op.eps, r = 1e-30, 1e15
    c.x[3] = 0
    c.block[3] = 0
    y, h = c.forward()
    assert (h[3] == 0).all() and (y[3] == 0).all()
    out = c.backward(y)
    dy = c.dy[3].double() + r * c.pre.double() * c.dh[3].double()
    within(out["dx"][3], c.scale * dy, c.scale * (E + P) * (c.dy[3].abs().double() + r * (c.pre.double() * c.dh[3].double()).abs()), "dx")
    db = r * c.post.double() * c.gate.double() * dy
    within(out["dblock"][3], db, (U + 2 * P) * db.abs() + r * P * c.dy[3].abs().double(), "dblock")


def test_block_is_only_needed_for_what_it_takes_part_in(gpu):
    c = Case(gpu, 40, 264, gate_rows=7)
    y, _ = c.forward()
    whole, c.block = c.backward(y), None
    assert torch.equal(c.backward(y, "dx dpre")["dx"], whole["dx"]) and torch.equal(c.backward(y, "dpre")["dpre"], whole["dpre"])
    for want in ("dblock", "dpost", "dgate"):
        with pytest.raises(F.FiccoError) as e:
            c.backward(y, want)
        assert e.value.status == F.FICCO_ERR_ARG
    c = Case(gpu, 40, 264, gate_rows=7, post=False)
    y, _ = c.forward()
    whole, c.block = c.backward(y), None
    assert torch.equal(c.backward(y, "dx dblock")["dblock"], whole["dblock"])


def test_rows_whose_offsets_pass_32_bits(gpu):
    """2^31 values and some rows more: the last rows come out as by themselves."""
    rows, last = (1 << 18) + 12, 12
    c = Case(gpu, rows, 8192, gate=False)
    y, h = c.forward()
    out = c.backward(y, "dx dblock")
    small = Case(gpu, last, 8192, gate=False)
    small.post, small.pre = c.post, c.pre
    small.x, small.block, small.dy, small.dh = (t[rows - last:].clone() for t in (c.x, c.block, c.dy, c.dh))
    y1, h1 = small.forward()
    one = small.backward(y1, "dx dblock")
    for big, little in ((y, y1), (h, h1), (out["dx"], one["dx"]), (out["dblock"], one["dblock"])):
        assert torch.equal(big[rows - last:rows], little[:last])


def test_no_rows(gpu):
    for gate_rows in (0, 4):
        op = F.ficco_residual_norm_t(rows=0, width=64, gate_rows=gate_rows, residual_scale=1.0, eps=EPS)
        w = torch.ones(64, dtype=torch.bfloat16, device=gpu["dev"])
        sums = [torch.full((64,), 9.0, device=gpu["dev"]) for _ in range(3)]
        F.ficco_residual_norm(op, None, None, w, w, w, None, w, gpu["cs"])
        F.ficco_residual_norm_backward(op, None, None, w, w, w, None, None, None, None, *sums, None, 0, gpu["cs"])
        torch.cuda.synchronize()
        assert (sums[0] == 0).all() and (sums[2] == 0).all() and (sums[1] == (9 if gate_rows else 0)).all() and (w == 1).all()


def test_captured_calls_replay(gpu):
    c = Case(gpu, 400, 1024, gate_rows=100)
    (y, h), stream = c.forward(), torch.cuda.Stream()
    y, h = y[:-1], h[:-1]
    n = F.ficco_residual_norm_workspace(c.op)
    ws = torch.empty(n, dtype=torch.uint8, device=gpu["dev"])
    outs = lambda: [torch.empty_like(y), torch.empty_like(h), torch.empty_like(c.x), torch.empty_like(h), torch.empty(1024, device=gpu["dev"]), torch.empty(4, 1024, device=gpu["dev"]),  # noqa: E731
                    torch.empty(1024, device=gpu["dev"])]

    def step(o):
        F.ficco_residual_norm(c.op, c.x, c.block, c.post, c.gate, c.pre, o[0], o[1], stream)
        F.ficco_residual_norm_backward(c.op, o[0], c.block, c.post, c.gate, c.pre, c.dy, c.dh, *o[2:], ws, n, stream)
    eager, replayed = outs(), outs()
    torch.cuda.synchronize()
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(replayed)
    for turn in range(4):
        c.x.normal_()
        c.dh.normal_()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, replayed)), turn


def test_refusals_on_the_device(gpu):
    op = F.ficco_residual_norm_t(rows=8, width=64, residual_scale=1.0, eps=EPS)
    t, host = torch.zeros(4096, device=gpu["dev"]), torch.zeros(4096)
    for k in range(1, 8):
        args = [op, t, t, t, t, t, t, t, gpu["cs"]]
        args[k] = host
        with pytest.raises(F.FiccoError) as e:
            F.ficco_residual_norm(*args)
        assert e.value.status == F.FICCO_ERR_ARG
    n = F.ficco_residual_norm_workspace(op)
    with pytest.raises(F.FiccoError) as e:
        F.ficco_residual_norm_backward(op, t, t, t, t, t, t, t, t, t, t, t, t, t, n - 1, gpu["cs"])
    assert e.value.status == F.FICCO_ERR_ARG
