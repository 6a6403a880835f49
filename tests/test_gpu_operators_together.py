"""The operators around the pair as a layer uses them, one behind the other on a stream without waiting in between: forward and
backward of a block between a reduce-scatter and the next gather, and a router in front of an expert-parallel dispatch."""
import numpy as np
import pytest

import ficco_inputs as fi
import paper_2512_10236_amd as F
from oracle import gemm as og
from oracle import grouped as ogr

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS = 1e-5


def rms(v):
    return v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)


class Layer:
    """y1 = x + gate norm(block), h = norm(y1), u = gelu(h W1 + b1), v = u W2 + b2, y2 = y1 + norm(v); `block` is what a reduce-scatter
    delivers. The residual stream is fp32, W1 is [K,N] and W2 [N,K]."""

    def __init__(self, gpu, T=96, D=512, H=1024, seed=1):
        g = torch.Generator(device=gpu["dev"])
        g.manual_seed(seed)
        n = lambda *s, std=1.0, mean=0.0, t=torch.bfloat16: (torch.randn(*s, generator=g, device=gpu["dev"]) * std + mean).to(t)  # noqa: E731
        f, b = torch.float32, torch.bfloat16
        self.T, self.D, self.H, dev = T, D, H, gpu["dev"]
        self.x, self.dy2 = n(T, D, t=f), n(T, D, t=f)
        self.p = dict(gate=n(D, std=0.3, mean=0.7, t=f), post1=n(D, std=0.1, mean=1.0, t=f), pre=n(D, std=0.1, mean=1.0, t=f), post2=n(D, std=0.1, mean=1.0, t=f),
                      W1=n(D, H, std=D ** -0.5), b1=n(H, std=0.3), W2=n(D, H, std=H ** -0.5), b2=n(D, std=0.3))
        e = lambda *s, t=b: torch.full(s, float("nan"), dtype=t, device=dev)  # noqa: E731
        self.block, self.y1, self.h, self.z, self.u, self.v, self.y2 = e(T, D), e(T, D, t=f), e(T, D), e(T, H), e(T, H), e(T, D), e(T, D, t=f)
        self.grad = {k: e(*v.shape, t=b if k in ("W1", "W2") else f) for k, v in self.p.items()}
        self.grad.update(x=e(T, D, t=f), block=e(T, D))
        self.dv, self.du, self.dh, self.dy1 = e(T, D), e(T, H), e(T, D), e(T, D, t=f)
        self.norm = F.ficco_residual_norm_t(rows=T, width=D, stream_type=F.FICCO_F32, param_type=F.FICCO_F32, residual_scale=1.0, eps=EPS)
        self.up = F.ficco_linear_t(M=T, K=D, N=H, activation=F.FICCO_ACT_GELU)
        self.down = F.ficco_linear_t(M=T, K=H, N=D, weight_layout=F.FICCO_WEIGHT_NK)
        self.bytes = max(16, F.ficco_residual_norm_workspace(self.norm), *[F.ficco_linear_workspace(o, k) for o in (self.up, self.down) for k in (False, True)])
        self.ws = torch.full((self.bytes,), 0xFF, dtype=torch.uint8, device=dev)

    def step(self, s):
        p, g, w = self.p, self.grad, (self.ws, self.bytes)
        F.ficco_residual_norm(self.norm, self.x, self.block, p["post1"], p["gate"], p["pre"], self.y1, self.h, s)
        F.ficco_linear(self.up, self.h, p["W1"], p["b1"], None, self.z, self.u, *w, s)
        F.ficco_linear(self.down, self.u, p["W2"], p["b2"], None, None, self.v, *w, s)
        F.ficco_residual_norm(self.norm, self.y1, self.v, p["post2"], None, None, self.y2, None, s)
        F.ficco_residual_norm_backward(self.norm, None, self.v, p["post2"], None, None, self.dy2, None, self.dy1, self.dv, g["post2"], None, None, *w, s)
        F.ficco_linear_backward(self.down, self.u, p["W2"], None, self.dv, self.du, g["W2"], g["b2"], *w, s)
        F.ficco_linear_backward(self.up, self.h, p["W1"], self.z, self.du, self.dh, g["W1"], g["b1"], *w, s)
        F.ficco_residual_norm_backward(self.norm, self.y1, self.block, p["post1"], p["gate"], p["pre"], self.dy1, self.dh, g["x"], g["block"], g["post1"], g["gate"], g["pre"], *w, s)

    def reference(self):
        v = {k: t.double().requires_grad_() for k, t in dict(self.p, x=self.x, block=self.block).items()}
        y1 = v["x"] + v["gate"] * rms(v["block"]) * v["post1"]
        z = (rms(y1) * v["pre"]) @ v["W1"] + v["b1"]
        y2 = y1 + rms((z * torch.special.ndtr(z)) @ v["W2"].t() + v["b2"]) * v["post2"]
        grads = torch.autograd.grad(y2, list(v.values()), self.dy2.double())
        return y2.detach(), dict(zip(v, grads))

    def outputs(self):
        return [self.y2, *self.grad.values()]


def test_a_block_between_reduce_scatter_and_gather(gpu):
    """Forward and backward in one go against automatic differentiation of the definition in 64 bits. On the longest way there are
    nine roundings to bf16, each off by 2^-8 / sqrt(3) of a 2-norm at most and independent, with gains of the norms and products
    around them below 2: 1.4e-2."""
    G, T, D = 4, 96, 512
    layer = Layer(gpu, T, D)
    parts = torch.from_numpy(fi.make_partials(5, G, T, D).view(np.int16)).to(gpu["dev"])
    landing = torch.empty_like(parts)
    torch.cuda.synchronize()
    plan = F.ficco_plan(G * T, 64, D, G, 2, F.FICCO_FINE_FUSED)
    try:
        F.ficco_rs_reduce(plan, 1, parts, landing, parts[1], layer.block, gpu["cs"])
        layer.step(gpu["cs"])
        F.ficco_query_stats(plan)
    finally:
        F.ficco_destroy(plan)
    torch.cuda.synchronize()
    assert torch.isfinite(layer.block).all()
    y2, grads = layer.reference()
    assert (layer.y2.double() - y2).norm() <= 1.4e-2 * y2.norm()
    for k, ref in grads.items():
        got = layer.grad[k].double()
        assert torch.isfinite(got).all() and (got - ref).norm() <= 1.4e-2 * ref.norm(), (k, ((got - ref).norm() / ref.norm()).item())


def test_two_layers_on_two_streams(gpu):
    """Two calls at a time, each with a workspace of its own, give what they give alone; so do graphs of both, replayed in turn."""
    layers = [Layer(gpu, 300, 768, 1536, seed=2), Layer(gpu, 128, 512, 1024, seed=3)]
    for k in layers:
        k.block.copy_(torch.randn_like(k.x))
    torch.cuda.synchronize()
    alone = []
    for k in layers:
        k.step(gpu["cs"])
        torch.cuda.synchronize()
        alone.append([t.clone() for t in k.outputs()])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for k in layers:
            for t in k.outputs():
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(5):
            for k, s in zip(layers, streams):
                k.step(s)
        torch.cuda.synchronize()
        for k, ref in zip(layers, alone):
            assert all(torch.equal(a, b) for a, b in zip(k.outputs(), ref)), turn
    graphs = []
    for k, s in zip(layers, streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            k.step(s)
    for turn in range(3):
        for k in layers:
            for t in k.outputs():
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for k, ref in zip(layers, alone):
            assert all(torch.equal(a, b) for a, b in zip(k.outputs(), ref)), turn


def test_a_router_in_front_of_a_dispatch(gpu):
    """Three peers' tokens, five experts, the best one of each: the counts are the dispatch's `rows`, and the rows of the dispatch that they
    describe come out multiplied by their own experts' weights."""
    dev, peers, E, K, N = gpu["dev"], 3, 5, 128, 72
    T = 200
    g = torch.Generator(device=dev)
    g.manual_seed(9)
    logits = torch.randn(peers * T, E, generator=g, device=dev) + torch.randn(E, generator=g, device=dev)
    ids = logits.argmax(1, keepdim=True).to(torch.int32)
    valid = torch.ones(peers * T, dtype=torch.uint8, device=dev)
    valid[T - 30:T] = 0                                   # the first peer's last tokens are padding
    op = F.ficco_expert_balance_t(tokens=peers * T, group_tokens=T, experts=E, top_k=1, logits_type=F.FICCO_F32, coefficient=1.0)
    counts, n, loss = torch.empty(peers, E, dtype=torch.int32, device=dev), torch.empty(peers, dtype=torch.int32, device=dev), torch.empty(1, device=dev)
    ws = torch.empty(max(16, F.ficco_expert_balance_workspace(op)), dtype=torch.uint8, device=dev)
    dlogits = torch.empty_like(logits)
    torch.cuda.synchronize()
    F.ficco_expert_balance(op, logits, ids, valid, counts, n, loss, ws, ws.numel(), gpu["cs"])
    F.ficco_expert_balance_backward(op, logits, valid, counts, n, None, dlogits, gpu["cs"])
    torch.cuda.synchronize()
    rows = counts.cpu().tolist()
    assert n.tolist() == [T - 30, T, T] and [sum(r) for r in rows] == n.tolist()
    # the loss falls along its gradient
    step = logits - 0.1 / dlogits.abs().max() * dlogits
    lower = torch.empty(1, device=dev)
    F.ficco_expert_balance(op, step, ids, valid, counts, n, lower, ws, ws.numel(), gpu["cs"])
    torch.cuda.synchronize()
    assert lower.item() < loss.item()
    # tokens in the dispatch's order: expert by expert, peer by peer
    A, W = fi.normal_bf16(3, fi.TENSOR_A, peers * T, K), np.stack([fi.normal_bf16(7 + e, fi.TENSOR_W, K, N, K ** -0.5) for e in range(E)])
    of, ok = ids.cpu().numpy()[:, 0], valid.cpu().numpy() != 0
    order = np.concatenate([np.flatnonzero((of == e) & ok & (np.arange(peers * T) // T == p)) for e in range(E) for p in range(peers)])
    A = np.ascontiguousarray(A[order])
    M = A.shape[0]
    A_src, W_dev = torch.from_numpy(A.view(np.int16)).to(dev), torch.from_numpy(W.view(np.int16)).to(dev)
    A_dev, C_dev = torch.empty_like(A_src), torch.empty(M, N, dtype=torch.int16, device=dev)
    torch.cuda.synchronize()
    plan = F.ficco_plan_grouped(K, N, rows, 1, F.FICCO_FINE_PERSISTENT)
    try:
        F.ficco_run(plan, A_src, A_dev, W_dev, C_dev, None, gpu["cs"], gpu["xs"])
        F.ficco_query_stats(plan)
    finally:
        F.ficco_destroy(plan)
    ref = ogr.grouped_gemm(A, W, np.asarray(rows).sum(axis=0))
    out = fi.bf16_bits_to_f32(C_dev.cpu().numpy().view(np.uint16)).astype(np.float64)
    assert og.rel_err(out, ref) <= 8e-3
