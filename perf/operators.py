"""The operators around the pair: their plain forms, and the calls a program makes of the library's.

A case is a dict of plain values; `op` says which operator it goes through:
  linear            C = act(A W + bias) + residual, operands in place (ficco_linear), `pre` = the value in front of the
                    activation is stored for the backward pass
  linear_backward   dA, dW and dbias from dC and the stored value (ficco_linear_backward)
  norm              y = scale x + gate norm(block) and h = norm(y): what stands between one block of a layer and the next
                    (ficco_residual_norm); `post` / `pre` / `gate`: which of the norms and the gate there are
  norm_backward     the gradients of all of its inputs (ficco_residual_norm_backward)
  balance           counts of tokens per expert and the balance loss (ficco_expert_balance), with `grad` the gradient of the
                    router's logits as well (ficco_expert_balance_backward)

Matrices are bf16; activations N(0,1), weights N(0,1/K), so that outputs have unit variance. The weight of a linear case is
[K,N] (`layout` "kn") or [N,K] ("nk") and is taken as it is by every pass.
"""
import math
import random

import torch

own = False

# The largest products and the largest streams listed below; drawn cases stay under them.
MOST_FLOPS = 2 * 16384 * 8192 * 3584
MOST_ROWS = 16384 * 4096


def listed():
    return [
        # one token of a decode step through a QKV share of an 8B-class model at TP=8
        dict(name="linear_token", op="linear", M=1, K=4096, N=768, layout="nk", activation="silu", bias="bf16", residual=False, pre=False),
        # a decode batch through the same share, the weight as the library's other entry points take it
        dict(name="linear_batch", op="linear", M=64, K=4096, N=768, layout="kn", activation="none", bias="bf16", residual=True, pre=False),
        # odd token count, column and k extents that fill no tile
        dict(name="linear_ragged", op="linear", M=8 * 371, K=2880, N=1160, layout="nk", activation="gelu", bias="f32", residual=True, pre=False),
        # FFN-up share of a 70B-class model at TP=8, the benchmark's default, in a training step's forward pass
        dict(name="linear_ffn", op="linear", M=16384, K=8192, N=3584, layout="kn", activation="gelu_tanh", bias="bf16", residual=False, pre=True),
        # the backward pass of the same layer over half as many tokens
        dict(name="linear_backward_ffn", op="linear_backward", M=8192, K=8192, N=3584, layout="kn", activation="gelu_tanh"),
        # ... and of a small one of odd extents
        dict(name="linear_backward_ragged", op="linear_backward", M=1187, K=2880, N=1160, layout="nk", activation="silu"),
        # a decode batch of eight rows between two blocks, both norms
        dict(name="norm_batch", op="norm", rows=8, width=8192, gate_rows=0, gate=False, post=True, pre=True, stream="bf16", param="bf16", scale=1.0),
        # the row block that a GPU owns behind a reduce-scatter of 16384 tokens over eight, residual stream in fp32
        dict(name="norm_block", op="norm", rows=2048, width=8192, gate_rows=0, gate=True, post=True, pre=True, stream="f32", param="f32", scale=0.75),
        # a training step: all gradients, a gate for each sequence of 2048 tokens
        dict(name="norm_backward", op="norm_backward", rows=16384, width=4096, gate_rows=2048, gate=True, post=True, pre=True, stream="bf16", param="f32", scale=1.0),
        # ... with an odd number of rows and a narrow width, only the norm in front of the next block
        dict(name="norm_backward_ragged", op="norm_backward", rows=8 * 371, width=1160, gate_rows=0, gate=False, post=False, pre=True, stream="f32", param="f32", scale=1.0),
        # the router of a decode batch
        dict(name="balance_batch", op="balance", tokens=64, experts=8, top_k=2, group=0, logits="f32", padded=False, grad=False),
        # a training batch of 16 sequences, many experts, sequences padded at their ends
        dict(name="balance_train", op="balance", tokens=65536, experts=256, top_k=8, group=4096, logits="f32", padded=True, grad=True),
    ]


def _log(rng, low, high):
    return math.exp(rng.uniform(math.log(low), math.log(high)))


def _step(rng, low, high, steps):
    step = rng.choice(steps)
    return max(step, int(_log(rng, low, high)) // step * step)


def draw(rng):
    while True:
        op = rng.choice(["linear", "linear", "linear_backward", "norm", "norm_backward", "balance"])
        if op in ("linear", "linear_backward"):
            c = dict(op=op, M=_step(rng, 1, 16384, [1, 1, 64]), K=_step(rng, 512, 16384, [64]), N=_step(rng, 64, 14336, [8, 64]), layout=rng.choice(["kn", "nk"]),
                     activation=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]))
            if op == "linear":
                c.update(bias=rng.choice(["none", "bf16", "f32"]), residual=rng.random() < 0.5, pre=c["activation"] != "none" and rng.random() < 0.5)
            if work(c)["flops"] <= MOST_FLOPS and c["K"] * c["N"] <= 1 << 26:
                return c
        elif op in ("norm", "norm_backward"):
            c = dict(op=op, rows=_step(rng, 1, 16384, [1, 1, 64]), width=_step(rng, 64, 16384, [8, 64]), gate_rows=0, gate=rng.random() < 0.6, post=rng.random() < 0.6,
                     pre=True, stream=rng.choice(["bf16", "f32"]), param=rng.choice(["bf16", "f32"]), scale=rng.choice([1.0, 0.75, 1.5]))
            if c["gate"] and rng.random() < 0.5:
                c["gate_rows"] = max(1, c["rows"] // rng.choice([1, 2, 3, 8, 16]))
            if c["rows"] * c["width"] <= MOST_ROWS:
                return c
        else:
            E = int(_log(rng, 4, 512))
            c = dict(op=op, tokens=int(_log(rng, 1, 65536)), experts=E, top_k=rng.randint(1, min(8, E)), group=0, logits=rng.choice(["bf16", "f32"]),
                     padded=rng.random() < 0.5, grad=rng.random() < 0.6)
            if rng.random() < 0.5:
                c["group"] = max(1, c["tokens"] // rng.choice([1, 2, 3, 8, 16]))
            if c["tokens"] * E <= 65536 * 256:
                return c


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once, the products' flops."""
    op = case["op"]
    if op in ("linear", "linear_backward"):
        M, K, N = case["M"], case["K"], case["N"]
        if op == "linear":
            return {"bytes": 2 * (M * K + K * N + M * N * (1 + case["residual"] + case["pre"])), "flops": 2 * M * K * N}
        # the value in front of the activation is not needed where there is no activation
        return {"bytes": 2 * (2 * M * K + 2 * K * N + M * N * (1 + (case["activation"] != "none"))), "flops": 4 * M * K * N}
    if op in ("norm", "norm_backward"):
        n, s = case["rows"] * case["width"], 2 if case["stream"] == "bf16" else 4
        if op == "norm":
            return {"bytes": n * (2 * s + 2 + 2 * case["pre"]), "flops": 10 * n}
        # dy, y, dx; block and its gradient (block is read only where a norm or a gate needs it); dh
        return {"bytes": n * (3 * s + 2 + 2 * (case["post"] or case["gate"]) + 2 * case["pre"]), "flops": 30 * n}
    n, s = case["tokens"] * case["experts"], 2 if case["logits"] == "bf16" else 4
    return {"bytes": n * s * (3 if case["grad"] else 1) + case["tokens"] * (4 * case["top_k"] + case["padded"]), "flops": n * (12 if case["grad"] else 6)}


# ---------------------------------------------------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g, device=dev) * std + mean).to(dtype)

    op = case["op"]
    s = {"case": case}
    if op in ("linear", "linear_backward"):
        M, K, N = case["M"], case["K"], case["N"]
        s["A"] = normal(M, K)
        s["W"] = normal(K, N, std=K ** -0.5) if case["layout"] == "kn" else normal(N, K, std=K ** -0.5)
        if op == "linear":
            s["bias"] = None if case["bias"] == "none" else normal(N, std=0.5, dtype=_TYPES[case["bias"]])
            s["residual"] = normal(M, N) if case["residual"] else None
        else:
            s["z"] = None if case["activation"] == "none" else normal(M, N)
            s["dC"] = normal(M, N)
    elif op in ("norm", "norm_backward"):
        T, D = case["rows"], case["width"]
        stream, param = _TYPES[case["stream"]], _TYPES[case["param"]]
        gates = (-(-T // case["gate_rows"]),) if case["gate_rows"] else ()
        s["block"] = normal(T, D)
        s["post"] = normal(D, std=0.1, mean=1.0, dtype=param) if case["post"] else None
        s["gate"] = normal(*gates, D, std=0.5, mean=0.5, dtype=param) if case["gate"] else None
        s["pre"] = normal(D, std=0.1, mean=1.0, dtype=param) if case["pre"] else None
        if op == "norm":
            s["x"] = normal(T, D, std=2.0, dtype=stream)
        else:
            s["y"] = normal(T, D, std=2.0, dtype=stream)
            s["dy"] = normal(T, D, dtype=stream)
            s["dh"] = normal(T, D) if case["pre"] else None
    else:
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        # some experts are preferred, as they are before a balance loss has done its work
        s["logits"] = (torch.randn(T, E, generator=g, device=dev) + 0.5 * torch.randn(E, generator=g, device=dev)).to(_TYPES[case["logits"]])
        s["ids"] = torch.topk(s["logits"].float() + torch.randn(T, E, generator=g, device=dev), k, dim=1).indices.to(torch.int32)
        group = case["group"] or T
        s["valid"] = None
        if case["padded"]:      # the last tokens of a sequence are padding, up to half of them
            used = torch.rand(-(-T // group), generator=g, device=dev) * 0.5 + 0.5
            at = torch.arange(T, device=dev)
            s["valid"] = (at % group < (used[at // group] * group)).to(torch.uint8)
        s["dloss"] = torch.full((1,), 1.0, device=dev)
    return s


COEFFICIENT, EPS = 0.01, 1e-6


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2512_10236_amd as F
    s["F"] = F
    op, dev = case["op"], torch.device("cuda")
    types = {"bf16": F.FICCO_BF16, "f32": F.FICCO_F32}
    if op in ("linear", "linear_backward"):
        M, K, N = case["M"], case["K"], case["N"]
        s["op"] = F.ficco_linear_t(M=M, K=K, N=N, weight_layout={"kn": F.FICCO_WEIGHT_KN, "nk": F.FICCO_WEIGHT_NK}[case["layout"]],
                                   activation=getattr(F, "FICCO_ACT_" + case["activation"].upper()), bias_type=types.get(case.get("bias"), F.FICCO_BF16))
        if op == "linear":
            s["C"] = torch.empty(M, N, dtype=torch.bfloat16, device=dev)
            s["z"] = torch.empty_like(s["C"]) if case["pre"] else None
        else:
            s["dA"], s["dW"], s["dbias"] = torch.empty_like(s["A"]), torch.empty_like(s["W"]), torch.empty(N, device=dev)
        s["bytes"] = F.ficco_linear_workspace(s["op"], op == "linear_backward")
    elif op in ("norm", "norm_backward"):
        s["op"] = F.ficco_residual_norm_t(rows=case["rows"], width=case["width"], gate_rows=case["gate_rows"], stream_type=types[case["stream"]],
                                          param_type=types[case["param"]], residual_scale=case["scale"], eps=EPS)
        s["bytes"] = 0
        if op == "norm":
            s["out_y"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["block"]) if case["pre"] else None
        else:
            s["dx"], s["dblock"] = torch.empty_like(s["y"]), torch.empty_like(s["block"])
            s["dparams"] = [torch.empty_like(s[p], dtype=torch.float32) if s[p] is not None else None for p in ("post", "gate", "pre")]
            s["bytes"] = F.ficco_residual_norm_workspace(s["op"])
    else:
        groups = -(-case["tokens"] // (case["group"] or case["tokens"]))
        s["op"] = F.ficco_expert_balance_t(tokens=case["tokens"], group_tokens=case["group"], experts=case["experts"], top_k=case["top_k"],
                                           logits_type=types[case["logits"]], coefficient=COEFFICIENT)
        s["counts"] = torch.empty(groups, case["experts"], dtype=torch.int32, device=dev)
        s["group_valid"] = torch.empty(groups, dtype=torch.int32, device=dev)
        s["loss"] = torch.empty(1, device=dev)
        s["dlogits"] = torch.empty_like(s["logits"]) if case["grad"] else None
        s["bytes"] = F.ficco_expert_balance_workspace(s["op"])
    s["workspace"] = torch.empty(s["bytes"], dtype=torch.uint8, device=dev) if s["bytes"] else None
    return s


# ------------------------------------------------------------------------------------------------------ plain forms
def _act(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return z.clamp_min(0)
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z))


def _act_slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if kind == "gelu_tanh":
        t = torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (2 / math.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    e = 1 / (1 + torch.exp(-z))
    return e * (1 + z * (1 - e))


def _plain_linear(s):
    c = s["case"]
    W = s["W"].float()
    z = s["A"].float() @ (W if c["layout"] == "kn" else W.t())
    if s["bias"] is not None:
        z = z + s["bias"].float()
    C = _act(z, c["activation"])
    if s["residual"] is not None:
        C = C + s["residual"].float()
    return {"C": C.bfloat16(), "pre": z.bfloat16() if c["pre"] else None}


def _plain_linear_backward(s):
    c = s["case"]
    A, W, dz = s["A"].float(), s["W"].float(), s["dC"].float()
    if c["activation"] != "none":
        dz = dz * _act_slope(s["z"].float(), c["activation"])
    kn = c["layout"] == "kn"
    dA = dz @ (W.t() if kn else W)
    dW = A.t() @ dz if kn else dz.t() @ A
    return {"dA": dA.bfloat16(), "dW": dW.bfloat16(), "dbias": dz.sum(0)}


def _rows_of_gate(s):
    """The gate of every row, in 32 bits, or 1."""
    c, g = s["case"], s["gate"]
    if g is None:
        return 1.0
    return g.float().repeat_interleave(c["gate_rows"], 0)[:c["rows"]] if c["gate_rows"] else g.float()


def _plain_norm(s):
    c, b = s["case"], s["block"].float()
    if s["post"] is not None:
        b = b * torch.rsqrt((b * b).mean(1, keepdim=True) + EPS) * s["post"].float()
    y = c["scale"] * s["x"].float() + _rows_of_gate(s) * b
    h = (y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * s["pre"].float()).bfloat16() if s["pre"] is not None else None
    return {"y": y.to(s["x"].dtype), "h": h}


def _plain_norm_backward(s):
    c, b, y, gate = s["case"], s["block"].float(), s["y"].float(), _rows_of_gate(s)
    out = {"dpost": None, "dgate": None, "dpre": None}
    dy = s["dy"].float()
    if s["pre"] is not None:
        dh, r = s["dh"].float(), torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
        yh = y * r
        out["dpre"] = (dh * yh).sum(0)
        u = dh * s["pre"].float()
        dy = dy + r * (u - yh * (u * yh).mean(1, keepdim=True))
    if s["post"] is not None:
        r = torch.rsqrt((b * b).mean(1, keepdim=True) + EPS)
        bh, w = b * r, s["post"].float()
        n = bh * w
    else:
        n = b
    if s["gate"] is not None:
        dg = dy * n
        if c["gate_rows"]:
            groups = s["gate"].shape[0]
            dg = torch.nn.functional.pad(dg, (0, 0, 0, groups * c["gate_rows"] - c["rows"])).view(groups, c["gate_rows"], -1)
            out["dgate"] = dg.sum(1)
        else:
            out["dgate"] = dg.sum(0)
    dn = dy * gate
    if s["post"] is not None:
        out["dpost"] = (dn * bh).sum(0)
        u = dn * w
        dn = r * (u - bh * (u * bh).mean(1, keepdim=True))
    return {"dx": (c["scale"] * dy).to(s["y"].dtype), "dblock": dn.bfloat16(), **out}


def _plain_balance(s):
    c = s["case"]
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    group = c["group"] or T
    groups = -(-T // group)
    valid = s["valid"].float() if s["valid"] is not None else torch.ones(T, device=s["logits"].device)
    of = torch.arange(T, device=valid.device) // group
    flat = (of[:, None] * E + s["ids"]).reshape(-1)
    counts = torch.zeros(groups * E, device=valid.device).index_add_(0, flat, valid[:, None].expand(T, k).reshape(-1)).view(groups, E)
    n = torch.zeros(groups, device=valid.device).index_add_(0, of, valid)
    # products and sums of probabilities with counts in 64 bits: what is left of them is small next to their parts
    p = torch.exp(s["logits"].double() - s["logits"].double().amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True) * valid[:, None]
    per = COEFFICIENT * E / (groups * k) / torch.clamp_min(n, 1).double() ** 2
    weighted = (p * counts.double()[of]).sum(1)
    loss = (weighted * per[of]).sum().float().reshape(1)
    out = {"counts": counts.to(torch.int32), "valid": n.to(torch.int32), "loss": loss}
    if c["grad"]:
        d = p * (counts.double()[of] - weighted[:, None]) * per[of][:, None] * s["dloss"]
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "norm": _plain_norm, "norm_backward": _plain_norm_backward, "balance": _plain_balance}[op](s)
    F, stream, work_, size = s["F"], torch.cuda.current_stream(), s["workspace"], s["bytes"]
    if op == "linear":
        F.ficco_linear(s["op"], s["A"], s["W"], s["bias"], s["residual"], s["z"], s["C"], work_, size, stream)
        return {"C": s["C"], "pre": s["z"]}
    if op == "linear_backward":
        F.ficco_linear_backward(s["op"], s["A"], s["W"], s["z"], s["dC"], s["dA"], s["dW"], s["dbias"], work_, size, stream)
        return {"dA": s["dA"], "dW": s["dW"], "dbias": s["dbias"]}
    if op == "norm":
        F.ficco_residual_norm(s["op"], s["x"], s["block"], s["post"], s["gate"], s["pre"], s["out_y"], s["h"], stream)
        return {"y": s["out_y"], "h": s["h"]}
    if op == "norm_backward":
        dpost, dgate, dpre = s["dparams"]
        F.ficco_residual_norm_backward(s["op"], s["y"], s["block"], s["post"], s["gate"], s["pre"], s["dy"], s["dh"], s["dx"], s["dblock"], dpost, dgate, dpre, work_, size, stream)
        return {"dx": s["dx"], "dblock": s["dblock"], "dpost": dpost, "dgate": dgate, "dpre": dpre}
    F.ficco_expert_balance(s["op"], s["logits"], s["ids"], s["valid"], s["counts"], s["group_valid"], s["loss"], work_, size, stream)
    out = {"counts": s["counts"], "valid": s["group_valid"], "loss": s["loss"]}
    if c["grad"]:
        F.ficco_expert_balance_backward(s["op"], s["logits"], s["valid"], s["counts"], s["group_valid"], s["dloss"], s["dlogits"], stream)
        out["dlogits"] = s["dlogits"]
    return out


# --------------------------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    """The same outputs from the definitions in 64 bits. Gradients come from automatic differentiation of the forward
    definition, not from the formulas of the plain forms."""
    s = _inputs(case, seed)
    d = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    op = case["op"]

    def activation(z):
        kind = case["activation"]
        if kind == "relu":
            return torch.where(z > 0, z, torch.zeros_like(z))
        if kind == "gelu":
            return z * torch.special.ndtr(z)
        if kind == "gelu_tanh":
            return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        if kind == "silu":
            return z * torch.sigmoid(z)
        return z

    if op == "linear":
        W = d["W"] if case["layout"] == "kn" else d["W"].t()
        z = torch.mm(d["A"], W)
        if d["bias"] is not None:
            z += d["bias"]
        C = activation(z)
        if d["residual"] is not None:
            C = C + d["residual"]
        return {"C": C, "pre": z if case["pre"] else None}
    if op == "linear_backward":
        if d["z"] is not None:
            z = d["z"].requires_grad_()
            dz, = torch.autograd.grad(activation(z), z, d["dC"])
        else:
            dz = d["dC"]
        if case["layout"] == "kn":
            return {"dA": torch.mm(dz, d["W"].t()), "dW": torch.mm(d["A"].t(), dz), "dbias": torch.sum(dz, 0)}
        return {"dA": torch.mm(dz, d["W"]), "dW": torch.mm(dz.t(), d["A"]), "dbias": torch.sum(dz, 0)}

    def rms(v):
        return v / torch.sqrt(torch.mean(v ** 2, dim=1, keepdim=True) + EPS)

    if op in ("norm", "norm_backward"):
        rows = torch.arange(case["rows"], device="cuda")
        row_gate = (lambda g: 1.0 if g is None else g[rows // case["gate_rows"]] if case["gate_rows"] else g[None, :])
        branch = lambda b, post, gate: row_gate(gate) * (b if post is None else rms(b) * post)  # noqa: E731
        if op == "norm":
            y = case["scale"] * d["x"] + branch(d["block"], d["post"], d["gate"])
            return {"y": y, "h": None if d["pre"] is None else rms(y) * d["pre"]}
        # y is an input of the backward pass: its own gradient first, then the branch's with that
        out = {"dpost": None, "dgate": None, "dpre": None}
        dy = d["dy"]
        if d["pre"] is not None:
            y, w = d["y"].requires_grad_(), d["pre"].requires_grad_()
            gy, out["dpre"] = torch.autograd.grad(rms(y) * w, [y, w], d["dh"])
            dy = dy + gy
        leaves = {k: d[n].requires_grad_() for k, n in (("dblock", "block"), ("dpost", "post"), ("dgate", "gate")) if d[n] is not None}
        grads = torch.autograd.grad(branch(d["block"], d["post"], d["gate"]) + torch.zeros_like(dy), list(leaves.values()), dy)
        out.update(zip(leaves, grads))
        return {"dx": case["scale"] * dy, **out}
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    group = case["group"] or T
    groups = -(-T // group)
    device = s["logits"].device
    valid = torch.ones(T, dtype=torch.bool, device=device) if s["valid"] is None else s["valid"].bool()
    lines = torch.arange(T, device=device) // group
    where = (lines[:, None] * E + s["ids"].long())[valid].reshape(-1)
    counts = torch.bincount(where, minlength=groups * E).view(groups, E)
    n = torch.bincount(lines[valid], minlength=groups)
    x = d["logits"].requires_grad_()
    p = torch.softmax(x, 1) * valid[:, None]
    mean = torch.zeros(groups, E, dtype=torch.float64, device=device).index_add(0, lines, p) / n.clamp(min=1)[:, None]
    share = counts / (k * n.clamp(min=1))[:, None]
    loss = COEFFICIENT * E * (share * mean).sum() / groups
    out = {"counts": None, "valid": None, "loss": loss.detach().reshape(1)}
    if case["grad"]:
        out["dlogits"], = torch.autograd.grad(loss, x)
    return out
