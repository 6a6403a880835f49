"""What the binding takes as an operand of the operators around the pair: a tensor that is what the struct says, or an address. The C function
is replaced by one that notes its arguments, so that what is taken is seen as well as what is refused."""
import ctypes

import pytest

import paper_2512_10236_amd as F
from paper_2512_10236_amd import binding

torch = pytest.importorskip("torch")
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Noted:
    def __init__(self, lib):
        self.lib, self.args = lib, None

    def __getattr__(self, name):
        if name.startswith("ficco_str") or name.startswith("ficco_last"):
            return getattr(self.lib, name)

        def call(*args):
            self.args = args
            return F.FICCO_OK
        return call


@pytest.fixture
def noted(monkeypatch):
    n = Noted(F.load())
    monkeypatch.setattr(binding, "load", lambda: n)
    return n


M, K, N = 6, 128, 72
T, E = 10, 24
t = lambda *shape, dtype=BF: torch.zeros(*shape, dtype=dtype)  # noqa: E731

LINEAR = dict(A=(M, K), W=(K, N), bias=(N,), residual=(M, N), pre=(M, N), C=(M, N), workspace=(64,))
LINEAR_BACK = dict(A=(M, K), W=(K, N), pre=(M, N), dC=(M, N), dA=(M, K), dW=(K, N), dbias=(N,), workspace=(64,))
NORM = dict(x=(M, N), block=(M, N), post=(N,), gate=(M, N), pre=(N,), y=(M, N), h=(M, N))
NORM_BACK = dict(y=(M, N), block=(M, N), post=(N,), gate=(M, N), pre=(N,), dy=(M, N), dh=(M, N), dx=(M, N), dblock=(M, N), dpost=(N,), dgate=(M, N), dpre=(N,), workspace=(64,))
BALANCE = dict(logits=(T, E), ids=(T, 2), valid=(T,), counts=(1, E), group_valid=(1,), loss=(1,), workspace=(64,))
BALANCE_BACK = dict(logits=(T, E), valid=(T,), counts=(1, E), group_valid=(1,), dloss=(1,), dlogits=(T, E))
SUMS = ("dbias", "dpost", "dgate", "dpre", "loss", "dloss")
CALLS = {"linear": (F.ficco_linear, LINEAR, lambda **k: F.ficco_linear_t(M=M, K=K, N=N, **k)), "linear_backward": (F.ficco_linear_backward, LINEAR_BACK, lambda **k: F.ficco_linear_t(M=M, K=K, N=N, **k)),
         "norm": (F.ficco_residual_norm, NORM, lambda **k: F.ficco_residual_norm_t(rows=M, width=N, gate_rows=1, eps=1e-6, **k)),
         "norm_backward": (F.ficco_residual_norm_backward, NORM_BACK, lambda **k: F.ficco_residual_norm_t(rows=M, width=N, gate_rows=1, eps=1e-6, **k)),
         "balance": (F.ficco_expert_balance, BALANCE, lambda **k: F.ficco_expert_balance_t(tokens=T, experts=E, top_k=2, coefficient=1.0, **k)),
         "balance_backward": (F.ficco_expert_balance_backward, BALANCE_BACK, lambda **k: F.ficco_expert_balance_t(tokens=T, experts=E, top_k=2, coefficient=1.0, **k))}
STRIDED = {("linear", "A"): "lda", ("linear", "residual"): "ld_residual", ("linear", "pre"): "ld_pre", ("linear", "C"): "ldc", ("linear_backward", "A"): "lda", ("linear_backward", "pre"): "ld_pre",
           ("linear_backward", "dC"): "ldc", ("balance", "logits"): "ld_logits", ("balance_backward", "logits"): "ld_logits"}
OPERANDS = [(c, o) for c, (_, names, _) in CALLS.items() for o in names]


def right_type(name):
    return F32 if name in SUMS else I32 if name in ("ids", "counts", "group_valid") else torch.uint8 if name in ("valid", "workspace") else BF


def call(noted, name, op=None, **given):
    """Calls with zeros of the right shapes, but for `given`; the addresses that the C function got, by operand."""
    fn, shapes, make = CALLS[name]
    noted.args = None
    args = {k: given.get(k, t(*s, dtype=right_type(k))) for k, s in shapes.items()}
    fn(op if op is not None else make(), *args.values(), *([64] if "workspace" in shapes else []), None)
    return dict(zip(shapes, noted.args[1:]))


def refused(noted, name, op=None, **given):
    with pytest.raises(F.FiccoError) as e:
        call(noted, name, op, **given)
    assert e.value.status == F.FICCO_ERR_ARG and noted.args is None
    assert next(iter(given)) in str(e.value)


@pytest.mark.parametrize("name,operand", OPERANDS)
def test_dense_tensors_addresses_and_none(noted, name, operand):
    shape = CALLS[name][1][operand]
    x = t(*shape, dtype=right_type(operand))
    assert call(noted, name, **{operand: x})[operand] == x.data_ptr()
    flat = t(x.numel() + 64, dtype=x.dtype)[8:]
    assert call(noted, name, **{operand: flat})[operand] == flat.data_ptr()
    assert call(noted, name, **{operand: 4096})[operand] == 4096
    assert call(noted, name, **{operand: None})[operand] is None
    raw = t(x.numel() * 4, dtype=torch.uint8)
    assert call(noted, name, **{operand: raw})[operand] == raw.data_ptr()


@pytest.mark.parametrize("name,operand", [o for o in OPERANDS if len(CALLS[o[0]][1][o[1]]) == 2])
def test_a_slice_of_columns_needs_its_stride(noted, name, operand):
    """Columns of a wider buffer: refused as dense rows, and where the struct has a stride for them, taken with that one and refused with another;
    so is the wider buffer itself, which begins at the same address."""
    rows, width = CALLS[name][1][operand]
    wide = t(rows, width + 40, dtype=right_type(operand))
    if rows == 1:
        assert call(noted, name, **{operand: wide[:, :width]})[operand] == wide.data_ptr()
        return
    refused(noted, name, **{operand: wide[:, :width]})
    refused(noted, name, **{operand: wide[:, 8:]})
    ld = STRIDED.get((name, operand))
    if ld:
        make = CALLS[name][2]
        same = {"ldc": {"C": wide[:, :width], "dC": wide[:, :width]}}.get(ld, {})
        same = {k: v for k, v in {**same, operand: wide[:, :width]}.items() if k in CALLS[name][1]}
        if name == "balance_backward":
            same["dlogits"] = wide[:, :width]
        got = call(noted, name, make(**{ld: width + 40}), **same)
        assert got[operand] == wide.data_ptr()
        assert call(noted, name, make(**{ld: width + 40}), **{**same, operand: wide})[operand] == wide.data_ptr()
        refused(noted, name, make(**{ld: width + 48}), **{operand: wide[:, :width]})
        refused(noted, name, **{operand: wide})
        refused(noted, name, make(**{ld: width + 40}), **{operand: t(rows, width)} if operand != "logits" else {operand: t(rows, width, dtype=BF)})


@pytest.mark.parametrize("name,operand", [o for o in OPERANDS if len(CALLS[o[0]][1][o[1]]) == 2])
def test_transposed_and_skipping_views(noted, name, operand):
    rows, width = CALLS[name][1][operand]
    x = t(width, width, dtype=right_type(operand))
    refused(noted, name, **{operand: x.t()})
    refused(noted, name, **{operand: t(rows, 2 * width, dtype=right_type(operand))[:, ::2]})
    if rows > 1:
        refused(noted, name, **{operand: t(2 * rows, width, dtype=right_type(operand))[::2]})


def test_rows_in_more_than_two_dimensions(noted):
    x = t(2, 3, K)
    assert call(noted, "linear", A=x)["A"] == x.data_ptr()
    heads = t(M * 4, K // 4)
    assert call(noted, "linear", A=heads)["A"] == heads.data_ptr()
    wide = t(2, 3, 2 * K)
    assert call(noted, "linear", F.ficco_linear_t(M=M, K=K, N=N, lda=2 * K), A=wide[..., K:])["A"] == wide[..., K:].data_ptr()
    split = t(M, 2, 4, K // 4)[:, 1]                          # heads of the second half of a row
    assert call(noted, "linear", F.ficco_linear_t(M=M, K=K, N=N, lda=2 * K), A=split)["A"] == split.data_ptr()
    refused(noted, "linear", A=split)
    last = t(M, 5, K)[:, -1:]                                 # the last position of each sequence
    assert call(noted, "linear", F.ficco_linear_t(M=M, K=K, N=N, lda=5 * K), A=last)["A"] == last.data_ptr()
    refused(noted, "linear", A=last)
    refused(noted, "linear", A=t(2, 5, K)[:, :3])             # rows that are not evenly apart
    one = t(4, 3 * K)[1:2, K:2 * K]
    assert call(noted, "linear", F.ficco_linear_t(M=1, K=K, N=N), A=one, residual=t(1, N), pre=t(1, N), C=t(1, N))["A"] == one.data_ptr()


@pytest.mark.parametrize("name,operand", [o for o in OPERANDS if o[1] != "workspace"])
def test_types(noted, name, operand):
    shape, right = CALLS[name][1][operand], right_type(operand)
    same = {BF: (torch.int16,), F32: (), I32: (), torch.uint8: (torch.bool,)}[right]
    for dtype in same:
        x = t(*shape, dtype=dtype)
        assert call(noted, name, **{operand: x})[operand] == x.data_ptr()
    wrong = {BF: (torch.float16, F32, torch.float64), F32: (BF, torch.float16, torch.float64), I32: (torch.int64, F32, torch.int16), torch.uint8: (I32, F32, torch.int64)}[right]
    for dtype in wrong:
        refused(noted, name, **{operand: t(*shape, dtype=dtype)})


def test_types_that_the_struct_names(noted):
    assert call(noted, "linear", F.ficco_linear_t(M=M, K=K, N=N, bias_type=F.FICCO_F32), bias=t(N, dtype=F32))
    refused(noted, "linear", F.ficco_linear_t(M=M, K=K, N=N, bias_type=F.FICCO_F32), bias=t(N))
    op = F.ficco_residual_norm_t(rows=M, width=N, gate_rows=1, eps=1e-6, stream_type=F.FICCO_F32)
    assert call(noted, "norm", op, x=t(M, N, dtype=F32), y=t(M, N, dtype=F32))
    refused(noted, "norm", op, x=t(M, N))
    op = F.ficco_expert_balance_t(tokens=T, experts=E, top_k=2, logits_type=F.FICCO_F32)
    assert call(noted, "balance", op, logits=t(T, E, dtype=F32))
    refused(noted, "balance", op, logits=t(T, E))


def test_what_topk_returns_is_refused_as_ids(noted):
    ids = torch.topk(torch.randn(T, E), 2, dim=1).indices
    refused(noted, "balance", ids=ids)
    refused(noted, "balance", ids=ids.to(I32).repeat(1, 2)[:, :2])
    assert call(noted, "balance", ids=ids.to(I32))


def test_pointers_to_the_struct(noted):
    op = F.ficco_linear_t(M=M, K=K, N=N, lda=2 * K)
    for o in (op, ctypes.byref(op), ctypes.pointer(op)):
        assert call(noted, "linear", o, A=t(M, 2 * K)[:, :K])
        refused(noted, "linear", o, A=t(M, 3 * K)[:, :K])


def test_no_rows(noted):
    assert call(noted, "linear", F.ficco_linear_t(M=0, K=K, N=N), A=t(0, K), residual=t(0, N), pre=None, C=t(0, N))["pre"] is None
    assert call(noted, "linear", F.ficco_linear_t(M=0, K=K, N=N), A=t(4, 2 * K)[:, :K])


def test_a_number(noted):
    """A tensor without dimensions, as a loss often is."""
    one = torch.zeros((), dtype=F32)
    assert call(noted, "balance", loss=one)["loss"] == one.data_ptr()
    op = F.ficco_expert_balance_t(tokens=1, experts=1, top_k=1, logits_type=F.FICCO_F32)
    assert call(noted, "balance", op, logits=one)["logits"] == one.data_ptr()
