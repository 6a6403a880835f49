"""The alignment that the interface asks for of every operand of the operators around the pair, and no more: an address that has it and no more is taken,
half of it is refused."""
import pytest

import standin

BASE = 1 << 20
LINEAR = dict(M=8, K=64, N=64, activation=4)
NORM = dict(rows=8, width=64, eps=1e-6, residual_scale=1.0)
BALANCE = dict(tokens=6000, experts=64, top_k=2, coefficient=1.0)
# bytes by operand, of (op, fields of its struct)
RULES = [("linear", LINEAR, dict(A=16, W=16, bias=2, residual=16, pre=16, C=16)), ("linear", dict(LINEAR, bias_type=1), dict(bias=4)),
         ("linear_backward", LINEAR, dict(A=16, W=16, pre=16, dC=16, dA=16, dW=16, dbias=4, workspace=16))]
for types in (dict(stream_type=0, param_type=0), dict(stream_type=1, param_type=1)):
    RULES += [("norm", dict(NORM, **types), dict.fromkeys("x block post gate pre y h".split(), 16)),
              ("norm_backward", dict(NORM, **types), dict.fromkeys("y block post gate pre dy dh dx dblock dpost dgate dpre workspace".split(), 16))]
for kind, size in ((0, 2), (1, 4)):
    RULES += [("balance", dict(BALANCE, logits_type=kind), dict(logits=size, ids=4, valid=1, counts=4, group_valid=4, loss=4, workspace=16)),
              ("balance_backward", dict(BALANCE, logits_type=kind), dict(logits=size, valid=1, counts=4, group_valid=4, dloss=4, dlogits=size))]


def test_alignment(tmp_path):
    calls, right = [], []
    for op, fields, rules in RULES:
        for name, size in rules.items():
            calls.append(dict(op=op, fields=fields, given={name: BASE + size}))
            right.append(0)
            if size > 1:
                calls.append(dict(op=op, fields=fields, given={name: BASE + size // 2}))
                right.append(-1)
    out, _ = standin.run(standin.build(str(tmp_path)), calls)
    wrong = [(c["op"], c["given"], r["status"]) for c, r, status in zip(calls, out, right) if r["status"] != status or bool(r["launches"]) != (status == 0)]
    assert not wrong, wrong


@pytest.mark.parametrize("ld,status", [(1 << 22, 0), ((1 << 22) + 8, -2)])
def test_the_largest_stride_of_logits(tmp_path, ld, status):
    out, _ = standin.run(standin.build(str(tmp_path)), [dict(op=op, fields=dict(tokens=8, experts=4, top_k=2, coefficient=1.0, ld_logits=ld)) for op in ("balance", "balance_backward")])
    assert [c["status"] for c in out] == [status] * 2
