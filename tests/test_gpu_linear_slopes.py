"""The activations' slopes over every bf16 number up to 300, to their own size where they are small: dbias of one row is dC act'(z) in fp32.

Tolerance. With q the exponent that an activation's exponential takes (z^2 / 2, 2 |u|, |z|), rounded in fp32 three times at most, the exponential is
off by 3 q e of itself, e = 2^-24; the instructions for it and for the reciprocal by 2 e each, a handful of products and sums by e each: 16 e; the
normal tail's polynomial by 1e-6. Each part of the slope is off by that of itself. Below 2^-126 numbers are flushed, before they are multiplied by
up to 2^14."""
import pytest

import paper_2512_10236_amd as F

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def parts(z, kind):
    """(the slope, the size of its parts, q), in 64 bits."""
    if kind == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * torch.sigmoid(-z)), s * (1 + z.abs() * torch.sigmoid(-z)), z.abs()
    if kind == "gelu_tanh":
        c, k = (8 / torch.pi) ** 0.5, 0.044715
        s, t, dk = torch.sigmoid(c * (z + k * z ** 3)), torch.sigmoid(-c * (z + k * z ** 3)), c * (1 + 3 * k * z * z)
        return s + z * s * t * dk, s + (z * s * t * dk).abs(), (c * (z + k * z ** 3)).abs()
    phi, Phi = torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5, 0.5 * torch.special.erfc(-z / 2 ** 0.5)
    return Phi + z * phi, Phi + (z * phi).abs(), z * z / 2


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_slopes(gpu, kind):
    dev = gpu["dev"]
    bits = torch.arange(0, 0x4396, dtype=torch.int32, device=dev).to(torch.int16)          # 0 to 300
    z = torch.cat([bits.view(torch.bfloat16), -bits.view(torch.bfloat16)])
    z = torch.cat([z, z.new_zeros(-z.numel() % 8)])[None]
    N = z.shape[1]
    op = F.ficco_linear_t(M=1, K=64, N=N, activation=getattr(F, "FICCO_ACT_" + kind.upper()))
    n = F.ficco_linear_workspace(op, True)
    ws, db = torch.empty(n, dtype=torch.uint8, device=dev), torch.empty(N, device=dev)
    dC = torch.ones_like(z)
    torch.cuda.synchronize()
    F.ficco_linear_backward(op, None, None, z, dC, None, None, db, ws, n, gpu["cs"])
    torch.cuda.synchronize()
    slope, size, q = parts(z[0].double(), kind)
    assert torch.isfinite(db).all()
    over = (db.double() - slope).abs() - (size * (3 * q * E + 16 * E + (1e-6 if kind == "gelu" else 0)) + 2.0 ** -112)
    worst = over.argmax()
    assert over[worst] <= 0, (z[0, worst].item(), db[worst].item(), slope[worst].item())
