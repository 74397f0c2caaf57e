"""Gradients of packed attention against differences of the definition in 64 bits."""
import math

import pytest
import torch

import packed_reference as ref

B = pytest.importorskip("paper_2406_08756_amd.binding")
pytestmark = pytest.mark.gpu
F64 = torch.float64


def loss(p, q, k, v, table):
    """sum of out d_out, and the largest |logit's change| is the caller's matter."""
    total = torch.zeros((), dtype=F64)
    g = p.d_out.detach().cpu().to(F64).reshape(p.tokens, p.heads, p.d)
    group = p.heads // p.kv
    for a, b in zip(p.at, p.at[1:]):
        i = torch.arange(b - a)
        apart = i[:, None] - i
        for h in range(p.heads):
            z = p.scale * (q[a:b, h] @ k[a:b, h // group].t())
            if table is not None:
                z = z + table[torch.searchsorted(torch.tensor(p.starts), apart.clamp(min=0), right=True) - 1, h]
            z = z.masked_fill(apart < 0, -math.inf)
            total = total + ((torch.softmax(z, 1) @ v[a:b, h // group]) * g[a:b, h]).sum()
    return total


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d,lens,starts", [(4, 2, 64, [37, 70, 1], [0, 1, 2, 9, 40]), (3, 1, 104, [90, 33], None), (8, 1, 32, [20, 45], [0, 4])],
                         ids=["grouped_bias", "wide", "pack8"])
def test_gradients_against_differences(heads, kv, d, lens, starts, dtype):
    p = ref.Problem(dtype, heads, kv, d, lens, starts=starts, seed=31)
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    bounds = ref.reference(p)
    values = {"q": p.q, "k": p.k, "v": p.v}
    if starts is not None:
        values["table"] = p.table
    values = {n: t.detach().cpu().to(F64) for n, t in values.items()}
    count = {"q": heads, "k": kv, "v": kv}
    shaped = {n: t.reshape(p.tokens, count[n], d) if n in count else t for n, t in values.items()}
    gen = torch.Generator().manual_seed(32)
    step = 2.0 ** -14
    size = float((p.d_out.detach().cpu().to(F64).abs().sum()) * values["v"].abs().max())
    for n in shaped:
        for _ in range(4):
            # a direction along which no logit changes by more than 1 per unit: |scale u k| <= scale sum |k| max |u|
            u = torch.rand(shaped[n].shape, generator=gen, dtype=F64) * 2 - 1
            if n == "q":
                u = u / (p.scale * shaped["k"].abs().sum(2).max())
            elif n == "k":
                u = u / (p.scale * shaped["q"].abs().sum(2).max())
            at = [loss(p, *(shaped[m] + (sign * step * u if m == n else 0.0) if m in shaped else None for m in ("q", "k", "v", "table"))) for sign in (1, -1)]
            by_difference = float(at[0] - at[1]) / (2 * step)
            gradient = getattr(p, "d_table" if n == "table" else "d" + n).detach().cpu().to(F64).reshape(u.shape)
            # off by what the elements may be; the third derivative of a softmax's mean over values of size x is at most
            # 6 x where logits move by 1 per unit, and the sums in 64 bits lose 2^-40 of their terms
            most = float((u.abs() * bounds["d_table" if n == "table" else "d" + n][1].reshape(u.shape)).sum())
            most += size * (6 * step ** 2 / 6 + 2.0 ** -40 / step)
            assert abs(float((gradient * u).sum()) - by_difference) <= most, n
