"""Attention over packed sequences in 64 bits, straight from the formulas, and how far kernels that hold sums in fp32 and
round probabilities and ds to the storage type may be from it, element by element."""
from __future__ import annotations

import ctypes as C
import math

import torch

F64 = torch.float64
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
FP32 = 2.0 ** -24


class Problem:
    """Inputs of one call, with fused or separate tensors; everything derives from the arguments."""

    def __init__(self, dtype, heads, kv, d, lens, gap=0, tail=0, starts=None, fused=True, pad=0, seed=0, device="cuda"):
        self.dtype, self.heads, self.kv, self.d, self.lens, self.starts = dtype, heads, kv, d, list(lens), starts
        self.scale = d ** -0.5
        self.tokens = gap + sum(lens) + tail
        self.device = device
        at = [gap]
        for n in lens:
            at.append(at[-1] + n)
        self.at = at
        gen = torch.Generator().manual_seed(seed * 7919 + heads * 131 + d)

        def normal(*shape):
            return torch.randn(*shape, generator=gen).to(dtype).to(device)

        self.offsets = torch.tensor(at, dtype=torch.int32, device=device)
        widths = (heads * d, kv * d, kv * d)
        if fused:
            block = normal(self.tokens, sum(widths) + pad)
            d_block = torch.full_like(block, 7.0)
            cut = [0, widths[0], widths[0] + widths[1], sum(widths)]
            self.q, self.k, self.v = (block[:, a:b] for a, b in zip(cut, cut[1:]))
            self.dq, self.dk, self.dv = (d_block[:, a:b] for a, b in zip(cut, cut[1:]))
        else:
            self.q, self.k, self.v = (normal(self.tokens, w + pad * (i + 1))[:, :w] for i, w in enumerate(widths))
            self.dq, self.dk, self.dv = (torch.full((self.tokens, w + pad * (3 - i)), 7.0, dtype=dtype, device=device)[:, :w]
                                         for i, w in enumerate(widths))
        self.out = torch.full((self.tokens, heads * d + pad), 7.0, dtype=dtype, device=device)[:, :heads * d]
        self.d_out = normal(self.tokens, heads * d + pad)[:, :heads * d]
        self.lse = torch.full((heads, self.tokens), 7.0, device=device)
        self.table = self.d_table = None
        if starts is not None:
            self.table = normal(len(starts), heads)
            self.d_table = torch.full_like(self.table, 7.0)

    def config(self, B):
        starts = None if self.starts is None else (C.c_int32 * len(self.starts))(*self.starts)
        return B.lynx_attention_config(
            dtype=B.LYNX_BF16 if self.dtype == torch.bfloat16 else B.LYNX_F32, heads=self.heads, kv_heads=self.kv, head_dim=self.d,
            tokens=self.tokens, sequences=len(self.lens), scale=self.scale, num_buckets=0 if self.starts is None else len(self.starts),
            bucket_starts=starts, q_stride=self.q.stride(0), k_stride=self.k.stride(0), v_stride=self.v.stride(0),
            out_stride=self.out.stride(0), dq_stride=self.dq.stride(0), dk_stride=self.dk.stride(0), dv_stride=self.dv.stride(0))

    def forward(self, B, stream=None):
        self.cfg = self.config(B)
        B.lynx_attention_forward(self.cfg, self.q, self.k, self.v, self.offsets, self.table, self.out, self.lse, stream)

    def backward(self, B, stream=None):
        if not hasattr(self, "workspace"):
            n = B.lynx_attention_backward_bytes(self.cfg)
            assert n > 0
            self.workspace = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=self.device)
            self.ws = (self.workspace.data_ptr() + 255) // 256 * 256
            self.ws_bytes = n
        B.lynx_attention_backward(self.cfg, self.q, self.k, self.v, self.offsets, self.table, self.out, self.lse, self.d_out,
                                  self.dq, self.dk, self.dv, self.d_table, self.ws, self.ws_bytes, stream)

    def results(self):
        names = ["out", "lse", "dq", "dk", "dv"] + (["d_table"] if self.table is not None else [])
        return {n: getattr(self, n).clone() for n in names}


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def reference(p):
    """{name: (value, tolerance)} in 64 bits, NaN in rows of no sequence."""
    u = HALF_STEP[p.dtype]
    u_mid = u if p.dtype == torch.bfloat16 else 0.0  # rounding of probabilities and ds ahead of a product
    q, k, v, g = (t.detach().cpu().to(F64).reshape(p.tokens, -1, p.d) for t in (p.q, p.k, p.v, p.d_out))
    table = None if p.table is None else p.table.detach().cpu().to(F64)
    group = p.heads // p.kv
    val = {"out": torch.full((p.tokens, p.heads, p.d), math.nan, dtype=F64), "lse": torch.full((p.heads, p.tokens), math.nan, dtype=F64)}
    val["dq"] = val["out"].clone()
    val["dk"] = torch.full((p.tokens, p.kv, p.d), math.nan, dtype=F64)
    val["dv"] = val["dk"].clone()
    tol = {n: t.clone() for n, t in val.items()}
    if table is not None:
        val["d_table"], tol["d_table"] = torch.zeros_like(table), torch.zeros_like(table)
        edges = torch.tensor(p.starts)
    for a, b in zip(p.at, p.at[1:]):
        n = b - a
        if n == 0:
            continue
        i = torch.arange(n)
        apart = i[:, None] - i
        hidden = apart < 0
        for kh in range(p.kv):
            K, V = k[a:b, kh], v[a:b, kh]
            for name in ("dk", "dv"):
                val[name][a:b, kh] = 0.0
                tol[name][a:b, kh] = 0.0
            for h in range(kh * group, (kh + 1) * group):
                Q, G = q[a:b, h], g[a:b, h]
                z = p.scale * (Q @ K.t())
                reach = p.scale * (Q.abs() @ K.abs().t())
                if table is not None:
                    which = torch.searchsorted(edges, apart.clamp(min=0), right=True) - 1
                    bias = table[which, h]
                    z = z + bias
                    reach = reach + torch.where(bias.isfinite(), bias.abs(), torch.zeros((), dtype=F64))
                z = z.masked_fill(hidden, -math.inf)
                reach = reach.masked_fill(hidden, 0.0).amax(1)
                lse = torch.logsumexp(z, 1)
                P = torch.where(torch.isinf(lse)[:, None], torch.zeros((), dtype=F64), torch.exp(z - lse[:, None]))
                # a logit is off by the d products and sums that it is formed of; its own probability and the sum by that
                # each, the sum by its n additions, and the exponentials, the scaling and the logarithm by a few steps
                fp = FP32 * (2 * (p.d + 8) * reach + n + 64)
                out = P @ V
                size = P @ V.abs()
                out_tol = (u_mid + fp[:, None]) * size + u * out.abs()
                val["out"][a:b, h], tol["out"][a:b, h] = out, out_tol
                val["lse"][h, a:b] = lse
                tol["lse"][h, a:b] = fp + 4 * FP32 * torch.where(torch.isinf(lse), torch.zeros((), dtype=F64), lse.abs())
                dP = G @ V.t()
                delta = (G * out).sum(1, keepdim=True)
                ds = P * (dP - delta)
                # delta comes from the stored out
                delta_tol = (G.abs() * out_tol).sum(1, keepdim=True) + FP32 * (p.d + 4) * (G.abs() * out.abs()).sum(1, keepdim=True)
                # (the exponent also carries the rounding of the stored statistic)
                wide = fp[:, None] + 4 * FP32 * torch.where(torch.isinf(lse), torch.zeros((), dtype=F64), lse.abs())[:, None]
                ds_tol = P * (wide * (dP - delta).abs() + FP32 * (p.d + 4) * (G.abs() @ V.abs().t()) + delta_tol)
                ds_all = ds_tol + (u_mid + FP32 * (group * n + 8)) * ds.abs()
                val["dq"][a:b, h] = p.scale * ds @ K
                tol["dq"][a:b, h] = p.scale * ds_all @ K.abs() + u * val["dq"][a:b, h].abs()
                val["dk"][a:b, kh] += p.scale * ds.t() @ Q
                tol["dk"][a:b, kh] += p.scale * ds_all.t() @ Q.abs()
                val["dv"][a:b, kh] += P.t() @ G
                tol["dv"][a:b, kh] += ((u_mid + wide + FP32 * (group * n + 8)) * P).t() @ G.abs()
                if table is not None:
                    for t, x in ((val, ds), (tol, ds_tol + FP32 * 4096 * ds.abs())):  # (at most so many additions in a row)
                        t["d_table"][:, h] += torch.bincount(which[~hidden], x[~hidden], len(p.starts))
            for name in ("dk", "dv"):
                tol[name][a:b, kh] += u * val[name][a:b, kh].abs()
    if table is not None:
        tol["d_table"] += u * val["d_table"].abs()
    tiny = 2.0 ** -126  # (below the smallest normal number a storage type's steps are absolute)
    return {n: (val[n], tol[n] + tiny) for n in val}


def check(p, names, got=None):
    """The named results of `p` against the reference; rows of no sequence are as they were."""
    ref = reference(p)
    for n in names:
        value, bound = ref[n]
        x = (getattr(p, n) if got is None else got[n]).detach().cpu().to(F64).reshape(value.shape)
        outside = value.isnan()
        if n != "d_table":
            untouched = torch.ones(p.tokens, dtype=torch.bool)
            untouched[p.at[0]:p.at[-1]] = False
            rows = outside.all(0) if n == "lse" else outside.flatten(1).all(1)
            assert torch.equal(rows, untouched), n
        assert bool((x[outside] == 7.0).all()), n + ": a row of no sequence was written"
        same = (x == value) | outside
        off = torch.where(same, torch.zeros((), dtype=F64), (x - value).abs() / bound)
        assert not bool((off.isnan() | (off > 1)).any()), "%s: %.3g of the tolerance" % (n, float(off.nan_to_num(nan=math.inf).max()))
