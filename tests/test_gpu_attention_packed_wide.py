"""Packed attention with many heads: launches of enough workgroups that each takes 128 rows or keys, whose waves share tiles
(fewer give every wave tiles of its own).  Rows: (tokens << pack) / 128 + sequences tiles times heads >> pack are 400 or more;
keys: tokens / 128 + sequences tiles times kv_heads are 1024 (head_dim <= 64) or 512 or more, of 96 tokens a sequence or more."""
import math

import pytest
import torch

import packed_reference as ref

B = pytest.importorskip("paper_2406_08756_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

LENS = [300, 1, 129, 128, 127, 64, 300, 0, 33, 257]  # 1339 tokens, 10 + 10 tiles
FEWER = [97, 290, 128, 1, 0, 200]  # 716 tokens, 5 + 6 tiles: 704 of 64 heads


def usual(buckets, far):
    return list(B.lynx_position_buckets(buckets, far))


# heads, kv, d, lens, bias, what else
SHAPES = [
    (64, 64, 64, LENS, None, dict(gap=2, tail=5)),
    (128, 64, 40, LENS, (32, 128), dict(fused=False, pad=8)),
    (192, 64, 16, LENS, (5, 40), {}),
    (256, 64, 64, LENS, (16, 64), {}),
    (512, 64, 32, LENS, None, {}),
    (64, 64, 128, FEWER, (64, 1024), dict(gap=1)),
    (64, 64, 104, FEWER, None, dict(fused=False, pad=16)),
    (128, 64, 128, FEWER, None, {}),
    (256, 64, 72, FEWER, (32, 128), dict(tail=9)),
    (128, 16, 104, FEWER, (32, 128), {}),  # (dQ with fewer heads to a tile than the others)
    (5, 5, 64, [96 + 7 * (i % 5) for i in range(130)], (32, 128), {}),  # (more sequences than are ordered by size)
    (5, 5, 96, [96 + 7 * (i % 5) for i in range(130)], None, {}),
    (6, 1, 48, [3] * 520 + [0] + [70, 1], (9, 2048), {}),  # (rows alone are enough)
]


def both(p):
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    ref.check(p, ["out", "lse", "dq", "dk", "dv"] + (["d_table"] if p.table is not None else []))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "h%d_k%d_d%d_n%d_%s" % (s[0], s[1], s[2], len(s[3]), "bias" if s[4] else "plain"))
def test_shapes(shape, dtype):
    heads, kv, d, lens, bias, more = shape
    both(ref.Problem(dtype, heads, kv, d, lens, starts=usual(*bias) if bias else None, seed=21, **more))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("masked", [[0], [0, 1, 2, 3], [2, 3]], ids=str)
def test_buckets_of_minus_infinity(masked, dtype):
    p = ref.Problem(dtype, 128, 64, 64, LENS, starts=[0, 1, 5, 60], seed=22)
    p.table[masked, 3:90] = -math.inf
    both(p)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,d,starts,lens", [(64, 64, 64, None, LENS), (128, 64, 48, [0, 1, 9, 70], LENS), (128, 64, 128, None, FEWER)],
                         ids=["plain", "bias", "wide"])
def test_infinities_and_nan(heads, kv, d, starts, lens, dtype):
    make = lambda: ref.Problem(dtype, heads, kv, d, lens, starts=starts, seed=23)  # noqa: E731
    clean = make()
    both(clean)
    want = clean.results()
    group = heads // kv
    a, b = max(zip(clean.at, clean.at[1:]), key=lambda s: s[1] - s[0])
    at = a + 170
    h0 = slice((kv - 1) * group, heads)
    views = {"out": heads, "dq": heads, "dk": kv, "dv": kv}

    def run(name, column, value, **touched):
        p = make()
        getattr(p, name)[at, column] = value
        p.forward(B)
        p.backward(B)
        torch.cuda.synchronize()
        got = p.results()
        for n, count in views.items():
            keep = torch.ones(p.tokens, count, dtype=torch.bool, device="cuda")
            if n in touched:
                keep[touched[n]] = False
            keep = keep.repeat_interleave(d, 1)
            assert torch.equal(ref.bits(got[n])[keep], ref.bits(want[n])[keep]), (name, n)
        keep = torch.ones(heads, p.tokens, dtype=torch.bool, device="cuda")
        if "lse" in touched:
            keep[touched["lse"]] = False
        assert torch.equal(ref.bits(got["lse"])[keep], ref.bits(want["lse"])[keep]), (name, "lse")
        return got

    after, all_keys, seen, row = (slice(at, b), h0), (slice(a, b), kv - 1), (slice(a, at + 1), kv - 1), (at, heads - 1)
    for value in (math.inf, math.nan):
        got = run("v", (kv - 1) * d + 3, value, out=after, dq=after, dk=all_keys)
        assert bool((~torch.isfinite(got["out"].view(-1, heads, d)[at:b, h0, 3])).all())
        assert bool(torch.isfinite(got["out"].view(-1, heads, d)[at:b, h0, 4]).all())
        run("k", (kv - 1) * d + 3, value, lse=(h0, slice(at, b)), out=after, dq=after, dk=all_keys, dv=all_keys)
        run("q", (heads - 1) * d + 3, value, lse=(heads - 1, at), out=row, dq=row, dk=seen, dv=seen)
        got = run("d_out", (heads - 1) * d + 3, value, dq=row, dk=seen, dv=seen)
        assert bool((~torch.isfinite(got["dv"].view(-1, kv, d)[a:at + 1, kv - 1, 3])).all())
        assert bool(torch.isfinite(got["dv"].view(-1, kv, d)[a:at + 1, kv - 1, 4]).all())


def test_captured_with_lengths_that_change():
    p = ref.Problem(BF16, 128, 64, 64, LENS, starts=usual(32, 128), seed=24, tail=30)
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        p.forward(B, s)
        p.backward(B, s)
    for lens in (LENS, [1, 2, 0, 0, 0, 0, 0, 0, 0, 1336], [130] * 10, LENS):
        at = [0]
        for n in lens:
            at.append(at[-1] + n)
        p.lens, p.at = lens, at
        p.offsets.copy_(torch.tensor(at, dtype=torch.int32))
        for n in ("out", "lse", "dq", "dk", "dv"):
            getattr(p, n).fill_(7.0)
        p.workspace.fill_(0x7F)
        graph.replay()
        torch.cuda.synchronize()
        got = p.results()
        p.forward(B)
        p.backward(B)
        torch.cuda.synchronize()
        for n, t in p.results().items():
            assert torch.equal(ref.bits(t), ref.bits(got[n])), n
        if lens[0] != 1:
            ref.check(p, list(got))


def test_offsets_that_are_out_of_range_reach_nothing_outside():
    p = ref.Problem(BF16, 64, 64, 64, [150] * 9, seed=25)
    big = {}
    for n in ("out", "dq", "dk", "dv"):
        big[n] = torch.full((1750, 4096), 7.0, dtype=BF16, device="cuda")
        setattr(p, n, big[n][200:1550])
    p.offsets.copy_(torch.tensor([-5, 1 << 30, 60, 300, 200, 700, -(1 << 30), 1000, 1351, 1 << 30], dtype=torch.int32))
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    for n, t in big.items():
        assert bool((t[:200] == 7.0).all()) and bool((t[1550:] == 7.0).all()), n
