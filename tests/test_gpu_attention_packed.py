"""Packed attention with grouped heads and the position bias on the GPU, against the 64-bit reference."""
import math

import pytest
import torch

import packed_reference as ref

B = pytest.importorskip("paper_2406_08756_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def usual(buckets, far):
    return list(B.lynx_position_buckets(buckets, far))


# heads, kv, d, lens, what else
SHAPES = [
    (1, 1, 8, [1], {}),
    (1, 1, 64, [1, 1, 1, 2], dict(gap=3, tail=5)),
    (2, 1, 64, [31, 32, 33], {}),
    (4, 4, 64, [128, 127, 129, 256], dict(fused=False, pad=8)),
    (5, 5, 128, [300, 0, 0, 77, 1], dict(tail=9)),
    (6, 3, 40, [65, 200, 7], dict(gap=1)),
    (8, 2, 128, [513], dict(fused=False, pad=16)),
    (8, 1, 128, [64, 3, 190], {}),
    (16, 1, 64, [70, 5, 130], dict(tail=2)),
    (24, 2, 72, [45, 90], {}),
    (7, 7, 104, [263, 129], dict(gap=2, tail=2)),
    (3, 1, 96, [150, 151], {}),
    (32, 8, 64, [20, 40, 1, 1, 60], {}),
    (2, 2, 120, [1030], {}),
    (1, 1, 16, [0, 0, 5, 0], {}),
    (4, 1, 64, [2] * 150 + [0] * 30 + [9], {}),
]
BIASES = [None, ("usual", 32, 128), ("starts", [0]), ("starts", [0, 0, 1, 1, 40]), ("usual", 64, 1024), ("usual", 9, 2048)]


def starts_of(bias):
    return None if bias is None else usual(*bias[1:]) if bias[0] == "usual" else bias[1]


def both(p):
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    ref.check(p, ["out", "lse", "dq", "dk", "dv"] + (["d_table"] if p.table is not None else []))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "h%d_k%d_d%d_n%d" % (s[0], s[1], s[2], len(s[3])))
def test_shapes(shape, dtype):
    heads, kv, d, lens, more = shape
    both(ref.Problem(dtype, heads, kv, d, lens, **more))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bias", BIASES[1:], ids=str)
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (1, 3, 5, 7, 8, 10, 13, 15)], ids=lambda s: "h%d_k%d_d%d_n%d" % (s[0], s[1], s[2], len(s[3])))
def test_bias(shape, bias, dtype):
    heads, kv, d, lens, more = shape
    both(ref.Problem(dtype, heads, kv, d, lens, starts=starts_of(bias), seed=1, **more))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_large_logits(dtype):
    p = ref.Problem(dtype, 4, 2, 64, [200, 90], starts=usual(32, 128), seed=2)
    p.q.mul_(16.0)
    p.table.mul_(8.0)
    both(p)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("masked", [[0], [3], [0, 1, 2, 3], [2, 3]], ids=str)
def test_buckets_of_minus_infinity(masked, dtype):
    # bucket 0 alone leaves the first row of each sequence nothing; all of them leave nothing to any
    p = ref.Problem(dtype, 4, 2, 64, [140, 1, 300], starts=[0, 1, 5, 60], seed=3)
    p.table[masked, 1:3] = -math.inf
    both(p)
    got = p.results()
    for h in (1, 2):
        if 0 in masked:
            assert bool((got["lse"][h, [0, 140, 141]] == -math.inf).all())
            assert bool((got["out"].view(p.tokens, 4, 64)[[0, 140, 141], h] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,d,starts", [(2, 2, 64, None), (4, 1, 104, [0, 1, 9, 70]), (3, 3, 128, None)])
def test_infinities_and_nan(heads, kv, d, starts, dtype):
    """An element that is not finite reaches what it is a term of; every other result keeps its bits."""
    lens = [200, 60, 140]
    make = lambda: ref.Problem(dtype, heads, kv, d, lens, starts=starts, seed=4)  # noqa: E731
    clean = make()
    both(clean)
    want = clean.results()
    group, a, b = heads // kv, 200, 260  # the middle sequence is spoilt at its token 35
    at = a + 35

    def spoilt(name, column, value):
        p = make()
        getattr(p, name)[at, column] = value
        p.forward(B)
        p.backward(B)
        torch.cuda.synchronize()
        return p.results()

    def same(got, touched):
        for n, t in want.items():
            if n == "d_table":
                continue
            keep = ~touched[n].reshape(t.shape)
            assert torch.equal(ref.bits(got[n])[keep], ref.bits(t)[keep]), n

    def nothing():
        return {n: torch.zeros(t.shape if n == "lse" else (t.shape[0], t.shape[1] // d, d), dtype=torch.bool, device="cuda") for n, t in want.items() if n != "d_table"}

    h0 = slice((kv - 1) * group, heads)  # the query heads of the last key head
    for value in (math.inf, -math.inf, math.nan):
        # V: the rows that see it, and (through delta) their dQ and what they give to dK; its own dV depends on no V
        t = nothing()
        t["out"][at:b, h0] = t["dq"][at:b, h0] = True
        t["dk"][a:b, kv - 1] = True
        got = spoilt("v", (kv - 1) * d + 3, value)
        same(got, t)
        assert bool((~torch.isfinite(got["out"].view(-1, heads, d)[at:b, h0, 3])).all())
        assert bool(torch.isfinite(got["out"].view(-1, heads, d)[at:b, h0, 4]).all())
        # K: the rows that see it have no statistic (or leave the key out: minus infinity), all their results with it
        t = nothing()
        t["lse"][h0, at:b] = t["out"][at:b, h0] = t["dq"][at:b, h0] = True
        t["dk"][a:b, kv - 1] = t["dv"][a:b, kv - 1] = True
        same(spoilt("k", (kv - 1) * d + 3, value), t)
        # Q and d_out: the row, and the keys that it sees
        t = nothing()
        t["lse"][heads - 1, at] = t["out"][at, heads - 1] = t["dq"][at, heads - 1] = True
        t["dk"][a:at + 1, kv - 1] = t["dv"][a:at + 1, kv - 1] = True
        got = spoilt("q", (heads - 1) * d + 3, value)
        same(got, t)
        assert bool((~torch.isfinite(got["out"].view(-1, heads, d)[at, heads - 1])).all())
        t = nothing()
        t["dq"][at, heads - 1] = True
        t["dk"][a:at + 1, kv - 1] = t["dv"][a:at + 1, kv - 1] = True
        got = spoilt("d_out", (heads - 1) * d + 3, value)
        same(got, t)
        assert bool((~torch.isfinite(got["dv"].view(-1, kv, d)[a:at + 1, kv - 1, 3])).all())
        assert bool(torch.isfinite(got["dv"].view(-1, kv, d)[a:at + 1, kv - 1, 4]).all())
        # a neighbour's values, rows of no sequence: nobody's
    p = ref.Problem(dtype, heads, kv, d, lens, starts=starts, seed=4, gap=0, tail=40)
    for n in ("q", "k", "v", "d_out"):
        getattr(p, n)[400:] = math.nan
    both(p)


def test_same_bits_every_time_and_on_other_streams():
    p = ref.Problem(BF16, 8, 2, 128, [700, 20, 411, 3], starts=usual(32, 128), seed=6)
    both(p)
    want = p.results()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for again in range(4):
        for n in want:
            getattr(p, n).fill_(7.0)
        p.workspace.fill_(0x7F)
        torch.cuda.synchronize()
        s = streams[again % 2]
        p.forward(B, s)
        p.backward(B, s)
        torch.cuda.synchronize()
        for n, t in p.results().items():
            assert torch.equal(ref.bits(t), ref.bits(want[n])), n


def test_two_calls_at_once():
    """Two problems of their own workspaces, each on a stream, have the results that they have alone."""
    ps = [ref.Problem(BF16, 4, 2, 64, lens, starts=usual(16, 64), seed=8 + i) for i, lens in enumerate(([900, 100], [33, 800, 5]))]
    alone = []
    for p in ps:
        both(p)
        alone.append(p.results())
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(3):
        for p, s in zip(ps, streams):
            p.forward(B, s)
            p.backward(B, s)
    torch.cuda.synchronize()
    for p, want in zip(ps, alone):
        for n, t in p.results().items():
            assert torch.equal(ref.bits(t), ref.bits(want[n])), n


def test_captured_with_lengths_that_change():
    p = ref.Problem(BF16, 8, 4, 64, [150, 350, 12], starts=usual(32, 128), seed=9, tail=30)
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        p.forward(B, s)
        p.backward(B, s)
    for lens in ([150, 350, 12], [1, 500, 30], [0, 542, 0], [150, 350, 12], [170, 171, 172]):
        at = [0]
        for n in lens:
            at.append(at[-1] + n)
        p.lens, p.at = lens, at
        p.offsets.copy_(torch.tensor(at, dtype=torch.int32))
        for n in ("out", "lse", "dq", "dk", "dv"):
            getattr(p, n).fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = p.results()
        ref.check(p, list(got))
        p.forward(B)
        p.backward(B)
        torch.cuda.synchronize()
        for n, t in p.results().items():
            assert torch.equal(ref.bits(t), ref.bits(got[n])), n


def test_offsets_that_are_out_of_range_reach_nothing_outside():
    """Offsets beyond the tensors and decreasing ones: the tensors' surroundings keep their bits."""
    p = ref.Problem(BF16, 2, 2, 64, [40, 50, 10], seed=10)
    big = {}
    for n in ("out", "dq", "dk", "dv"):
        big[n] = torch.full((300, 128), 7.0, dtype=BF16, device="cuda")
        setattr(p, n, big[n][100:200])
    p.offsets.copy_(torch.tensor([-5, 1 << 30, 60, 101], dtype=torch.int32))
    p.forward(B)
    p.backward(B)
    torch.cuda.synchronize()
    for n, t in big.items():
        assert bool((t[:100] == 7.0).all()) and bool((t[200:] == 7.0).all()), n


def test_rows_far_apart():
    """Offsets of elements beyond 32 bits."""
    rows, stride = 1040, 1 << 21
    block = torch.empty(rows * stride, dtype=BF16, device="cuda")
    p = ref.Problem(BF16, 2, 1, 64, [1000, 40], seed=11, starts=[0, 1, 30], fused=False)
    wide = block.view(rows, stride)
    for i, n in enumerate(("q", "k", "v", "dq", "dk", "dv", "out", "d_out")):
        t = getattr(p, n)
        w = wide[:, 1024 * i:1024 * i + t.shape[1]]
        w.copy_(t)
        setattr(p, n, w)
    both(p)


def test_a_longer_prompt_of_many_heads():
    both(ref.Problem(BF16, 4, 1, 128, [2500], starts=usual(32, 128), seed=12))
