"""Packed attention on the host: buckets of the position bias, sizes, refusals (nothing is launched by a refused call), and the
64-bit reference of the GPU tests against automatic differentiation and differences."""
import ctypes as C
import math

import pytest
import torch

import packed_reference as ref

B = pytest.importorskip("paper_2406_08756_amd.binding")


def config(**kw):
    c = dict(dtype=B.LYNX_BF16, heads=4, kv_heads=2, head_dim=64, tokens=100, sequences=3, scale=0.125, num_buckets=0, q_stride=256,
             k_stride=128, v_stride=128, out_stride=256, dq_stride=256, dk_stride=128, dv_stride=128)
    c.update(kw)
    if "starts" in c:
        starts = c.pop("starts")
        c["num_buckets"] = len(starts)
        c["bucket_starts"] = (C.c_int32 * len(starts))(*starts)
    return B.lynx_attention_config(**c)


@pytest.mark.parametrize("buckets,far", [(2, 2), (2, 2048), (3, 2), (16, 128), (24, 200), (32, 128), (33, 2048), (64, 33), (64, 64), (64, 2048)])
def test_buckets(buckets, far):
    starts = list(B.lynx_position_buckets(buckets, far))
    low = buckets // 2
    assert starts[:low] == list(range(low)) and starts[low] == low
    steps = buckets - low
    for b in range(1, steps):
        n = starts[low + b]
        assert n ** steps * low ** b >= far ** b * low ** steps
        assert (n - 1) ** steps * low ** b < far ** b * low ** steps


def test_buckets_on_borders():
    # ratio 16 over 8 buckets: every second border is a whole number, where a rounded logarithm may fall short
    starts = list(B.lynx_position_buckets(16, 128))
    assert [starts[8 + b] for b in (0, 2, 4, 6)] == [8, 16, 32, 64]


@pytest.mark.parametrize("buckets,far", [(0, 8), (1, 8), (65, 128), (32, 16), (32, 2049), (-3, 8)])
def test_buckets_refused(buckets, far):
    with pytest.raises(B.LynxError) as e:
        B.lynx_position_buckets(buckets, far)
    assert e.value.status == B.LYNX_ERR_INVALID_ARG


SHAPE, ARG = B.LYNX_ERR_SHAPE, B.LYNX_ERR_INVALID_ARG
REFUSED = [
    (dict(dtype=2), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(heads=-4, kv_heads=-2), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(head_dim=60), SHAPE), (dict(head_dim=136, q_stride=1088, k_stride=544, v_stride=544, out_stride=1088), SHAPE),
    (dict(tokens=0), SHAPE), (dict(tokens=(1 << 24) + 1), SHAPE), (dict(sequences=0), SHAPE), (dict(sequences=(1 << 20) + 1), SHAPE),
    (dict(q_stride=248), SHAPE), (dict(k_stride=132), SHAPE), (dict(v_stride=-128), SHAPE), (dict(out_stride=(1 << 21) + 8), SHAPE),
    (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG),
    (dict(num_buckets=4), ARG), (dict(starts=[0] * 65), SHAPE), (dict(num_buckets=-1), SHAPE), (dict(starts=[1, 2]), ARG),
    (dict(starts=[0, 3, 2]), ARG), (dict(starts=[0, -1]), ARG), (dict(starts=[0, 2049]), SHAPE),
    (dict(heads=1 << 18, kv_heads=1 << 18, head_dim=8, q_stride=1 << 21, k_stride=1 << 21, v_stride=1 << 21, out_stride=1 << 21, dq_stride=1 << 21,
          dk_stride=1 << 21, dv_stride=1 << 21, tokens=1 << 24), SHAPE),
]
FAKE = [256 * (i + 1) for i in range(14)]


def forward(cfg, **change):
    a = dict(q=FAKE[0], k=FAKE[1], v=FAKE[2], offsets=FAKE[3], table=FAKE[4], out=FAKE[5], lse=FAKE[6])
    a.update(change)
    B.lynx_attention_forward(cfg, *a.values())


def backward(cfg, **change):
    a = dict(zip(["q", "k", "v", "offsets", "table", "out", "lse", "d_out", "d_q", "d_k", "d_v", "d_table", "workspace"], FAKE))
    a["n"] = B.lynx_attention_backward_bytes(cfg)
    a.update(change)
    B.lynx_attention_backward(cfg, *a.values())


@pytest.mark.parametrize("change,status", REFUSED, ids=lambda v: str(v)[:40])
def test_refused_configs(change, status):
    cfg = config(**change)
    assert B.lynx_attention_backward_bytes(cfg) == 0
    for call in (forward, backward):
        with pytest.raises(B.LynxError) as e:
            call(cfg)
        assert e.value.status == status


@pytest.mark.parametrize("change", [dict(dq_stride=248), dict(dk_stride=64), dict(dv_stride=129)])
def test_gradient_strides_are_the_backward_pass_s(change):
    with pytest.raises(B.LynxError) as e:
        backward(config(**change))
    assert e.value.status == SHAPE


@pytest.mark.parametrize("name", ["q", "k", "v", "offsets", "table", "out", "lse"])
@pytest.mark.parametrize("bad", [None, 258])
def test_refused_pointers_forward(name, bad):
    with pytest.raises(B.LynxError) as e:
        forward(config(starts=[0, 1]), **{name: bad})
    assert e.value.status == ARG


@pytest.mark.parametrize("name", ["q", "k", "v", "offsets", "table", "out", "lse", "d_out", "d_q", "d_k", "d_v", "d_table", "workspace"])
@pytest.mark.parametrize("bad", [None, 258])
def test_refused_pointers_backward(name, bad):
    with pytest.raises(B.LynxError) as e:
        backward(config(starts=[0, 1]), **{name: bad})
    assert e.value.status == ARG


def test_workspace():
    plain, biased = config(), config(starts=list(range(32)))
    assert B.lynx_attention_backward_bytes(plain) >= 4 * 100 * 4
    assert B.lynx_attention_backward_bytes(biased) > B.lynx_attention_backward_bytes(plain)
    for cfg in (plain, biased):
        with pytest.raises(B.LynxError) as e:
            backward(cfg, n=B.lynx_attention_backward_bytes(cfg) - 1)
        assert e.value.status == B.LYNX_ERR_OOM


def test_null_config():
    assert B._lib.lynx_attention_backward_bytes(None) == 0
    assert B._lib.lynx_attention_forward(None, *FAKE[:8]) == ARG
    assert B._lib.lynx_attention_backward(None, *FAKE[:13], 1 << 30, None) == ARG
    assert B._lib.lynx_position_buckets(4, 8, None) == ARG


def _loss(p, q, k, v, table):
    total = 0.0
    group = p.heads // p.kv
    for a, b in zip(p.at, p.at[1:]):
        i = torch.arange(b - a)
        for h in range(p.heads):
            z = p.scale * q[a:b].reshape(b - a, p.heads, p.d)[:, h] @ k[a:b].reshape(b - a, p.kv, p.d)[:, h // group].t()
            which = torch.searchsorted(torch.tensor(p.starts), (i[:, None] - i).clamp(min=0), right=True) - 1
            z = (z + table[which, h]).masked_fill(i > i[:, None], -math.inf)
            out = torch.softmax(z, 1) @ v[a:b].reshape(b - a, p.kv, p.d)[:, h // group]
            total = total + (out * p.d_out[a:b].reshape(b - a, p.heads, p.d)[:, h].to(ref.F64)).sum()
    return total


def test_reference_gradients():
    p = ref.Problem(torch.float32, 4, 2, 8, [5, 0, 1, 9], starts=[0, 1, 2, 4], device="cpu")
    leaves = [t.to(ref.F64).clone().requires_grad_() for t in (p.q, p.k, p.v, p.table)]
    loss = _loss(p, *leaves)
    loss.backward()
    want = {n: t.grad for n, t in zip(("dq", "dk", "dv", "d_table"), leaves)}
    got = ref.reference(p)
    gen = torch.Generator().manual_seed(5)
    for (n, grad), leaf in zip(want.items(), leaves):
        mine = got[n][0].reshape(grad.shape)
        assert float((mine - grad).abs().max()) < 1e-12
        # along a direction: central differences in 64 bits, off by h^2 of the third derivative and by rounding / h
        way = torch.randn(leaf.shape, generator=gen, dtype=ref.F64)
        h = 1e-5
        with torch.no_grad():
            ends = [float(_loss(p, *[t + s * h * way if t is leaf else t for t in leaves])) for s in (1, -1)]
        assert abs((ends[0] - ends[1]) / (2 * h) - float((mine * way).sum())) < 1e-7
