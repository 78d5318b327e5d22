"""Rotary positions against 64 bits: amplitude (u cos - w sin) is off by the roundings of cosine, sine (each 2^-22: angle and function in fp32),
two products and a sum (2^-23), and half a step of the storage type."""
import ctypes
import math

import pytest
import torch

import paper_2201_11990_amd as M
from paper_2201_11990_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
SCALED = {"none": (M.ROTARY_UNSCALED, {}), "linear": (M.ROTARY_LINEAR, {"factor": 4.0}), "base": (M.ROTARY_BASE, {"factor": 3.0}),
          "parts": (M.ROTARY_PARTS, {"factor": 8.0, "original_positions": 2048, "slow": 1.0, "fast": 32.0})}


def frequencies(n, scaling, base):
    i = torch.arange(n // 2, dtype=torch.float64)
    how = SCALED[scaling][1]
    if scaling == "base" and n > 2:
        base = base * how["factor"] ** (n / (n - 2))
    f = base ** (-2 * i / n)
    if scaling == "linear":
        f = f / how["factor"]
    if scaling == "parts":
        turns = how["original_positions"] * f / (2 * math.pi)
        keep = ((turns - how["slow"]) / (how["fast"] - how["slow"])).clamp(0, 1)
        f = keep * f + (1 - keep) * f / how["factor"]
    return f, (0.1 * math.log(how["factor"]) + 1 if scaling == "parts" else 1.0)


def turned(x, positions, n, layout, scaling, base=10000.0, sign=1.0):
    """(value, sum of the magnitudes of the two products)"""
    f, amplitude = frequencies(n, scaling, base)
    angle = positions.double().cpu()[:, None] * f
    cos, sin = (t.view(t.shape[0], *[1] * (x.dim() - 2), t.shape[1]) for t in (angle.cos() * amplitude, sign * angle.sin() * amplitude))
    x = x.double().cpu()
    u, w = (x[..., :n // 2], x[..., n // 2:n]) if layout == M.ROTARY_HALF else (x[..., 0:n:2], x[..., 1:n:2])
    both = []
    for a, b, c, d in ((u * cos, w * sin, -1, u), (u * sin, w * cos, 1, u)):
        both.append((a + c * b, u.abs() * amplitude + w.abs() * amplitude))
    join = (lambda p: torch.cat(p, -1)) if layout == M.ROTARY_HALF else (lambda p: torch.stack(p, -1).flatten(-2))
    value = torch.cat([join([b[0] for b in both]), x[..., n:]], -1)
    size = torch.cat([join([b[1] for b in both]), torch.zeros_like(x[..., n:])], -1)
    return value, size


def check(got, want, dtype, what):
    value, size = want
    bound = 2.0 ** -21 * size + HALF_STEP[dtype] * value.abs()
    off = (got.double().cpu() - value).abs() - bound
    assert (off <= 0).all(), (what, float(off.max()))


def heads(tokens, kv, group, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((tokens, kv, group, d), generator=g, device="cuda").to(DT[dtype]), torch.randn((tokens, kv, d), generator=g, device="cuda").to(DT[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", [M.ROTARY_HALF, M.ROTARY_INTERLEAVED])
@pytest.mark.parametrize("d,n", [(128, 128), (64, 16), (160, 160), (96, 40), (72, 72), (256, 256), (64, 2), (8, 6), (80, 52), (256, 2)])
def test_forward_and_backward(dtype, layout, d, n):
    q, k = heads(37, 2, 3, d, dtype, d + n)
    positions = torch.randint(0, 40000, (37,), dtype=torch.int32, device="cuda")
    desc = M.rotary_desc(n, layout=layout)
    out = [torch.full_like(t, float("nan")) for t in (q, k)]
    for fn, sign in ((M.mtnlg_rotary_fwd, 1.0), (M.mtnlg_rotary_bwd, -1.0)):
        fn(desc, q, k, *out, positions=positions)
        for got, x in zip(out, (q, k)):
            check(got, turned(x, positions, n, layout, "none", sign=sign), dtype, fn.__name__)


@pytest.mark.parametrize("scaling", list(SCALED))
@pytest.mark.parametrize("n", [2, 64, 128])
def test_scalings_and_far_positions(scaling, n):
    q, k = heads(9, 1, 2, 128, "fp32", 3)
    positions = torch.tensor([0, 1, 2, 4095, 4096, 131071, 1 << 20, (1 << 24) + 1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    how, args = SCALED[scaling]
    out = [torch.empty_like(t) for t in (q, k)]
    M.mtnlg_rotary_fwd(M.rotary_desc(n, base=500000.0, scaling=how, **args), q, k, *out, positions=positions)
    for got, x in zip(out, (q, k)):
        check(got, turned(x, positions, n, M.ROTARY_HALF, scaling, base=500000.0), "fp32", scaling)


@pytest.mark.parametrize("layout", [M.ROTARY_HALF, M.ROTARY_INTERLEAVED])
@pytest.mark.parametrize("tokens", [1, 7, 8, 9, 1000])
def test_in_place_parts_of_a_fused_matrix_and_no_positions(layout, tokens):
    kv, group, d, n = 2, 3, 64, 32
    g = torch.Generator(device="cuda").manual_seed(tokens)
    qkv = torch.randn((tokens, kv, group + 2, d), generator=g, device="cuda").to(torch.bfloat16)
    before = qkv.clone()
    q, k = qkv[:, :, :group], qkv[:, :, group]
    M.mtnlg_rotary_fwd(M.rotary_desc(n, layout=layout), q, k, q, k)
    positions = torch.arange(tokens)
    check(q, turned(before[:, :, :group], positions, n, layout, "none"), "bf16", "q")
    check(k, turned(before[:, :, group], positions, n, layout, "none"), "bf16", "k")
    assert torch.equal(qkv[:, :, group + 1], before[:, :, group + 1])
    assert torch.equal(qkv[..., :group + 1, n:], before[..., :group + 1, n:])


def test_queries_alone_rows_of_padding_and_many_heads():
    g = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn((40, 96, 40), generator=g, device="cuda")
    out = torch.full_like(q, 7.0)
    positions = torch.arange(40, dtype=torch.int32, device="cuda") - 5
    q[:5] = float("nan")
    M.mtnlg_rotary_fwd(M.rotary_desc(40), q, None, out, None, positions=positions)
    assert (out[:5] == 7.0).all()
    check(out[5:], turned(q[5:], positions[5:], 40, M.ROTARY_HALF, "none"), "fp32", "q")


def test_turning_back_gives_the_heads_again_and_the_products_go_by_distance():
    q, k = heads(50, 1, 1, 64, "fp32", 8)
    desc = M.rotary_desc(64)
    one, two = [torch.empty_like(t) for t in (q, k)], [torch.empty_like(t) for t in (q, k)]
    M.mtnlg_rotary_fwd(desc, q, k, *one)
    M.mtnlg_rotary_bwd(desc, *one, *two)
    for got, x in zip(two, (q, k)):
        assert (got - x).abs().max() <= 2.0 ** -20 * 4 * x.abs().max()
    far = [torch.empty_like(t) for t in (q, k)]
    M.mtnlg_rotary_fwd(desc, q, k, *far, positions=torch.arange(50, dtype=torch.int32, device="cuda") + 100000)
    near_products = one[0][:, 0, 0].double() @ one[1][:, 0].double().T
    far_products = far[0][:, 0, 0].double() @ far[1][:, 0].double().T
    sizes = one[0][:, 0, 0].double().norm(dim=-1)[:, None] * one[1][:, 0].double().norm(dim=-1)
    assert ((near_products - far_products).abs() <= 2.0 ** -19 * sizes).all()


@pytest.mark.parametrize("tokens,kv", [(5, 1), (1, 2), (1, 1)])
def test_in_place_with_strides_that_are_not_looked_at(tokens, kv):
    # of dimensions of one, and a head of keys' heads: whatever stands there, the same matrix is the same
    q, k = heads(tokens, kv, 1, 64, "bf16", 12)
    before = q.clone(), k.clone()
    desc = B.RotaryDesc(B.BF16, kv, kv, 64, 64, M.ROTARY_HALF, M.ROTARY_UNSCALED, 0, tokens, 1e4, 1.0, 1.0, 32.0, 0.0)
    m = lambda t, other: B.Heads(t.data_ptr(), 64 * kv if tokens > 1 else 24 * other, 64 if kv > 1 else 40 * other, 8 * other)   # noqa: E731
    args = [m(q, 1), m(k, 2), m(q, 3), m(k, 4)]
    status = B.lib().mtnlg_rotary_fwd(ctypes.byref(desc), *(ctypes.byref(a) for a in args), None, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    for got, x in ((q, before[0]), (k, before[1])):
        check(got, turned(x, torch.arange(tokens), 64, M.ROTARY_HALF, "none"), "bf16", "in place")


def test_more_tokens_than_a_launch_has():
    # 64 tokens to a workgroup of 256: 2^30 of them are 2^32 work items.  Rows look alike, and so do the positions of all tokens but the ones that are looked at
    tokens = (1 << 30) + 100
    row = torch.randn((1, 1, 8), generator=torch.Generator(device="cuda").manual_seed(11), device="cuda").bfloat16()
    q, out = row.expand(tokens, 1, 8).contiguous(), torch.zeros((tokens, 1, 8), dtype=torch.bfloat16, device="cuda")
    for given in (True, False):
        positions = torch.full((tokens,), 77, dtype=torch.int32, device="cuda") if given else None
        at = [0, 1, (1 << 29) - 1, 1 << 29, (1 << 29) + 1, (1 << 30) - 1, 1 << 30, tokens - 1]
        if given:
            positions[at] = torch.arange(len(at), dtype=torch.int32, device="cuda") + 1000
        M.mtnlg_rotary_fwd(M.rotary_desc(2), q, None, out, None, positions=positions)
        check(out[at], turned(q[at], positions[at] if given else torch.tensor(at), 2, M.ROTARY_HALF, "none"), "bf16", "q")
        if given:
            others = (out == out[5]).all(-1)[:, 0]
            others[at] = True
            assert others.all()
        out.zero_()
    del q, out, positions
    torch.cuda.empty_cache()


def test_a_captured_call_replays():
    q, k = heads(300, 2, 4, 128, "bf16", 4)
    positions = torch.arange(300, dtype=torch.int32, device="cuda")
    desc = M.rotary_desc(128)
    out = [torch.empty_like(t) for t in (q, k)]
    M.mtnlg_rotary_fwd(desc, q, k, *out, positions=positions)
    want = [t.clone() for t in out]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mtnlg_rotary_fwd(desc, q, k, *out, positions=positions)
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
