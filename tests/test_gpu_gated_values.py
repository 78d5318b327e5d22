"""The gated feed-forward block's activations and slopes by value: rows of weights with a single one, so that pre-activations are exact, the other half is 1, and
g and both halves of dz are act(x), act'(x) and act(x), rounded once."""
import pytest
import torch

import paper_2201_11990_amd as M
from test_gpu_gated import DT, GATES, HALF_STEP, backward, forward, inputs, room, within

pytestmark = pytest.mark.gpu
# tokens, hidden, ffn: bf16 few tokens, 32 / 64 tiles, streaming tiles (cut along K, ragged, whole); fp32 32 / 64 tiles, in parts
SIZES = [(3, 64, 64), (90, 256, 512), (300, 512, 2048), (512, 2048, 2048)]


def one_hot(T, h, ffn, dtype, kind):
    """A call whose z is [+- x[:, 0], 1] and whose dg is 1: columns alternate in sign."""
    s = inputs(T, h, ffn, dtype)
    for k in ("x", "w_fc1", "w_fc2", "dy"):
        s[k].zero_()
    s["x"][:, 1] = 1.0
    s["w_fc1"][:ffn, 0] = torch.tensor([1.0, -1.0], device="cuda").repeat(ffn // 2)
    s["w_fc1"][ffn:, 1] = 1.0
    s["dy"][:, 0] = 1.0
    s["w_fc2"][0] = 1.0
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    return s, desc, room(desc)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", list(GATES))
@pytest.mark.parametrize("T,h,ffn", SIZES)
def test_infinite_pre_activations_are_not_hidden(dtype, kind, T, h, ffn):
    # sums that pass the largest value: inf act(z) is inf, at -inf it is -inf times 0, and so is the second term of both slopes
    s, desc, ws = one_hot(T, h, ffn, dtype, kind)
    s["x"][::2, 0] = s["x"][::2, 2] = 3e38
    s["w_fc1"][:ffn, 2] = s["w_fc1"][:ffn, 0]
    forward(desc, s, ws)
    backward(desc, s, ws)
    z, g, dz = (s[k].float() for k in ("z", "g", "dz"))
    assert (z[::2, :ffn:2] == float("inf")).all() and (z[::2, 1:ffn:2] == -float("inf")).all() and (z[:, ffn:] == 1).all()
    assert (g[::2, ::2] == float("inf")).all() and torch.isnan(g[::2, 1::2]).all()
    assert (dz[::2, ffn::2] == float("inf")).all() and torch.isnan(dz[::2, ffn + 1::2]).all()
    assert torch.isnan(dz[::2, :ffn]).all()
    # the other tokens (x = 0)
    assert (g[1::2] == 0).all() and (dz[1::2, :ffn] == 0.5).all() and (dz[1::2, ffn:] == 0).all()


F = 2.0 ** -23
REACH = {"silu": 60.0, "gelu_tanh": 9.0, "gelu_erf": 12.5}   # how far either way: everything that is worked out stays a normal number


def by_value(kind, x):
    """act(x), act'(x) in 64 bits without cancellation, and how far either may be off in fp32, in f = 2^-23 and before it is stored.

    The argument of an exponential is off by f for each of two operations, which moves the exponential by that times the argument: SiLU |x|, the tanh form 3 |2 u| (u of five
    operations), the erf form x^2 (a square, a product; of erfc(y) x^2 = 2 y^2 times what y = |x| / sqrt 2 is off).  A few operations more of f each, the hardware's
    exponential and reciprocal included; 24 in the polynomial of the erf form: 11 for its steps, 7 for what its argument is off, 2 for its fit.  A slope is s + t of two such terms with the exponential twice
    in t, off by that of |s| + |t|; SiLU's in fp32 takes 1 - s, which is off by f, from s."""
    if kind == "silu":
        s, r = torch.sigmoid(x), torch.sigmoid(-x)
        t, e = x * s * r, x.abs()
        return x * s, s + t, F * (e + 8) * (x * s).abs(), F * (2 * e + 16) * (s + t.abs()) + 8 * F * x.abs() * s * (x > 0)
    if kind == "gelu_tanh":
        k = (2 / torch.pi) ** 0.5
        w = 2 * k * (x + 0.044715 * x ** 3)
        s, r = torch.sigmoid(w), torch.sigmoid(-w)
        t, e = x * 2 * k * (1 + 3 * 0.044715 * x * x) * s * r, 3 * w.abs()
        return x * s, s + t, F * (e + 8) * (x * s).abs(), F * (2 * e + 16) * (s + t.abs())
    s = 0.5 * torch.special.erfc(-x * 0.5 ** 0.5)
    t = x * torch.exp(-0.5 * x * x) * (0.5 / torch.pi) ** 0.5
    return x * s, s + t, F * (x * x + 25) * (x * s).abs(), F * (x * x + 25) * (s + t.abs())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", list(GATES))
@pytest.mark.parametrize("T,h,ffn", SIZES)
def test_activations_and_slopes_by_value(dtype, kind, T, h, ffn):
    # relative to the value, as far as 1e-29 from zero: nothing cancels where x is negative
    s, desc, ws = one_hot(T, h, ffn, dtype, kind)
    most = REACH[kind]
    if dtype == "bf16":   # values of 8 bits
        at = torch.arange(ffn, device="cuda") * 37 % 200 * (most / 200)
        at = at.bfloat16().float()
    else:
        at = torch.rand(ffn, generator=torch.Generator(device="cuda").manual_seed(T), device="cuda") * most
    s["w_fc1"][:ffn, 0] = at
    s["x"][:, 0] = torch.tensor([1.0, -1.0], device="cuda").repeat(T)[:T]
    forward(desc, s, ws)
    backward(desc, s, ws)
    z = s["x"][:, :1].double() * at.double()
    assert torch.equal(s["z"][:, :ffn].double(), z) and (s["z"][:, ffn:] == 1).all()
    u = HALF_STEP[DT[dtype]]
    a, slope, ea, es = by_value(kind, z)
    for got, value, e, what in ((s["g"], a, ea, "act"), (s["dz"][:, ffn:], a, ea, "act of the backward pass"), (s["dz"][:, :ffn], slope, es, "slope")):
        within(got, value, e + u * (value.abs() + e), what)
