"""The gated feed-forward block's activations and slopes by value: rows of weights with a single one, so that pre-activations are exact, the other half is 1, and
g and both halves of dz are act(x), act'(x) and act(x), rounded once."""
import pytest
import torch

import paper_2201_11990_amd as M
from test_gpu_gated import DT, GATES, backward, forward, inputs, room

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
