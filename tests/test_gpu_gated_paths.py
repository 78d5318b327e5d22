"""The gated feed-forward block on every kernel that takes one of its products (gated_paths.py), against 64 bits with the bounds of test_gpu_gated.py."""
import pytest
import torch

import paper_2201_11990_amd as M
from gated_paths import PATHS
from test_gpu_gated import GATES, backward, check_backward, check_forward, check_weights, forward, inputs, room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(GATES))
@pytest.mark.parametrize("size", list(PATHS), ids=str)
def test_forward_and_backward_on_every_kernel(size, kind):
    dtype, T, h, ffn = size
    s = inputs(T, h, ffn, dtype, 11)
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    ws = room(desc)
    forward(desc, s, ws)
    check_forward(kind, s)
    kept = {k: s[k].clone() for k in ("z", "g", "y")}
    backward(desc, s, ws)
    check_backward(kind, s)
    check_weights(s, s["dw_fc1"], s["dw_fc2"])
    # the products of the inputs' gradients alone, which may be other kernels
    s["dz"].fill_(float("nan")), s["dx"].fill_(float("nan"))
    backward(desc, s, ws, dw_fc1=None, dw_fc2=None)
    check_backward(kind, s)
    # without z the same g and y, bit for bit
    s["g"].fill_(float("nan")), s["y"].fill_(float("nan"))
    forward(desc, s, ws, z=False)
    for k in kept:
        assert torch.equal(s[k], kept[k]), k
