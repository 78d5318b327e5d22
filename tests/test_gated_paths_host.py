"""Which kernels the gated feed-forward block's tests reach: every size goes to the kernels that its entry names, and together they are all that there are."""
import pytest

from gated_paths import PATHS, PRODUCTS, path
from test_gpu_gated import SIZES


@pytest.mark.parametrize("size", list(PATHS), ids=str)
def test_sizes_go_to_the_kernels_that_they_were_chosen_for(size):
    assert tuple(path(*size, product) for product in PRODUCTS) == PATHS[size]


def test_every_kernel_is_reached():
    stream = {"256x256", "256x256, cut", "256x320", "ragged 256", "ragged 256, cut", "ragged 128", "ragged 128 deep", "cut 128"}
    every = {("bf16", "g"): stream | {"tokens", "wave 32", "wave 64"}, ("bf16", "y"): {"tokens", "cut 128", "plain"},
             ("bf16", "dz"): stream | {"wave 32", "wave 64", "group 32", "group 64"}, ("bf16", "dx"): {"cut 128", "group 32", "group 64", "plain"},
             ("fp32", "g"): {"wave 32", "wave 64", "parts"}, ("fp32", "y"): {"plain"}, ("fp32", "dz"): {"wave 32", "wave 64", "parts", "group 32"},
             ("fp32", "dx"): {"group 32", "plain"}}
    sizes = [(dtype, *s) for s in SIZES for dtype in ("bf16", "fp32")] + list(PATHS)
    for (dtype, product), want in every.items():
        assert {path(*s, product) for s in sizes if s[0] == dtype} == want, (dtype, product)
