"""Which kernels the gated feed-forward block's tests reach: every size goes to the kernels that its entry names, and together they are all that there are."""
import ctypes

import pytest

from gated_paths import NAMES, PATHS, PRODUCTS, path
from paper_2201_11990_amd import binding as B
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


def test_more_work_items_than_a_launch_has_are_refused():
    # fp32 in parts: 512 to a tile of 128 x 128, less than 2^32 in all
    fn = B.lib()._ZN5mtnlg10gated_pathEPK16mtnlg_gated_descii
    fn.argtypes, fn.restype = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int], ctypes.c_int

    def ask(dtype, ffn):
        desc = B.GatedDesc(dtype, 0, 2 ** 22 - 64, 8, ffn, 0)
        return fn(ctypes.addressof(desc), 0, 0)

    assert NAMES[ask(B.F32, 255 * 64)] == "parts" and ask(B.F32, 255 * 64 + 8) == -3 and ask(B.BF16, 255 * 64 + 8) > 0
    desc = B.GatedDesc(B.F32, 0, 2 ** 22 - 64, 8, 255 * 64 + 8, 0)
    assert B.lib().mtnlg_gated_ffn_workspace(ctypes.byref(desc)) == 0
    assert B.lib().mtnlg_gated_ffn_fwd(ctypes.byref(desc), *((i + 1) << 46 for i in range(7)), 1 << 40, None) == -3
