"""Sizes of the gated feed-forward block chosen by the kernels that take its products, and the question which kernel that is."""
import ctypes

from paper_2201_11990_amd import binding as B

NAMES = {0: "plain", 1: "tokens", 2: "wave 32", 3: "wave 64", 4: "parts", 5: "group 32", 6: "group 64", 16: "256x256", 17: "256x320", 18: "ragged 256", 19: "ragged 128",
         20: "ragged 128 deep", 24: "cut 128"}   # enum gated_kernel, with enum gemm_tile from 16 on
PRODUCTS = ("g", "y", "dz", "dx")
DTYPES = {"bf16": B.BF16, "fp32": B.F32}


def path(dtype, T, h, ffn, product, with_dw=True):
    fn = B.lib()._ZN5mtnlg10gated_pathEPK16mtnlg_gated_descii
    fn.argtypes, fn.restype = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int], ctypes.c_int
    desc = B.GatedDesc(DTYPES[dtype], 0, T, h, ffn, 0)
    name = NAMES[fn(ctypes.addressof(desc), PRODUCTS.index(product), int(with_dw))]
    if name in ("256x256", "ragged 256") and last_round_is_cut(T, 2 * ffn if product == "g" else ffn, h):
        name += ", cut"
    return name


def last_round_is_cut(rows, columns, k):
    """Of 256 x 256 tiles, room for the partial ones given: up to 128 tiles in the last of less than four rounds, in parts of 8 slabs at least."""
    tiles, slabs = -(-rows // 256) * -(-columns // 256), -(-k // 64)
    return 0 < tiles % 256 <= 128 and tiles < 1024 and slabs >= 16


# tokens, hidden, ffn: the kernels of g, y, dz and dx, both weights' gradients wanted
PATHS = {
    ("bf16", 2048, 64, 10240): ("256x320", "plain", "256x320", "group 32"),
    ("bf16", 2048, 64, 5120): ("256x320", "plain", "256x256", "group 32"),
    ("bf16", 2560, 256, 3200): ("256x256", "plain", "ragged 128", "group 64"),
    ("bf16", 768, 4096, 1408): ("256x256, cut", "plain", "cut 128", "plain"),
    ("bf16", 256, 4096, 8448): ("256x256, cut", "plain", "256x256, cut", "cut 128"),
    ("bf16", 77, 5488, 3024): ("cut 128", "plain", "wave 32", "cut 128"),
    ("bf16", 77, 64, 4104): ("ragged 128", "plain", "group 32", "group 32"),
    ("bf16", 130, 512, 6240): ("ragged 128 deep", "plain", "ragged 128 deep", "cut 128"),
    ("bf16", 512, 4096, 4104): ("ragged 256, cut", "cut 128", "ragged 256, cut", "cut 128"),
    ("bf16", 700, 136, 11208): ("ragged 128", "cut 128", "ragged 256", "group 32"),
    ("bf16", 2816, 128, 4800): ("ragged 256", "plain", "ragged 256", "group 64"),
    ("bf16", 3000, 72, 2056): ("ragged 256", "plain", "ragged 128", "group 64"),
    ("fp32", 34, 64, 8000): ("wave 64", "plain", "group 32", "group 32"),
    ("fp32", 1500, 136, 2056): ("parts", "plain", "parts", "group 32"),
    ("fp32", 1100, 256, 2304): ("parts", "plain", "parts", "group 32"),
}
