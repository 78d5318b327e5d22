"""AdamW over many tensors at the edges of what its calls allow: the least alignment, as many tensors as may be, more chunks than workgroups."""
import pytest
import torch

import paper_2201_11990_amd as M
from test_gpu_adam_many import BLOCK, E4M3, check, copies, model, norm_of, run_norm, with_states

pytestmark = pytest.mark.gpu


def moved(t, by):
    """The same values `by` bytes behind a boundary of 256 bytes."""
    room = torch.zeros(t.numel() * t.element_size() + 256 + by, dtype=torch.uint8, device="cuda")
    return room[by:by + t.numel() * t.element_size()].view(t.dtype).copy_(t)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grads", ["fp32", "bf16"])
def test_the_least_alignment(grads, bits):
    rows = with_states(model([1, 3, 257, 4096, 4099, 70_001, 131_072 + 5], grads), bits)
    for t in rows:
        for k, by in (("master", 16), ("m", 4 if bits == 8 else 16), ("v", 4 if bits == 8 else 16), ("m_scale", 4), ("v_scale", 4),
                      ("grad", 8 if grads == "bf16" else 16), ("weight_bf16", 8)):
            if t.get(k) is not None:
                t[k] = moved(t[k], by)
    before = copies(rows)
    for some in (rows, rows[:4]):   # many chunks, and few in one launch
        sq, _ = run_norm(some)
        want = norm_of(some)
        assert abs(float(sq) - want) <= 2.0 ** -24 * want * 1.01
    sq, _ = run_norm(rows)
    M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=5, seed=21)
    check(before, rows, bits, float(sq), 5, seed=21)


@pytest.mark.parametrize("bits", [32, 8])
def test_as_many_tensors_as_may_be(bits):
    # 2^16 tensors of one to four elements, 16 bytes apart in fp32 (a block of scales each)
    n = 1 << 16
    flat = with_states(model([4 * n], "fp32"), 32)[0]
    if bits == 8:
        flat.update({k: with_states(model([4 * n], "fp32"), 8)[0][k] for k in ("m", "v")})
        flat.update({k: torch.full((n,), 1e-5, device="cuda") for k in ("m_scale", "v_scale")})
    count = [i * 7 % 4 + 1 for i in range(n)]
    part = lambda k, i: flat[k][i:i + 1] if k.endswith("scale") else flat[k][4 * i:4 * i + count[i]]   # noqa: E731
    keys = ("master", "m", "v", "grad", "weight_bf16") + (("m_scale", "v_scale") if bits == 8 else ())
    rows = [{k: part(k, i) for k in keys} | {"decay": i % 2 == 0} for i in range(n)]
    some = [0, 55, 56, 57, 159, 160, 161, 40_000, n - 1]
    before = [copies([rows[i]])[0] for i in some]
    beside = flat["master"].view(n, 4)[:, 3][torch.tensor(count, device="cuda") < 4].clone()
    table = M.AdamTensors(rows)
    sq, _ = run_norm(table)
    inside = torch.arange(4, device="cuda") < torch.tensor(count, device="cuda")[:, None]
    want = float((flat["grad"].double().view(n, 4) * inside).square().sum())
    assert abs(float(sq) - want) <= 2.0 ** -24 * want * 1.01
    M.mtnlg_adam_step_many(table, sq, lr=1e-3, step=3, seed=2)
    for old, i in zip(before, some):
        check([old], [rows[i]], bits, float(sq), 3, seed=2, block=i)
    assert torch.equal(flat["master"].view(n, 4)[:, 3][torch.tensor(count, device="cuda") < 4], beside)
    with pytest.raises(RuntimeError):
        M.mtnlg_adam_step_many(rows + [rows[0]], sq, lr=1e-3, step=3)


def test_more_chunks_than_workgroups():
    # 2^20 chunks of 4096 elements and some: workgroups come around
    n = (1 << 32) + 4096 * 5 + 300
    g = torch.Generator(device="cuda").manual_seed(7)
    part = torch.randn(1 << 20, generator=g, device="cuda") * 1e-3
    whole = lambda x: x.repeat(-(-n // x.numel()))[:n]   # noqa: E731
    codes = torch.randint(1, 127, (1 << 20,), generator=g, device="cuda", dtype=torch.uint8)
    row = {"master": whole(part * 20), "grad": whole(part.bfloat16()), "weight_bf16": None, "m": whole(codes).view(E4M3), "v": whole(codes.flip(0)).view(E4M3),
           "m_scale": torch.full((-(-n // BLOCK),), 1e-6, device="cuda"), "v_scale": torch.full((-(-n // BLOCK),), 1e-6, device="cuda")}
    spans = [(0, 20 * BLOCK), ((1 << 32) - 4096, (1 << 32) + 4096), ((n // BLOCK - 9) * BLOCK, n)]
    cut = lambda a, b: {k: (v[a // BLOCK:-(-b // BLOCK)] if k.endswith("scale") else v[a:b]).clone() for k, v in row.items() if v is not None}   # noqa: E731
    before = [cut(a, b) for a, b in spans]
    M.mtnlg_adam_step_many([row], lr=1e-3, step=4, seed=6)
    for old, (a, b) in zip(before, spans):
        check([old], [cut(a, b)], 8, None, 4, seed=6, block=a // BLOCK)
    del row, before
    torch.cuda.empty_cache()
