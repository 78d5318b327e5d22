"""Host-side checks of the gated feed-forward block and of the optimizer step over many tensors that need no GPU: arguments are refused before any
launch, size queries answer, the binding looks at shapes and types."""
import ctypes

import pytest
import torch

import paper_2201_11990_amd as M
from paper_2201_11990_amd import binding as B

INVALID, NULL, SHAPE, SMALL = -1, -2, -3, -4
BIG = 1 << 50


def gated(**kw):
    d = dict(dtype=B.BF16, gate=B.GATE_SILU, tokens=100, hidden=64, ffn=128, flags=0)
    d.update(kw)
    return B.GatedDesc(*d.values())


NAMES = {False: ("x", "w_fc1", "w_fc2", "z", "g", "y"), True: ("x", "w_fc1", "w_fc2", "z", "g", "dy", "dz", "dx", "dw_fc1", "dw_fc2")}


def call_gated(desc, backward, ws=BIG, **kw):
    """status of a call whose matrices lie apart (never dereferenced: argument checks come first), `kw` put in their places"""
    at = {n: (i + 1) << 36 for i, n in enumerate(NAMES[backward] + ("workspace",))}
    at.update(kw)
    fn = B.lib().mtnlg_gated_ffn_bwd if backward else B.lib().mtnlg_gated_ffn_fwd
    return fn(None if desc is None else ctypes.byref(desc), *(at[n] for n in NAMES[backward]), at["workspace"], ws, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad,status", [(dict(dtype=2), INVALID), (dict(gate=-1), INVALID), (dict(gate=3), INVALID), (dict(tokens=0), INVALID),
                                        (dict(tokens=-5), INVALID), (dict(hidden=0), INVALID), (dict(ffn=0), INVALID), (dict(flags=1), INVALID),
                                        (dict(flags=8), INVALID), (dict(hidden=60), SHAPE), (dict(ffn=4), SHAPE), (dict(hidden=32776), SHAPE),
                                        (dict(ffn=(1 << 20) + 8), SHAPE), (dict(tokens=(1 << 22) - 63), SHAPE),
                                        (dict(hidden=32768, ffn=(1 << 16) - 248), SHAPE), (dict(dtype=B.F32, hidden=32768, ffn=(1 << 15) - 120), SHAPE)])
def test_gated_descriptors_that_are_refused(bad, status, backward):
    assert call_gated(gated(**bad), backward) == status
    assert M.mtnlg_gated_ffn_workspace(gated(**bad)) == 0


@pytest.mark.parametrize("backward", [False, True])
def test_gated_pointers_that_are_refused(backward):
    nullable = {"z"} if not backward else {"dx", "dw_fc1", "dw_fc2"}
    assert call_gated(None, backward) == NULL
    for n in NAMES[backward]:
        if n not in nullable:
            assert call_gated(gated(), backward, **{n: None}) == NULL, n
        assert call_gated(gated(), backward, **{n: (1 << 41) + 8}) == INVALID, n   # not of 16 bytes
    for desc in (gated(), gated(dtype=B.F32), gated(tokens=1), gated(tokens=512, hidden=2048, ffn=512)):
        need = M.mtnlg_gated_ffn_workspace(desc)
        if need:
            assert call_gated(desc, backward, workspace=None) == NULL
            assert call_gated(desc, backward, ws=need - 1) == SMALL
            assert call_gated(desc, backward, workspace=(1 << 41) + 8) == INVALID


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("backward", [False, True])
def test_gated_outputs_on_other_arguments_are_refused(backward, dtype):
    es = 4 if dtype == B.F32 else 2
    T, h, F = 100, 64, 128
    size = {"x": T * h, "w_fc1": 2 * F * h, "w_fc2": h * F, "z": 2 * T * F, "g": T * F, "y": T * h, "dy": T * h, "dz": 2 * T * F, "dx": T * h,
            "dw_fc1": 2 * F * h, "dw_fc2": h * F}
    outs = ("dz", "dx", "dw_fc1", "dw_fc2") if backward else ("z", "g", "y")
    for a in outs:
        for b in NAMES[backward]:
            if a == b:
                continue
            base = 1 << 42
            for shift in (0, size[b] * es - 16, 16 - size[a] * es):   # the same place; a's first bytes on b's last; a's last on b's first
                assert call_gated(gated(dtype=dtype), backward, **{b: base, a: base + shift}) == INVALID, (a, b, shift)


def test_gated_binding_refuses_shapes_and_types():
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)   # noqa: E731
    with pytest.raises(ValueError):
        M.gated_desc(t(3, 8), t(10, 16))
    with pytest.raises(ValueError):
        M.gated_desc(t(3, 8), t(9, 8))
    with pytest.raises(ValueError):
        M.gated_desc(t(2, 3, 8), t(16, 8))
    with pytest.raises(TypeError):
        M.gated_desc(t(3, 8, dt=torch.float16), t(16, 8, dt=torch.float16))
    desc = M.gated_desc(t(3, 8), t(16, 8), M.GATE_GELU_ERF, M.WGRAD_FP32)
    assert (desc.dtype, desc.gate, desc.tokens, desc.hidden, desc.ffn, desc.flags) == (B.BF16, 2, 3, 8, 8, 4)
    for x, w1, w2 in ((t(4, 8), t(16, 8), t(8, 8)), (t(3, 8), t(8, 8), t(8, 8)), (t(3, 8), t(16, 8), t(8, 16)), (t(3, 8, dt=torch.float32), t(16, 8), t(8, 8)),
                      (t(3, 8), t(16, 8, dt=torch.float32), t(8, 8))):
        with pytest.raises(ValueError):
            B._gated(desc, x, w1, w2)


def tensor(i=0, count=1000, **kw):
    d = dict(count=count, master=(8 * i + 1) << 40, m=(8 * i + 2) << 40, v=(8 * i + 3) << 40, m_scale=(8 * i + 4) << 40, v_scale=(8 * i + 5) << 40,
             grad=(8 * i + 6) << 40, weight_bf16=(8 * i + 7) << 40, decay=1)
    d.update(kw)
    return B.AdamTensor(*d.values())


def call_step(rows, sqnorm=None, desc=True, of=True, adam=None, **kw):
    d = dict(tensors=len(rows), grad_dtype=B.F32, state_bits=32, seed=0)
    d.update(kw)
    table = (B.AdamTensor * max(1, len(rows)))(*rows)
    many = B.AdamManyDesc(B.AdamDesc(*(adam or (1e-3, 0.9, 0.95, 1e-8, 0.1, 1.0, 1))), *d.values())
    return B.lib().mtnlg_adam_step_many(ctypes.byref(many) if desc else None, table if of else None, sqnorm, None)


def test_struct_sizes_are_those_of_the_header():
    assert ctypes.sizeof(B.AdamTensor) == 72 and ctypes.sizeof(B.AdamManyDesc) == 48 and ctypes.sizeof(B.GatedDesc) == 32


def test_step_arguments_that_are_refused():
    one = [tensor()]
    assert call_step(one, desc=False) == NULL and call_step(one, of=False) == NULL
    assert call_step(one, tensors=0) == INVALID and call_step(one, tensors=(1 << 16) + 1) == SHAPE
    for kw in (dict(grad_dtype=2), dict(state_bits=16), dict(state_bits=0)):
        assert call_step(one, **kw) == INVALID
    for adam in ((1e-3, 1.0, 0.95, 1e-8, 0.1, 1.0, 1), (1e-3, 0.9, -0.1, 1e-8, 0.1, 1.0, 1), (1e-3, 0.9, 0.95, 0.0, 0.1, 1.0, 1), (1e-3, 0.9, 0.95, 1e-8, 0.1, 1.0, 0),
                 (1e-3, float("nan"), 0.95, 1e-8, 0.1, 1.0, 1)):
        assert call_step(one, adam=adam) == INVALID
    for name in ("master", "m", "v", "grad"):
        assert call_step([tensor(), tensor(1, **{name: None})]) == NULL
        assert call_step([tensor(1, **{name: (1 << 45) + 8}), tensor()]) == INVALID
    assert call_step([tensor(weight_bf16=(1 << 45) + 4)]) == INVALID
    assert call_step([tensor(grad=(1 << 45) + 4)], grad_dtype=B.BF16) == INVALID
    for name in ("m_scale", "v_scale"):
        assert call_step([tensor(**{name: None})], state_bits=8) == NULL
        assert call_step([tensor(**{name: (1 << 45) + 2})], state_bits=8) == INVALID
    assert call_step([tensor(m=(1 << 45) + 2)], state_bits=8) == INVALID
    assert call_step(one, sqnorm=(1 << 45) + 2) == INVALID
    assert call_step([tensor(count=0)]) == INVALID and call_step([tensor(count=-1)]) == INVALID
    assert call_step([tensor(count=(1 << 39) + 1)]) == SHAPE
    # blocks of 256 are counted in 32 bits: two tensors of 2^39 elements have 2^32
    assert call_step([tensor(i, count=1 << 39) for i in range(2)]) == SHAPE


@pytest.mark.parametrize("bits", [32, 8])
def test_step_tensors_on_one_another_are_refused(bits):
    state = 4 if bits == 32 else 1
    size = {"master": 4000, "m": 1000 * state, "v": 1000 * state, "weight_bf16": 2000, "grad": 4000}
    if bits == 8:
        size.update(m_scale=16, v_scale=16)
    for a in size:
        for b in size:
            if a == "grad" and b == "grad":
                continue   # gradients may be shared: they are read only
            base = 1 << 46
            for shift in (0, size[b] // 16 * 16 - 16, 16 - size[a] // 16 * 16 if size[a] >= 16 else 0):
                first, second = {b: base}, {a: base + shift}
                if a == b:
                    assert call_step([tensor(0, **first), tensor(1, **second)], state_bits=bits) == INVALID, (a, b, shift)
                else:
                    assert call_step([tensor(0, **first, **second)], state_bits=bits) == INVALID, (a, b, shift)
                    assert call_step([tensor(0, **first), tensor(1), tensor(2, **second)], state_bits=bits) == INVALID, (a, b, shift)
        if a != "grad":
            assert call_step([tensor(0, **{a: 1 << 46})], sqnorm=1 << 46, state_bits=bits) == INVALID
    assert call_step([tensor(), tensor()], state_bits=bits) == INVALID


def test_norm_arguments_that_are_refused():
    def call(tensors, n=None, dtype=B.F32, workspace=1 << 50, size=BIG, sqnorm=1 << 51, of=True):
        table = (B.AdamTensor * max(1, len(tensors)))(*tensors)
        return B.lib().mtnlg_grad_sqnorm_many(len(tensors) if n is None else n, table if of else None, dtype, workspace, size, sqnorm, 0, None)

    one = [tensor()]
    assert call(one, of=False) == NULL and call(one, workspace=None) == NULL and call(one, sqnorm=None) == NULL
    assert call(one, n=0) == INVALID and call(one, n=(1 << 16) + 1) == SHAPE and call(one, dtype=3) == INVALID
    assert call(one, workspace=(1 << 50) + 4) == INVALID and call(one, sqnorm=(1 << 51) + 2) == INVALID
    assert call(one, size=M.mtnlg_grad_sqnorm_many_workspace() - 1) == SMALL
    assert call([tensor(), tensor(1, grad=None)]) == NULL
    assert call([tensor(grad=(1 << 45) + 8)]) == INVALID and call([tensor(grad=(1 << 45) + 4)], dtype=B.BF16) == INVALID
    assert call([tensor(count=0)]) == INVALID and call([tensor(count=(1 << 39) + 1)]) == SHAPE
    size, at = M.mtnlg_grad_sqnorm_many_workspace(), 1 << 45
    for kw in (dict(sqnorm=at), dict(sqnorm=at + 3996), dict(workspace=at), dict(workspace=at + 3984), dict(workspace=at - size + 16)):
        assert call([tensor(), tensor(1, grad=at)], **kw) == INVALID, kw
    for sqnorm in (1 << 50, (1 << 50) + size - 4):
        assert call(one, sqnorm=sqnorm) == INVALID


def test_tables_refuse_what_does_not_fit():
    t = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)   # noqa: E731
    with pytest.raises(ValueError):
        M.AdamTensors([])
    with pytest.raises(ValueError):   # not on a GPU
        M.AdamTensors([{"grad": t(5)}])
    with pytest.raises(TypeError):
        M.AdamTensors([{"grad": t(5, torch.float16)}])
