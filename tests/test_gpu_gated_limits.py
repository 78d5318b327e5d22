"""The gated feed-forward block with the largest weights that it takes (h F just under 2^31 - 2^23 elements, in fp32 2^30 - 2^22), where the byte offsets between the two
halves of w_fc1 pass 2^31 on every kernel: first, middle and last columns against 64 bits with the bounds of test_gpu_gated.py, all of the rest written."""
import pytest
import torch

import paper_2201_11990_amd as M
from gated_paths import path
from test_gpu_gated import DT, GATES, HALF_STEP, act, backward, check_backward, check_forward, check_weights, forward, product, room, within
from test_gpu_gated import F as STEP

# tokens, hidden, ffn, kernel of g
LIMITS = [("bf16", 5, 32768, 65280, "tokens"), ("bf16", 3, 2048, 1044480, "tokens"), ("bf16", 65, 32768, 65280, "ragged 128"), ("bf16", 100, 20480, 104448, "ragged 128 deep"),
          ("bf16", 130, 32768, 65280, "ragged 256"), ("bf16", 256, 32768, 65280, "256x256"), ("bf16", 256, 20480, 104448, "256x256, cut"),
          ("bf16", 256, 2048, 1044480, "256x320"), ("bf16", 33, 2040, 1048576, "tokens"), ("fp32", 5, 32768, 32640, "wave 32"), ("fp32", 40, 32768, 32640, "wave 64"), ("fp32", 70, 32768, 32640, "parts")]


@pytest.mark.parametrize("dtype,T,h,ffn,kernel", LIMITS)
def test_sizes_at_the_limit_go_to_their_kernels(dtype, T, h, ffn, kernel):
    most = 2 ** 31 - 2 ** 23 if dtype == "bf16" else 2 ** 30 - 2 ** 22
    assert most - 64 * h <= h * ffn <= most and path(dtype, T, h, ffn, "g") == kernel


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T,h,ffn,kernel", LIMITS)
def test_weights_at_the_limit(dtype, T, h, ffn, kernel):
    gen, dt = torch.Generator(device="cuda").manual_seed(T), DT[dtype]
    r = lambda *s, f=1.0: torch.randn(s, generator=gen, device="cuda", dtype=dt).mul_(f)   # noqa: E731
    nan = lambda *s: torch.full(s, float("nan"), dtype=dt, device="cuda")   # noqa: E731
    s = {"x": r(T, h), "w_fc1": r(2 * ffn, h, f=h ** -0.5), "w_fc2": r(h, ffn, f=ffn ** -0.5), "dy": r(T, h), "z": nan(T, 2 * ffn), "g": nan(T, ffn),
         "y": nan(T, h), "dz": nan(T, 2 * ffn), "dx": nan(T, h), "dw_fc1": nan(2 * ffn, h), "dw_fc2": nan(h, ffn)}
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES["silu"])
    ws, u = room(desc), HALF_STEP[dt]
    forward(desc, s, ws)
    backward(desc, s, ws)
    some = lambda n: torch.cat([torch.arange(a, a + 40, device="cuda") for a in (0, n // 2 - 20, n - 40)])   # noqa: E731
    cols, units = some(ffn), some(h)
    close = lambda got, want, e, what: within(got, want, e + u * (want.abs() + e), what)   # noqa: E731
    # z and g
    (za, ea), (zb, eb) = product(s["x"], s["w_fc1"][cols]), product(s["x"], s["w_fc1"][ffn + cols])
    close(s["z"][:, cols], za, ea, "z of the gate"), close(s["z"][:, ffn + cols], zb, eb, "z of the other")
    a, _ = act("silu", za)
    error = (1.13 * ea + 4 * STEP * (za.abs() + ea)) * (zb.abs() + eb) + a.abs() * eb + STEP * (a * zb).abs()
    close(s["g"][:, cols], a * zb, error, "g")
    close(s["y"][:, units], *product(s["g"], s["w_fc2"][units]), "y")
    # dz from the z that is stored
    za, zb = s["z"][:, cols].double(), s["z"][:, ffn + cols].double()
    a, slope = act("silu", za)
    dg, e = product(s["dy"], s["w_fc2"][:, cols].T)
    ea = (e * (slope.abs() + 40 * STEP) + dg.abs() * 40 * STEP) * zb.abs() + 2 * STEP * (dg * zb * slope).abs()
    eb = (e + STEP * dg.abs()) * (a.abs() + 4 * STEP * za.abs()) + dg.abs() * 4 * STEP * za.abs()
    close(s["dz"][:, cols], dg * zb * slope, ea, "dz of the gate"), close(s["dz"][:, ffn + cols], dg * a, eb, "dz of the other")
    close(s["dx"][:, units], *product(s["dz"], s["w_fc1"][:, units].T), "dx")
    for rows in (cols, ffn + cols):
        close(s["dw_fc1"][rows], *product(s["dz"][:, rows].T, s["x"].T), "dw_fc1")
    close(s["dw_fc2"][units], *product(s["dy"][:, units].T, s["g"].T), "dw_fc2")
    for k in ("z", "g", "y", "dz", "dx", "dw_fc1", "dw_fc2"):
        assert not torch.isnan(s[k]).any(), k
    del s, ws, a, za, zb, ea, eb, dg, e, slope, error
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,h,ffn", [("bf16", 8, 8), ("bf16", 16, 8), ("fp32", 8, 8), ("fp32", 8, 16)])
def test_as_many_tokens_as_may_be(dtype, h, ffn):
    # a thousand of 2^22 - 64 tokens are not zero, the first and the last among them: sums over tokens are sums of a thousand
    T, n = 2 ** 22 - 64, 1000
    gen, dt = torch.Generator(device="cuda").manual_seed(h + ffn), DT[dtype]
    at = torch.randint(0, T, (n,), generator=gen, device="cuda").index_fill_(0, torch.tensor([0], device="cuda"), T - 1).unique()
    s = {k: torch.zeros(shape, dtype=dt, device="cuda") for k, shape in (("x", (T, h)), ("dy", (T, h)))}
    for k in s:
        s[k][at] = torch.randn((len(at), h), generator=gen, device="cuda").to(dt)
    r = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(dt)   # noqa: E731
    nan = lambda *shape: torch.full(shape, float("nan"), dtype=dt, device="cuda")   # noqa: E731
    s.update(w_fc1=r(2 * ffn, h), w_fc2=r(h, ffn), z=nan(T, 2 * ffn), g=nan(T, ffn), y=nan(T, h), dz=nan(T, 2 * ffn), dx=nan(T, h), dw_fc1=nan(2 * ffn, h),
             dw_fc2=nan(h, ffn))
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES["gelu_tanh"])
    ws = room(desc)
    forward(desc, s, ws)
    backward(desc, s, ws)
    some = {k: (t[at] if t.shape[0] == T else t) for k, t in s.items()}
    check_forward("gelu_tanh", some)
    check_backward("gelu_tanh", some)
    check_weights(some, s["dw_fc1"], s["dw_fc2"])
    rest = torch.ones(T, dtype=torch.bool, device="cuda").index_fill_(0, at, False)
    for k in ("z", "g", "y", "dz", "dx"):
        assert (s[k][rest] == 0).all(), k
