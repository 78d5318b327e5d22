"""The gated feed-forward block against 64 bits.

u: half a step of the storage type (bf16 2^-8, fp32 2^-24); f = 2^-23 for every operation and addition of an fp32 sum.  A sum of n products is off by
f (n + 2) sum |a||b| at most (in whatever order, a matrix instruction may round down).  Activations have slopes of at most 1.13 and are worked out to
4 f |x| (x (1 + tanh) cancels for negative x, and its factors are off by f each), slopes to 40 f (the tanh form's second factor, x u'(x) (1 - tanh^2), reaches
17 times the error of tanh where it still moves).  What is stored rounded (g, dz) is what the next product takes: the reference takes the kernel's own."""
import pytest
import torch

import paper_2201_11990_amd as M

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F = 2.0 ** -23
GATES = {"silu": M.GATE_SILU, "gelu_tanh": M.GATE_GELU_TANH, "gelu_erf": M.GATE_GELU_ERF}
# tokens, hidden, ffn: one token to many, widths that no tile divides, whole tiles of every kernel, and rows on either side of where the kernels change
SIZES = [(1, 8, 8), (1, 2048, 1024), (2, 64, 40), (5, 1032, 520), (16, 512, 1368), (17, 520, 344), (24, 2560, 1024), (32, 776, 264), (33, 1024, 2048), (61, 520, 344),
         (64, 2048, 776), (65, 264, 128), (130, 264, 136), (128, 4096, 256), (256, 512, 1024), (300, 2048, 1000), (130, 1032, 5464), (777, 2048, 5464), (200, 4096, 4104), (106, 5664, 1648), (70, 8192, 520), (257, 1024, 776), (512, 640, 1280),
         (1024, 2048, 2048), (2048, 1280, 2560)]


def act(kind, x):
    x = x.detach().requires_grad_()
    a = torch.nn.functional.silu(x) if kind == "silu" else torch.nn.functional.gelu(x, approximate="tanh" if kind == "gelu_tanh" else "none")
    (slope,) = torch.autograd.grad(a.sum(), x)
    return a.detach(), slope


def within(got, value, bound, what):
    off = (got.double() - value).abs() - bound
    assert (off <= 0).all(), (what, float(off.max()), float(bound.max()))


def product(a, b, extra=0.0):
    """a b^T in 64 bits, and how far an fp32 sum may be from it"""
    a, b = a.double(), b.double()
    return a @ b.T, F * (a.shape[1] + 2) * (a.abs() @ b.abs().T) + extra


def inputs(T, h, ffn, dtype, seed=0, wide=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, f=1.0: (torch.randn(s, generator=g, device="cuda") * f).to(DT[dtype])   # noqa: E731
    nan = lambda *s, dt=DT[dtype]: torch.full(s, float("nan"), dtype=dt, device="cuda")   # noqa: E731
    wt = torch.float32 if wide else DT[dtype]
    return {"x": r(T, h), "w_fc1": r(2 * ffn, h, f=h ** -0.5), "w_fc2": r(h, ffn, f=ffn ** -0.5), "dy": r(T, h), "z": nan(T, 2 * ffn), "g": nan(T, ffn),
            "y": nan(T, h), "dz": nan(T, 2 * ffn), "dx": nan(T, h), "dw_fc1": nan(2 * ffn, h, dt=wt), "dw_fc2": nan(h, ffn, dt=wt)}


def room(desc):
    return torch.full((M.mtnlg_gated_ffn_workspace(desc),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN, whatever reads it


def forward(desc, s, ws, z=True):
    M.mtnlg_gated_ffn_fwd(desc, s["x"], s["w_fc1"], s["w_fc2"], s["z"] if z else None, s["g"], s["y"], ws)


def backward(desc, s, ws, **kw):
    a = {**s, **kw}
    M.mtnlg_gated_ffn_bwd(desc, *(a[k] for k in ("x", "w_fc1", "w_fc2", "z", "g", "dy", "dz", "dx", "dw_fc1", "dw_fc2")), ws)


def check_forward(kind, s, z=True, rows=slice(None)):
    u, ffn = HALF_STEP[s["x"].dtype], s["g"].shape[1]
    want, e = product(s["x"][rows], s["w_fc1"])
    if z:
        within(s["z"][rows], want, e + u * (want.abs() + e), "z")
    za, zb, ea, eb = want[:, :ffn], want[:, ffn:], e[:, :ffn], e[:, ffn:]
    a, _ = act(kind, za)
    g = a * zb
    error = (1.13 * ea + 4 * F * (za.abs() + ea)) * (zb.abs() + eb) + a.abs() * eb + F * g.abs()
    within(s["g"][rows], g, error + u * (g.abs() + error), "g")
    y, e = product(s["g"][rows], s["w_fc2"])
    within(s["y"][rows], y, e + u * (y.abs() + e), "y")


def check_backward(kind, s, rows=slice(None), dx=True):
    """dz and dx of some rows; values of dw_fc1, dw_fc2 with their bounds, roundings aside"""
    u, ffn = HALF_STEP[s["x"].dtype], s["g"].shape[1]
    z = s["z"][rows].double()
    a, slope = act(kind, z[:, :ffn])
    dg, e = product(s["dy"][rows], s["w_fc2"].T)
    da, db = dg * z[:, ffn:] * slope, dg * a
    ea = (e * (slope.abs() + 40 * F) + dg.abs() * 40 * F) * z[:, ffn:].abs() + 2 * F * da.abs()
    eb = (e + F * dg.abs()) * (a.abs() + 4 * F * z[:, :ffn].abs()) + dg.abs() * 4 * F * z[:, :ffn].abs()
    within(s["dz"][rows, :ffn], da, ea + u * (da.abs() + ea), "dz of the gate")
    within(s["dz"][rows, ffn:], db, eb + u * (db.abs() + eb), "dz of the other")
    if dx:
        want, e = product(s["dz"][rows], s["w_fc1"].T)
        within(s["dx"][rows], want, e + u * (want.abs() + e), "dx")


def check_weights(s, got1, got2, turns=1, start=0.0):
    for got, (want, e), what in ((got1, product(s["dz"].T, s["x"].T), "dw_fc1"), (got2, product(s["dy"].T, s["g"].T), "dw_fc2")):
        if got is None:
            continue
        u = HALF_STEP[got.dtype]
        within(got, turns * want + start, turns * (e + 2 * u * (turns * want.abs() + abs(start) + e)), what)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,ffn", SIZES)
def test_forward_and_backward(dtype, T, h, ffn):
    kind = ("silu", "gelu_tanh", "gelu_erf")[(T + h + ffn // 8) % 3]
    s = inputs(T, h, ffn, dtype)
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    ws = room(desc)
    forward(desc, s, ws)
    check_forward(kind, s)
    kept = {k: s[k].clone() for k in ("z", "g", "y")}
    backward(desc, s, ws)
    check_backward(kind, s)
    check_weights(s, s["dw_fc1"], s["dw_fc2"])
    # without z the same g and y, bit for bit
    s["g"].fill_(float("nan")), s["y"].fill_(float("nan"))
    forward(desc, s, ws, z=False)
    check_forward(kind, s, z=False)
    for k in kept:
        assert torch.equal(s[k], kept[k]), k


# A model in use: few tokens, no z.  Weights of all sizes, so that a workgroup has 16 to 96 of their rows; slabs of 64 for some of the eight waves, for all,
# several with a tail; token counts around whole groups; more tokens where the weights are many
@pytest.mark.parametrize("T,h,ffn", [(1, 8, 16), (1, 136, 10240), (3, 1032, 10248), (8, 20480, 328), (9, 72, 5120), (9, 1032, 10240), (15, 4096, 2048), (16, 2048, 8192),
                                     (17, 520, 12288), (20, 2048, 10240), (24, 4104, 7168), (31, 1544, 4096), (32, 20480, 640), (32, 600, 1304), (40, 2048, 16384),
                                     (48, 4096, 10240), (49, 8200, 4600), (64, 2048, 16392), (64, 5120, 14336), (41, 10240, 3584), (57, 2040, 1008), (33, 264, 520)])
def test_few_tokens(T, h, ffn):
    kind = ("silu", "gelu_tanh", "gelu_erf")[T % 3]
    s = inputs(T, h, ffn, "bf16", T)
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    ws = room(desc)
    forward(desc, s, ws, z=False)
    check_forward(kind, s, z=False)
    assert torch.isnan(s["z"]).all()
    want = s["g"].clone(), s["y"].clone()
    forward(desc, s, ws)
    check_forward(kind, s)
    assert torch.equal(s["g"], want[0]) and torch.equal(s["y"], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", list(GATES))
@pytest.mark.parametrize("T", [3, 90, 512])
def test_gates_far_from_zero(dtype, kind, T):
    # pre-activations up to 60 either way: exponentials that overflow, slopes that vanish
    s = inputs(T, 256, 512, dtype, 3)
    s["x"] *= 12
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    ws = room(desc)
    forward(desc, s, ws)
    check_forward(kind, s)
    backward(desc, s, ws)
    check_backward(kind, s)


@pytest.mark.parametrize("dtype,wide", [("bf16", False), ("bf16", True), ("fp32", False), ("fp32", True)])
@pytest.mark.parametrize("T,h,ffn", [(7, 72, 40), (130, 264, 136), (512, 512, 1024)])
def test_weight_gradients_added_up_and_in_fp32(dtype, wide, T, h, ffn):
    s = inputs(T, h, ffn, dtype, 1, wide)
    flags = M.WGRAD_FP32 if wide else 0
    ws = room(M.gated_desc(s["x"], s["w_fc1"]))
    forward(M.gated_desc(s["x"], s["w_fc1"]), s, ws)
    backward(M.gated_desc(s["x"], s["w_fc1"], flags=flags), s, ws)
    check_weights(s, s["dw_fc1"], s["dw_fc2"])
    s["dw_fc1"].fill_(3.0), s["dw_fc2"].fill_(3.0)
    for turn in (1, 2):
        backward(M.gated_desc(s["x"], s["w_fc1"], flags=flags | M.ACCUMULATE_WGRAD), s, ws)
        check_weights(s, s["dw_fc1"], s["dw_fc2"], turn, 3.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [5, 200, 512])
def test_gradients_that_are_not_wanted(dtype, T):
    s = inputs(T, 512, 256, dtype, 2)
    desc = M.gated_desc(s["x"], s["w_fc1"])
    ws = room(desc)
    forward(desc, s, ws)
    backward(desc, s, ws)
    outs = ("dz", "dx", "dw_fc1", "dw_fc2")
    for left_out in (("dx",), ("dw_fc1",), ("dw_fc2",), ("dw_fc1", "dw_fc2"), ("dx", "dw_fc1", "dw_fc2")):
        for k in outs:
            s[k].fill_(float("nan"))
        backward(desc, s, ws, **{k: None for k in left_out})
        assert all(torch.isnan(s[k]).all() for k in left_out)
        # (not bit for bit what all of them give: products that are one launch together may be other kernels alone, with sums in another order)
        check_backward("silu", s, dx="dx" not in left_out)
        check_weights(s, s["dw_fc1"] if "dw_fc1" not in left_out else None, s["dw_fc2"] if "dw_fc2" not in left_out else None)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,ffn", [(6, 512, 256), (40, 264, 128), (200, 520, 136), (512, 512, 512)])
def test_infinities_and_nan_of_a_token_stay_with_it(dtype, T, h, ffn):
    s = inputs(T, h, ffn, dtype, 4)
    desc = M.gated_desc(s["x"], s["w_fc1"], M.GATE_GELU_TANH)
    ws = room(desc)
    forward(desc, s, ws)
    backward(desc, s, ws)
    want = {k: s[k].clone() for k in ("z", "g", "y", "dz", "dx")}
    s["x"][2, 5], s["x"][3, 1], s["dy"][1, 7] = float("nan"), float("inf"), float("-inf")
    forward(desc, s, ws)
    backward(desc, s, ws)
    rows = [t for t in range(T) if t not in (1, 2, 3)]
    for k in want:
        if dtype == "bf16":
            assert torch.equal(s[k][rows], want[k][rows]), k
        else:   # (fp32: a tile beside an infinity is taken on other instructions, with sums in another order)
            near = (s[k][rows].double() - want[k][rows].double()).abs()
            assert (near <= 2 * F * (max(h, 2 * ffn) + 40) * want[k].abs()[rows].amax() * 30).all(), k
    assert torch.isnan(s["z"][2]).all() and torch.isnan(s["y"][2]).all()
    if dtype == "bf16":
        assert torch.equal(s["y"][1], want["y"][1])


def test_matrices_of_more_than_32_bits_of_elements():
    # z and dz of 2^31 and more elements: the last rows as those of a call of them alone, which the test above holds to 64 bits
    T, h, ffn = 70_000, 64, 16_384
    s = inputs(T, h, ffn, "bf16", 6)
    desc = M.gated_desc(s["x"], s["w_fc1"])
    ws = room(desc)
    forward(desc, s, ws)
    backward(desc, s, ws, dw_fc1=None)
    last = slice(T - 40, T)
    check_forward("silu", s, rows=last)
    check_backward("silu", s, rows=last)
    check_forward("silu", s, rows=slice(0, 40))
    check_backward("silu", s, rows=slice(0, 40))
    del s, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", list(GATES))
def test_gradients_against_differences(kind):
    T, h, ffn = 9, 72, 40
    s = inputs(T, h, ffn, "fp32", 5)
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    ws = room(desc)
    forward(desc, s, ws)
    backward(desc, s, ws)

    def y(x, w1, w2):
        z = x @ w1.T
        return ((act(kind, z[:, :ffn])[0] * z[:, ffn:]) @ w2.T * s["dy"].double()).sum()

    at = [s[k].double() for k in ("x", "w_fc1", "w_fc2")]
    e = 2.0 ** -10   # central differences: off by e^2 of a third derivative, of the slope's size
    for i, name in enumerate(("dx", "dw_fc1", "dw_fc2")):
        way = torch.randn(at[i].shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").double()
        move = lambda sign: y(*(t + sign * e * way if j == i else t for j, t in enumerate(at)))   # noqa: E731
        slope = (move(1) - move(-1)) / (2 * e)
        along, size = (s[name].double() * way).sum(), (s[name].double() * way).abs().sum()
        assert abs(slope - along) <= 1e-5 * size, name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,ffn", [(1, 2048, 512), (20, 520, 264), (48, 1024, 512), (300, 512, 520), (512, 512, 1024)])
def test_runs_are_identical_and_replays_too(dtype, T, h, ffn):
    s = inputs(T, h, ffn, dtype, 7)
    desc = M.gated_desc(s["x"], s["w_fc1"])
    ws = room(desc)
    outs = ("z", "g", "y", "dz", "dx", "dw_fc1", "dw_fc2")

    def run():
        forward(desc, s, ws)
        backward(desc, s, ws)

    run()
    want = {k: s[k].clone() for k in outs}
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):   # two graphs that share the workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
    for i in range(4):
        for k in outs:
            s[k].zero_()
        ws.fill_(0xFF)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s[k], want[k]) for k in outs)
        run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in outs:
            s[k].zero_()
        run()
    side.synchronize()
    assert all(torch.equal(s[k], want[k]) for k in outs)
    forward(desc, s, ws, z=False)
    assert torch.equal(s["z"], want["z"])


def test_rows_behind_the_outputs_are_left_as_they_were():
    for T, h, ffn in ((1, 264, 136), (15, 264, 136), (33, 520, 264), (130, 264, 136)):
        for dtype in ("bf16", "fp32"):
            s = inputs(T, h, ffn, dtype, 8)
            desc = M.gated_desc(s["x"], s["w_fc1"])
            ws = room(desc)
            whole = {k: torch.full((s[k].shape[0] + 70, s[k].shape[1]), 7.0, dtype=s[k].dtype, device="cuda") for k in ("z", "g", "y", "dz", "dx", "dw_fc1", "dw_fc2")}
            for k, t in whole.items():
                s[k] = t[:s[k].shape[0]]
            forward(desc, s, ws)
            backward(desc, s, ws)
            forward(desc, s, ws, z=False)
            assert all((t[s[k].shape[0]:] == 7).all() for k, t in whole.items())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", list(GATES))
@pytest.mark.parametrize("T", [16, 300])
def test_gates_at_their_limits(dtype, kind, T):
    h, ffn = 64, 128
    s = inputs(T, h, ffn, dtype)
    # z = [+- x0, x1] by weights of one value a row
    s["w_fc1"].zero_()
    s["w_fc1"][:ffn, 0] = torch.tensor([1.0, -1.0], device="cuda").repeat(ffn // 2)
    s["w_fc1"][ffn:, 1] = 1.0
    s["x"][:, 0] = torch.tensor([9.0, 12.0, 79.0, 81.0, 90.0, 1e4, 1e10, 1e12, 1e14, 1e20, 1e30, 1e36], device="cuda").repeat(T // 12 + 1)[:T]
    desc = M.gated_desc(s["x"], s["w_fc1"], GATES[kind])
    ws = room(desc)
    forward(desc, s, ws)
    check_forward(kind, s)
    backward(desc, s, ws)
    check_backward(kind, s)
    negative = s["z"][:, 1:ffn:2].double()
    assert (s["g"][:, 1::2].double().abs() <= 80 * torch.exp(-negative.abs().clamp(max=70))).all()   # act(-r) < r exp(-r)
    far = s["z"][:, :ffn].double().abs() >= 1e4   # slopes of 0 and 1
    dg, e = product(s["dy"], s["w_fc2"].T)
    one = (s["z"][:, :ffn] > 0).double() * dg * s["z"][:, ffn:].double()
    error = (e + 2 * F * dg.abs()) * s["z"][:, ffn:].double().abs() + 1e-20
    within(s["dz"][:, :ffn][far], one[far], (error + HALF_STEP[s["x"].dtype] * (one.abs() + error))[far], "dz far from zero")


def test_matrices_that_are_not_dense_or_elsewhere_are_refused():
    s = inputs(6, 64, 128, "bf16")
    desc = M.gated_desc(s["x"], s["w_fc1"])
    for k, bad in (("x", torch.empty(64, 6, dtype=torch.bfloat16, device="cuda").T), ("w_fc2", torch.empty(128, 64, dtype=torch.bfloat16, device="cuda").T),
                   ("g", torch.empty(6, 256, dtype=torch.bfloat16, device="cuda")[:, :128]), ("y", torch.empty(6, 64, dtype=torch.bfloat16)),
                   ("z", torch.empty(6, 128, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            forward(desc, {**s, k: bad}, None)
