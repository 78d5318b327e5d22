"""The root-mean-square norm with the residual's addition against 64 bits.

f = 2^-23 for every operation in fp32 (a step: sums over h columns in some order are off by f log2(h) at most when summed as a tree
over lanes of up to 32 terms, taken as f * 64), u: half a step of the storage type."""
import pytest
import torch

import paper_2201_11990_amd as M

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
F, EPS = 2.0 ** -23, 1e-5
SIZES = [(1, 8), (3, 64), (5, 520), (61, 1032), (9, 2048), (7, 2056), (130, 4096), (301, 1024), (37, 4104), (600, 8192), (5, 8200), (6, 16392), (3, 20480), (2, 24584), (2, 32768)]


def inputs(T, h, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    return {"x": r(T, h).to(DT[dtype]), "residual": (3 * r(T, h)).to(DT[dtype]), "gamma": (1 + 0.2 * r(h)).to(DT[dtype]), "dout": r(T, h).to(DT[dtype]),
            "dres": r(T, h).to(DT[dtype])}


def within(got, value, bound, what):
    off = (got.double() - value).abs() - bound
    assert (off <= 0).all(), (what, float(off.max()))


def norm64(x, gamma):
    x = x.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    return r, x * r * gamma.double()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h", SIZES)
@pytest.mark.parametrize("with_residual", [True, False])
def test_forward(dtype, T, h, with_residual):
    s = inputs(T, h, dtype)
    u = HALF_STEP[dtype]
    out, xsum, rstd = torch.full_like(s["x"], float("nan")), torch.full_like(s["x"], 7.0), torch.empty(T, device="cuda")
    M.mtnlg_rmsnorm_fwd(s["x"], s["gamma"], EPS, out, rstd, residual=s["residual"] if with_residual else None, xsum=xsum if with_residual else None)
    if with_residual:
        total = s["x"].double() + s["residual"].double()
        within(xsum, total, u * total.abs() + F * total.abs(), "xsum")
    r, y = norm64(xsum if with_residual else s["x"], s["gamma"])
    within(rstd, r[:, 0], 40 * F * r[:, 0], "rstd")
    within(out, y, (u + 45 * F) * y.abs(), "out")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h", SIZES + [(3000, 512), (1500, 2048)])
@pytest.mark.parametrize("with_dres", [True, False])
def test_backward(dtype, T, h, with_dres):
    s = inputs(T, h, dtype, 1)
    u = HALF_STEP[dtype]
    r, _ = norm64(s["x"], s["gamma"])
    rstd = r[:, 0].float()
    x, g, d = s["x"].double(), s["gamma"].double(), s["dout"].double()
    n = x * r
    dot = (d * g * n).mean(-1, keepdim=True)
    size = (d * g * n).abs().mean(-1, keepdim=True)
    dx = r * (d * g - n * dot)
    error = r * ((d * g).abs() * 8 * F + n.abs() * (dot.abs() * 8 * F + size * 64 * F))
    if with_dres:
        dx = dx + s["dres"].double()
        error = error + dx.abs() * F
    dgamma, dg_size = (d * n).sum(0), (d * n).abs().sum(0)
    ws = torch.full((M.mtnlg_rmsnorm_bwd_workspace(T, h),), 0xFF, dtype=torch.uint8, device="cuda")
    for grad_dtype in {torch.float32, DT[dtype]}:
        got, got_g = torch.full_like(s["x"], float("nan")), torch.zeros(h, dtype=grad_dtype, device="cuda")
        for turn in (1, 2):   # overwritten, then added to
            M.mtnlg_rmsnorm_bwd(s["x"], s["gamma"], rstd, s["dout"], got, got_g, ws, dres=s["dres"] if with_dres else None, accumulate=turn == 2)
            within(got, dx, error + u * dx.abs(), "dx")
            step = turn * (2.0 ** -8 if grad_dtype == torch.bfloat16 else 2.0 ** -24)
            within(got_g, turn * dgamma, turn * step * dgamma.abs() + turn * 64 * F * dg_size, "dgamma")


def test_gradient_of_both_summands_in_place_and_against_differences():
    T, h = 6, 264
    s = inputs(T, h, "fp32", 5)
    x = s["x"].clone()
    rstd, out = torch.empty(T, device="cuda"), torch.empty_like(x)
    M.mtnlg_rmsnorm_fwd(x, s["gamma"], EPS, out, rstd, residual=s["residual"], xsum=x)   # the sum over one of its summands
    ws = torch.empty(M.mtnlg_rmsnorm_bwd_workspace(T, h), dtype=torch.uint8, device="cuda")
    dx, dgamma = s["dout"].clone(), torch.empty(h, device="cuda")
    M.mtnlg_rmsnorm_bwd(x, s["gamma"], rstd, dx, dx, dgamma, ws)   # over dout
    # central differences of step e: off by e^2 of a third derivative, which is of the slope's size for unit rows
    e = 2.0 ** -10
    for name, grad in (("x", dx), ("gamma", dgamma)):
        way = torch.randn(grad.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").double()
        at = lambda sign: norm64(x.double() + (sign * e * way if name == "x" else 0), s["gamma"].double() + (sign * e * way if name == "gamma" else 0))[1]   # noqa: E731
        slope = ((at(1) - at(-1)) * s["dout"].double()).sum() / (2 * e)
        along, size = (grad.double() * way).sum(), (grad.double() * way).abs().sum()
        assert abs(slope - along) <= 1e-5 * size


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,columns", [(1, 8, 0), (5, 520, 128), (61, 1032, 0), (9, 2048, 128), (7, 2056, 512), (5, 8200, 64), (3, 20480, 128), (2, 32768, 0),
                                         (4, 72, 8), (3, 136, 32)])
def test_eight_bits(dtype, T, h, columns):
    s = inputs(T, h, dtype, 2)
    n = columns or h
    scale, rstd = torch.full((T, -(-h // n)), float("nan"), device="cuda"), torch.empty(T, device="cuda")
    out, xsum = torch.empty((T, h), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty_like(s["x"])
    s["gamma"][:n] = 0 if h > n else s["gamma"][:n]   # a whole group of zeros
    M.mtnlg_rmsnorm_fwd_e4m3(s["x"], s["gamma"], EPS, out, scale, rstd, columns=columns, residual=s["residual"], xsum=xsum)
    r, y = norm64(xsum, s["gamma"])
    within(rstd, r[:, 0], 40 * F * r[:, 0], "rstd")
    parts = y.split(n, -1)
    most = torch.stack([p.abs().amax(-1) for p in parts], -1)
    want_scale = torch.where(most > 0, most / 448, 1.0)
    within(scale, want_scale, 50 * F * want_scale, "scale")
    wide = torch.repeat_interleave(scale.double(), n, -1)[:, :h]
    code = y / wide
    # half a step: 2^-4 of a normal value (from 2^-6 on), else 2^-10; and where the fp32 value lies across a border from the exact one, 50 f more
    within(out, code, torch.maximum(2.0 ** -4 * code.abs(), torch.full_like(code, 2.0 ** -10)) + 50 * F * code.abs(), "out")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,columns", [(2000, 2048, 128), (1500, 1000, 0), (70, 20480, 8)])
def test_codes_and_scales_bit_by_bit(dtype, T, h, columns):
    # from the norm's rstd on every operation rounds once to fp32, here as there: two products, the largest magnitude / 448, the quotient by that scale; then to the nearest code
    s = inputs(T, h, dtype, 7)
    n = columns or h
    scale, rstd = torch.empty((T, -(-h // n)), device="cuda"), torch.empty(T, device="cuda")
    out, xsum = torch.empty((T, h), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty_like(s["x"])
    M.mtnlg_rmsnorm_fwd_e4m3(s["x"], s["gamma"], EPS, out, scale, rstd, columns=columns, residual=s["residual"], xsum=xsum)
    y = xsum.cpu().float() * rstd.cpu()[:, None] * s["gamma"].cpu().float()
    want_scale = torch.stack([p.abs().amax(-1) for p in y.split(n, -1)], -1) / 448
    assert torch.equal(scale.cpu(), want_scale)
    codes = (y / torch.repeat_interleave(want_scale, n, -1)[:, :h]).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert torch.equal(out.cpu().view(torch.uint8), codes.view(torch.uint8))


@pytest.mark.parametrize("columns", [0, 32])
def test_eight_bits_beside_an_infinity(columns):
    # an infinite scale: quotients of what is finite are zeros, of the infinity itself not a number; other groups are as they were
    x, gamma = torch.randn((3, 64), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda"), torch.ones(64, device="cuda")
    new = lambda: (torch.empty((3, 64), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((3, 2 if columns else 1), device="cuda"))   # noqa: E731
    (codes, scale), (want, want_scale), rstd = new(), new(), torch.empty(3, device="cuda")
    M.mtnlg_rmsnorm_fwd_e4m3(x, gamma, EPS, want, want_scale, rstd, columns=columns)
    gamma[5] = float("inf")
    M.mtnlg_rmsnorm_fwd_e4m3(x, gamma, EPS, codes, scale, rstd, columns=columns)
    assert torch.isposinf(scale[:, 0]).all() and torch.isnan(codes[:, 5].float()).all()
    others = [i for i in range(columns or 64) if i != 5]
    assert (codes.float()[:, others] == 0).all()
    if columns:
        assert torch.equal(scale[:, 1], want_scale[:, 1]) and torch.equal(codes.float()[:, columns:], want.float()[:, columns:])


def test_rows_of_zeros_infinities_and_nan():
    x = torch.randn((5, 64), device="cuda")
    x[1], x[2, 5], x[3, 7] = 0, float("nan"), float("inf")
    gamma, out, rstd = torch.ones(64, device="cuda"), torch.empty_like(x), torch.empty(5, device="cuda")
    M.mtnlg_rmsnorm_fwd(x, gamma, 0.0, out, rstd)
    assert torch.isfinite(out[[0, 4]]).all() and torch.isnan(out[1]).all() and torch.isnan(out[2]).all() and torch.isnan(out[3, 7]) and (out[3, :7] == 0).all()
    M.mtnlg_rmsnorm_fwd(x, gamma, EPS, out, rstd)
    assert (out[1] == 0).all()
    codes, scale = torch.empty((5, 64), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((5, 1), device="cuda")
    M.mtnlg_rmsnorm_fwd_e4m3(x, gamma, EPS, codes, scale, rstd)
    assert (codes[1].float() == 0).all() and scale[1] == 1 and torch.isnan(codes[2].float()).all()


@pytest.mark.parametrize("columns", [0, 32])
def test_eight_bits_of_results_too_small_for_their_scale(columns):
    # magnitudes / 448 below 2^-126: that is the scale then.  (F: half a step of the smallest fp32 numbers, 2^-150, many times over)
    x = torch.randn((6, 64), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    x[:, 40] = 0
    gamma = torch.full((64,), 2.0 ** -120, device="cuda")
    codes, scale, rstd = torch.empty((6, 64), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((6, 2 if columns else 1), device="cuda"), torch.empty(6, device="cuda")
    M.mtnlg_rmsnorm_fwd_e4m3(x, gamma, EPS, codes, scale, rstd, columns=columns)
    assert (scale == 2.0 ** -126).all()
    code = norm64(x, gamma)[1] * 2.0 ** 126
    within(codes, code, torch.maximum(2.0 ** -4 * code.abs(), torch.full_like(code, 2.0 ** -10)) + 50 * F * code.abs() + F, "codes")


@pytest.mark.parametrize("T,h", [((1 << 21) + 5, 16), ((1 << 22) + 3, 4104), ((1 << 26) + 5, 8)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_more_rows_than_a_launch_has(T, h, with_residual):
    # with a workgroup of 16 waves to a row, or four rows to one of 256 threads, 2^22 and 2^26 rows are 2^32 work items.  Rows that all look alike but for their sign and a factor of 2
    g = torch.Generator(device="cuda").manual_seed(8)
    one, gamma = torch.randn(h, generator=g, device="cuda").bfloat16(), (1 + 0.2 * torch.randn(h, generator=g, device="cuda")).bfloat16()
    rows = torch.arange(T, device="cuda") % 3
    factor = torch.tensor([1.0, -1.0, 2.0], device="cuda").bfloat16()
    x = factor[rows][:, None] * one
    residual = x if with_residual else None
    out, rstd = torch.empty_like(x), torch.full((T,), float("nan"), device="cuda")
    out.fill_(float("nan"))
    xsum = torch.empty_like(x) if with_residual else None
    M.mtnlg_rmsnorm_fwd(x, gamma, EPS, out, rstd, residual=residual, xsum=xsum)
    three = factor[:, None] * one * (2 if with_residual else 1)
    r, y = norm64(three, gamma)
    within(out[-3:], y[rows[-3:]], (2.0 ** -8 + 45 * F) * y[rows[-3:]].abs(), "out")
    within(rstd[-3:], r[rows[-3:], 0], 40 * F * r[rows[-3:], 0], "rstd")
    same = lambda t: (t[:T // 3 * 3].unflatten(0, (-1, 3)) == t[:3]).all() and torch.equal(t[T // 3 * 3:], t[:T % 3])   # noqa: E731
    within(out[:3], y, (2.0 ** -8 + 45 * F) * y.abs(), "out")
    assert same(rstd) and same(out)
    if with_residual:
        assert torch.equal(xsum[:3], three) and same(xsum)
    del out, x, residual
    codes, scale = torch.zeros((T, h), dtype=torch.uint8, device="cuda"), torch.zeros((T, 1), device="cuda")
    x = factor[rows][:, None] * one
    M.mtnlg_rmsnorm_fwd_e4m3(x, gamma, EPS, codes.view(torch.float8_e4m3fn), scale, rstd)
    assert same(codes) and same(scale) and (scale > 0).all()
    del x, codes, xsum
    torch.cuda.empty_cache()


def test_runs_are_identical_and_replays_too():
    s = inputs(700, 2048, "bf16", 3)
    rstd, out, dx, dgamma = torch.empty(700, device="cuda"), torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(2048, device="cuda")
    xsum = torch.empty_like(s["x"])
    ws = torch.empty(M.mtnlg_rmsnorm_bwd_workspace(700, 2048), dtype=torch.uint8, device="cuda")

    def run():
        M.mtnlg_rmsnorm_fwd(s["x"], s["gamma"], EPS, out, rstd, residual=s["residual"], xsum=xsum)
        M.mtnlg_rmsnorm_bwd(xsum, s["gamma"], rstd, s["dout"], dx, dgamma, ws, dres=s["dres"])

    run()
    want = [t.clone() for t in (out, rstd, dx, dgamma)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in (out, rstd, dx, dgamma):
            t.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, rstd, dx, dgamma), want))
