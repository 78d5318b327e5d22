"""The operators of a packed batch's decoder layer one after the other, as a layer uses them: norm, product, rotary positions in place, attention on the
fused matrix, product, residual and norm; then all of it backwards.  Against the same chain in 64 bits with automatic gradients.

Distances are of whole matrices, relative.  bf16: each matrix stored on the way (and the weights and score gradients that attention rounds for its products) moves
what follows by at most half a step of its own size, 2^-8; the way to the output stores 6 (norm, product, turned heads, weights, attention, product), and the
gradients store 8 more (the sum for the second norm, its gradient, attention's, score gradients, head gradients, turned back, product, norm).  These
movements are of different elements' own and do not line up, so that their plain sum leaves room for what products pass on enlarged.
fp32: 2^-24 for each of those, and 2^-23 for each addition of the longest sum of each step, which a row of every product has.
"""
import math

import pytest
import torch

import paper_2201_11990_amd as M

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
LENGTHS, H, KV, GROUP, D, TURNED, EPS = [70, 1, 129, 0, 56], 256, 2, 2, 64, 48, 1e-5


def chain(x, gamma, w_qkv, w_out, gamma2, positions):
    """(out, second norm), all in 64 bits"""
    norm = lambda t, g: t * torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS) * g   # noqa: E731
    qkv = (norm(x, gamma) @ w_qkv.T).view(-1, KV, GROUP + 2, D)
    angle = positions.double()[:, None] * 10000.0 ** (-torch.arange(0, TURNED, 2, dtype=torch.float64, device=x.device) / TURNED)
    cos, sin = angle.cos()[:, None, None], angle.sin()[:, None, None]

    def turn(t):
        u, w = t[..., :TURNED // 2], t[..., TURNED // 2:TURNED]
        return torch.cat([u * cos - w * sin, u * sin + w * cos, t[..., TURNED:]], -1)

    heads = turn(qkv[:, :, :GROUP + 1])
    rows, at = [], 0
    for n in LENGTHS:
        q, k, v = heads[at:at + n, :, :GROUP], heads[at:at + n, :, GROUP], qkv[at:at + n, :, GROUP + 1]
        s = torch.einsum("tjgd,sjd->jgts", q, k) / math.sqrt(D)
        p = torch.where(torch.ones(n, n, dtype=torch.bool, device=x.device).tril(), s, -math.inf).softmax(-1)
        rows.append(torch.einsum("jgts,sjd->tjgd", p, v))
        at += n
    out = torch.cat(rows).flatten(1) @ w_out.T
    return out, norm(out + x, gamma2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_layer_forward_and_backward(dtype):
    dt, T, ATT = DT[dtype], sum(LENGTHS), KV * GROUP * D
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s, f=1.0: (torch.randn(s, generator=g, device="cuda") * f).to(dt)   # noqa: E731
    new = lambda *s, t=dt: torch.full(s, float("nan"), dtype=t, device="cuda")   # noqa: E731
    x, gamma, gamma2 = rand(T, H), 1 + rand(H, f=0.1), 1 + rand(H, f=0.1)
    w_qkv, w_out, dy = rand(KV * (GROUP + 2) * D, H, f=H ** -0.5), rand(H, ATT, f=ATT ** -0.5), rand(T, H)
    off = torch.tensor([0] + [sum(LENGTHS[:i + 1]) for i in range(len(LENGTHS))], dtype=torch.int32, device="cuda")
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in LENGTHS]).cuda()
    desc, longest = M.rotary_desc(TURNED), max(LENGTHS)
    split = lambda t: (t[:, :, :GROUP], t[:, :, GROUP], t[:, :, GROUP + 1])   # noqa: E731

    # forward
    n1, n2, xsum, out, a = new(T, H), new(T, H), new(T, H), new(T, H), new(T, KV, GROUP, D)
    rstd, rstd2, lse = (new(*s, t=torch.float32) for s in ((T,), (T,), (KV * GROUP, T)))
    qkv, dqkv = (new(T, KV, GROUP + 2, D) for _ in range(2))
    M.mtnlg_rmsnorm_fwd(x, gamma, EPS, n1, rstd)
    M.mtnlg_gemm(M.GEMM_NT, n1, w_qkv, qkv.view(T, -1))
    q, k, v = split(qkv)
    M.mtnlg_rotary_fwd(desc, q, k, q, k, positions)
    sizes = M.packed_desc(q, k, len(LENGTHS), longest, longest)
    room = lambda n: torch.empty((n,), dtype=torch.uint8, device="cuda") if n else None   # noqa: E731
    M.mtnlg_packed_attention_fwd(q, k, v, a, lse, off, off, longest, longest, workspace=room(M.mtnlg_packed_attention_fwd_workspace(sizes)))
    M.mtnlg_gemm(M.GEMM_NT, a.view(T, ATT), w_out, out)
    M.mtnlg_rmsnorm_fwd(out, gamma2, EPS, n2, rstd2, residual=x, xsum=xsum)
    # backward
    dxsum, dx, dn1, da, dg, dg2 = new(T, H), new(T, H), new(T, H), new(T, KV, GROUP, D), new(H, t=torch.float32), new(H, t=torch.float32)
    norm_room = room(M.mtnlg_rmsnorm_bwd_workspace(T, H))
    M.mtnlg_rmsnorm_bwd(xsum, gamma2, rstd2, dy, dxsum, dg2, norm_room)
    M.mtnlg_gemm(M.GEMM_NN, dxsum, w_out, da.view(T, ATT))
    dq, dk, dv = split(dqkv)
    M.mtnlg_packed_attention_bwd(q, k, v, a, lse, da, dq, dk, dv, off, off, longest, longest, room(M.mtnlg_packed_attention_bwd_workspace(sizes)))
    M.mtnlg_rotary_bwd(desc, dq, dk, dq, dk, positions)
    M.mtnlg_gemm(M.GEMM_NN, dqkv.view(T, -1), w_qkv, dn1)
    M.mtnlg_rmsnorm_bwd(x, gamma, rstd, dn1, dx, dg, norm_room, dres=dxsum)
    dw_qkv, dw_out = new(*w_qkv.shape), new(*w_out.shape)
    M.mtnlg_gemm(M.GEMM_TN, dqkv.view(T, -1), n1, dw_qkv)
    M.mtnlg_gemm(M.GEMM_TN, dxsum, a.view(T, ATT), dw_out)

    leaves = [t.double().requires_grad_() for t in (x, gamma, w_qkv, w_out, gamma2)]
    want_out, want_n2 = chain(*leaves, positions)
    want_n2.backward(dy.double())
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    sums = 2.0 ** -23 * (2 * H + D + longest + ATT)   # norms and first product, scores, attention, second product
    forward, both = 6 * u + sums, 14 * u + 2 * sums + 2.0 ** -23 * (longest * GROUP + T + KV * (GROUP + 2) * D)
    far = lambda got, want: float((got.double() - want).norm() / want.norm())   # noqa: E731
    for name, got, want, bound in (("out", out, want_out, forward), ("second norm", n2, want_n2, forward + 2 * u),
                                   *zip(("dx", "dgamma", "dw_qkv", "dw_out", "dgamma2"), (dx, dg, dw_qkv, dw_out, dg2), (t.grad for t in leaves), [both] * 5)):
        assert far(got, want) <= bound, (name, far(got, want), bound)
