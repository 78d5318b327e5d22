"""Attention over packed sequences with grouped heads, forward and backward, against 64 bits (packed_reference.py: the bounds)."""
import math

import pytest
import torch

import paper_2201_11990_amd as M
from packed_reference import assert_within, reference, spans

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
SENTINEL = 7.0


def offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def i32(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


class Case:
    """One call's tensors: q, k, v, da random, outputs full of a sentinel, the workspace of NaN."""

    def __init__(self, ql, kl, kv, group, d, dtype, layout="apart", q_off=None, k_off=None, q_len=None, k_len=None, seed=0, backward=True,
                 spread=1.0, scale=0.0, tq=None, tk=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = DT[dtype]
        self.q_off, self.k_off = q_off or offsets(ql), k_off or offsets(kl)
        self.q_len, self.k_len, self.scale = q_len, k_len, scale
        tq, tk = tq or self.q_off[-1], tk or self.k_off[-1]
        self.tq, self.tk, self.kv, self.group, self.d = tq, tk, kv, group, d
        fill = lambda t: t.copy_(torch.randn(t.shape, generator=g, device="cuda") * spread)   # noqa: E731

        def heads(tokens, n, fused=None):
            """[tokens, kv, n, d] in this case's layout"""
            if layout == "heads first":
                return torch.empty((kv, n, tokens, d), dtype=dt, device="cuda").permute(2, 0, 1, 3)
            if layout == "wide rows":
                return torch.empty((tokens, kv * n + 1, d + 8), dtype=dt, device="cuda")[:, 1:, 8:].unflatten(1, (kv, n))
            return torch.empty((tokens, kv, n, d), dtype=dt, device="cuda")

        if layout == "fused":
            assert tq == tk
            both = [torch.empty((tq, kv, group + 2, d), dtype=dt, device="cuda") for _ in range(2)]
            (self.q, self.k, self.v), (self.dq, self.dk, self.dv) = ((t[:, :, :group], t[:, :, group], t[:, :, group + 1]) for t in both)
        else:
            self.q, self.dq = heads(tq, group), heads(tq, group)
            self.k, self.v, self.dk, self.dv = (heads(tk, 1)[:, :, 0] for _ in range(4))
        self.a, self.da = heads(tq, group), heads(tq, group)
        for t in (self.q, self.k, self.v, self.da):
            fill(t)
        self.lse = torch.full((kv * group, tq), SENTINEL, device="cuda")
        self.backward = backward
        for t in (self.a, self.dq, self.dk, self.dv):
            t.fill_(SENTINEL)
        self.q_spans, self.k_spans = spans(self.q_off, q_len), spans(self.k_off, k_len)
        self.max_q, self.max_k = (max(1, *(n for _, n in s)) for s in (self.q_spans, self.k_spans))
        self.where = (i32(self.q_off), i32(self.k_off), self.max_q, self.max_k)
        self.lengths = {"q_lengths": i32(q_len), "k_lengths": i32(k_len)}

    def workspaces(self):
        desc = M.packed_desc(self.q, self.k, len(self.q_off) - 1, self.max_q, self.max_k, self.scale)
        full = lambda n: torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None   # noqa: E731
        return full(M.mtnlg_packed_attention_fwd_workspace(desc)), full(M.mtnlg_packed_attention_bwd_workspace(desc))

    def run(self, with_workspace=True):
        fwd, bwd = self.workspaces()
        M.mtnlg_packed_attention_fwd(self.q, self.k, self.v, self.a, self.lse, *self.where, scale=self.scale, workspace=fwd if with_workspace else None,
                                     **self.lengths)
        if self.backward:
            M.mtnlg_packed_attention_bwd(self.q, self.k, self.v, self.a, self.lse, self.da, self.dq, self.dk, self.dv, *self.where, bwd,
                                         scale=self.scale, **self.lengths)
        return self.results()

    def results(self):
        names = ("a", "lse", "dq", "dk", "dv") if self.backward else ("a", "lse")
        return {n: getattr(self, n) for n in names}

    def want(self):
        return reference(self.q, self.k, self.v, self.da if self.backward else None, self.q_spans, self.k_spans, self.scale or None)

    def check(self, want=None):
        """Rows of a sequence within their bounds, all others as they were."""
        want = want or self.want()
        for name, got in self.results().items():
            value, bound = want[name]
            rows = torch.zeros(self.tq if name in ("a", "lse", "dq") else self.tk, dtype=torch.bool, device="cuda")
            for first, n in self.q_spans if name in ("a", "lse", "dq") else self.k_spans:
                rows[first:first + n] = True
            if name == "lse":
                got, value, bound = got.T, value.T, bound.T
            assert (got[~rows] == SENTINEL).all(), f"{name}: rows of no sequence were written"
            assert_within(got[rows], (value[rows], bound[rows]), name)


RAGGED = [1, 0, 33, 130, 64, 17]


@pytest.mark.parametrize("d", [8, 40, 64, 72, 96, 104, 128, 144, 160, 192, 200, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_head_sizes(dtype, d):
    c = Case(RAGGED, RAGGED, 2, 2, d, dtype, seed=d)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv,group", [(1, 1), (1, 8), (2, 3), (3, 7), (8, 1), (1, 40)])
def test_groups(dtype, kv, group):
    c = Case([70, 129, 3], [70, 129, 3], kv, group, 64, dtype, seed=group)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["fused", "heads first", "wide rows"])
def test_layouts(dtype, layout):
    c = Case([33, 150, 1], [33, 150, 1], 2, 3, 72, dtype, layout=layout, seed=5)
    c.run()
    c.check()


def test_heads_of_a_matrix_with_three_dimensions_are_those_of_groups():
    c = Case([33, 150], [33, 150], 2, 3, 64, "bf16")
    a, lse, dq, dk, dv = (t.clone() for t in c.run().values())
    flat = lambda t: t.flatten(1, 2)   # noqa: E731
    for t in (c.a, c.dq, c.dk, c.dv, c.lse):
        t.fill_(SENTINEL)
    fwd, bwd = c.workspaces()
    M.mtnlg_packed_attention_fwd(flat(c.q), c.k, c.v, flat(c.a), c.lse, *c.where, workspace=fwd)
    M.mtnlg_packed_attention_bwd(flat(c.q), c.k, c.v, flat(c.a), c.lse, flat(c.da), flat(c.dq), c.dk, c.dv, *c.where, bwd)
    for got, want in ((c.a, a), (c.lse, lse), (c.dq, dq), (c.dk, dk), (c.dv, dv)):
        assert torch.equal(got, want)


# more queries than keys (the first see none), fewer, no keys at all, no queries
LQ, LK = [5, 1, 64, 40, 3, 0, 130, 1], [5, 300, 200, 12, 0, 50, 129, 1]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,group", [(64, 2), (128, 5)])
def test_queries_and_keys_of_different_lengths(dtype, d, group):
    c = Case(LQ, LK, 2, group, d, dtype, seed=3)
    c.run()
    c.check()
    assert torch.isneginf(c.lse).any() and not torch.isnan(c.lse).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_regions_that_are_not_full_and_rows_of_no_sequence(dtype):
    # sequences begin after row 0 and end before the last; regions hold more than their lengths; lengths beyond a region end with it
    c = Case(None, None, 2, 2, 64, dtype, q_off=[3, 40, 40, 200], k_off=[10, 110, 150, 420], q_len=[30, 7, 500], k_len=[90, 0, 250], tq=211, tk=500)
    for t in (c.q, c.k, c.v, c.da):   # what is not of a sequence is never looked at
        spans_of = c.q_spans if t.shape[0] == c.tq else c.k_spans
        rows = torch.ones(t.shape[0], dtype=torch.bool, device="cuda")
        for first, n in spans_of:
            rows[first:first + n] = False
        t[rows] = float("nan")
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_query_does_not_see_does_not_reach_it(dtype, bad, d):
    # keys and values of a late token, then queries and gradients of an early one, hold infinities or NaN: what earlier queries and later keys get lies within
    # the bounds of finite inputs (not bit by bit the same: products with such rows are taken in another order)
    n, at, early = 150, 117, 40
    c = Case([n, 40], [n, 40], 1, 2, d, dtype, seed=9)
    want = c.want()
    rows = lambda t, which: tuple(x[which] for x in t)   # noqa: E731
    c.k[at], c.v[at] = bad, bad
    c.run()
    for which in (slice(0, at), slice(n, None)):
        for name in ("a", "dq"):
            assert_within(getattr(c, name)[which], rows(want[name], which), name)
        assert_within(c.lse.T[which], tuple(x.T[which] for x in want["lse"]), "lse")
    assert not torch.isfinite(c.a[at:n]).any()
    c = Case([n, 40], [n, 40], 1, 2, d, dtype, seed=9)
    c.da[early], c.q[early] = bad, bad
    c.run()
    for name in ("dk", "dv"):
        assert_within(getattr(c, name)[early + 1:], rows(want[name], slice(early + 1, None)), name)
        assert not torch.isfinite(getattr(c, name)[:early + 1]).any()


def test_a_row_by_row_product_matches_the_matrix_instructions():
    # an infinity that one query sees: the others of its tile are computed without matrix instructions, to the same bounds
    for dtype in ("bf16", "fp32"):
        c = Case([64], [64], 1, 3, 96, dtype, seed=2)
        want = c.want()
        c.v[63] = float("inf")
        c.backward = False
        c.run()
        assert_within(c.a[:63], tuple(t[:63] for t in want["a"]), "a")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("keys,group,d", [([3000, 1, 777, 2048], 4, 128), ([5001], 1, 64), ([1500, 0, 900], 8, 192), ([700] * 9, 7, 256)])
def test_single_tokens_over_long_caches(dtype, keys, group, d):
    c = Case([1] * len(keys), keys, 2, group, d, dtype, backward=False, seed=len(keys))
    fwd, _ = c.workspaces()
    assert fwd is not None or max(keys) < 1000   # the keys are cut where they are long enough
    c.run()
    want = c.want()
    c.check(want)
    c.a.fill_(SENTINEL), c.lse.fill_(SENTINEL)
    c.run(with_workspace=False)
    c.check(want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("queries,keys", [([1], [16384]), ([1], [16385]), ([1], [16447]), ([1, 1], [300, 20481]), ([1], [32769]), ([3], [16400])])
def test_a_cache_in_as_many_chunks_as_there_are(dtype, queries, keys):
    # the last key, which a further chunk would hold alone or with a few others, has most of the first head's weight
    c = Case(queries, keys, 1, 2, 64, dtype, backward=False, seed=61)
    c.k[-1, 0] = 3 * c.q[-1, 0, 0]
    fwd, _ = c.workspaces()
    assert fwd is not None
    want = c.want()
    c.run()
    c.check(want)
    c.a.fill_(SENTINEL), c.lse.fill_(SENTINEL)
    c.run(with_workspace=False)
    c.check(want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompts_continued_behind_a_cache(dtype):
    c = Case(None, None, 2, 2, 128, dtype, q_off=[0, 100, 133, 133], k_off=[0, 1536, 2048, 2304], k_len=[1400, 33, 100], backward=False)
    c.run()
    c.check()


@pytest.mark.parametrize("count", [63, 64, 65, 200, 4097])
def test_many_sequences(count):
    g = torch.Generator().manual_seed(count)
    lengths = torch.randint(0, 4, (count,), generator=g).tolist()
    lengths[-1] = 70
    c = Case(lengths, lengths, 1, 2, 64, "bf16", seed=1)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count", [32, 33, 64, 65, 150])
def test_single_tokens_of_many_sequences_over_long_caches(dtype, count):
    # cut keys and their join, with the sequences counted one to a lane, and several
    g = torch.Generator().manual_seed(count)
    keys = torch.randint(0, 3000, (count,), generator=g).tolist()
    keys[count // 2], keys[-1] = 6000, 1
    c = Case([1] * count, keys, 1, 2, 64, dtype, backward=False, seed=71)
    fwd, _ = c.workspaces()
    assert fwd is not None
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("count", [32, 33, 80])
def test_work_of_many_sequences_that_is_cut_and_joined(dtype, count):
    g = torch.Generator().manual_seed(count)
    lengths = torch.randint(0, 9, (count,), generator=g).tolist()
    lengths[count - 2] = 1200
    c = Case(lengths, lengths, 1, 3, 64, dtype, seed=72)
    desc = M.packed_desc(c.q, c.k, count, c.max_q, c.max_k)
    assert M.mtnlg_packed_attention_bwd_workspace(desc) > 8 * c.lse.numel()   # more than a sum for each row
    c.run()
    c.check()


def test_scores_of_any_size():
    # weights from 1 down to nothing, sums that hold one weight only, and maxima that move from tile to tile
    for dtype in ("bf16", "fp32"):
        c = Case([300], [300], 1, 2, 64, dtype, spread=3.0, seed=4)
        c.k.copy_(c.k * torch.linspace(0.2, 3, 300, device="cuda")[:, None, None])
        c.run()
        c.check()


def test_scale_is_a_parameter():
    c = Case([90, 20], [90, 20], 2, 2, 64, "fp32", scale=0.03)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_larger_workgroups(dtype):
    # enough rows for 128 to a workgroup, enough keys that a group is not dealt out
    c = Case([300, 900, 1400], [300, 900, 1400], 8, 4, 64, dtype, seed=8)
    c.run()
    c.check()


def test_runs_are_identical_and_replays_too():
    c = Case([130, 700, 64], [130, 700, 64], 2, 4, 128, "bf16", seed=6)
    eager = {k: v.clone() for k, v in c.run().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # another stream than the tensors'
        again = c.run()
    torch.cuda.current_stream().wait_stream(side)
    for k in eager:
        assert torch.equal(eager[k], again[k]), k
    one = Case([1, 1, 1], [3000, 70, 900], 2, 4, 128, "bf16", seed=7, backward=False)
    one_eager = {k: v.clone() for k, v in one.run().items()}
    (fwd, bwd), (one_fwd, _) = c.workspaces(), one.workspaces()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        M.mtnlg_packed_attention_fwd(c.q, c.k, c.v, c.a, c.lse, *c.where, workspace=fwd)
        M.mtnlg_packed_attention_bwd(c.q, c.k, c.v, c.a, c.lse, c.da, c.dq, c.dk, c.dv, *c.where, bwd)
        M.mtnlg_packed_attention_fwd(one.q, one.k, one.v, one.a, one.lse, *one.where, workspace=one_fwd)
    for turn in range(4):
        for t in (c.a, c.dq, c.dk, c.dv, c.lse, one.a, one.lse):
            t.fill_(SENTINEL)
        bwd.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(getattr(c, k), eager[k]), (turn, k)
        for k in one_eager:
            assert torch.equal(getattr(one, k), one_eager[k]), (turn, k)


def test_a_captured_call_takes_new_lengths():
    # the arrays are read on the device: a replay goes by what they hold then
    c = Case([130, 70, 56], [130, 70, 56], 2, 2, 64, "bf16")
    c.max_q = c.max_k = 256
    c.where = (*c.where[:2], 256, 256)
    c.run()
    fwd, bwd = c.workspaces()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mtnlg_packed_attention_fwd(c.q, c.k, c.v, c.a, c.lse, *c.where, workspace=fwd)
        M.mtnlg_packed_attention_bwd(c.q, c.k, c.v, c.a, c.lse, c.da, c.dq, c.dk, c.dv, *c.where, bwd)
    for lengths in ([1, 250, 5], [256, 0, 0], [100, 20, 30]):
        off = offsets(lengths)
        for t in c.where[:2]:
            t.copy_(i32(off))
        c.q_spans = c.k_spans = spans(off, None)
        for t in (c.a, c.dq, c.dk, c.dv, c.lse):
            t.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        c.check()


def test_offsets_beyond_the_matrices_touch_nothing_outside():
    # rows that the arrays name and the matrices do not have: taken for the nearest that they have
    c = Case([100], [100], 1, 2, 64, "bf16", q_off=[0, 60, 100], k_off=[0, 60, 100])
    c.run()
    for t, v in zip(c.where[:2], ([-5, 60, 1000], [0, 60, 2 ** 31 - 1])):
        t.copy_(i32(v))
    for t in (c.a, c.dq, c.dk, c.dv, c.lse):
        t.fill_(SENTINEL)
    c.run()
    c.check()


def test_a_cache_beyond_32_bits_of_elements():
    # keys and values of 2^31 elements each, the sequence in the last rows
    tk, kv, d = 2 ** 22 + 600, 4, 128
    k, v = (torch.zeros((tk, kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = Case([70], [500], kv, 2, d, "bf16", backward=False)
    k[-500:], v[-500:] = small.k, small.v
    off = i32([tk - 500, tk])
    M.mtnlg_packed_attention_fwd(small.q, k, v, small.a, small.lse, small.where[0], off, 70, 500)
    small.check()


def test_a_cache_of_nearly_as_many_keys_as_there_may_be():
    # their number and a chunk's add up to more than 2^31.  All scores are 0 but the last one, that key's value 3 where all others are 1
    tk, d = (1 << 31) - 300, 8
    k, v = torch.zeros((tk, 1, d), dtype=torch.bfloat16, device="cuda"), torch.ones((tk, 1, d), dtype=torch.bfloat16, device="cuda")
    q, a, lse = torch.ones((1, 1, d), dtype=torch.bfloat16, device="cuda"), torch.full((1, 1, d), SENTINEL, dtype=torch.bfloat16, device="cuda"), torch.full((1, 1), SENTINEL, device="cuda")
    k[-1], v[-1] = 8, 3
    score = 64 / math.sqrt(d)
    desc = M.packed_desc(q, k, 1, 1, tk)
    ws = torch.full((M.mtnlg_packed_attention_fwd_workspace(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    M.mtnlg_packed_attention_fwd(q, k, v, a, lse, i32([0, 1]), i32([0, tk]), 1, tk, workspace=ws)
    total = tk - 1 + math.exp(score)
    # sums of equal weights are whole numbers up to 2^24 for each part of a chunk, exact; the other weights' exponent, 33, is off by 2^-18, and the score by 2^-18 as well
    assert abs(float(lse) - math.log(total)) <= 2.0 ** -16
    want = (tk - 1 + 3 * math.exp(score)) / total
    assert (a.double() - want).abs().max() <= 2.0 ** -8 * want * 1.01 + 2.0 ** -15


def test_gradients_against_differences():
    # the sum of da . a and its change with each input along a random direction, in fp32 with 64-bit sums; central differences of step h are off by
    # h^2 times a third derivative, and by the fp32 roundings of a over 2 h
    c = Case([40, 25], [40, 25], 2, 2, 64, "fp32", spread=0.5, seed=12)
    c.run()
    h = 2.0 ** -5
    for name in ("q", "k", "v"):
        t, grad = getattr(c, name), getattr(c, "d" + name).double()
        way = torch.randn(t.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
        keep, sums = t.clone(), []
        for sign in (1, -1):
            t.copy_(keep + sign * h * way)
            want = reference(c.q, c.k, c.v, None, c.q_spans, c.k_spans)["a"][0]
            sums.append((want * c.da.double()).sum())
        t.copy_(keep)
        slope, along = (sums[0] - sums[1]) / (2 * h), (grad * way.double()).sum()
        size = (grad.abs() * way.double().abs()).sum()
        assert abs(slope - along) <= 2e-3 * size, (name, float(slope), float(along))


@pytest.mark.parametrize("dtype,ql,kl,kv,group,d", [
    ("fp32", [3, 40, 1], [900, 1300, 0], 2, 2, 96), ("fp32", [700], [700], 1, 1, 64), ("fp32", [130, 600, 0, 33], [130, 600, 70, 20], 2, 3, 128),
    ("bf16", [700], [700], 1, 1, 64), ("bf16", [700, 64, 1], [900, 30, 700], 1, 8, 128), ("bf16", [520, 257], [520, 257], 2, 4, 160),
    ("bf16", [600], [600], 1, 5, 192), ("bf16", [600, 100], [600, 100], 1, 4, 256)])
def test_work_that_is_cut_and_joined(dtype, ql, kl, kv, group, d):
    # few workgroups: dq's keys (fp32) and the queries of dk and dv are dealt out over more of them, whose parts a further launch adds
    c = Case(ql, kl, kv, group, d, dtype, seed=21)
    desc = M.packed_desc(c.q, c.k, len(ql), c.max_q, c.max_k)
    assert M.mtnlg_packed_attention_bwd_workspace(desc) > 8 * c.lse.numel()   # more than a sum for each row
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 160), ("bf16", 256), ("fp32", 64)])
def test_what_a_query_does_not_see_in_work_that_is_cut(dtype, d):
    n, at, early = 1100, 901, 300
    c = Case([n], [n], 1, 2, d, dtype, seed=22)
    want = c.want()
    part = lambda t, which: tuple(x[which] for x in t)   # noqa: E731
    c.k[at], c.v[at] = float("nan"), float("inf")
    c.run()
    for name in ("a", "dq"):
        assert_within(getattr(c, name)[:at], part(want[name], slice(0, at)), name)
    assert not torch.isfinite(c.a[at:]).any()
    c = Case([n], [n], 1, 2, d, dtype, seed=22)
    c.da[early], c.q[early] = float("inf"), float("nan")
    c.run()
    for name in ("dk", "dv"):
        assert_within(getattr(c, name)[early + 1:], part(want[name], slice(early + 1, None)), name)
        assert not torch.isfinite(getattr(c, name)[:early + 1]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("at", [0, 5, 70, 299])
def test_an_infinity_that_is_seen_stays_one(dtype, d, at):
    # one column of a value, or of an output's gradient: that column of what sees it is infinite, no other changes (weights are positive)
    c = Case([300], [300], 1, 2, d, dtype, seed=23)
    want = c.want()
    c.v[at, 0, 3] = float("inf")
    c.backward = False
    c.run()
    assert torch.isposinf(c.a[at:, ..., 3]).all()
    others = torch.arange(d, device="cuda") != 3
    assert_within(c.a[..., others], tuple(t[..., others] for t in want["a"]), "a")
    assert_within(c.a[:at], tuple(t[:at] for t in want["a"]), "a")
    c = Case([300], [300], 1, 2, d, dtype, seed=23)
    c.da[at, 0, 1, 3] = float("inf")
    c.run()
    assert torch.isposinf(c.dv[:at + 1, 0, 3]).all()
    assert_within(c.dv[..., others], tuple(t[..., others] for t in want["dv"]), "dv")
    assert_within(c.dv[at + 1:], tuple(t[at + 1:] for t in want["dv"]), "dv")


def test_two_calls_at_once():
    # on two streams, each with its own workspace
    cases = [Case([130, 700, 64], [130, 700, 64], 2, 4, 128, "bf16", seed=31), Case([500, 90], [500, 90], 1, 4, 64, "bf16", seed=32)]
    alone = [{k: v.clone() for k, v in c.run().items()} for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c, want in zip(cases, alone):
        for k, v in c.results().items():
            assert torch.equal(v, want[k]), k


@pytest.mark.parametrize("d", [64, 72, 128, 152, 192])
def test_larger_workgroups_of_every_width(d):
    # 128 rows to a workgroup; then with a token that is infinite, or not a number, and hidden from those before it
    lengths, at = [300, 900, 1400], 700
    c = Case(lengths, lengths, 8, 4, d, "bf16", seed=41)
    want = c.want()
    c.run()
    c.check(want)
    part = lambda t, which: tuple(x[which] for x in t)   # noqa: E731
    c.k[at], c.v[at] = float("-inf"), float("nan")
    c.run()
    for which in (slice(0, at), slice(1200, None)):
        for name in ("a", "dq"):
            assert_within(getattr(c, name)[which], part(want[name], which), name)
    assert not torch.isfinite(c.a[at:1200]).any()
    c = Case(lengths, lengths, 8, 4, d, "bf16", seed=41)
    c.q[at], c.da[at] = float("nan"), float("inf")
    c.run()
    for name in ("dk", "dv"):
        for which in (slice(0, 300), slice(at + 1, None)):
            assert_within(getattr(c, name)[which], part(want[name], which), name)
        assert not torch.isfinite(getattr(c, name)[300:at + 1]).any()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 192), ("fp32", 64)])
@pytest.mark.parametrize("keys", [3, 70])
def test_many_queries_that_see_no_key(dtype, d, keys):
    # all rows of some workgroups and of some waves; 128 rows to a workgroup
    c = Case([400, 5], [keys, 5], 170, 1, d, dtype, seed=51)
    c.run()
    c.check()
    assert torch.isneginf(c.lse[:, :400 - keys]).all() and (c.a[:400 - keys] == 0).all() and (c.dq[:400 - keys] == 0).all()
