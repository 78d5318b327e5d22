// Attention over packed sequences with grouped heads: how calls are cut into workgroups, the kernels that join what was cut, and the entry points.
#include "packed.h"

namespace mtnlg {

namespace {

constexpr int MOST_CHUNKS = 64;   // of a row: a lane of the wave that joins them to each
constexpr int64_t MOST_ROWS = ((int64_t)1 << 31) - 256;

// A row's results from those of its chunks: a wave to a row, four columns to a lane.
template <typename E>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedFwdArgs w) {
  const int lane = threadIdx.x & 63, r = w.group, d = w.d, j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lq * r + 3) / 4); }, s, at)) return;
  const int row = at * 4 + (threadIdx.x >> 6);
  if (row >= s.lq * r) return;
  const int tok = row / r, g = row - tok * r, head = j * r + g, limit = min(tok + s.lk - s.lq, s.lk - 1);
  const int nc = min(limit < 0 ? 0 : limit / w.chunk + 1, w.chunks);
  const int64_t all = (int64_t)w.where.q_tokens * w.kv_heads * r, id = (int64_t)(s.q0 + tok) * ((int64_t)w.kv_heads * r) + head;
  float m = -INFINITY, l = 0.0f;
  if (lane < nc) {
    const float2 t = *reinterpret_cast<const float2 *>(w.stat + 2 * (lane * all + id));
    m = t.x;
    l = t.y;
  }
  const float most = wave_max(m), ref = most == -INFINITY ? 0.0f : most;
  const float mul = sizeof(E) == 4 ? exact_exp(product_of(m, w.scale) - product_of(ref, w.scale)) : fast_exp2((m - ref) * (w.scale * kLog2e));
  const float total = wave_sum(l * mul);
  f32x4 o = {};
  const float *from = w.part + id * d + (lane * 4 < d ? lane * 4 : 0);   // lanes past the columns go along: the others take the chunks' factors from them
  for (int i = 0; i < nc; i += 4) {   // four reads in flight (of the last chunk again past the end, where the factors are 0)
    f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const f32x4 *>(from + min(i + u, nc - 1) * all * d);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = __shfl(mul, i + u, 64);
      if (i + u < nc) o += v[u] * f;   // (an infinity there is read again: not times 0)
    }
  }
  if (lane * 4 < d) put4(row_at<E>(w.a, s.q0 + tok, j, g) + lane * 4, o * (nc ? 1.0f / total : 0.0f));
  if (lane == 0) w.lse[(int64_t)head * w.where.q_tokens + s.q0 + tok] = nc ? plus_log(product_of(most, w.scale), total) : -INFINITY;
}

// dq from its chunks of keys: a wave to a row, four columns to a lane.
template <typename E>
__global__ __launch_bounds__(256) void packed_dq_join_kernel(PackedBwdArgs w) {
  const int lane = threadIdx.x & 63, r = w.group, d = w.d, j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lq * r + 3) / 4); }, s, at)) return;
  const int row = at * 4 + (threadIdx.x >> 6);
  if (row >= s.lq * r || lane * 4 >= d) return;
  const int tok = row / r, g = row - tok * r, limit = min(tok + s.lk - s.lq, s.lk - 1);
  const int nc = min(limit < 0 ? 0 : limit / w.chunk + 1, w.chunks);
  const int64_t all = (int64_t)w.where.q_tokens * w.kv_heads * r;
  const float *from = w.dq_part + ((int64_t)(s.q0 + tok) * ((int64_t)w.kv_heads * r) + j * r + g) * d + lane * 4;
  f32x4 sum = {};
#pragma unroll 4
  for (int i = 0; i < nc; ++i) sum += *reinterpret_cast<const f32x4 *>(from + i * all * d);
  put4(row_at<E>(w.dq, s.q0 + tok, j, g) + lane * 4, sum * w.scale);
}

// The parts of dk and dv added up: a wave to a key, four columns of dv (lower half of the lanes' columns) and dk to a lane in turn.  (Sixteen keys to a workgroup and a
// part at a time: 8.5 us for 5 parts of 1536 keys, 4 heads of 96, and 12 for 11.)
constexpr int DKV_JOINED = 4;   // keys of a workgroup
template <typename E>
__global__ __launch_bounds__(256) void packed_dkv_join_kernel(PackedBwdArgs w) {
  const int lane = threadIdx.x & 63, d = w.d, j = blockIdx.x % w.kv_heads;
  Span s;
  unsigned at;
  if (!find_piece(w.where, blockIdx.x / w.kv_heads, [&](const Span &s) { return (unsigned)((s.lk + DKV_JOINED - 1) / DKV_JOINED); }, s, at)) return;
  const int64_t all = (int64_t)w.where.k_tokens * w.kv_heads * (2 * d);
  const int key = at * DKV_JOINED + (threadIdx.x >> 6);
  if (key >= s.lk) return;
  const float *from = w.part + ((int64_t)(s.k0 + key) * w.kv_heads + j) * (2 * d);
  for (int col = lane * 4; col < 2 * d; col += 256) {
    f32x4 v = {};
    for (int p = 0; p < w.splits; p += 4) {   // four reads in flight (of the last part again past the end)
      f32x4 part[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) part[u] = *reinterpret_cast<const f32x4 *>(from + min(p + u, w.splits - 1) * all + col);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (p + u < w.splits) v += part[u];
    }
    put4(col < d ? row_at<E>(w.dv, s.k0 + key, j, 0) + col : row_at<E>(w.dk, s.k0 + key, j, 0) + (col - d), v);
  }
}

// How the keys are cut where the rows alone leave most of the chip idle.
struct FwdPlan {
  int owned;
  int64_t pieces;   // workgroups of a head of keys at most, without cuts
  int chunk, chunks;
  size_t part_bytes, bytes;
};
struct Cut {
  int chunk, chunks;
};
// all pieces with their chunks: all keys in chunks and the last ones of each sequence, for every block that a sequence can have
int64_t cut_pieces(const PackedShape &S, const Cut &c, int64_t pieces, int owned) {
  if (c.chunks == 1) return pieces;
  const int64_t blocks_of = ((int64_t)S.max_q * S.group + owned - 1) / owned, by_keys = blocks_of * (S.where.k_tokens / c.chunk + S.where.count);
  return pieces * c.chunks < by_keys ? pieces * c.chunks : by_keys;
}
// Estimated microseconds with and without: a workgroup takes `tile` us for 64 keys where all `slots` for workgroups are in use, 3.5 us to start (3 to find that there is
// nothing for it), and a cut call 8 us and the way of its parts through memory (at 4 TB/s) to join them.  Cut where that is
// half as much again faster, into about 1024 pieces.  Measured: 32 single tokens, 64 to 15872 keys, 32 heads of 128 on 8: 280 us whole, 96 cut (104 into 512 pieces, 112 into
// 2048); 973 tokens behind up to 4608 keys, 60 us whole, 89 and 102 in chunks of 2304 and 1152; heads of 256: 806 and 110 tokens behind up to 1899 keys, 12 on 4, 172 us whole and 121
// cut, 16 sequences of up to 968 tokens and 2058 keys, 16 on 8, 209 and 350 (most of 5120 workgroups find nothing).
constexpr int CUT_LEAST = 256;   // keys of a chunk at least
Cut cut_keys(const PackedShape &S, int64_t pieces, int owned, double tile, int slots, int least, int into) {
  const double wide = (double)(pieces * S.kv_heads), mean = (double)S.where.k_tokens / S.where.count;
  if (S.max_k < 2 * least || wide >= 1024) return Cut{0, 1};
  const double work = wide * mean / 64 / slots;   // tiles of a slot where all come out even
  // (rounded up: 16385 keys in chunks of 256 are 65)
  const double want = fmax(least, fmax((S.max_k + (int64_t)MOST_CHUNKS - 1) / MOST_CHUNKS, wide * mean / into));
  if (want >= S.max_k) return Cut{0, 1};
  const int64_t chunk = ((int64_t)want + 63) / 64 * 64;
  if (chunk >= S.max_k) return Cut{0, 1};
  const Cut c{(int)chunk, (int)((S.max_k + chunk - 1) / chunk)};
  const double each = fmax(1.0, mean / chunk);   // chunks of a sequence
  const double idle = fmax(0.0, (double)(cut_pieces(S, c, pieces, owned) * S.kv_heads) - wide * each);
  const double whole = tile * fmax(S.max_k / 64.0, work);
  const double cut = tile * fmax(chunk / 64.0, work) + (3.5 * wide * each + 3.0 * idle) / slots + 8.0 + (double)S.where.q_tokens * S.heads * each * S.d * 8.0 / 4.0e6;
  return 1.5 * cut >= whole ? Cut{0, 1} : c;
}
// us of 64 keys of the forward kernels, and how many of their workgroups run at once
double fwd_tile(const PackedShape &S) { return S.dtype == MTNLG_F32 ? (S.d <= 160 ? 0.11 : 0.07) * S.d : S.d > PACKED_TUNED ? 5.0 : 0.9; }
int fwd_slots(const PackedShape &S) { return S.d <= 160 ? 512 : 256; }
FwdPlan fwd_plan(const PackedShape &S) {
  FwdPlan p{};
  const int64_t rows = (int64_t)S.where.q_tokens * S.group, most = (int64_t)S.max_q * S.group;
  p.owned = 128;
  p.pieces = pieces_bound(rows, most, S.where.count, p.owned);
  if (packed_tuned(S.dtype, S.d) && p.pieces * S.kv_heads < packed_fwd_places(S.d)) {
    p.owned = 64;
    p.pieces = pieces_bound(rows, most, S.where.count, p.owned);
  }
  const Cut c = cut_keys(S, p.pieces, p.owned, fwd_tile(S), fwd_slots(S), CUT_LEAST, 1024);
  p.chunk = c.chunk;
  p.chunks = c.chunks;
  if (p.chunks > 1) {
    const size_t all = (size_t)S.where.q_tokens * S.heads;
    p.part_bytes = align_up(p.chunks * all * S.d * sizeof(float), 256);
    p.bytes = p.part_bytes + align_up(p.chunks * all * 2 * sizeof(float), 256);
  }
  return p;
}

bool unaligned(const mtnlg_packed_sequences *w) {
  return (((uintptr_t)w->q_offsets | (uintptr_t)w->k_offsets | (uintptr_t)w->q_lengths | (uintptr_t)w->k_lengths) & 3) != 0;
}

struct BwdPlan {
  int owned, key_owned, splits;   // rows of a dq workgroup, keys of one of dk / dv; parts of its tiles
  Cut cut;                        // of the keys of dq (packed_plain.hip)
  int64_t pieces, key_pieces;
  size_t d_bytes, part_bytes, bytes;
};
BwdPlan bwd_plan(const PackedShape &S) {
  BwdPlan p{};
  const int64_t rows = (int64_t)S.where.q_tokens * S.group, most = (int64_t)S.max_q * S.group;
  p.owned = 128;
  p.pieces = pieces_bound(rows, most, S.where.count, p.owned);
  if (packed_tuned(S.dtype, S.d) && p.pieces * S.kv_heads < packed_dq_places(S.d)) {
    p.owned = 64;
    p.pieces = pieces_bound(rows, most, S.where.count, p.owned);
  }
  p.key_owned = packed_tuned(S.dtype, S.d) ? packed_dkv_tuned_owned(S.d) : packed_dkv_plain_owned(S.dtype, S.d);
  p.key_pieces = pieces_bound(S.where.k_tokens, S.max_k, S.where.count, p.key_owned);
  // Where the keys leave units idle, a workgroup's tiles of queries (of all heads of the group) are dealt out: about 512 workgroups, of 8 tiles at least, which the
  // joining launch and the parts' way through memory cost.  fp32: of 4, a tile takes longer (1536 tokens in 4 documents, 8 heads of 96 on 4: 73 and 7 us with 8
  // tiles at least, 59 and 8 with 4, 61 and 11 with 2).
  const int64_t wide = p.key_pieces * S.kv_heads, tiles = (int64_t)S.group * ((S.max_q + 31) / 32);
  int64_t splits = wide >= 512 ? 1 : (512 + wide - 1) / wide;
  const int64_t most_splits = tiles / (S.dtype == MTNLG_F32 ? 4 : 8);
  if (splits > most_splits) splits = most_splits;
  p.splits = (int)(splits < 1 ? 1 : splits > 64 ? 64 : splits);
  p.d_bytes = align_up((size_t)S.where.q_tokens * S.heads * sizeof(float), 256);
  p.part_bytes = p.splits > 1 ? align_up((size_t)p.splits * S.where.k_tokens * S.kv_heads * 2 * S.d * sizeof(float), 256) : 0;
  // fp32: a tile of dq is long, and few rows are few workgroups (1536 tokens in 4 documents, 8 heads of 96 on 4: 114 us whole, 53 and 8 for the join so)
  p.cut = S.dtype == MTNLG_F32 ? cut_keys(S, p.pieces, p.owned, 0.16 * S.d, 512, 64, 512) : Cut{0, 1};
  p.pieces = cut_pieces(S, p.cut, p.pieces, p.owned);
  p.bytes = p.d_bytes + p.part_bytes + (p.cut.chunks > 1 ? (size_t)p.cut.chunks * S.where.q_tokens * S.heads * S.d * sizeof(float) : 0);
  return p;
}

}  // namespace

int packed_shape(const mtnlg_packed_desc *D, PackedShape *S) {
  if (!D) return MTNLG_NULL_POINTER;
  if (D->dtype != MTNLG_F32 && D->dtype != MTNLG_BF16) return MTNLG_INVALID_ARG;
  if (D->heads <= 0 || D->kv_heads <= 0 || D->heads % D->kv_heads || D->head_dim <= 0 || D->sequences <= 0) return MTNLG_INVALID_ARG;
  if (D->q_tokens <= 0 || D->k_tokens <= 0 || D->max_q <= 0 || D->max_k <= 0) return MTNLG_INVALID_ARG;
  if (!(D->scale >= 0.0f && D->scale < INFINITY)) return MTNLG_INVALID_ARG;
  if (D->head_dim % 8 || D->head_dim > 256 || D->heads > 65535 || D->sequences > 1 << 16) return MTNLG_UNSUPPORTED_SHAPE;
  if (D->q_tokens > 0x7FFFFFFF || D->k_tokens > 0x7FFFFFFF) return MTNLG_UNSUPPORTED_SHAPE;
  // rows are counted in 32 bits, up to the end of the block that has the last one
  if (D->q_tokens * D->heads > MOST_ROWS || D->k_tokens * D->kv_heads > MOST_ROWS) return MTNLG_UNSUPPORTED_SHAPE;
  *S = PackedShape{D->dtype, D->heads, D->kv_heads, D->heads / D->kv_heads, D->head_dim, D->scale > 0.0f ? D->scale : 1.0f / sqrtf((float)D->head_dim),
                   Sequences{nullptr, nullptr, nullptr, nullptr, D->sequences, (int)D->q_tokens, (int)D->k_tokens}, D->max_q, D->max_k};
  // no sequence is longer than the matrix
  if (S->max_q > S->where.q_tokens) S->max_q = S->where.q_tokens;
  if (S->max_k > S->where.k_tokens) S->max_k = S->where.k_tokens;
  return MTNLG_OK;
}

}  // namespace mtnlg

using namespace mtnlg;

extern "C" {

size_t mtnlg_packed_attention_fwd_workspace(const mtnlg_packed_desc *desc) {
  PackedShape S;
  return packed_shape(desc, &S) == MTNLG_OK ? fwd_plan(S).bytes : 0;
}

int mtnlg_packed_attention_fwd(const mtnlg_packed_desc *desc, const mtnlg_packed_sequences *where, const mtnlg_heads *q, const mtnlg_heads *k,
                               const mtnlg_heads *v, const mtnlg_heads *a, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  if (!where || !where->q_offsets || !where->k_offsets || !q || !k || !v || !a || !q->data || !k->data || !v->data || !a->data || !lse) return MTNLG_NULL_POINTER;
  PackedShape S;
  MTNLG_TRY(packed_shape(desc, &S));
  MTNLG_TRY(heads_check(q, S.where.q_tokens, S.kv_heads, S.group, S.d, S.dtype));
  MTNLG_TRY(heads_check(a, S.where.q_tokens, S.kv_heads, S.group, S.d, S.dtype));
  MTNLG_TRY(heads_check(k, S.where.k_tokens, S.kv_heads, 1, S.d, S.dtype));
  MTNLG_TRY(heads_check(v, S.where.k_tokens, S.kv_heads, 1, S.d, S.dtype));
  if (a->data == q->data || a->data == k->data || a->data == v->data) return MTNLG_INVALID_ARG;
  if (((uintptr_t)lse & 3) || ((uintptr_t)workspace & 15) || unaligned(where)) return MTNLG_INVALID_ARG;
  FwdPlan plan = fwd_plan(S);
  if (!workspace || plan.bytes == 0) {   // without scratch: no cuts
    plan.chunk = 0;
    plan.chunks = 1;
  } else if (workspace_bytes < plan.bytes) {
    return MTNLG_WORKSPACE_TOO_SMALL;
  }
  PackedFwdArgs w{};
  w.where = Sequences{where->q_offsets, where->k_offsets, where->q_lengths, where->k_lengths, S.where.count, S.where.q_tokens, S.where.k_tokens};
  w.kv_heads = S.kv_heads;
  w.group = S.group;
  w.d = S.d;
  w.chunk = plan.chunk;
  w.chunks = plan.chunks;
  w.scale = S.scale;
  w.q = heads_of(q, S.where.q_tokens, S.d);
  w.k = heads_of(k, S.where.k_tokens, S.d);
  w.v = heads_of(v, S.where.k_tokens, S.d);
  w.a = heads_of(a, S.where.q_tokens, S.d);
  w.lse = lse;
  w.part = (float *)workspace;
  w.stat = (float *)((char *)workspace + plan.part_bytes);
  const int64_t pieces = cut_pieces(S, Cut{plan.chunk, plan.chunks}, plan.pieces, plan.owned);
  const int64_t blocks = pieces * S.kv_heads;
  if (!grid_fits(blocks, 256)) return MTNLG_UNSUPPORTED_SHAPE;
  const hipStream_t st = (hipStream_t)stream;
  LaunchScope scope(MTNLG_K_ATTN_FWD, st);
  MTNLG_TRY(packed_tuned(S.dtype, S.d) ? packed_fwd_tuned(w, plan.owned, blocks, st) : packed_fwd_plain(S.dtype, w, blocks, st));
  if (plan.chunks == 1) return MTNLG_OK;
  const unsigned joins = (unsigned)(pieces_bound((int64_t)S.where.q_tokens * S.group, (int64_t)S.max_q * S.group, S.where.count, 4) * S.kv_heads);
  if (S.dtype == MTNLG_F32) packed_join_kernel<float><<<joins, 256, 0, st>>>(w);
  else packed_join_kernel<bf16><<<joins, 256, 0, st>>>(w);
  return check_launch();
}


size_t mtnlg_packed_attention_bwd_workspace(const mtnlg_packed_desc *desc) {
  PackedShape S;
  return packed_shape(desc, &S) == MTNLG_OK ? bwd_plan(S).bytes : 0;
}

int mtnlg_packed_attention_bwd(const mtnlg_packed_desc *desc, const mtnlg_packed_sequences *where, const mtnlg_heads *q, const mtnlg_heads *k,
                               const mtnlg_heads *v, const mtnlg_heads *a, const float *lse, const mtnlg_heads *da, const mtnlg_heads *dq,
                               const mtnlg_heads *dk, const mtnlg_heads *dv, void *workspace, size_t workspace_bytes, void *stream) {
  if (!where || !where->q_offsets || !where->k_offsets || !lse || !workspace) return MTNLG_NULL_POINTER;
  for (const mtnlg_heads *m : {q, k, v, a, da, dq, dk, dv})
    if (!m || !m->data) return MTNLG_NULL_POINTER;
  PackedShape S;
  MTNLG_TRY(packed_shape(desc, &S));
  for (const mtnlg_heads *m : {q, a, da, dq}) MTNLG_TRY(heads_check(m, S.where.q_tokens, S.kv_heads, S.group, S.d, S.dtype));
  for (const mtnlg_heads *m : {k, v, dk, dv}) MTNLG_TRY(heads_check(m, S.where.k_tokens, S.kv_heads, 1, S.d, S.dtype));
  for (const mtnlg_heads *m : {dq, dk, dv})
    for (const mtnlg_heads *in : {q, k, v, a, da})
      if (m->data == in->data) return MTNLG_INVALID_ARG;
  if (dq->data == dk->data || dq->data == dv->data || dk->data == dv->data) return MTNLG_INVALID_ARG;
  if (((uintptr_t)lse & 3) || ((uintptr_t)workspace & 15) || unaligned(where)) return MTNLG_INVALID_ARG;
  const BwdPlan plan = bwd_plan(S);
  if (workspace_bytes < plan.bytes) return MTNLG_WORKSPACE_TOO_SMALL;
  const int key_threads = packed_tuned(S.dtype, S.d) ? 512 : 4 * plan.key_owned;   // of a dk / dv workgroup
  if (!grid_fits(plan.pieces * S.kv_heads, 256) || !grid_fits(plan.key_pieces * plan.splits * S.kv_heads, key_threads)) return MTNLG_UNSUPPORTED_SHAPE;
  PackedBwdArgs w{};
  w.where = Sequences{where->q_offsets, where->k_offsets, where->q_lengths, where->k_lengths, S.where.count, S.where.q_tokens, S.where.k_tokens};
  w.kv_heads = S.kv_heads;
  w.group = S.group;
  w.d = S.d;
  w.splits = plan.splits;
  w.scale = S.scale;
  w.q = heads_of(q, S.where.q_tokens, S.d);
  w.k = heads_of(k, S.where.k_tokens, S.d);
  w.v = heads_of(v, S.where.k_tokens, S.d);
  w.a = heads_of(a, S.where.q_tokens, S.d);
  w.da = heads_of(da, S.where.q_tokens, S.d);
  w.dq = heads_of(dq, S.where.q_tokens, S.d);
  w.dk = heads_of(dk, S.where.k_tokens, S.d);
  w.dv = heads_of(dv, S.where.k_tokens, S.d);
  w.lse = lse;
  w.D = (float *)workspace;
  w.part = (float *)((char *)workspace + plan.d_bytes);
  w.chunk = plan.cut.chunk;
  w.chunks = plan.cut.chunks;
  w.dq_part = (float *)((char *)workspace + plan.d_bytes + plan.part_bytes);
  const hipStream_t st = (hipStream_t)stream;
  LaunchScope scope(MTNLG_K_ATTN_BWD, st);
  MTNLG_TRY(packed_tuned(S.dtype, S.d) ? packed_bwd_tuned(w, plan.owned, plan.pieces, plan.key_pieces, st)
                                       : packed_bwd_plain(S.dtype, w, plan.pieces, plan.key_pieces, st));
  if (plan.cut.chunks > 1) {
    const unsigned joins = (unsigned)(pieces_bound((int64_t)S.where.q_tokens * S.group, (int64_t)S.max_q * S.group, S.where.count, 4) * S.kv_heads);
    packed_dq_join_kernel<float><<<joins, 256, 0, st>>>(w);   // (bf16 is not cut)
    MTNLG_TRY(check_launch());
  }
  if (plan.splits == 1) return MTNLG_OK;
  const unsigned joins = (unsigned)(pieces_bound(S.where.k_tokens, S.max_k, S.where.count, DKV_JOINED) * S.kv_heads);
  if (S.dtype == MTNLG_F32) packed_dkv_join_kernel<float><<<joins, 256, 0, st>>>(w);
  else packed_dkv_join_kernel<bf16><<<joins, 256, 0, st>>>(w);
  return check_launch();
}

}  // extern "C"
