// Rotary positions (Su et al., "RoFormer: Enhanced transformer with rotary position embedding", 2021): pair i of a head's first n columns turns by
//   angle = position * f_i,  f_i = base^(-2 i / n):   (u, w) -> amplitude (u cos - w sin, u sin + w cos),
// the backward pass by -angle.  Pairs are columns (i, n/2 + i) or (2 i, 2 i + 1).  Scaled for contexts longer than the trained one: positions divided by a factor
// (Chen et al., "Extending context window of large language models via positional interpolation", 2023), base times factor^(n / (n - 2)), or by parts (Peng et
// al., "YaRN: Efficient context window extension of large language models", 2023).
//
// Bound by memory: queries and keys are read and written once, in one launch.  A workgroup takes the rows of a few tokens; it works out their sines and
// cosines once, for all heads, and shares them through LDS.  Angles are worked out in 64 bits, in turns: at position 10^6 the fp32 product of position and
// frequency is off by up to 0.06 radians.
#include <math.h>

#include "common.h"

namespace mtnlg {

namespace {

struct RotaryArgs {
  int64_t tokens;
  int heads, kv_heads, group, d, n;   // rows of a token: its query heads, then its key heads
  const void *q, *k;
  void *q_out, *k_out;
  int64_t qs[3], ks[3], qos[3], kos[3];   // strides in elements: token, group, head in the group
  const int32_t *positions;
  double base_log2, factor, original, slow, fast;
  int scaling;
  float amplitude, sign;
  int copied;   // items of a head that are copied
  int tile;     // tokens of a workgroup
};

constexpr int THREADS = 256, MAX_PAIRS = 1024, MAX_TILE = 8;   // pairs and tokens of a tile

// turns of pair i for one position
__device__ double frequency(const RotaryArgs &a, int i) {
  double f = exp2(-2.0 * i / a.n * a.base_log2) * 0.15915494309189533577;
  if (a.scaling == MTNLG_ROTARY_LINEAR) f /= a.factor;
  if (a.scaling == MTNLG_ROTARY_PARTS) {   // turns in the original context: few, the pair is stretched; many, it stays
    const double keep = fmin(fmax((a.original * f - a.slow) / (a.fast - a.slow), 0.0), 1.0);
    f = f * keep + f / a.factor * (1.0 - keep);
  }
  return f;
}

template <typename E, int V> struct Piece { E v[V]; };
template <typename E, int V>
__device__ __forceinline__ void load_piece(const E *p, float (&x)[V]) {
  struct alignas(sizeof(E) * V < 16 ? sizeof(E) * V : 16) Raw { E v[V]; };
  const Raw t = *reinterpret_cast<const Raw *>(p);
#pragma unroll
  for (int e = 0; e < V; ++e) x[e] = to_f32(t.v[e]);
}
template <typename E, int V>
__device__ __forceinline__ void store_piece(E *p, const float (&x)[V]) {
  struct alignas(sizeof(E) * V < 16 ? sizeof(E) * V : 16) Raw { E v[V]; };
  Raw t;
#pragma unroll
  for (int e = 0; e < V; ++e) t.v[e] = from_f32<E>(x[e]);
  *reinterpret_cast<Raw *>(p) = t;
}

// An item is V pairs of a head (HALF: V columns of either half) or V columns (interleaved: V / 2 pairs), or V columns that are copied.
template <typename E, int V, bool HALF>
__global__ __launch_bounds__(THREADS) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 turn[MAX_PAIRS];   // [token of the tile][pair]
  __shared__ int place[MAX_TILE];      // positions of the tile's tokens
  const int pairs = a.n / 2;
  const int64_t first = (int64_t)blockIdx.x * a.tile;
  const int tokens = (int)(a.tokens - first < a.tile ? a.tokens - first : a.tile);
  for (int t = threadIdx.x; t < tokens; t += THREADS) place[t] = a.positions ? a.positions[first + t] : (int)(first + t);
  __syncthreads();
  for (int p = threadIdx.x; p < tokens * pairs; p += THREADS) {
    const int t = p / pairs, i = p - t * pairs;
    double x = place[t] * frequency(a, i);
    x -= rint(x);
    float s, c;
    sincospif(2.0f * (float)x, &s, &c);
    turn[p] = float2{c * a.amplitude, s * a.amplitude * a.sign};
  }
  __syncthreads();
  const int turned = HALF ? pairs / V : a.n / V, items = turned + a.copied, at_once = THREADS / items;
  const int item = threadIdx.x % items, row0 = threadIdx.x / items;
  if (row0 >= at_once) return;
  const int rows = a.heads + a.kv_heads;
  const bool copy = item >= turned;
  const int col = copy ? a.n + (item - turned) * V : item * V;
  int t = row0 / rows, head = row0 % rows;
  for (; t < tokens;) {
    if (place[t] >= 0) {   // a negative position: a row of padding, left as it is
      const bool query = head < a.heads;
      const int j = query ? head / a.group : head - a.heads, g = query ? head - j * a.group : 0;
      const int64_t *is = query ? a.qs : a.ks, *os = query ? a.qos : a.kos;
      const E *in = static_cast<const E *>(query ? a.q : a.k) + (first + t) * is[0] + j * is[1] + g * is[2] + col;
      E *out = static_cast<E *>(query ? a.q_out : a.k_out) + (first + t) * os[0] + j * os[1] + g * os[2] + col;
      float x[V];
      load_piece<E, V>(in, x);
      if (copy) {
        store_piece<E, V>(out, x);
      } else if constexpr (HALF) {
        float y[V], u[V], w[V];
        load_piece<E, V>(in + pairs, y);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 cs = turn[t * pairs + col + e];
          u[e] = x[e] * cs.x - y[e] * cs.y;
          w[e] = x[e] * cs.y + y[e] * cs.x;
        }
        store_piece<E, V>(out, u);
        store_piece<E, V>(out + pairs, w);
      } else {
        float u[V];
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float2 cs = turn[t * pairs + (col + e) / 2];
          u[e] = x[e] * cs.x - x[e + 1] * cs.y;
          u[e + 1] = x[e] * cs.y + x[e + 1] * cs.x;
        }
        store_piece<E, V>(out, u);
      }
    }
    head += at_once;
    while (head >= rows) {
      head -= rows;
      ++t;
    }
  }
}

template <typename E, bool HALF>
int launch(RotaryArgs &a, bool in_place, hipStream_t st) {
  // widest pieces that the halves, the head's other columns and 16-byte accesses allow
  const int unit = HALF ? a.n / 2 : a.n;
  const int V = unit % 8 == 0 ? 8 : unit % 4 == 0 ? 4 : HALF ? 1 : 2;
  a.copied = in_place ? 0 : (a.d - a.n) / V;
  const int pairs = a.n / 2, rows = a.heads + a.kv_heads;
  a.tile = MAX_PAIRS / pairs < MAX_TILE ? MAX_PAIRS / pairs : MAX_TILE;
  if (rows > 64) a.tile = (a.tile + 3) / 4;
  const unsigned blocks = (unsigned)((a.tokens + a.tile - 1) / a.tile);
  LaunchScope scope(MTNLG_K_ELEMENTWISE, st);
  if (V == 8) rotary_kernel<E, 8, HALF><<<blocks, THREADS, 0, st>>>(a);
  else if (V == 4) rotary_kernel<E, 4, HALF><<<blocks, THREADS, 0, st>>>(a);
  else rotary_kernel<E, HALF ? 1 : 2, HALF><<<blocks, THREADS, 0, st>>>(a);
  return check_launch();
}

int rotary(const mtnlg_rotary_desc *D, const mtnlg_heads *q, const mtnlg_heads *k, const mtnlg_heads *q_out, const mtnlg_heads *k_out,
           const int32_t *positions, float sign, hipStream_t st) {
  if (!D || !q || !q_out || !q->data || !q_out->data || !k != !k_out || (k && (!k->data || !k_out->data))) return MTNLG_NULL_POINTER;
  if (D->dtype != MTNLG_F32 && D->dtype != MTNLG_BF16) return MTNLG_INVALID_ARG;
  if (D->layout != MTNLG_ROTARY_HALF && D->layout != MTNLG_ROTARY_INTERLEAVED) return MTNLG_INVALID_ARG;
  if (D->tokens <= 0 || D->heads <= 0 || D->kv_heads <= 0 || D->heads % D->kv_heads || D->head_dim <= 0) return MTNLG_INVALID_ARG;
  if (D->rotary_dim <= 0 || D->rotary_dim % 2 || D->rotary_dim > D->head_dim) return MTNLG_INVALID_ARG;
  if (!(D->base > 0.0 && D->base < INFINITY) || !(D->amplitude >= 0.0 && D->amplitude < INFINITY)) return MTNLG_INVALID_ARG;
  if (D->scaling < MTNLG_ROTARY_UNSCALED || D->scaling > MTNLG_ROTARY_PARTS) return MTNLG_INVALID_ARG;
  if (D->scaling != MTNLG_ROTARY_UNSCALED && !(D->factor >= 1.0 && D->factor < INFINITY)) return MTNLG_INVALID_ARG;
  if (D->scaling == MTNLG_ROTARY_PARTS && (D->original_positions <= 0 || !(D->slow >= 0.0 && D->fast > D->slow && D->fast < INFINITY))) return MTNLG_INVALID_ARG;
  if (D->head_dim % 8 || D->head_dim > 256 || D->tokens > 0x7FFFFFFF || D->heads > 65535) return MTNLG_UNSUPPORTED_SHAPE;
  if ((uintptr_t)positions & 3) return MTNLG_INVALID_ARG;
  const int group = D->heads / D->kv_heads;
  MTNLG_TRY(heads_check(q, D->tokens, D->kv_heads, group, D->head_dim, D->dtype));
  MTNLG_TRY(heads_check(q_out, D->tokens, D->kv_heads, group, D->head_dim, D->dtype));
  if (k) {
    MTNLG_TRY(heads_check(k, D->tokens, D->kv_heads, 1, D->head_dim, D->dtype));
    MTNLG_TRY(heads_check(k_out, D->tokens, D->kv_heads, 1, D->head_dim, D->dtype));
  }
  auto same = [](const mtnlg_heads *x, const mtnlg_heads *y) { return x->data == y->data && x->token == y->token && x->group == y->group && x->head == y->head; };
  // in place or apart; the same address with other strides would read what another row has written
  if ((q->data == q_out->data && !same(q, q_out)) || (k && k->data == k_out->data && !same(k, k_out))) return MTNLG_INVALID_ARG;
  RotaryArgs a{};
  a.tokens = D->tokens;
  a.heads = D->heads;
  a.kv_heads = k ? D->kv_heads : 0;
  a.group = group;
  a.d = D->head_dim;
  a.n = D->rotary_dim;
  auto take = [](const mtnlg_heads *m, int64_t (&s)[3]) {
    s[0] = m->token;
    s[1] = m->group;
    s[2] = m->head;
    return m->data;
  };
  a.q = take(q, a.qs);
  a.q_out = take(q_out, a.qos);
  if (k) {
    a.k = take(k, a.ks);
    a.k_out = take(k_out, a.kos);
  }
  a.positions = positions;
  double base = D->base;
  if (D->scaling == MTNLG_ROTARY_BASE && a.n > 2) base *= pow(D->factor, (double)a.n / (a.n - 2));
  a.base_log2 = log2(base);
  a.scaling = D->scaling;
  a.factor = D->factor;
  a.original = D->original_positions;
  a.slow = D->slow;
  a.fast = D->fast;
  a.amplitude = (float)(D->amplitude > 0.0 ? D->amplitude : D->scaling == MTNLG_ROTARY_PARTS ? 0.1 * log(D->factor) + 1.0 : 1.0);
  a.sign = sign;
  const bool in_place = q->data == q_out->data && (!k || k->data == k_out->data);
  if (D->layout == MTNLG_ROTARY_HALF)
    return D->dtype == MTNLG_F32 ? launch<float, true>(a, in_place, st) : launch<bf16, true>(a, in_place, st);
  return D->dtype == MTNLG_F32 ? launch<float, false>(a, in_place, st) : launch<bf16, false>(a, in_place, st);
}

}  // namespace

// A matrix of heads that the kernels can take: rows of head_dim elements, aligned for 16-byte accesses, none on another.
int heads_check(const mtnlg_heads *m, int64_t tokens, int groups, int heads, int d, int dtype) {
  const int es = dtype == MTNLG_F32 ? 4 : 2, unit = 16 / es;
  if ((uintptr_t)m->data & 15) return MTNLG_INVALID_ARG;
  struct Dim { int64_t n, stride; } dim[3] = {{tokens, m->token}, {groups, m->group}, {heads, m->head}};
  for (auto &x : dim) {
    if (x.n == 1) x.stride = 0;   // never taken
    if (x.n > 1 && (x.stride <= 0 || x.stride % unit)) return MTNLG_INVALID_ARG;
    if (x.stride > ((int64_t)1 << 40)) return MTNLG_UNSUPPORTED_SHAPE;
  }
  // the DMA's offsets inside a tile of 64 rows have 32 bits
  if (tokens > 1 && m->token * es > ((int64_t)1 << 25)) return MTNLG_UNSUPPORTED_SHAPE;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (dim[j].stride < dim[i].stride) {
        const Dim t = dim[i];
        dim[i] = dim[j];
        dim[j] = t;
      }
  int64_t span = d;   // elements from the first to the end of the last
  for (auto &x : dim) {
    if (x.n == 1) continue;
    if (x.stride < span) return MTNLG_INVALID_ARG;
    span += (x.n - 1) * x.stride;
  }
  return MTNLG_OK;
}

}  // namespace mtnlg

using namespace mtnlg;

extern "C" {

int mtnlg_rotary_fwd(const mtnlg_rotary_desc *desc, const mtnlg_heads *q, const mtnlg_heads *k, const mtnlg_heads *q_out, const mtnlg_heads *k_out,
                     const int32_t *positions, void *stream) {
  return rotary(desc, q, k, q_out, k_out, positions, 1.0f, (hipStream_t)stream);
}
int mtnlg_rotary_bwd(const mtnlg_rotary_desc *desc, const mtnlg_heads *dq_out, const mtnlg_heads *dk_out, const mtnlg_heads *dq, const mtnlg_heads *dk,
                     const int32_t *positions, void *stream) {
  return rotary(desc, dq_out, dk_out, dq, dk, positions, -1.0f, (hipStream_t)stream);
}

}  // extern "C"
