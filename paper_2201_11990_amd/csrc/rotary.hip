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
  int64_t tokens, begin;   // begin: first token of the launch
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

// Pairs of a tile: one to a thread.  8192 tokens of 20 heads of 128 on buffers that no cache holds, halves, then side by side: 3 tokens to a tile 22.5 and 31 us, 6 and 3 22.5 and
// 27.5, 4 (side by side) 25.4, 8 27 and 28.7.
constexpr int THREADS = 256, MAX_PAIRS = THREADS, MAX_TILE = 64;
constexpr int MOST_BLOCKS = 1 << 23;   // of a launch, which has fewer than 2^32 work items
constexpr int AHEAD = 2;   // rows of a thread at once: 3 and 4 cost registers and with them waves (24.6, 27 us)

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

template <typename E, int V>
struct alignas(sizeof(E) * V < 16 ? sizeof(E) * V : 16) Piece { E v[V]; };

// A thread takes the same item of every head it works on: V pairs (HALF: V columns of either half), V columns (interleaved: V / 2 pairs), or V columns that are copied.
// The first AHEAD rows of each are read before the sines are worked out, which takes about as long as the reads; rows of padding with them (their positions first: 8192 tokens of 20 heads
// of 128, forward and backward, 41.9 us a pass, 43.1 so).
template <typename E, int V, bool HALF>
__global__ __launch_bounds__(THREADS) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 turn[MAX_PAIRS];   // [token of the tile][pair]
  __shared__ int place[MAX_TILE];      // positions of the tile's tokens
  __shared__ double rate[128];         // turns of each pair for one position
  const int pairs = a.n / 2;
  const int64_t first = a.begin + (int64_t)blockIdx.x * a.tile;
  const int tokens = (int)(a.tokens - first < a.tile ? a.tokens - first : a.tile);
  const int turned = HALF ? pairs / V : a.n / V, items = turned + a.copied, at_once = THREADS / items;
  const int item = threadIdx.x % items, row0 = threadIdx.x / items, heads = a.heads + a.kv_heads, rows = row0 < at_once ? tokens * heads : 0;
  const bool copy = item >= turned;
  const int col = copy ? a.n + (item - turned) * V : item * V;
  struct Spot {
    const E *in;
    E *out;
    int t;
  };
  auto spot = [&](int row) {
    Spot s;
    s.t = row / heads;
    const int head = row - s.t * heads;
    const bool query = head < a.heads;
    const int j = query ? head / a.group : head - a.heads, g = query ? head - j * a.group : 0;
    const int64_t *is = query ? a.qs : a.ks, *os = query ? a.qos : a.kos;
    s.in = static_cast<const E *>(query ? a.q : a.k) + (first + s.t) * is[0] + j * is[1] + g * is[2] + col;
    s.out = static_cast<E *>(query ? a.q_out : a.k_out) + (first + s.t) * os[0] + j * os[1] + g * os[2] + col;
    return s;
  };
  auto work_out_turns = [&] {
    if (threadIdx.x < pairs) rate[threadIdx.x] = frequency(a, threadIdx.x);
    else if (threadIdx.x >= 128 && threadIdx.x - 128 < tokens) place[threadIdx.x - 128] = a.positions ? a.positions[first + threadIdx.x - 128] : (int)(first + threadIdx.x - 128);
    __syncthreads();
    for (int p = threadIdx.x; p < tokens * pairs; p += THREADS) {
      const int t = p / pairs, i = p - t * pairs;
      double x = place[t] * rate[i];
      x -= rint(x);
      float s, c;
      sincospif(2.0f * (float)x, &s, &c);
      turn[p] = float2{c * a.amplitude, s * a.amplitude * a.sign};
    }
    __syncthreads();
  };
  bool begun = false;
  int row = row0;
  do {
    Piece<E, V> x[AHEAD], y[HALF ? AHEAD : 1];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (row + u * at_once < rows) {
        const Spot s = spot(row + u * at_once);
        x[u] = *reinterpret_cast<const Piece<E, V> *>(s.in);
        if (HALF && !copy) y[HALF ? u : 0] = *reinterpret_cast<const Piece<E, V> *>(s.in + pairs);
      }
    }
    if (!begun) work_out_turns();
    begun = true;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (row + u * at_once >= rows) continue;
      const Spot s = spot(row + u * at_once);
      if (place[s.t] < 0) continue;   // a row of padding, left as it is
      Piece<E, V> out[HALF ? 2 : 1];
      const float2 *const by = turn + s.t * pairs;
      if (copy) {
        out[0] = x[u];
      } else if constexpr (HALF) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 cs = by[col + e];
          const float v = to_f32(x[u].v[e]), w = to_f32(y[u].v[e]);
          out[0].v[e] = from_f32<E>(v * cs.x - w * cs.y);
          out[HALF].v[e] = from_f32<E>(v * cs.y + w * cs.x);
        }
        *reinterpret_cast<Piece<E, V> *>(s.out + pairs) = out[HALF];
      } else {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float2 cs = by[(col + e) / 2];
          const float v = to_f32(x[u].v[e]), w = to_f32(x[u].v[e + 1]);
          out[0].v[e] = from_f32<E>(v * cs.x - w * cs.y);
          out[0].v[e + 1] = from_f32<E>(v * cs.y + w * cs.x);
        }
      }
      *reinterpret_cast<Piece<E, V> *>(s.out) = out[0];
    }
    row += AHEAD * at_once;
  } while (row - row0 < tokens * heads);   // the same number of turns for all threads
}

template <typename E, bool HALF>
int launch(RotaryArgs &a, bool in_place, hipStream_t st) {
  // widest pieces that the halves, the head's other columns and 16-byte accesses allow
  const int unit = HALF ? a.n / 2 : a.n;
  const int V = unit % 8 == 0 ? 8 : unit % 4 == 0 ? 4 : HALF ? 1 : 2;
  a.copied = in_place ? 0 : (a.d - a.n) / V;
  const int pairs = a.n / 2, rows = a.heads + a.kv_heads;
  const int at_once = THREADS / ((HALF ? pairs / V : a.n / V) + a.copied), want = 2 * AHEAD * at_once / rows;   // two rounds of a workgroup's reads
  a.tile = MAX_PAIRS / pairs < MAX_TILE ? MAX_PAIRS / pairs : MAX_TILE;
  if (want < a.tile) a.tile = want < 1 ? 1 : want;
  if (a.tokens < 512 * (int64_t)a.tile) a.tile = (int)((a.tokens + 511) / 512);   // few tokens: more workgroups
  LaunchScope scope(MTNLG_K_ELEMENTWISE, st);
  for (a.begin = 0; a.begin < a.tokens; a.begin += (int64_t)MOST_BLOCKS * a.tile) {
    const int64_t tiles = (a.tokens - a.begin + a.tile - 1) / a.tile;
    const unsigned blocks = (unsigned)(tiles < MOST_BLOCKS ? tiles : MOST_BLOCKS);
    if (V == 8) rotary_kernel<E, 8, HALF><<<blocks, THREADS, 0, st>>>(a);
    else if (V == 4) rotary_kernel<E, 4, HALF><<<blocks, THREADS, 0, st>>>(a);
    else rotary_kernel<E, HALF ? 1 : 2, HALF><<<blocks, THREADS, 0, st>>>(a);
    MTNLG_TRY(check_launch());
  }
  return MTNLG_OK;
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
  // (strides of a dimension of one are not looked at)
  auto same = [&](const mtnlg_heads *x, const mtnlg_heads *y, int heads) {
    return x->data == y->data && (D->tokens == 1 || x->token == y->token) && (D->kv_heads == 1 || x->group == y->group) && (heads == 1 || x->head == y->head);
  };
  // in place or apart; the same address with other strides would read what another row has written
  if ((q->data == q_out->data && !same(q, q_out, group)) || (k && k->data == k_out->data && !same(k, k_out, 1))) return MTNLG_INVALID_ARG;
  // ... and so would an output that is the other one, or the other one's input
  if (k && (q_out->data == k->data || k_out->data == q->data || q_out->data == k_out->data)) return MTNLG_INVALID_ARG;
  double base = D->base;
  if (D->scaling == MTNLG_ROTARY_BASE && D->rotary_dim > 2) base *= pow(D->factor, (double)D->rotary_dim / (D->rotary_dim - 2));
  const double amplitude = D->amplitude > 0.0 ? D->amplitude : D->scaling == MTNLG_ROTARY_PARTS ? 0.1 * log(D->factor) + 1.0 : 1.0;
  if (!(base < INFINITY) || !((float)amplitude < INFINITY)) return MTNLG_INVALID_ARG;   // (their products would be NaN)
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
  a.base_log2 = log2(base);
  a.scaling = D->scaling;
  a.factor = D->factor;
  a.original = D->original_positions;
  a.slow = D->slow;
  a.fast = D->fast;
  a.amplitude = (float)amplitude;
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
