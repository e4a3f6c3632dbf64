// Exact attention of one token per sequence over a prefix that the batch shares and over the sequence's own rows.
//
// Both parts are the same stream: a wave holds a tile of query rows as the columns of its matrix products and goes
// through key and value rows with a running maximum and sum of the softmax.  Keys enter S = K Q^T straight from
// memory in the operand's layout, and what a lane holds of S is, with the contraction index permuted alike on both
// sides, already the operand of O^T += V^T P^T: no value crosses a lane between the two products.
#include "wave_common.h"

namespace wave {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// The reference of the exponentials follows the maximum only when that has grown by more than 2^8 over it: a weight is
// then at most 2^8, far from the end of any type here, and most steps leave the accumulators alone.
constexpr float kSlack = 8.f;

__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }

// ----------------------------------------------------------------------------
// A step: KEYS key and value rows against 16 query columns a tile.  Lane = 16 * g + c: column c of every product, and of
// a product's rows g * 4 .. g * 4 + 3.
// ----------------------------------------------------------------------------
template <typename T, int D>
struct Step;

// bf16: v_mfma_f32_16x16x32_bf16.  S has two tiles of 16 keys; a lane has the keys t * 16 + g * 4 + i of its column.  The
// contraction of the second product takes them in the order t * 4 + i, so a lane reads CH neighbouring channels of those
// eight value rows (16 lanes: a whole row) and pairs up the rows of each channel with v_perm.
template <int D>
struct Step<bf16_t, D> {
  static constexpr int KEYS = 32, NS = 8, KC = D / 32, CH = D / 16, ACC = CH;
  struct Q { bf16x8 x[KC]; };
  struct K { uint4 x[2][KC]; };
  struct V { uint32_t x[8][CH / 2]; };
  static __device__ __forceinline__ int key(int g, int s) { return (s >> 2) * 16 + g * 4 + (s & 3); }
  // channel of value i of accumulator a; a lane's are contiguous in (i, a)
  static __device__ __forceinline__ int channel(int g, int a, int i) { return (g * 4 + i) * CH + a; }

  static __device__ __forceinline__ Q load_q(const char* row, int g) {
    Q q;
#pragma unroll
    for (int s = 0; s < KC; ++s) q.x[s] = __builtin_bit_cast(bf16x8, load16(row + (s * 32 + g * 8) * 2));
    return q;
  }
  static __device__ __forceinline__ K load_k(const char* base, int k0, int last, int g, int c) {
    K k;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const char* row = base + (size_t)min(k0 + t * 16 + c, last) * (D * 2);
#pragma unroll
      for (int s = 0; s < KC; ++s) k.x[t][s] = load16(row + (s * 32 + g * 8) * 2);
    }
    return k;
  }
  static __device__ __forceinline__ V load_v(const char* base, int k0, int last, int g, int c) {
    V v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* at = base + (size_t)min(k0 + key(g, j), last) * (D * 2) + c * (CH * 2);
      if constexpr (CH == 8) {
        const uint4 u = load16(at);
        v.x[j][0] = u.x; v.x[j][1] = u.y; v.x[j][2] = u.z; v.x[j][3] = u.w;
      } else {
        const uint2 u = *reinterpret_cast<const uint2*>(at);
        v.x[j][0] = u.x; v.x[j][1] = u.y;
      }
    }
    return v;
  }
  // rows from `last` on count as zero: what lies there may be anything
  static __device__ __forceinline__ void mask_v(V& v, int k0, int last, int g) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k0 + key(g, j) > last)
#pragma unroll
        for (int u = 0; u < CH / 2; ++u) v.x[j][u] = 0;
  }
  static __device__ __forceinline__ void scores(const K& k, const Q& q, float (&s)[NS]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KC; ++i)
        a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.x[t][i]), q.x[i], a, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t * 4 + i] = a[i];
    }
  }
  // V^T as the left operand, channel a of every lane's chunk
  struct Vt { bf16x8 x[CH]; };
  static __device__ __forceinline__ Vt transpose(const V& v) {
    Vt r;
#pragma unroll
    for (int a = 0; a < CH; ++a) {
      const uint32_t sel = (a & 1) ? 0x07060302u : 0x05040100u;
      uint4 u;
      u.x = __builtin_amdgcn_perm(v.x[1][a / 2], v.x[0][a / 2], sel);
      u.y = __builtin_amdgcn_perm(v.x[3][a / 2], v.x[2][a / 2], sel);
      u.z = __builtin_amdgcn_perm(v.x[5][a / 2], v.x[4][a / 2], sel);
      u.w = __builtin_amdgcn_perm(v.x[7][a / 2], v.x[6][a / 2], sel);
      r.x[a] = __builtin_bit_cast(bf16x8, u);
    }
    return r;
  }
  // A weight's 24 bits as three bf16 numbers of eight, cut off from the top: their sum is the weight, so the product with
  // the values loses nothing.  (Two numbers, each the nearest, hold 16 bits; outputs are then off by 2e-6 of their norm,
  // twice what the fp32 sums cost.)
  static __device__ __forceinline__ void accumulate(const Vt& v, const float (&p)[NS], f32x4 (&o)[ACC]) {
    uint32_t w[3][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x = p[2 * j], y = p[2 * j + 1];
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        w[n][j] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
        x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
      }
    }
#pragma unroll
    for (int n = 2; n >= 0; --n) {
      const bf16x8 b = __builtin_bit_cast(bf16x8, make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]));
#pragma unroll
      for (int a = 0; a < CH; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.x[a], b, o[a], 0, 0, 0);
    }
  }
};

// f32: v_mfma_f32_16x16x4_f32, one tile of 16 keys; a lane has the keys g * 4 + i.  Product number i of the second
// contraction takes key g * 4 + i from lane group g.
template <int D>
struct Step<float, D> {
  static constexpr int KEYS = 16, NS = 4, KC = D / 16, CV = D / 64, ACC = D / 16;
  struct Q { f32x4 x[KC]; };
  struct K { f32x4 x[KC]; };
  struct V { f32x4 x[4][CV]; };
  typedef V Vt;
  static __device__ __forceinline__ int key(int g, int s) { return g * 4 + s; }
  static __device__ __forceinline__ int channel(int g, int a, int i) { return (a >> 2) * 64 + (g * 4 + i) * 4 + (a & 3); }
  static __device__ __forceinline__ f32x4 load(const char* p) { return *reinterpret_cast<const f32x4*>(p); }

  static __device__ __forceinline__ Q load_q(const char* row, int g) {
    Q q;
#pragma unroll
    for (int s = 0; s < KC; ++s) q.x[s] = load(row + (s * 16 + g * 4) * 4);
    return q;
  }
  static __device__ __forceinline__ K load_k(const char* base, int k0, int last, int g, int c) {
    K k;
    const char* row = base + (size_t)min(k0 + c, last) * (D * 4);
#pragma unroll
    for (int s = 0; s < KC; ++s) k.x[s] = load(row + (s * 16 + g * 4) * 4);
    return k;
  }
  static __device__ __forceinline__ V load_v(const char* base, int k0, int last, int g, int c) {
    V v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < CV; ++u)
        v.x[i][u] = load(base + (size_t)min(k0 + g * 4 + i, last) * (D * 4) + (u * 64 + c * 4) * 4);
    return v;
  }
  static __device__ __forceinline__ void mask_v(V& v, int k0, int last, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k0 + g * 4 + i > last)
#pragma unroll
        for (int u = 0; u < CV; ++u) v.x[i][u] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  static __device__ __forceinline__ void scores(const K& k, const Q& q, float (&s)[NS]) {
    // four chains: a sum of 128 products in one is off by twice as much
    f32x4 a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) a[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[i][j], q.x[i][j], a[j], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = (a[0][i] + a[1][i]) + (a[2][i] + a[3][i]);
  }
  static __device__ __forceinline__ Vt transpose(const V& v) { return v; }
  static __device__ __forceinline__ void accumulate(const Vt& v, const float (&p)[NS], f32x4 (&o)[ACC]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < CV; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[u * 4 + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x[i][u][j], p[i], o[u * 4 + j], 0, 0, 0);
  }
};

// The softmax state of a tile of 16 query columns.
template <typename T, int D>
struct State {
  typedef Step<T, D> S;
  float m, l;  // reference (log2 units, one for the column's four lanes) and this lane's share of the sum
  f32x4 o[S::ACC];
  __device__ __forceinline__ void init() {
    m = neg_inf();
    l = 0.f;
#pragma unroll
    for (int a = 0; a < S::ACC; ++a) o[a] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // s: products q . k; becomes the weights exp(s / sqrt(d)) over the reference.  scale: log2(e) / sqrt(d), applied inside
  // the difference, which is then rounded once.
  __device__ __forceinline__ void weigh(float (&s)[S::NS], float scale) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < S::NS; ++i) top = fmaxf(top, s[i]);
    top *= scale;
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float grown = fmaxf(m, top);
      const float f = m == neg_inf() ? 0.f : exp2f(m - grown);
      m = grown;
      l *= f;
#pragma unroll
      for (int a = 0; a < S::ACC; ++a) o[a] *= f;
    }
    const float ref = m == neg_inf() ? 0.f : m;  // (every score -infinity so far)
#pragma unroll
    for (int i = 0; i < S::NS; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -ref));
      l += s[i];
    }
  }
};

// ----------------------------------------------------------------------------
// The stream of one wave: the rows k0, k0 + stride, .. below `end` against MQ tiles of query columns.  z: where a lane
// leaves the scores of its column (NULL: nowhere).
// ----------------------------------------------------------------------------
template <typename T, int D, int MQ>
__device__ __forceinline__ void stream_rows(const char* K, const char* V, int k0, int stride, int end, float scale,
                                            const typename Step<T, D>::Q (&q)[MQ], State<T, D> (&st)[MQ], float* z, int g,
                                            int c) {
  typedef Step<T, D> S;
  const int last = end - 1;
  if (k0 >= end) return;
  typename S::K k = S::load_k(K, k0, last, g, c);
  typename S::V v = S::load_v(V, k0, last, g, c);
  for (;;) {
    const int next = k0 + stride;
    const bool ragged = k0 + S::KEYS > end;
    float s[MQ][S::NS];
#pragma unroll
    for (int t = 0; t < MQ; ++t) S::scores(k, q[t], s[t]);
    // The next rows' loads go out as soon as the registers are free: a wave has loads in flight all the time.  They are made
    // behind the end too (the last row again), since a wait behind a load that may not have been made waits for all of them.
    k = S::load_k(K, next, last, g, c);
    if (ragged) {
      S::mask_v(v, k0, last, g);
#pragma unroll
      for (int t = 0; t < MQ; ++t)
#pragma unroll
        for (int i = 0; i < S::NS; ++i)
          if (k0 + S::key(g, i) > last) s[t][i] = neg_inf();
    }
    if (MQ == 1 && z) {
#pragma unroll
      for (int i = 0; i < S::NS; i += 4)
        *reinterpret_cast<f32x4*>(z + k0 + S::key(g, i)) = f32x4{s[0][i], s[0][i + 1], s[0][i + 2], s[0][i + 3]};
    }
    const typename S::Vt vt = S::transpose(v);
    v = S::load_v(V, next, last, g, c);
#pragma unroll
    for (int t = 0; t < MQ; ++t) {
      st[t].weigh(s[t], scale);
      S::accumulate(vt, s[t], st[t].o);
    }
    if (next >= end) return;
    k0 = next;
  }
}

// What a partial result leaves of its softmax.  A sum that is no number may have no reference, where every score was none:
// it has to survive the joining.
__device__ __forceinline__ float2 partial_ml(float m, float l) { return make_float2(l == l ? m : -neg_inf(), l); }

// The four waves' states of one tile of columns joined in LDS; columns below `cols` are left by all 256 threads as one
// partial result each: (m, l) at ml[col], the sum at acc + col * D.
struct __attribute__((aligned(16))) JoinShared {
  float m[4][16], l[4][16];
};
template <typename T, int D>
__device__ __forceinline__ void join_waves(const State<T, D>& st, int cols, JoinShared& js, float* lds, int wave, int g, int c,
                                           float2* ml, float* acc) {
  typedef Step<T, D> S;
  constexpr int PITCH = D + 4;  // floats a column: lanes of a column's four groups and of neighbouring columns on other banks
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    js.m[wave][c] = st.m;
    js.l[wave][c] = l;
  }
  if (c < cols) {
    float* at = lds + ((size_t)wave * 16 + c) * PITCH;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int a = 0; a < S::ACC; a += 4) {
        // four neighbouring channels
        const f32x4 x = {st.o[a][i], st.o[a + 1][i], st.o[a + 2][i], st.o[a + 3][i]};
        *reinterpret_cast<f32x4*>(at + S::channel(g, a, i)) = x;
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < cols * D; i += 256) {
    const int col = i / D, ch = i % D;
    float m = js.m[0][col];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, js.m[w][col]);
    float sum = 0.f, tot = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = js.m[w][col] == neg_inf() ? 0.f : exp2f(js.m[w][col] - m);
      sum += f * lds[((size_t)w * 16 + col) * PITCH + ch];
      tot += f * js.l[w][col];
    }
    acc[(size_t)col * D + ch] = sum;
    if (ch == 0) ml[col] = partial_ml(m, tot);
  }
}

// ----------------------------------------------------------------------------
// How the own rows are cut: pieces of `rows` rows, a multiple of 128 that makes about `target` of them per KV head.  Piece
// w of a KV head belongs to the sequence whose pieces it falls among.  All lanes of a wave call this together.
// ----------------------------------------------------------------------------
struct Pieces {
  int rows;               // rows of a piece
  int b, first, length;   // the sequence, its first piece, its rows (b = B: there is no piece w)
};
__device__ __forceinline__ int cache_length(const int32_t* lengths, int b, int capacity) {
  return min(max(lengths[b], 0), capacity);
}
__device__ __forceinline__ int piece_rows(const int32_t* lengths, int B, int capacity, int target) {
  long long total = 0;
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int len = b0 + lane < B ? cache_length(lengths, b0 + lane, capacity) : 0;
    // (64 lengths of up to 2^30 in two sums of 16 bits and more each)
    total += ((long long)wave_sum_i(len >> 12) << 12) + wave_sum_i(len & 4095);
  }
  const long long r = (total + target - 1) / target;
  return (int)((r + 127) / 128 > 0 ? (r + 127) / 128 * 128 : 128);
}
__device__ __forceinline__ Pieces find_piece(const int32_t* lengths, int B, int capacity, int target, int w) {
  const int lane = threadIdx.x & 63;
  Pieces p;
  p.rows = piece_rows(lengths, B, capacity, target);
  p.b = B;
  p.first = p.length = 0;
  int before = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int len = b0 + lane < B ? cache_length(lengths, b0 + lane, capacity) : 0;
    const int n = (len + p.rows - 1) / p.rows;
    const int incl = before + wave_incl_scan(n);
    const uint64_t hit = __ballot(w < incl);
    if (hit) {
      const int at = __ffsll((unsigned long long)hit) - 1;
      p.b = b0 + at;
      p.first = __builtin_amdgcn_readlane(incl - n, at);
      p.length = __builtin_amdgcn_readlane(len, at);
      return p;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return p;
}
// The first piece of sequence b.
__device__ __forceinline__ int first_piece(const int32_t* lengths, int b, int capacity, int rows) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < b; b0 += 64) {
    const int len = b0 + lane < b ? cache_length(lengths, b0 + lane, capacity) : 0;
    before += wave_sum_i((len + rows - 1) / rows);
  }
  return before;
}

struct AttendArgs {
  const char *q, *k, *v, *prefix_k, *prefix_v;
  const int32_t* lengths;
  const float* weights;
  float *weights_out, *out, *lse;
  float *z, *acc, *pacc;   // products q . k [B * Hq][zrow]; sums of the own pieces [Hkv][pieces][G][D], of the prefix [splits][B * Hq][D]
  float2 *ml, *pml;        // their references and normalisers
  int B, Hq, Hkv, G, capacity, P;
  int target, pieces, prefix_rows, splits, zrow;
  float scale, decay;
};

// Own rows: one workgroup per piece, all G heads of its unit as columns; the four waves take every fourth step.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void own_rows_kernel(const AttendArgs a) {
  typedef Step<T, D> S;
  __shared__ JoinShared js;
  __shared__ __attribute__((aligned(16))) float lds[4 * 16 * (D + 4)];
  const int w = blockIdx.x / a.Hkv, h = blockIdx.x % a.Hkv;
  const Pieces p = find_piece(a.lengths, a.B, a.capacity, a.target, w);
  if (p.b == a.B) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int start = (w - p.first) * p.rows, end = min(p.length, start + p.rows);
  const size_t unit = (size_t)p.b * a.Hkv + h, row = D * sizeof(T);
  const int head = h * a.G + min(c, a.G - 1);  // (columns behind the G heads repeat the last one)
  const size_t bh = (size_t)p.b * a.Hq + head;
  typename S::Q q[1] = {S::load_q(a.q + bh * row, g)};
  State<T, D> st[1];
  st[0].init();
  float* z = a.weights_out && c < a.G ? a.z + bh * a.zrow : nullptr;
  stream_rows<T, D, 1>(a.k + unit * a.capacity * row, a.v + unit * a.capacity * row, start + wave * S::KEYS, 4 * S::KEYS, end,
                       a.scale, q, st, z, g, c);
  const size_t at = ((size_t)h * a.pieces + w) * a.G;
  join_waves<T, D>(st[0], a.G, js, lds, wave, g, c, a.ml + at, a.acc + at * D);
}

// Prefix: one workgroup per (KV head, range of prefix rows, MQ tiles of the B * G query rows).
template <typename T, int D, int MQ>
__global__ __launch_bounds__(256, MQ == 1 ? 2 : 1) void prefix_rows_kernel(const AttendArgs a) {
  typedef Step<T, D> S;
  __shared__ JoinShared js;
  __shared__ __attribute__((aligned(16))) float lds[4 * 16 * (D + 4)];
  const int hs = blockIdx.x % (a.Hkv * a.splits), tile = blockIdx.x / (a.Hkv * a.splits);
  const int h = hs % a.Hkv, split = hs / a.Hkv;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int M = a.B * a.G, m0 = tile * MQ * 16;
  const size_t row = D * sizeof(T);
  typename S::Q q[MQ];
  State<T, D> st[MQ];
#pragma unroll
  for (int t = 0; t < MQ; ++t) {
    const int m = min(m0 + t * 16 + c, M - 1), b = m / a.G;
    q[t] = S::load_q(a.q + ((size_t)b * a.Hq + h * a.G + (m - b * a.G)) * row, g);
    st[t].init();
  }
  const int start = split * a.prefix_rows, end = min(a.P, start + a.prefix_rows);
  stream_rows<T, D, MQ>(a.prefix_k + (size_t)h * a.P * row, a.prefix_v + (size_t)h * a.P * row, start + wave * S::KEYS,
                        4 * S::KEYS, end, a.scale, q, st, nullptr, g, c);
#pragma unroll
  for (int t = 0; t < MQ; ++t) {
    const int first = m0 + t * 16;
    if (first < M) {
      // partial results by KV head and query row
      const size_t at = ((size_t)split * a.Hkv + h) * M + first;
      join_waves<T, D>(st[t], min(16, M - first), js, lds, wave, g, c, a.pml + at, a.pacc + at * D);
    }
    __syncthreads();
  }
}

// Prefix with more query rows than a tile (bf16): four waves with MQ tiles of columns each go through the same rows, which
// they share in LDS.  While they work on a tile of 64 rows the next one is on its way there, straight from memory.  Chunk
// x (16 bytes) of row r lies at x ^ f(r): the lanes of an operand read, which have one chunk of sixteen key rows, or two
// neighbouring chunks of eight value rows, then hit all banks.  The values' operand comes transposed (ds_read_b64_tr_b16:
// sixteen lanes read four rows of sixteen channels, and each gets the four values of its channel).
template <int D>
struct SharedTile {
  static constexpr int ROWS = 64, ROW = D * 2, CHUNKS = ROW / 16, BYTES = ROWS * ROW;
  static constexpr int FILLS = BYTES / 1024 / 4;  // wave-wide loads of each wave
  static __device__ __forceinline__ int fk(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int fv(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
  // rows r0 .. of src (the last one again behind the end) into lds; V: which of the two arrangements
  template <bool V>
  static __device__ __forceinline__ void fill(char* lds, const char* src, int r0, int last, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < FILLS; ++i) {
      const int piece = wave * FILLS + i, r = piece * (1024 / ROW) + lane / CHUNKS;
      const int x = lane % CHUNKS ^ (V ? fv(r) : fk(r));
      const char* from = src + (size_t)min(r0 + r, last) * ROW + x * 16;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                       (__attribute__((address_space(3))) void*)(lds + piece * 1024), 16, 0, 0);
    }
  }
};

template <int D, int MQ>
__global__ __launch_bounds__(256, 2) void prefix_shared_kernel(const AttendArgs a) {
  typedef Step<bf16_t, D> S;
  typedef SharedTile<D> L;
  constexpr int BLOCKS = D / 16;  // of sixteen channels
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(1024))) char lk0[L::BYTES], lk1[L::BYTES], lv0[L::BYTES], lv1[L::BYTES];
  const int hs = blockIdx.x % (a.Hkv * a.splits), tile = blockIdx.x / (a.Hkv * a.splits);
  const int h = hs % a.Hkv, split = hs / a.Hkv;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int M = a.B * a.G, m0 = (tile * 4 + wave) * MQ * 16;
  typename S::Q q[MQ];
  State<bf16_t, D> st[MQ];
#pragma unroll
  for (int t = 0; t < MQ; ++t) {
    const int m = min(m0 + t * 16 + c, M - 1), b = m / a.G;
    q[t] = S::load_q(a.q + ((size_t)b * a.Hq + h * a.G + (m - b * a.G)) * L::ROW, g);
    st[t].init();
  }
  const int start = split * a.prefix_rows, end = min(a.P, start + a.prefix_rows), last = end - 1;
  const char* K = a.prefix_k + (size_t)h * a.P * L::ROW;
  const char* V = a.prefix_v + (size_t)h * a.P * L::ROW;
  int ka[S::KC], va[BLOCKS];  // this lane's places in a tile, of row c and of row g * 4 + c / 4
#pragma unroll
  for (int x = 0; x < S::KC; ++x) ka[x] = c * L::ROW + ((x * 4 + g) ^ L::fk(c)) * 16;
#pragma unroll
  for (int x = 0; x < BLOCKS; ++x) {
    const int r = g * 4 + (c >> 2);
    va[x] = r * L::ROW + ((x * 2 + ((c & 3) >> 1)) ^ L::fv(r)) * 16 + (c & 1) * 8;
  }
  auto fill = [&](char* lk, char* lv, int r0) {
    L::template fill<false>(lk, K, r0, last, wave, lane);
    L::template fill<true>(lv, V, r0, last, wave, lane);
  };
  auto filled = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // this wave's loads into LDS (vmcnt 0)
    __syncthreads();
  };
  auto work = [&](const char* lk, const char* lv, int r0) {
#pragma unroll
    for (int half = 0; half < L::ROWS; half += 32) {
      const int k0 = r0 + half;
      if (k0 >= end) break;
      typename S::K k;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < S::KC; ++x) k.x[t][x] = load16(lk + ka[x] + (half + t * 16) * L::ROW);
      s16x4 v[BLOCKS][2];
#pragma unroll
      for (int x = 0; x < BLOCKS; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          v[x][t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(lv + va[x] + (half + t * 16) * L::ROW));
      float s[MQ][S::NS];
#pragma unroll
      for (int t = 0; t < MQ; ++t) S::scores(k, q[t], s[t]);
      if (k0 + 32 > end) {
        // (rows behind the end are the last row again: their weight is zero, and zero times a number that is none must not
        // show, so the values go too)
#pragma unroll
        for (int x = 0; x < BLOCKS; ++x)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (k0 + S::key(g, j) > last) v[x][j >> 2][j & 3] = 0;
#pragma unroll
        for (int t = 0; t < MQ; ++t)
#pragma unroll
          for (int i = 0; i < S::NS; ++i)
            if (k0 + S::key(g, i) > last) s[t][i] = neg_inf();
      }
      typename S::Vt vt;
#pragma unroll
      for (int x = 0; x < BLOCKS; ++x) {
        const uint2 lo = __builtin_bit_cast(uint2, v[x][0]), hi = __builtin_bit_cast(uint2, v[x][1]);
        vt.x[x] = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
      }
#pragma unroll
      for (int t = 0; t < MQ; ++t) {
        st[t].weigh(s[t], a.scale);
        S::accumulate(vt, s[t], st[t].o);
      }
    }
  };
  fill(lk0, lv0, start);
  filled();
  for (int r0 = start;; r0 += 2 * L::ROWS) {
    if (r0 + L::ROWS < end) fill(lk1, lv1, r0 + L::ROWS);
    work(lk0, lv0, r0);
    if (r0 + L::ROWS >= end) break;
    filled();
    if (r0 + 2 * L::ROWS < end) fill(lk0, lv0, r0 + 2 * L::ROWS);
    work(lk1, lv1, r0 + L::ROWS);
    if (r0 + 2 * L::ROWS >= end) break;
    filled();
  }
#pragma unroll
  for (int t = 0; t < MQ; ++t) {
    const int m = m0 + t * 16 + c;
    float l = st[t].l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (m < M) {
      const size_t at = ((size_t)split * a.Hkv + h) * M + m;
      if (g == 0) a.pml[at] = partial_ml(st[t].m, l);
#pragma unroll
      for (int x = 0; x < BLOCKS; ++x) *reinterpret_cast<f32x4*>(a.pacc + at * D + x * 16 + g * 4) = st[t].o[x];
    }
  }
}

// ----------------------------------------------------------------------------
// Merge.  The first B * Hq workgroups join a head's partial results.  With weights, the others have 1024 rows of a unit
// each: they form the G heads' normalisers from the partial (m, l) again, which is less than waiting for them, and add up
// the softmax weights.
// ----------------------------------------------------------------------------
struct HeadParts {
  const float2 *ml, *pml;
  int splits, own, stride, pstride;  // partials of the prefix and of own pieces, and what lies between them
  __device__ __forceinline__ float2 at(int i) const {
    return i < splits ? pml[(size_t)i * pstride] : ml[(size_t)(i - splits) * stride];
  }
};
__device__ __forceinline__ HeadParts head_parts(const AttendArgs& a, int b, int h, int gq, int first, int own) {
  HeadParts p;
  p.splits = a.splits;
  p.own = own;
  p.stride = a.G;
  p.pstride = a.Hkv * a.B * a.G;
  p.ml = a.ml + ((size_t)h * a.pieces + first) * a.G + gq;
  p.pml = a.pml + (size_t)h * a.B * a.G + (size_t)b * a.G + gq;
  return p;
}
// (reference, normaliser) over the partials; all lanes of a wave together
__device__ __forceinline__ float2 normaliser(const HeadParts& p) {
  const int lane = threadIdx.x & 63, n = p.splits + p.own;
  float m = neg_inf(), l = 0.f;
  for (int i = lane; i < n; i += 64) {
    const float2 x = p.at(i);
    const float t = fmaxf(m, x.x);
    if (t != neg_inf()) l = (m == neg_inf() ? 0.f : l * exp2f(m - t)) + (x.x == neg_inf() ? 0.f : x.y * exp2f(x.x - t));
    m = t;
  }
  const float top = wave_max(m);
  l = m == neg_inf() ? 0.f : l * exp2f(m - top);
  return make_float2(top, wave_sum_f(l));
}

constexpr int WEIGHT_ROWS = 1024;

template <int D>
__global__ __launch_bounds__(256) void join_kernel(const AttendArgs a) {
  const int heads = a.B * a.Hq, tid = threadIdx.x, wave = tid >> 6;
  const int rows = piece_rows(a.lengths, a.B, a.capacity, a.target);
  __shared__ float2 norm[8];
  if ((int)blockIdx.x < heads) {
    __shared__ float part[256 / (D / 4)][D];
    const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, h = hq / a.G, gq = hq % a.G;
    const int len = cache_length(a.lengths, b, a.capacity), own = (len + rows - 1) / rows;
    const int first = first_piece(a.lengths, b, a.capacity, rows);
    const HeadParts p = head_parts(a, b, h, gq, first, own);
    const float2 n = normaliser(p);
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    const int lane = tid % LANES, group = tid / LANES;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = group; i < p.splits + own; i += GROUPS) {
      const float2 x = p.at(i);
      const float f = x.x == neg_inf() ? 0.f : exp2f(x.x - n.x);
      const float* acc = i < p.splits
                             ? a.pacc + ((size_t)i * p.pstride + (size_t)h * a.B * a.G + (size_t)b * a.G + gq) * D
                             : a.acc + (((size_t)h * a.pieces + first + i - p.splits) * a.G + gq) * D;
      sum += f * *reinterpret_cast<const f32x4*>(acc + lane * 4);
    }
    *reinterpret_cast<f32x4*>(&part[group][lane * 4]) = sum;
    __syncthreads();
    for (int ch = tid; ch < D; ch += 256) {
      float o = 0.f;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) o += part[i][ch];
      a.out[(size_t)blockIdx.x * D + ch] = n.x == neg_inf() ? 0.f : o / n.y;
    }
    if (tid == 0) a.lse[blockIdx.x] = n.x == neg_inf() ? neg_inf() : (n.x + log2f(n.y)) * kLn2;
    return;
  }
  const int chunks = (a.capacity + WEIGHT_ROWS - 1) / WEIGHT_ROWS;
  const int at = blockIdx.x - heads, unit = at / chunks, r0 = at % chunks * WEIGHT_ROWS;
  const int b = unit / a.Hkv, h = unit % a.Hkv;
  const int len = cache_length(a.lengths, b, a.capacity);
  if (r0 >= len) return;
  const int own = (len + rows - 1) / rows, first = first_piece(a.lengths, b, a.capacity, rows);
  for (int gq = wave; gq < a.G; gq += 4) {
    const float2 n = normaliser(head_parts(a, b, h, gq, first, own));
    if ((tid & 63) == 0) norm[gq] = make_float2(n.x == neg_inf() ? 0.f : n.x, n.x == neg_inf() ? 1.f : 1.f / n.y);
  }
  __syncthreads();
  const size_t base = (size_t)unit * a.capacity;
  const float* z = a.z + ((size_t)b * a.Hq + h * a.G) * a.zrow;
  for (int j = r0 + tid; j < min(len, r0 + WEIGHT_ROWS); j += 256) {
    float w = 0.f;
    for (int gq = 0; gq < a.G; ++gq) w += __builtin_amdgcn_exp2f(fmaf(z[(size_t)gq * a.zrow + j], a.scale, -norm[gq].x)) * norm[gq].y;
    a.weights_out[base + j] = a.decay > 0.f ? a.decay * a.weights[base + j] + w : w;
  }
}

template <typename T, int D>
wave_status attend_td(const AttendArgs& a, const CacheAttendGeom& g, hipStream_t st) {
  if (a.P > 0) {
    const unsigned grid = a.Hkv * a.splits * g.mtiles;
    if (g.mtile == 16) WAVE_LAUNCH("prefix_rows", (prefix_rows_kernel<T, D, 1>), grid, 256, 0, st, a);
    if (g.mtile == 32) WAVE_LAUNCH("prefix_rows", (prefix_rows_kernel<T, D, 2>), grid, 256, 0, st, a);
    if constexpr (sizeof(T) == 2) {
      if (g.mtile == 64) WAVE_LAUNCH("prefix_shared", (prefix_shared_kernel<D, 1>), grid, 256, 0, st, a);
      if (g.mtile == 128) WAVE_LAUNCH("prefix_shared", (prefix_shared_kernel<D, 2>), grid, 256, 0, st, a);
    }
  }
  WAVE_LAUNCH("own_rows", (own_rows_kernel<T, D>), a.Hkv * g.pieces, 256, 0, st, a);
  const long long chunks = ((long long)a.capacity + WEIGHT_ROWS - 1) / WEIGHT_ROWS;
  const unsigned grid = a.B * a.Hq + (a.weights_out ? (unsigned)(a.B * a.Hkv * chunks) : 0u);
  WAVE_LAUNCH("cache_join", join_kernel<D>, grid, 256, 0, st, a);
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

}  // namespace

CacheAttendGeom cache_attend_geometry(const wave_cache& c, int Hq, int P, bool accumulate) {
  CacheAttendGeom g{};
  const int G = Hq / c.Hkv;
  // Own rows: about six pieces a CU over all KV heads; every sequence may end in a piece that is not full.
  g.target = 1536 / c.Hkv > 1 ? 1536 / c.Hkv : 1;
  const long long most = (long long)c.B * (((long long)c.capacity + 127) / 128);
  g.pieces = (int)((long long)g.target + c.B < most ? g.target + c.B : most);
  const int M = c.B * G;
  g.mtile = M <= 16 ? 16 : c.dtype == WAVE_F32 ? 32 : M <= 64 ? 64 : 128;
  g.mtiles = (M + g.mtile - 1) / g.mtile;
  if (P > 0) {
    const int want = 512 / (c.Hkv * g.mtiles) > 1 ? 512 / (c.Hkv * g.mtiles) : 1;
    const long long rows = ((long long)P + want - 1) / want;
    g.prefix_rows = (int)((rows + 127) / 128 * 128);
    g.splits = (int)(((long long)P + g.prefix_rows - 1) / g.prefix_rows);
  }
  g.zrow = (c.capacity + 31) / 32 * 32;  // whole steps
  size_t o = 0;
  g.off_z = o;     o = align_up(o + (accumulate ? sizeof(float) * (size_t)c.B * Hq * g.zrow : 0));
  g.off_ml = o;    o = align_up(o + sizeof(float) * 2 * (size_t)Hq * g.pieces);
  g.off_acc = o;   o = align_up(o + sizeof(float) * c.d * (size_t)Hq * g.pieces);
  g.off_pml = o;   o = align_up(o + sizeof(float) * 2 * (size_t)c.B * Hq * g.splits);
  g.off_pacc = o;  o = align_up(o + sizeof(float) * c.d * (size_t)c.B * Hq * g.splits);
  g.total = o;
  return g;
}

wave_status launch_cache_attend(const void* q, int Hq, const wave_cache& c, const void* prefix_k, const void* prefix_v,
                                int P, float decay, float* weights_out, float* out, float* lse, void* ws,
                                hipStream_t st) {
  const CacheAttendGeom g = cache_attend_geometry(c, Hq, P, weights_out != nullptr);
  char* w = static_cast<char*>(ws);
  AttendArgs a{};
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(c.k);
  a.v = static_cast<const char*>(c.v);
  a.prefix_k = static_cast<const char*>(prefix_k);
  a.prefix_v = static_cast<const char*>(prefix_v);
  a.lengths = c.lengths;
  a.weights = c.weights;
  a.weights_out = weights_out;
  a.out = out;
  a.lse = lse;
  a.z = reinterpret_cast<float*>(w + g.off_z);
  a.ml = reinterpret_cast<float2*>(w + g.off_ml);
  a.acc = reinterpret_cast<float*>(w + g.off_acc);
  a.pml = reinterpret_cast<float2*>(w + g.off_pml);
  a.pacc = reinterpret_cast<float*>(w + g.off_pacc);
  a.B = c.B;
  a.Hq = Hq;
  a.Hkv = c.Hkv;
  a.G = Hq / c.Hkv;
  a.capacity = c.capacity;
  a.P = P;
  a.target = g.target;
  a.pieces = g.pieces;
  a.prefix_rows = g.prefix_rows;
  a.splits = g.splits;
  a.zrow = g.zrow;
  a.scale = kLog2e / sqrtf((float)c.d);
  a.decay = decay;
  if (c.dtype == WAVE_BF16) return c.d == 128 ? attend_td<bf16_t, 128>(a, g, st) : attend_td<bf16_t, 64>(a, g, st);
  return c.d == 128 ? attend_td<float, 128>(a, g, st) : attend_td<float, 64>(a, g, st);
}

}  // namespace wave
