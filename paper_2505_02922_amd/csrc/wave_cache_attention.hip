// Exact attention of one token per sequence over a prefix that the batch shares and over the sequence's own rows, both the
// same stream (wave_attend.h).
#include <type_traits>

#include "wave_attend.h"

namespace wave {

namespace {

// Own rows: one workgroup per piece, all G heads of its unit as columns; the four waves take every fourth step.
template <typename T, int D>
__device__ __forceinline__ void own_rows(const AttendArgs& a, int block, JoinShared& js, const Areas areas) {
  typedef Step<T, D> S;
  const int w = block / a.Hkv, h = block % a.Hkv;
  const Piece p = find_piece(a.lengths, a.B, a.capacity, a.target, a.few, w);
  if (p.b == a.B) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int rows = ((p.length + p.count - 1) / p.count + 31) / 32 * 32;
  const int start = (w - p.first) * rows, end = min(p.length, start + rows);
  if (w == p.first && h == 0 && threadIdx.x == 0) a.info[p.b] = make_int2(w, p.count);
  const size_t unit = (size_t)p.b * a.Hkv + h, row = D * sizeof(T);
  const int head = h * a.G + min(c, a.G - 1);  // (columns behind the G heads repeat the last one)
  const size_t bh = (size_t)p.b * a.Hq + head;
  const typename S::Q q = S::load_q(a.q + bh * row, g);
  State<T, D> st;
  st.init();
  float* z = a.weights_out && c < a.G ? a.z + bh * a.zrow : nullptr;
  auto leave = [&](int r, const f32x4& x) {
    if (z) *reinterpret_cast<f32x4*>(z + r) = x;
  };
  stream_rows<T, D, true>(a.k + unit * a.capacity * row, a.v + unit * a.capacity * row, start + wave * S::KEYS, 4 * S::KEYS, end,
                          a.scale, q, st, leave, areas.of(wave), lane);
  const size_t at = ((size_t)h * a.pieces + w) * a.G;
  join_waves<T, D>(st, a.G, js, areas, wave, g, c, a.ml + at, a.acc + at * D);
}

// Prefix with the own rows' stream: one workgroup per (KV head, range of prefix rows, tile of 16 of the B * G query rows).
// Up to 16 query rows, a matter of memory (eight KV heads, 65536 rows for 16 query rows each: 45 us and 5 for the join, 5.5 TB/s),
// and fp32: its products bind it from about 64 query rows on (32768 rows, eight KV heads: 47 us for 16, 85 for 32, 192 .. 231 for
// 128: at best 91 TFLOP/s of the 134 that a large fp32 product reaches), so rows shared in LDS could only help between, where
// the second tile's rows come from the caches.
template <typename T, int D>
__device__ __forceinline__ void prefix_rows(const AttendArgs& a, int block, JoinShared& js, const Areas areas) {
  typedef Step<T, D> S;
  const int hs = block % (a.Hkv * a.splits), tile = block / (a.Hkv * a.splits);
  const int h = hs % a.Hkv, split = hs / a.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int M = a.B * a.G, m0 = tile * 16;
  const size_t row = D * sizeof(T);
  const int m = min(m0 + c, M - 1), b = m / a.G;
  const typename S::Q q = S::load_q(a.q + ((size_t)b * a.Hq + h * a.G + (m - b * a.G)) * row, g);
  State<T, D> st;
  st.init();
  const int start = split * a.prefix_rows, end = min(a.P, start + a.prefix_rows);
  stream_rows<T, D, false>(a.prefix_k + (size_t)h * a.P * row, a.prefix_v + (size_t)h * a.P * row, start + wave * S::KEYS,
                           4 * S::KEYS, end, a.scale, q, st, [](int, const f32x4&) {}, areas.of(wave), lane);
  const size_t at = ((size_t)split * a.Hkv + h) * M + m0;  // by KV head and query row
  join_waves<T, D>(st, min(16, M - m0), js, areas, wave, g, c, a.pml + at, a.pacc + at * D);
}

// Prefix with more query rows than a tile (bf16): four waves with MQ tiles of columns each go through the same rows, which
// they share in LDS.  A step is 32 rows; a ring of four steps holds the one that is worked on and the next, while two more
// are on their way.  The values' operand comes transposed (ds_read_b64_tr_b16: sixteen lanes read four rows of sixteen
// channels, and each gets the four values of its channel; a read takes two neighbouring chunks of eight rows).
// The scores of the next step are formed beside the softmax of this one, so that matrix and vector work of a wave do not
// wait for each other.  Measured (64K rows, 448 query rows on each of four KV heads, 60 GFLOP): 153 us back to back.  The card
// lowers its clock to 1.7 .. 1.8 GHz under this mixture (2.5 GHz in the own rows; products of random numbers alone: 2.0
// PFLOP/s instead of 2.4), and the time follows the work itself: of 144 us on a cooler card, sixteen products fewer a step are 23, no
// loads into LDS 14, no exponentials 7, no LDS reads of the keys or of the values 4 each, while other orders of the same
// instructions, a third fewer vector instructions, or two workgroups a CU instead of one change nothing.  (448 columns are three and
// a half tiles of 128: two of the last tile's waves have none and only fetch, an eighth of the waves in all.)
template <int D>
struct SharedStep {
  static constexpr int ROWS = 32, ROW = D * 2, CHUNKS = ROW / 16, HALF = ROWS * ROW, BYTES = 2 * HALF;  // keys, then values
  static constexpr int FILLS = HALF / 1024 / 4;  // wave-wide loads of each wave, for each of the two
  static __device__ __forceinline__ int fv(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
  // a wave's part of the rows r0 .. of K and V
  static __device__ __forceinline__ void fill(char* lds, const char* K, const char* V, int r0, int last, int wave, int lane) {
    rows_to_lds<ROW, FILLS, false>(lds, step_rows<ROW>(K, r0, last), wave * FILLS, lane, key_place<ROW>);
    rows_to_lds<ROW, FILLS, false>(lds + HALF, step_rows<ROW>(V, r0, last), wave * FILLS, lane, fv);
  }
};

template <int D, int MQ>
__device__ __forceinline__ void prefix_shared(const AttendArgs& a, int block, char* ring0, char* ring1, char* ring2, char* ring3) {
  typedef Step<bf16_t, D> S;
  typedef SharedStep<D> L;
  constexpr int BLOCKS = D / 16;  // of sixteen channels
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const int hs = block % (a.Hkv * a.splits), tile = block / (a.Hkv * a.splits);
  const int h = hs % a.Hkv, split = hs / a.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
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
  int ka[S::KC], va[BLOCKS];  // this lane's places in a step, of row c and of row g * 4 + c / 4
#pragma unroll
  for (int x = 0; x < S::KC; ++x) ka[x] = c * L::ROW + ((x * 4 + g) ^ key_place<L::ROW>(c)) * 16;
#pragma unroll
  for (int x = 0; x < BLOCKS; ++x) {
    const int r = g * 4 + (c >> 2);
    va[x] = L::HALF + r * L::ROW + ((x * 2 + ((c & 3) >> 1)) ^ L::fv(r)) * 16 + (c & 1) * 8;
  }
  auto read_k = [&](const char* lds) {
    typename S::K k;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int x = 0; x < S::KC; ++x) k.x[t][x] = load16(lds + ka[x] + t * 16 * L::ROW);
    return k;
  };
  auto read_v = [&](const char* lds) {
    typename S::Vt v;
#pragma unroll
    for (int x = 0; x < BLOCKS; ++x) {
      uint2 u[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        u[t] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((
                                             __attribute__((address_space(3))) s16x4*)(lds + va[x] + t * 16 * L::ROW)));
      v.x[x] = __builtin_bit_cast(bf16x8, make_uint4(u[0].x, u[0].y, u[1].x, u[1].y));
    }
    return v;
  };
  // `newest` steps' loads of this wave may be on their way still; then all waves are behind the step before
  auto arrive = [&](auto newest) {
    constexpr int N = decltype(newest)::value * 2 * L::FILLS;
    wait_for_loads<N>();
    __syncthreads();
  };
  L::fill(ring0, K, V, start, last, wave, lane);
  L::fill(ring1, K, V, start + 32, last, wave, lane);
  L::fill(ring2, K, V, start + 64, last, wave, lane);
  arrive(std::integral_constant<int, 2>());
  float s[MQ][S::NS];
  {
    const typename S::K k = read_k(ring0);
#pragma unroll
    for (int t = 0; t < MQ; ++t) S::scores(k, q[t], s[t]);
  }
  const int full = (end - start) / 32;
  const bool idle = m0 >= M;  // (a wave of the last tile may have no column at all: it only fetches)
  // step n: `now` holds it, `next` the step behind it, `free` the step before it
  auto step = [&](int n, const char* now, const char* next, char* free) {
    arrive(std::integral_constant<int, 1>());
    L::fill(free, K, V, start + (n + 3) * 32, last, wave, lane);
    if (idle) return;
#pragma unroll
    for (int t = 0; t < MQ; ++t) st[t].follow(s[t], a.scale);
    const typename S::K k = read_k(next);
    const typename S::Vt v = read_v(now);
    float p[MQ][S::NS];
    st[0].weights(s[0], p[0], a.scale);
    if (MQ > 1) st[MQ - 1].weights(s[MQ - 1], p[MQ - 1], a.scale);
#pragma unroll
    for (int t = 0; t < MQ; ++t) S::scores(k, q[t], s[t]);
#pragma unroll
    for (int t = 0; t < MQ; ++t) S::accumulate(v, p[t], st[t].o);
  };
  for (int n = 0;; n += 4) {
    if (n >= full) break;
    step(n, ring0, ring1, ring3);
    if (n + 1 >= full) break;
    step(n + 1, ring1, ring2, ring0);
    if (n + 2 >= full) break;
    step(n + 2, ring2, ring3, ring1);
    if (n + 3 >= full) break;
    step(n + 3, ring3, ring0, ring2);
  }
  if (start + full * 32 < end) {
    // Rows behind the end are the last row again.  Their weight is zero, and zero times a value that is no number must not
    // show, so the values go too.
    const int k0 = start + full * 32;
    const char* now = (full & 3) == 0 ? ring0 : (full & 3) == 1 ? ring1 : (full & 3) == 2 ? ring2 : ring3;
    typename S::Vt v = read_v(now);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k0 + S::key(g, j) > last) {
#pragma unroll
        for (int x = 0; x < BLOCKS; ++x) v.x[x][j] = (__bf16)0.f;
#pragma unroll
        for (int t = 0; t < MQ; ++t) s[t][j] = neg_inf();
      }
#pragma unroll
    for (int t = 0; t < MQ; ++t) {
      st[t].weigh(s[t], a.scale);
      S::accumulate(v, s[t], st[t].o);
    }
  }
  wait_for_loads<0>();  // none may write LDS behind the end of the workgroup
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
// Prefix and own rows in one launch: one is bound by the matrix units as soon as it has many query rows, the other by
// memory.  256 workgroups of the one (all, if there are fewer) and as many of the other alternate, so that a CU has one of
// each; what is left of the longer kind follows.  (64K prefix rows for 448 query rows per KV head with 160K own rows: 174 us, 153
// and 59 alone.  All of the prefix first 180 us; mixed in proportion, which leaves single prefix workgroups for the end, 206.)
// Tiles of one prefix range are a multiple of 8 workgroups apart, on one XCD, wherever Hkv * splits is one.
// ----------------------------------------------------------------------------
struct Role {
  int block;
  bool prefix, any;
};
__device__ __forceinline__ Role role_of(const AttendArgs& a) {
  const int group = blockIdx.x / a.turn, within = blockIdx.x % a.turn;
  Role r;
  r.prefix = !(group & 1) && (group >> 1) < a.prefix_turns;
  const int before = min((group + 1) >> 1, a.prefix_turns);
  r.block = (r.prefix ? group >> 1 : group - before) * a.turn + within;
  r.any = r.block < (r.prefix ? a.prefix_blocks : a.own_blocks);
  return r;
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(const AttendArgs a) {
  __shared__ JoinShared js;
  __shared__ __attribute__((aligned(16))) char lds[4][16 * (D + 4) * 4];
  const Areas areas{lds[0], lds[1], lds[2], lds[3]};
  const Role r = role_of(a);
  if (!r.any) return;
  if (r.prefix)
    prefix_rows<T, D>(a, r.block, js, areas);
  else
    own_rows<T, D>(a, r.block, js, areas);
}

template <int D, int MQ>
__global__ __launch_bounds__(256, 2) void attend_shared_kernel(const AttendArgs a) {
  typedef SharedStep<D> L;
  constexpr int AREA = L::BYTES > 16 * (D + 4) * 4 ? L::BYTES : 16 * (D + 4) * 4;
  __shared__ JoinShared js;
  __shared__ __attribute__((aligned(1024))) char ring0[AREA], ring1[AREA], ring2[AREA], ring3[AREA];
  const Role r = role_of(a);
  if (!r.any) return;
  if (r.prefix) {
    prefix_shared<D, MQ>(a, r.block, ring0, ring1, ring2, ring3);
  } else {
    const Areas areas{ring0, ring1, ring2, ring3};
    own_rows<bf16_t, D>(a, r.block, js, areas);
  }
}

// ----------------------------------------------------------------------------
// Merge.  The first workgroups join the heads' partial results: one head each, or four, a wave each, where there are many
// heads with few (256 sequences of 300 rows, 8192 heads: 8 us instead of 16; 4096 heads with nine each 9 instead of 13).  With weights, the others have weight_rows(G) rows
// of a unit each: they form the G heads' normalisers from the partial (m, l) again, which is less than waiting for them, and add up
// the softmax weights.
// ----------------------------------------------------------------------------
struct HeadParts {
  const float2 *ml, *pml;
  int splits, own, stride, pstride;  // partials of the prefix and of own pieces, and what lies between them
  __device__ __forceinline__ float2 at(int i) const {
    return i < splits ? pml[(size_t)i * pstride] : ml[(size_t)(i - splits) * stride];
  }
  template <int D>
  __device__ __forceinline__ const float* sum(const AttendArgs& a, int i, int b, int h, int gq, int first) const {
    return i < splits ? a.pacc + ((size_t)i * pstride + (size_t)h * a.B * a.G + (size_t)b * a.G + gq) * D
                      : a.acc + (((size_t)h * a.pieces + first + i - splits) * a.G + gq) * D;
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
  return make_float2(top, wave_add_f(l));
}

// ----------------------------------------------------------------------------
// Short caches: one launch, a workgroup of eight waves per unit, which go through the prefix and the unit's rows and join in
// LDS.  There the products of the own rows stay too, for the weights.
// ----------------------------------------------------------------------------
constexpr int SHORT_WAVES = 8, SHORT_THREADS = SHORT_WAVES * 64;
// rows that the waves take in one step each, and room for two
constexpr int short_step(int dtype) { return SHORT_WAVES * (dtype == WAVE_BF16 ? Step<bf16_t, 64>::KEYS : Step<float, 64>::KEYS); }

template <typename T, int D, int G>
__global__ __launch_bounds__(SHORT_THREADS) void attend_short_kernel(const AttendArgs a) {
  typedef Step<T, D> S;
  constexpr int PITCH = D + 4, ZROW = 2 * SHORT_WAVES * S::KEYS + 4;
  __shared__ __attribute__((aligned(16))) char lds[SHORT_WAVES][16 * PITCH * 4];
  __shared__ __attribute__((aligned(16))) float products[G][ZROW];
  __shared__ float sm[SHORT_WAVES][16], sl[SHORT_WAVES][16];
  const int unit = blockIdx.x, b = unit / a.Hkv, h = unit % a.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const size_t row = D * sizeof(T);
  const int len = cache_length(a.lengths, b, a.capacity), head = b * a.Hq + h * G;
  const typename S::Q q = S::load_q(a.q + (size_t)(head + min(c, G - 1)) * row, g);
  State<T, D> st;
  st.init();
  if (a.P > 0)
    stream_rows<T, D, false>(a.prefix_k + (size_t)h * a.P * row, a.prefix_v + (size_t)h * a.P * row, wave * S::KEYS,
                             SHORT_WAVES * S::KEYS, a.P, a.scale, q, st, [](int, const f32x4&) {}, lds[wave], lane);
  // the wave that the prefix leaves first takes the first own rows
  const int turn = (wave + SHORT_WAVES - (a.P + S::KEYS - 1) / S::KEYS % SHORT_WAVES) % SHORT_WAVES;
  const bool keep = a.weights_out && c < G;
  stream_rows<T, D, true>(a.k + (size_t)unit * a.capacity * row, a.v + (size_t)unit * a.capacity * row, turn * S::KEYS,
                          SHORT_WAVES * S::KEYS, len, a.scale, q, st,
                          [&](int r, const f32x4& x) { if (keep) *reinterpret_cast<f32x4*>(&products[c][r]) = x; },
                          lds[wave], lane);
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    sm[wave][c] = st.m;
    sl[wave][c] = l;
  }
  if (c < G) {
    float* at = reinterpret_cast<float*>(lds[wave]) + c * PITCH;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < S::ACC; x += 4)
        *reinterpret_cast<f32x4*>(at + S::channel(g, x, i)) = f32x4{st.o[x][i], st.o[x + 1][i], st.o[x + 2][i], st.o[x + 3][i]};
  }
  __syncthreads();
  // a head's reference and sum; none of its scores a number above -infinity: (0, 1), and no output
  auto normal = [&](int col, float& m, float& sum) {
    m = sm[0][col];
#pragma unroll
    for (int w = 1; w < SHORT_WAVES; ++w) m = fmaxf(m, sm[w][col]);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < SHORT_WAVES; ++w) sum += (sm[w][col] == neg_inf() ? 0.f : exp2f(sm[w][col] - m)) * sl[w][col];
    return !(m == neg_inf() && sum == 0.f);
  };
  for (int i = threadIdx.x; i < G * D; i += SHORT_THREADS) {
    const int col = i / D, ch = i % D;
    float m, sum, o = 0.f;
    const bool any = normal(col, m, sum);
#pragma unroll
    for (int w = 0; w < SHORT_WAVES; ++w)
      o += (sm[w][col] == neg_inf() ? 0.f : exp2f(sm[w][col] - m)) * reinterpret_cast<const float*>(lds[w])[col * PITCH + ch];
    a.out[(size_t)(head + col) * D + ch] = any ? o / sum : 0.f;
    if (ch == 0) a.lse[head + col] = any ? (m + log2f(sum)) * kLn2 : neg_inf();
  }
  if (!a.weights_out) return;
  float m[G], f[G];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    float sum;
    const bool any = normal(j, m[j], sum);
    m[j] = any ? m[j] : 0.f;
    f[j] = any ? 1.f / sum : 1.f;
  }
  const size_t base = (size_t)unit * a.capacity;
  for (int j = threadIdx.x; j < len; j += SHORT_THREADS) {
    float w = a.decay > 0.f ? a.decay * a.weights[base + j] : 0.f;
#pragma unroll
    for (int x = 0; x < G; ++x) w += __builtin_amdgcn_exp2f(fmaf(products[x][j], a.scale, -m[x])) * f[x];
    a.weights_out[base + j] = w;
  }
}

// rows of a unit per workgroup, by the registers that the heads' products take
constexpr int weight_rows(int G) { return G <= 4 ? 2048 : 1024; }

// The sequence's pieces as the launch before left them: the first one, and how many.  (Both loads side by side: a sequence without
// rows left nothing, and what is read then is not used.)
struct OwnPieces {
  int first, count, length;
};
__device__ __forceinline__ OwnPieces own_pieces(const AttendArgs& a, int b) {
  const int length = a.lengths[b];
  const int2 p = a.info[b];
  OwnPieces o;
  o.length = min(max(length, 0), a.capacity);
  o.first = o.length > 0 ? p.x : 0;
  o.count = o.length > 0 ? p.y : 0;
  return o;
}

template <int D, int G>
__global__ __launch_bounds__(256) void join_kernel(const AttendArgs a) {
  constexpr int WEIGHT_ROWS = weight_rows(G);
  const int heads = a.B * a.Hq, tid = threadIdx.x, wave = tid >> 6;
  __shared__ float2 norm[G];
  if (a.head_waves && (int)blockIdx.x < a.head_blocks) {
    const int bh = blockIdx.x * 4 + wave;
    if (bh >= heads) return;
    const int b = bh / a.Hq, hq = bh % a.Hq, h = hq / G, gq = hq % G;
    const OwnPieces own = own_pieces(a, b);
    const HeadParts p = head_parts(a, b, h, gq, own.first, own.count);
    const float2 n = normaliser(p);
    constexpr int LANES = D / 4, GROUPS = 64 / LANES;
    const int lane = tid % LANES, group = (tid & 63) / LANES;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = group; i < p.splits + own.count; i += GROUPS) {
      const float2 x = p.at(i);
      const float f = x.x == neg_inf() ? 0.f : exp2f(x.x - n.x);
      sum += f * *reinterpret_cast<const f32x4*>(p.sum<D>(a, i, b, h, gq, own.first) + lane * 4);
    }
#pragma unroll
    for (int off = LANES; off < 64; off *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], off);
    if (group == 0) {
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = n.x == neg_inf() ? 0.f : sum[e] / n.y;
      *reinterpret_cast<f32x4_of_floats*>(a.out + (size_t)bh * D + lane * 4) = o;
    }
    if ((tid & 63) == 0) a.lse[bh] = n.x == neg_inf() ? neg_inf() : (n.x + log2f(n.y)) * kLn2;
    return;
  }
  if ((int)blockIdx.x < a.head_blocks) {
    __shared__ float part[256 / (D / 4)][D];
    const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, h = hq / G, gq = hq % G;
    const OwnPieces own = own_pieces(a, b);
    const HeadParts p = head_parts(a, b, h, gq, own.first, own.count);
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    const int lane = tid % LANES, group = tid / LANES, parts = p.splits + own.count;
    // a thread's first partial results are on their way while the normaliser is formed, and JB of them together (one KV head
    // with 512 of them: 35 us one by one, 20 so)
    constexpr int JB = 4;
    float x[JB];
    f32x4 v[JB], sum = {0.f, 0.f, 0.f, 0.f};
    auto load = [&](int i0) {
#pragma unroll
      for (int e = 0; e < JB; ++e) {
        const int i = min(i0 + e * GROUPS, parts - 1);
        x[e] = p.at(i).x;
        v[e] = *reinterpret_cast<const f32x4*>(p.sum<D>(a, i, b, h, gq, own.first) + lane * 4);
      }
    };
    if (group < parts) load(group);
    const float2 n = normaliser(p);
    for (int i = group; i < parts;) {
#pragma unroll
      for (int e = 0; e < JB; ++e)
        if (i + e * GROUPS < parts) sum += (x[e] == neg_inf() ? 0.f : exp2f(x[e] - n.x)) * v[e];
      i += JB * GROUPS;
      if (i < parts) load(i);
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
  const int at = blockIdx.x - a.head_blocks, unit = at / chunks, r0 = at % chunks * WEIGHT_ROWS;
  const int b = unit / a.Hkv, h = unit % a.Hkv;
  const OwnPieces own = own_pieces(a, b);
  const int len = own.length;
  if (r0 >= len) return;
  // the products and the old weights are on their way while the normalisers are formed
  constexpr int PER = WEIGHT_ROWS / 256;
  const size_t base = (size_t)unit * a.capacity;
  const float* z = a.z + ((size_t)b * a.Hq + h * G) * a.zrow;
  float zz[G][PER], w[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = min(r0 + i * 256 + tid, len - 1);
#pragma unroll
    for (int gq = 0; gq < G; ++gq) zz[gq][i] = z[(size_t)gq * a.zrow + j];
    w[i] = a.decay > 0.f ? a.decay * a.weights[base + j] : 0.f;
  }
  for (int gq = wave; gq < G; gq += 4) {
    const float2 n = normaliser(head_parts(a, b, h, gq, own.first, own.count));
    if ((tid & 63) == 0) norm[gq] = make_float2(n.x == neg_inf() ? 0.f : n.x, n.x == neg_inf() ? 1.f : 1.f / n.y);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = r0 + i * 256 + tid;
#pragma unroll
    for (int gq = 0; gq < G; ++gq)
      w[i] += __builtin_amdgcn_exp2f(fmaf(zz[gq][i], a.scale, -norm[gq].x)) * norm[gq].y;
    if (j < len) a.weights_out[base + j] = w[i];
  }
}

template <int D>
wave_status join_td(AttendArgs a, hipStream_t st) {
  // (on the mean; fewer than 1024 heads leave CUs without work)
  a.head_waves = a.B * a.Hq >= 1024 && a.splits + a.pieces / a.B <= 16;
  a.head_blocks = a.head_waves ? (a.B * a.Hq + 3) / 4 : a.B * a.Hq;
  switch (a.G) {
#define WAVE_G(n)                                                                                              \
  case n: {                                                                                                    \
    const int chunks = (a.capacity + weight_rows(n) - 1) / weight_rows(n);                                     \
    const unsigned grid = a.head_blocks + (a.weights_out ? a.B * a.Hkv * chunks : 0);                             \
    WAVE_LAUNCH("cache_join", (join_kernel<D, n>), grid, 256, 0, st, a);                                       \
    break;                                                                                                     \
  }
    WAVE_G(1) WAVE_G(2) WAVE_G(3) WAVE_G(4) WAVE_G(5) WAVE_G(6) WAVE_G(7) WAVE_G(8)
#undef WAVE_G
    default: return WAVE_ERR_SHAPE;
  }
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

template <typename T, int D>
wave_status attend_td(AttendArgs a, const CacheAttendGeom& g, hipStream_t st) {
  if (g.one_launch) {
    switch (a.G) {
#define WAVE_G(n) \
  case n: WAVE_LAUNCH("cache_attend", (attend_short_kernel<T, D, n>), a.B * a.Hkv, SHORT_THREADS, 0, st, a); break;
      WAVE_G(1) WAVE_G(2) WAVE_G(3) WAVE_G(4) WAVE_G(5) WAVE_G(6) WAVE_G(7) WAVE_G(8)
#undef WAVE_G
      default: return WAVE_ERR_SHAPE;
    }
    return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
  }
  a.prefix_blocks = a.P > 0 ? a.Hkv * a.splits * g.mtiles : 0;
  a.own_blocks = a.Hkv * g.pieces;
  a.turn = a.prefix_blocks < 256 ? (a.prefix_blocks + 7) / 8 * 8 : 256;
  if (a.turn == 0) a.turn = 256;
  a.prefix_turns = (a.prefix_blocks + a.turn - 1) / a.turn;
  const int own_turns = (a.own_blocks + a.turn - 1) / a.turn;
  const unsigned blocks = own_turns >= a.prefix_turns ? a.turn * (a.prefix_turns - 1 + own_turns) + a.own_blocks - a.turn * (own_turns - 1)
                                                      : a.turn * (2 * a.prefix_turns - 2) + a.prefix_blocks - a.turn * (a.prefix_turns - 1);
  bool shared = false;
  if constexpr (sizeof(T) == 2) {
    shared = a.P > 0 && g.mtile > 16;
    if (shared) {
      if (g.mtile == 64)
        WAVE_LAUNCH("cache_attend", (attend_shared_kernel<D, 1>), blocks, 256, 0, st, a);
      else
        WAVE_LAUNCH("cache_attend", (attend_shared_kernel<D, 2>), blocks, 256, 0, st, a);
    }
  }
  if (!shared) WAVE_LAUNCH("cache_attend", (attend_rows_kernel<T, D>), blocks, 256, 0, st, a);
  return join_td<D>(a, st);
}

}  // namespace

wave_status launch_attend_join(const AttendArgs& a, int d, hipStream_t st) {
  return d == 128 ? join_td<128>(a, st) : join_td<64>(a, st);
}

// How a prefix is cut where `mtile` of its M query rows go together: workgroups side by side, and the ranges aimed at.
struct PrefixCut {
  int mtiles, want;
};
static PrefixCut prefix_cut(const wave_cache& c, int M, int mtile) {
  const int mtiles = (M + mtile - 1) / mtile;
  // One workgroup a CU where it is bound by the matrix units (its partial results cost more than a second one gains: 60 us
  // instead of 68 for 32K rows, 128 query rows and 500 own rows), two where it is bound by memory (100K rows, 64 query
  // rows: 88 us instead of 93).  No more than 256 ranges, each of which every head's joining reads (one KV head, 65536 rows:
  // 28 us with 512, 20).
  const int aim = mtile == 128 && c.d == 128 ? 256 : 512;
  const int even = aim / (c.Hkv * mtiles) > 1 ? aim / (c.Hkv * mtiles) : 1;
  return PrefixCut{mtiles, even < 256 ? even : 256};
}
// Pieces of own rows aimed at, as many as are resident: two a CU, four at d = 64 (or half of them, see find_piece).  Four, and never
// half of them, beside a prefix that its products bind: there many own rows gain, and few lose less (32K prefix rows for 128 query
// rows on eight KV heads with 100K own rows: 108 us, without this rule 117; with 16K 60 and 59; 64K for 448 on four with 160K: 161 and
// 159; d = 64, 50K for 192 and 80K: 42 both ways).
static bool binds(const wave_cache& c, int M, const PrefixCut& cut, long long splits) {
  return M > 16 && c.Hkv * splits * cut.mtiles >= 128;
}
static int pieces_aimed_at(const wave_cache& c, bool beside) {
  const int per_cu = beside || c.d == 64 ? 4 : 2;
  return per_cu * 256 / c.Hkv > 1 ? per_cu * 256 / c.Hkv : 1;
}
static int pieces_at_most(const wave_cache& c, int target) {
  const long long most = (long long)c.B * (((long long)c.capacity + 127) / 128);
  const long long cut = (long long)target + (cuts_fit(c.B, target) ? 0 : c.B);
  return (int)(cut < most ? cut : most);
}

CacheAttendGeom cache_attend_geometry(const wave_cache& c, int Hq, int P, bool accumulate) {
  CacheAttendGeom g{};
  const int G = Hq / c.Hkv;
  // One launch where a wave has one step to do, or two and the units do not fill the CUs twice over (62 sequences x 8 units of
  // 280 rows: 26 us, 23 in pieces) or reading all lengths to find a piece takes longer (2000 sequences x 2 of 165: 91 us, 162).
  // 64 rows for one sequence: 6.0 us instead of 8.3; 15 of 100 rows 7.2, 10.1; 22 of 200 behind 143 of a prefix 5.7, 10.6.
  // With four steps and few units it is slower: one sequence of 1000 rows 14.3 us instead of 10.2.
  const int steps = (int)(((long long)P + c.capacity + short_step(c.dtype) - 1) / short_step(c.dtype));
  g.one_launch = steps <= 1 || (steps <= 2 && (c.B * c.Hkv <= 256 || c.B > 512));
  const int M = c.B * G;
  // Two tiles of columns a wave share its reads of keys and values, and double what a workgroup has to do.  That pays where there
  // is work for most CUs at the smallest ranges (d = 128, 448 query rows on four KV heads: behind 500 rows 16.9 us, with one tile
  // 14.0; behind 2000 19.6 and 23.8; behind 8000 32 both ways); at d = 64, where a wave has half as much to read, not before that
  // grows far beyond, and then hardly (448 behind 8000 rows 24.0 us, 21.5; 800 behind 16000 45.4 and 43.3; 128 on eight KV heads behind
  // 64K 56.8 and 57.2).
  const long long tiles128 = (long long)c.Hkv * ((M + 127) / 128) * (((long long)P + 127) / 128);
  const bool wide = M > 64 && tiles128 >= (c.d == 128 ? 192 : 4096);
  const int narrow = M <= 16 || c.dtype == WAVE_F32 ? 16 : 64, widest = narrow == 64 && M > 64 ? 128 : narrow;
  g.mtile = wide ? widest : narrow;
  const PrefixCut cut = prefix_cut(c, M, g.mtile);
  g.mtiles = cut.mtiles;
  if (P > 0) {
    const long long rows = ((long long)P + cut.want - 1) / cut.want;
    g.prefix_rows = (int)((rows + 127) / 128 * 128);
    g.splits = (int)(((long long)P + g.prefix_rows - 1) / g.prefix_rows);
  }
  const bool beside = P > 0 && binds(c, M, cut, g.splits);
  g.target = pieces_aimed_at(c, beside);
  g.pieces = pieces_at_most(c, g.target);
  g.few = beside ? 0 : g.target / 2;
  // The workspace has room for every shorter prefix too, which may have more ranges than this one (they are whole steps of 128
  // rows), another tile of columns, and with it more pieces of own rows.
  int room_splits = 0, room_pieces = pieces_at_most(c, pieces_aimed_at(c, false));
  for (int mtile : {narrow, widest}) {
    if (P == 0) break;
    const PrefixCut x = prefix_cut(c, M, mtile);
    const int ranges = (int)(((long long)P + 127) / 128), splits = x.want < ranges ? x.want : ranges;
    if (splits > room_splits) room_splits = splits;
    const int pieces = pieces_at_most(c, pieces_aimed_at(c, binds(c, M, x, splits)));
    if (pieces > room_pieces) room_pieces = pieces;
  }
  g.zrow = (c.capacity + 31) / 32 * 32;  // whole steps
  size_t o = 0;
  g.off_info = o;  o = align_up(o + sizeof(int32_t) * 2 * (size_t)c.B);
  g.off_z = o;     o = align_up(o + (accumulate ? sizeof(float) * (size_t)c.B * Hq * g.zrow : 0));
  g.off_ml = o;    o = align_up(o + sizeof(float) * 2 * (size_t)Hq * room_pieces);
  g.off_acc = o;   o = align_up(o + sizeof(float) * c.d * (size_t)Hq * room_pieces);
  g.off_pml = o;   o = align_up(o + sizeof(float) * 2 * (size_t)c.B * Hq * room_splits);
  g.off_pacc = o;  o = align_up(o + sizeof(float) * c.d * (size_t)c.B * Hq * room_splits);
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
  a.info = reinterpret_cast<int2*>(w + g.off_info);
  a.B = c.B;
  a.Hq = Hq;
  a.Hkv = c.Hkv;
  a.G = Hq / c.Hkv;
  a.capacity = c.capacity;
  a.P = P;
  a.target = g.target;
  a.few = g.few;
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
