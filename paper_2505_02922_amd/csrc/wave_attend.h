// One token's attention over a stream of key and value rows: what the kernels that do it share.
//
// A wave holds a tile of query rows as the columns of its matrix products and goes through key and value rows with a
// running maximum and sum of the softmax.  What a lane holds of S = K Q^T is, with the contraction index permuted alike on
// both sides, already the operand of O^T += V^T P^T: no value crosses a lane between the two products.
#pragma once

#include "wave_common.h"

namespace wave {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
// four floats of a caller's array of floats, which need not lie on 16 bytes (one store all the same)
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_of_floats;

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

// Where key rows have their chunks in LDS: the sixteen lanes of an operand read, which take one chunk of sixteen rows, hit
// all banks.
template <int ROW>
__device__ __forceinline__ constexpr int key_place(int r) {
  return ROW >= 256 ? r & 15 : (r >> 1) & 7;
}
// A step of a stream: its first row and how many rows there are behind that one, at least; rows behind the last are the last
// again.  A lane's address is a base that the wave shares and 32 bits of its own.
struct StepRows {
  const char* base;
  int rest;
};
template <int ROW>
__device__ __forceinline__ StepRows step_rows(const char* base, int k0, int last) {
  const int row = min(k0, last);
  return StepRows{base + (size_t)row * ROW, last - row};
}
template <int ROW>
__device__ __forceinline__ const char* row_at(const StepRows& s, int r, int byte) {
  return s.base + (uint32_t)(min(r, s.rest) * ROW + byte);
}
// Pieces first .. first + COUNT - 1 of 1 KiB of a step's rows into LDS, one load instruction of a wave each, in the order of
// its lanes: chunk x (16 bytes) of row r lies at x ^ place(r).  ONCE: nobody else reads these rows, they pass by the caches
// (policy 2).
template <int ROW, int COUNT, bool ONCE, typename Place>
__device__ __forceinline__ void rows_to_lds(char* lds, const StepRows& s, int first, int lane, Place&& place) {
  constexpr int CHUNKS = ROW / 16;
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    const int r = (first + i) * (1024 / ROW) + lane / CHUNKS;
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)row_at<ROW>(s, r, (lane % CHUNKS ^ place(r)) * 16),
        (__attribute__((address_space(3))) void*)(lds + (first + i) * 1024), 16, 0, ONCE ? 2 : 0);
  }
}
__device__ __forceinline__ void wait_for_reads() { __builtin_amdgcn_s_waitcnt(0xc07f); }  // of LDS (lgkmcnt 0)
template <int N>
__device__ __forceinline__ void wait_for_loads() {  // until at most the newest N are on their way (vmcnt)
  static_assert(N < 16, "");
  __builtin_amdgcn_s_waitcnt(0x0f70 | N);
}

// bf16: v_mfma_f32_16x16x32_bf16.  S has two tiles of 16 keys; a lane has the keys t * 16 + g * 4 + i of its column.  The
// contraction of the second product takes them in the order t * 4 + i, so a lane reads CH neighbouring channels of those
// eight value rows (16 lanes: a whole row) and pairs up the rows of each channel with v_perm.
template <int D>
struct Step<bf16_t, D> {
  static constexpr int KEYS = 32, NS = 8, KC = D / 32, CH = D / 16, ACC = CH, VLOADS = 8, ROW = D * 2, KLOADS = KEYS * ROW / 1024;
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
  // from a step's key rows in LDS
  static __device__ __forceinline__ K read_k(const char* lds, int g, int c) {
    K k;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < KC; ++s)
        k.x[t][s] = load16(lds + (t * 16 + c) * (D * 2) + ((s * 4 + g) ^ key_place<D * 2>(c)) * 16);
    return k;
  }
  template <bool ONCE>
  static __device__ __forceinline__ V load_v(const StepRows& rows, int g, int c) {
    V v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* at = row_at<ROW>(rows, key(g, j), c * (CH * 2));
      if constexpr (CH == 8) {
        const uint4 u = ONCE ? load16_stream(at) : load16(at);
        v.x[j][0] = u.x; v.x[j][1] = u.y; v.x[j][2] = u.z; v.x[j][3] = u.w;
      } else {
        const uint2 u = ONCE ? load8_stream(at) : *reinterpret_cast<const uint2*>(at);
        v.x[j][0] = u.x; v.x[j][1] = u.y;
      }
    }
    return v;
  }
  // rows behind the last count as zero: their weight is zero, but the last row, which they repeat, may not be finite
  static __device__ __forceinline__ void mask_v(V& v, int rest, int g) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < CH / 2; ++u) v.x[j][u] = key(g, j) > rest ? 0u : v.x[j][u];
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
  // A weight's 24 bits as three bf16 numbers of eight, cut off from the top: their sum is the weight, so the product with the
  // values loses nothing.  (Two numbers, a third fewer products, keep 17 bits: with one heavy row behind a lighter one the output
  // is then off by 2^-18 of itself, sixty times what fp32 loses.)
  static __device__ __forceinline__ void accumulate(const Vt& v, const float (&p)[NS], f32x4 (&o)[ACC]) {
    uint32_t u[3][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x = p[2 * j], y = p[2 * j + 1];
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        u[n][j] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
        x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
      }
    }
    bf16x8 w[3];
#pragma unroll
    for (int n = 0; n < 3; ++n) w[n] = __builtin_bit_cast(bf16x8, make_uint4(u[n][0], u[n][1], u[n][2], u[n][3]));
#pragma unroll
    for (int n = 2; n >= 0; --n)
#pragma unroll
      for (int a = 0; a < CH; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.x[a], w[n], o[a], 0, 0, 0);
  }
};

// f32: v_mfma_f32_16x16x4_f32, one tile of 16 keys; a lane has the keys g * 4 + i.  Product number i of the second
// contraction takes key g * 4 + i from lane group g.
template <int D>
struct Step<float, D> {
  static constexpr int KEYS = 16, NS = 4, KC = D / 16, CV = D / 64, ACC = D / 16, VLOADS = 4 * CV, ROW = D * 4,
                       KLOADS = KEYS * ROW / 1024;
  struct Q { f32x4 x[KC]; };
  struct K { f32x4 x[KC]; };
  struct V { f32x4 x[4][CV]; };
  typedef V Vt;
  static __device__ __forceinline__ int key(int g, int s) { return g * 4 + s; }
  static __device__ __forceinline__ int channel(int g, int a, int i) { return (a >> 2) * 64 + (g * 4 + i) * 4 + (a & 3); }
  static __device__ __forceinline__ f32x4 load(const char* p) { return *reinterpret_cast<const f32x4*>(p); }
  static __device__ __forceinline__ f32x4 load_once(const char* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
  }

  static __device__ __forceinline__ Q load_q(const char* row, int g) {
    Q q;
#pragma unroll
    for (int s = 0; s < KC; ++s) q.x[s] = load(row + (s * 16 + g * 4) * 4);
    return q;
  }
  static __device__ __forceinline__ K read_k(const char* lds, int g, int c) {
    K k;
#pragma unroll
    for (int s = 0; s < KC; ++s) k.x[s] = load(lds + c * (D * 4) + ((s * 4 + g) ^ key_place<D * 4>(c)) * 16);
    return k;
  }
  template <bool ONCE>
  static __device__ __forceinline__ V load_v(const StepRows& rows, int g, int c) {
    V v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < CV; ++u) {
        const char* at = row_at<ROW>(rows, key(g, i), (u * 64 + c * 4) * 4);
        v.x[i][u] = ONCE ? load_once(at) : load(at);
      }
    return v;
  }
  static __device__ __forceinline__ void mask_v(V& v, int rest, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < CV; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) v.x[i][u][j] = key(g, i) > rest ? 0.f : v.x[i][u][j];
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
  // The reference follows the products s = q . k.  scale: log2(e) / sqrt(d).
  template <int N>
  __device__ __forceinline__ void follow(const float (&s)[N], float scale) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, s[i]);
    top *= scale;
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      raise(top);
    }
  }
  // to `top`, the same in all lanes of a column
  __device__ __forceinline__ void raise(float top) {
    const float grown = fmaxf(m, top);
    const float f = m == neg_inf() ? 0.f : exp2f(m - grown);
    m = grown;
    l *= f;
#pragma unroll
    for (int a = 0; a < S::ACC; ++a) o[a] *= f;
  }
  // p: the weights exp(s / sqrt(d)) over the reference.  The scale is applied inside the difference, which is then rounded
  // once.
  template <int N>
  __device__ __forceinline__ void weights(const float (&s)[N], float (&p)[N], float scale) {
    const float ref = m == neg_inf() ? 0.f : m;  // (every score -infinity so far)
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -ref));
#pragma unroll
    for (int i = 0; i < N; ++i) l += p[i];
  }
  template <int N>
  __device__ __forceinline__ void weigh(float (&s)[N], float scale) {
    follow(s, scale);
    weights(s, s, scale);
  }
};

// ----------------------------------------------------------------------------
// The stream of one wave: the rows k0, k0 + stride, .. below `end` against a tile of query columns.  leave: what happens to four
// neighbouring rows' products with a lane's column.  ONCE: nobody else reads these rows, so they pass by the caches.  lds: the
// wave's own place for a step's key rows.  Keys go through it because an operand has sixteen rows side by side, 64 bytes of
// each in a load: straight from memory every line is asked for twice, and must stay in the caches between.  A load of the
// values takes whole rows.  1.12 GB of own rows: 235 us with both straight from memory, 222 with the values passing by the
// caches, 209 us = 5.5 TB/s, what a plain read of 1 GiB reaches, so.  At d = 64, eight sequences of 3000 .. 65536 rows: 89 us, 92
// with the values in the caches.  (Values through LDS too: the same alone, but a tenth slower beside a long prefix, which
// needs LDS itself.)
// ----------------------------------------------------------------------------
template <typename T, int D, bool ONCE, typename Leave>
__device__ __forceinline__ void stream_rows(const char* K, const char* V, int k0, int stride, int end, float scale,
                                            const typename Step<T, D>::Q& q, State<T, D>& st, Leave&& leave, char* lds, int lane) {
  typedef Step<T, D> S;
  constexpr int ROW = S::ROW;
  const int last = end - 1, g = lane >> 4, c = lane & 15;
  if (k0 >= end) return;
  rows_to_lds<ROW, S::KLOADS, ONCE>(lds, step_rows<ROW>(K, k0, last), 0, lane, key_place<ROW>);
  __builtin_amdgcn_sched_barrier(0);
  typename S::V v = S::template load_v<ONCE>(step_rows<ROW>(V, k0, last), g, c);
  for (;;) {
    const int next = k0 + stride, rest = last - k0;
    __builtin_amdgcn_sched_barrier(0);
    wait_for_loads<S::VLOADS>();  // the keys are here; the values, asked for after them, may not be
    const typename S::K k = S::read_k(lds, g, c);
    wait_for_reads();  // they are in registers: their place is free
    __builtin_amdgcn_sched_barrier(0);
    // The next rows' loads go out as soon as there is room: a wave has loads in flight all the time.  They are made behind
    // the end too, since a wait behind a load that may not have been made waits for all of them.
    rows_to_lds<ROW, S::KLOADS, ONCE>(lds, step_rows<ROW>(K, next, last), 0, lane, key_place<ROW>);
    __builtin_amdgcn_sched_barrier(0);
    float s[S::NS];
    S::scores(k, q, s);
    if (rest < S::KEYS - 1) {
      S::mask_v(v, rest, g);
#pragma unroll
      for (int i = 0; i < S::NS; ++i) s[i] = S::key(g, i) > rest ? neg_inf() : s[i];
    }
#pragma unroll
    for (int i = 0; i < S::NS; i += 4) leave(k0 + S::key(g, i), f32x4{s[i], s[i + 1], s[i + 2], s[i + 3]});
    const typename S::Vt vt = S::transpose(v);
    __builtin_amdgcn_sched_barrier(0);
    v = S::template load_v<ONCE>(step_rows<ROW>(V, next, last), g, c);
    __builtin_amdgcn_sched_barrier(0);
    st.weigh(s, scale);
    S::accumulate(vt, s, st.o);
    if (next >= end) break;
    k0 = next;
  }
  wait_for_loads<0>();  // nothing may come into LDS behind this
}

// What a partial result leaves of its softmax.  A sum that is no number may have no reference, where every score was none:
// it has to survive the joining.
__device__ __forceinline__ float2 partial_ml(float m, float l) { return make_float2(l == l ? m : -neg_inf(), l); }

// The four waves' states of one tile of columns joined in LDS; columns below `cols` are left by all 256 threads as one
// partial result each: (m, l) at ml[col], the sum at acc + col * D.
// A place in LDS for each wave (no array: its elements have to stay known as LDS).
struct Areas {
  char *a, *b, *c, *d;
  __device__ __forceinline__ char* of(int wave) const { return wave == 0 ? a : wave == 1 ? b : wave == 2 ? c : d; }
};
struct JoinShared {
  float m[4][16], l[4][16];
};
template <typename T, int D>
__device__ __forceinline__ void join_waves(const State<T, D>& st, int cols, JoinShared& js, const Areas areas, int wave,
                                           int g, int c, float2* ml, float* acc) {
  typedef Step<T, D> S;
  constexpr int PITCH = D + 4;  // floats a column: a column's four groups and neighbouring columns lie on other banks
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    js.m[wave][c] = st.m;
    js.l[wave][c] = l;
  }
  if (c < cols) {
    float* at = reinterpret_cast<float*>(areas.of(wave)) + c * PITCH;
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
      sum += f * reinterpret_cast<const float*>(areas.of(w))[col * PITCH + ch];
      tot += f * js.l[w][col];
    }
    acc[(size_t)col * D + ch] = sum;
    if (ch == 0) ml[col] = partial_ml(m, tot);
  }
}

// ----------------------------------------------------------------------------
// How the own rows are cut: every sequence into equal pieces, by about the smallest number of rows (a multiple of 128) a piece
// with which there are no more than `target` of them per KV head, so that all workgroups run side by side and end together.
// With many sequences, where looking for it costs more than it gives, by the share of `target` pieces: then there may be one
// more for each sequence.  Piece w of a KV head belongs to the sequence whose pieces it falls among.  All lanes of a wave call
// this together.  (Pieces of one length for all sequences, six a CU: one sequence of 32000 rows 36 us, now 28; 16 of 1000 23
// and 19; 16 of 400 .. 4000 40 and 36; 62 of 280 33 and 25.)
// ----------------------------------------------------------------------------
__host__ __device__ constexpr bool cuts_fit(int B, int target) { return B <= 64 && 2 * B <= target; }
// Up to this many rows a piece (or for one sequence, which is cut evenly by any number), half as many pieces: less to start and
// to join (16 sequences x 8 units of 1000 rows 19.4 us, 18.6; one of 32000 30.1, 28.2); beyond, the two workgroups of a CU keep
// each other's loads in flight where sequences differ (8 of 7000 .. 65000 rows: 136 us with one, 132 with two).
constexpr long long FEW_ROWS = 256;
struct Piece {
  int b, first, count, length;  // the sequence, its first piece, its pieces, its rows (b = B: there is no piece w)
};
__device__ __forceinline__ int cache_length(const int32_t* lengths, int b, int capacity) {
  return min(max(lengths[b], 0), capacity);
}
__device__ __forceinline__ Piece find_piece(const int32_t* lengths, int B, int capacity, int target, int few, int w) {
  const int lane = threadIdx.x & 63;
  const int len0 = lane < B ? cache_length(lengths, lane, capacity) : 0;
  auto length = [&](int b0) { return b0 == 0 ? len0 : b0 + lane < B ? cache_length(lengths, b0 + lane, capacity) : 0; };
  long long total = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int len = length(b0);
    // (64 lengths of up to 2^30 in two sums of 16 bits and more each)
    total += ((long long)wave_sum_i(len >> 12) << 12) + wave_sum_i(len & 4095);
  }
  if (few > 0 && (B == 1 || total <= FEW_ROWS * target)) target = few;
  // pieces of a sequence where one has `steps` times 128 rows: never more than the rounded up quotient (a piece may get more)
  auto pieces = [](int len, int steps) { return (int)ceilf((float)len * ((1.f - 1e-6f) / (128.f * steps))); };
  auto fits = [&](int steps) {
    int n = 0;
    for (int b0 = 0; b0 < B; b0 += 64) n += wave_sum_i(pieces(length(b0), steps));
    return n <= target;
  };
  auto parts = [&](int n) { return max((int)ceil((double)total / (128.0 * n)), 1); };
  int steps = parts(target);
  if (cuts_fit(B, target) && !fits(steps)) {
    int low = steps;
    steps = parts(target - B);  // fits: a sequence has less than one piece more than its share
    for (int i = 0; i < 3 && steps - low > 1; ++i) {
      const int middle = (low + steps) / 2;
      if (fits(middle)) steps = middle; else low = middle;
    }
  }
  Piece p = {B, 0, 0, 0};
  int before = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int len = length(b0), n = pieces(len, steps);
    const int incl = before + wave_incl_scan(n);
    const uint64_t hit = __ballot(w < incl);
    if (hit) {
      const int at = __ffsll((unsigned long long)hit) - 1;
      p.b = b0 + at;
      p.count = __builtin_amdgcn_readlane(n, at);
      p.first = __builtin_amdgcn_readlane(incl, at) - p.count;
      p.length = __builtin_amdgcn_readlane(len, at);
      return p;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return p;
}
struct AttendArgs {
  const char *q, *k, *v, *prefix_k, *prefix_v;
  const int32_t* lengths;
  const float* weights;
  float *weights_out, *out, *lse;
  float *z, *acc, *pacc;   // products q . k [B * Hq][zrow]; sums of the own pieces [Hkv][pieces][G][D], of the prefix [splits][B * Hq][D]
  float2 *ml, *pml;        // their references and normalisers
  int2* info;              // [B] the first piece of a sequence and how many it has, for the joining
  int B, Hq, Hkv, G, capacity, P;
  int target, few, pieces, prefix_rows, splits, zrow;
  int prefix_blocks, own_blocks, turn, prefix_turns, head_blocks;
  bool head_waves;  // a head's joining is a wave's, not a workgroup's
  float scale, decay;
};
// Joins the partial results that a launch left by `pieces` (and `splits`): out and lse, and the weights where they are wanted.
wave_status launch_attend_join(const AttendArgs& a, int d, hipStream_t st);

}  // namespace wave
