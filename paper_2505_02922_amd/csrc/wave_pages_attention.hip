// Exact attention of one token per sequence over the paged cache: the stream of wave_attend.h over rows of 8 bits, and over
// the tail's rows in their own type.
#include "wave_attend.h"

namespace wave {

namespace {

// ----------------------------------------------------------------------------
// A step: 32 rows of one page against 16 query columns.  Codes are whole numbers up to 127, which bf16 holds, so the products
// are those of the plain cache's bf16 step with the codes widened on the way; the page's scales are the same for the whole
// step, one inside the exponent, the other on the weights.  An fp32 query is three bf16 numbers that hold all its bits.
// Eight sequences of 3001 .. 65536 rows, 32 and 8 heads, d = 128: 88.8 us, 562 MB (576 fetched), 6.3 TB/s, more than a plain
// read's 5.57.  A step is about 325 vector instructions, 128 of them the widening (one a code and one for two); they keep the vector
// units busy for 49 % of the time that a CU has work, 58 % at d = 64, 51 % for 64 sequences of 700 .. 4351 rows on four KV heads (39.8 us with
// the join, 169 MB; fp32, three products for one, 46 % of a longer time, 50.9), and 66 % where those begin alike and a third of the rows
// come from the caches (28.1 us, 165 MB of which 118 are fetched, 4.2 TB/s).  Neither the widening nor the products bound that: with the
// codes taken for bf16 as they are, and a product less a channel, the call took 31.4 us instead of 33.3.
// ----------------------------------------------------------------------------
template <typename T, int D>
struct Codes {
  typedef Step<bf16_t, D> B;
  static constexpr int KEYS = 32, NS = 8, ROW = D, KLOADS = KEYS * ROW / 1024, KC = D / 32, CHUNKS = D / 64;  // 16-code chunks a lane
  static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, WORDS = D / 64;  // of a value row in a lane
  // one load takes a lane's channels of a row where they are neighbours
  static constexpr int VLOADS = sizeof(T) == 4 ? 8 * WORDS : 8;
  struct Q { bf16x8 x[PARTS][KC]; };
  struct K { uint4 x[2][CHUNKS]; };
  struct V { uint32_t x[8][WORDS]; };
  static __device__ __forceinline__ constexpr int place(int r) { return D == 128 ? r & 7 : (r >> 1) & 3; }
  static __device__ __forceinline__ int key(int g, int s) { return B::key(g, s); }

  // product i takes from lane group g the channels 64 * (i / 2) + 16 * g + 8 * (i % 2) ..
  static __device__ __forceinline__ Q load_q(const char* row, int g) {
    Q q;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      const char* at = row + ((i >> 1) * 64 + g * 16 + (i & 1) * 8) * sizeof(T);
      if constexpr (PARTS == 1) {
        q.x[0][i] = __builtin_bit_cast(bf16x8, load16(at));
      } else {
        float f[8];
        unpack<float>(load16(at), reinterpret_cast<float(&)[4]>(f[0]));
        unpack<float>(load16(at + 16), reinterpret_cast<float(&)[4]>(f[4]));
#pragma unroll
        for (int n = 0; n < PARTS; ++n) {
          uint32_t u[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) u[j] = __builtin_amdgcn_perm(__float_as_uint(f[2 * j + 1]), __float_as_uint(f[2 * j]), 0x07060302u);
          q.x[n][i] = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] -= __uint_as_float(__float_as_uint(f[j]) & 0xffff0000u);
        }
      }
    }
    return q;
  }
  static __device__ __forceinline__ K read_k(const char* lds, int g, int c) {
    K k;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < CHUNKS; ++s) k.x[t][s] = load16(lds + (t * 16 + c) * ROW + ((s * 4 + g) ^ place(c)) * 16);
    return k;
  }
  // rows: the step's first row of values.  Nobody else reads them, so they pass by the caches; but where a row is half a line (d = 64),
  // two loads want it (16 sequences of 1000 .. 16000 rows: 30.8 us, past the caches 32.9)
  static __device__ __forceinline__ V load_v(const char* rows, int g, int c) {
    V v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* at = rows + key(g, j) * ROW;
      if constexpr (sizeof(T) == 2 && WORDS == 2) {
        const uint2 u = load8_stream(at + c * 8);
        v.x[j][0] = u.x;
        v.x[j][1] = u.y;
      } else {
#pragma unroll
        for (int u = 0; u < WORDS; ++u) {
          const uint32_t* word = reinterpret_cast<const uint32_t*>(at + u * 64 + c * 4);
          v.x[j][u] = D == 64 ? *word : __builtin_nontemporal_load(word);
        }
      }
    }
    return v;
  }
  static __device__ __forceinline__ float value(uint32_t word, int byte) { return (float)(int8_t)(word >> (8 * byte)); }
  static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
  }
  static __device__ __forceinline__ void scores(const K& k, const Q& q, float (&s)[NS]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        const uint4& u = k.x[t][i >> 1];
        const uint32_t lo = i & 1 ? u.z : u.x, hi = i & 1 ? u.w : u.y;
        const bf16x8 x = __builtin_bit_cast(bf16x8, make_uint4(pair(value(lo, 0), value(lo, 1)), pair(value(lo, 2), value(lo, 3)),
                                                               pair(value(hi, 0), value(hi, 1)), pair(value(hi, 2), value(hi, 3))));
#pragma unroll
        for (int n = PARTS - 1; n >= 0; --n) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q.x[n][i], a, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t * 4 + i] = a[i];
    }
  }
  // V^T as the left operand: channel a of every lane's
  static __device__ __forceinline__ typename B::Vt transpose(const V& v) {
    typename B::Vt r;
#pragma unroll
    for (int a = 0; a < D / 16; ++a) {
      uint32_t u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = pair(value(v.x[2 * j][a >> 2], a & 3), value(v.x[2 * j + 1][a >> 2], a & 3));
      r.x[a] = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
    }
    return r;
  }
};

// A unit has no more than eight heads, so columns 8 .. 15 of the scores are 0 .. 7 again: a column's scores lie in eight lanes, each
// forms the weights of four of its lane group's eight rows, and the lane eight away those of the other four.  Of a weight's three
// numbers columns 8 .. 15 of one product take the second, beside the first in columns 0 .. 7; a product with the third follows, and
// stream_codes adds the halves at its end.  So a step has two products a channel instead of three and half the work on its weights
// (64 sequences of up to 4351 rows that begin alike 33.8 -> 32.9 us, at d = 64 apart 38.0 -> 35.7, fp32 83.6 -> 80.9).
constexpr int DPP_ROW_ROR8 = 0x128;
__device__ __forceinline__ uint32_t from_other_half(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP_ROW_ROR8, 0xF, 0xF, true);
}
template <typename T, int D>
struct Weights {
  typedef Codes<T, D> C;
  uint32_t own[3][2];  // three bf16 numbers a weight, two rows each
  // the step's weights over the reference, times the values' scale
  __device__ __forceinline__ void form(const float (&s)[C::NS], State<T, D>& st, float scale, float vs, bool upper) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = upper ? s[4 + i] : s[i];
    float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) * scale;
    if (__any(top > st.m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 8));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      st.raise(top);
    }
    st.weights(x, x, scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= vs;
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        own[n][j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);
        x[2 * j] -= __uint_as_float(__float_as_uint(x[2 * j]) & 0xffff0000u);
        x[2 * j + 1] -= __uint_as_float(__float_as_uint(x[2 * j + 1]) & 0xffff0000u);
      }
  }
  __device__ __forceinline__ void accumulate(const typename Step<bf16_t, D>::Vt& v, f32x4 (&o)[D / 16], bool upper) const {
    // the upper half's first numbers go down, the lower half's second ones up
    uint32_t got[2], third[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      got[j] = from_other_half(upper ? own[0][j] : own[1][j]);
      third[j] = from_other_half(own[2][j]);
    }
    const bf16x8 one = __builtin_bit_cast(bf16x8, upper ? make_uint4(got[0], got[1], own[1][0], own[1][1]) : make_uint4(own[0][0], own[0][1], got[0], got[1]));
    const bf16x8 two = __builtin_bit_cast(bf16x8, upper ? make_uint4(0, 0, 0, 0) : make_uint4(own[2][0], own[2][1], third[0], third[1]));
#pragma unroll
    for (int a = 0; a < D / 16; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.x[a], two, o[a], 0, 0, 0);
#pragma unroll
    for (int a = 0; a < D / 16; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.x[a], one, o[a], 0, 0, 0);
  }
};

struct PagesAttendArgs {
  AttendArgs a;  // k and v: the tails
  const char *k_codes, *v_codes;
  const float *k_scales, *v_scales;
  const int32_t* table;
  int n_pages, max_pages, page, shift;
};

// The pages of a wave's next 64 steps, a step each lane.
struct StepPages {
  int id;
  float ks, vs;
  __device__ __forceinline__ void load(const PagesAttendArgs& p, const int32_t* table, int h, int k0, int stride, int end, int lane) {
    const int row = min((long long)k0 + (long long)lane * stride, (long long)end - 1);
    id = min(max(table[row >> p.shift], 0), p.n_pages - 1);
    const size_t at = (size_t)id * p.a.Hkv + h;
    ks = p.k_scales[at];
    vs = p.v_scales[at];
  }
};

// The stream of one wave over pages: steps k0, k0 + stride, .. below `end` (all of them whole).  As stream_rows: keys through
// LDS without registers, values straight, the next step's loads out before this one's products.
template <typename T, int D>
__device__ __forceinline__ void stream_codes(const PagesAttendArgs& p, int b, int h, int k0, int stride, int end,
                                             const typename Codes<T, D>::Q& q, State<T, D>& st, char* lds, int lane) {
  typedef Codes<T, D> C;
  if (k0 >= end) return;
  const int g = lane >> 4, c = lane & 15;
  const bool upper = c >= 8;
  const int32_t* table = p.table + (size_t)b * p.max_pages;
  StepPages pages;
  pages.load(p, table, h, k0, stride, end, lane);
  const auto place = [](int r) { return C::place(r); };
  auto rows = [&](const char* codes, int id, int row) {
    return codes + (((size_t)id * p.a.Hkv + h) * p.page + (row & (p.page - 1))) * D;
  };
  int n = 0;  // this step's lane
  int id = __builtin_amdgcn_readlane(pages.id, 0);
  rows_to_lds<C::ROW, C::KLOADS, true>(lds, StepRows{rows(p.k_codes, id, k0), 31}, 0, lane, place);
  __builtin_amdgcn_sched_barrier(0);
  typename C::V v = C::load_v(rows(p.v_codes, id, k0), g, c);
  for (;;) {
    const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(pages.ks), n));
    const float vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(pages.vs), n));
    const bool more = k0 < end - stride;
    const int next = more ? k0 + stride : k0;  // (behind the last step it comes again, and is not used)
    if (more && ++n == 64) {
      n = 0;
      pages.load(p, table, h, next, stride, end, lane);
    }
    id = __builtin_amdgcn_readlane(pages.id, n);
    __builtin_amdgcn_sched_barrier(0);
    wait_for_loads<C::VLOADS < 16 ? C::VLOADS : 15>();  // the keys are here; the values, asked for after them, may not be
    const typename C::K k = C::read_k(lds, g, c);
    wait_for_reads();
    __builtin_amdgcn_sched_barrier(0);
    rows_to_lds<C::ROW, C::KLOADS, true>(lds, StepRows{rows(p.k_codes, id, next), 31}, 0, lane, place);
    __builtin_amdgcn_sched_barrier(0);
    float s[C::NS];
    C::scores(k, q, s);
    const typename Step<bf16_t, D>::Vt vt = C::transpose(v);
    __builtin_amdgcn_sched_barrier(0);
    v = C::load_v(rows(p.v_codes, id, next), g, c);
    __builtin_amdgcn_sched_barrier(0);
    Weights<T, D> w;
    w.form(s, st, p.a.scale * ks, vs, upper);
    w.accumulate(vt, st.o, upper);
    if (!more) break;
    k0 = next;
  }
  wait_for_loads<0>();  // nothing may come into LDS behind this
  // both halves' sums
  st.l += __uint_as_float(from_other_half(__float_as_uint(st.l)));
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) st.o[x][i] += __uint_as_float(from_other_half(__float_as_uint(st.o[x][i])));
}

// Rows start .. end of a unit against its G heads, steps of 32 rows dealt out to WAVES waves.
template <typename T, int D, int WAVES>
__device__ __forceinline__ void stream_unit(const PagesAttendArgs& p, int b, int h, int start, int end, int length, State<T, D>& st,
                                            char* lds, int wave, int lane) {
  typedef Step<T, D> S;
  const AttendArgs& a = p.a;
  const int g = lane >> 4, c = lane & 15;
  const size_t row = D * sizeof(T), unit = (size_t)b * a.Hkv + h;
  const char* q = a.q + ((size_t)b * a.Hq + h * a.G + min(c & 7, a.G - 1)) * row;  // (columns from 8 on are the first ones' again)
  const int whole = length >> p.shift << p.shift, paged = min(end, whole);
  if (start < paged) {
    const typename Codes<T, D>::Q qc = Codes<T, D>::load_q(q, g);
    stream_codes<T, D>(p, b, h, start + wave * 32, WAVES * 32, paged, qc, st, lds, lane);
  }
  if (end > whole) {  // the tail, first by the waves that the pages leave first
    const int first = max(start, whole), steps = max(whole - start, 0) / 32;
    const int turn = (wave + WAVES - steps % WAVES) % WAVES;
    const typename S::Q qt = S::load_q(q, g);
    stream_rows<T, D, true>(a.k + unit * p.page * row, a.v + unit * p.page * row, first - whole + turn * S::KEYS, WAVES * S::KEYS,
                            end - whole, a.scale, qt, st, [](int, const f32x4&) {}, lds, lane);
  }
}

// One workgroup per piece of a sequence and KV head.  As many a CU as there are registers for: at d = 128 in bf16 three (168) leave
// 66.3 us of 70.7 with two (64 sequences of 700 .. 4351 rows on eight KV heads); fp32's three numbers a query need two's.
template <typename T, int D>
__global__ __launch_bounds__(256, D == 64 ? 4 : sizeof(T) == 2 ? 3 : 2) void pages_rows_kernel(const PagesAttendArgs p) {
  __shared__ JoinShared js;
  __shared__ __attribute__((aligned(16))) char lds[4][16 * (D + 4) * 4];
  const Areas areas{lds[0], lds[1], lds[2], lds[3]};
  const AttendArgs& a = p.a;
  const int w = blockIdx.x / a.Hkv, h = blockIdx.x % a.Hkv;
  const Piece piece = find_piece(a.lengths, a.B, a.capacity, a.target, a.few, w);
  if (piece.b == a.B) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int rows = ((piece.length + piece.count - 1) / piece.count + 31) / 32 * 32;
  const int start = (w - piece.first) * rows, end = min(piece.length, start + rows);
  if (w == piece.first && h == 0 && threadIdx.x == 0) a.info[piece.b] = make_int2(w, piece.count);
  State<T, D> st;
  st.init();
  stream_unit<T, D, 4>(p, piece.b, h, start, end, piece.length, st, areas.of(wave), wave, lane);
  const size_t at = ((size_t)h * a.pieces + w) * a.G;
  join_waves<T, D>(st, a.G, js, areas, wave, g, c, a.ml + at, a.acc + at * D);
}

// Short caches: one launch, a workgroup of eight waves per unit, which join in LDS.
constexpr int SHORT_WAVES = 8, SHORT_THREADS = SHORT_WAVES * 64;

template <typename T, int D>
__global__ __launch_bounds__(SHORT_THREADS) void pages_short_kernel(const PagesAttendArgs p) {
  typedef Step<T, D> S;
  constexpr int PITCH = D + 4;
  __shared__ __attribute__((aligned(16))) char lds[SHORT_WAVES][16 * PITCH * 4];
  __shared__ float sm[SHORT_WAVES][16], sl[SHORT_WAVES][16];
  const AttendArgs& a = p.a;
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x % a.Hkv;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int length = cache_length(a.lengths, b, a.capacity);
  State<T, D> st;
  st.init();
  stream_unit<T, D, SHORT_WAVES>(p, b, h, 0, length, length, st, lds[wave], wave, lane);
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    sm[wave][c] = st.m;
    sl[wave][c] = l;
  }
  if (c < a.G) {
    float* at = reinterpret_cast<float*>(lds[wave]) + c * PITCH;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < S::ACC; x += 4)
        *reinterpret_cast<f32x4*>(at + S::channel(g, x, i)) = f32x4{st.o[x][i], st.o[x + 1][i], st.o[x + 2][i], st.o[x + 3][i]};
  }
  __syncthreads();
  const int head = b * a.Hq + h * a.G;
  for (int i = threadIdx.x; i < a.G * D; i += SHORT_THREADS) {
    const int col = i / D, ch = i % D;
    float m = sm[0][col], sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 1; w < SHORT_WAVES; ++w) m = fmaxf(m, sm[w][col]);
#pragma unroll
    for (int w = 0; w < SHORT_WAVES; ++w) {
      const float f = sm[w][col] == neg_inf() ? 0.f : exp2f(sm[w][col] - m);
      sum += f * sl[w][col];
      o += f * reinterpret_cast<const float*>(lds[w])[col * PITCH + ch];
    }
    const bool any = !(m == neg_inf() && sum == 0.f);
    a.out[(size_t)(head + col) * D + ch] = any ? o / sum : 0.f;
    if (ch == 0) a.lse[head + col] = any ? (m + log2f(sum)) * kLn2 : neg_inf();
  }
}

template <typename T, int D>
wave_status pages_attend_td(const PagesAttendArgs& p, const PagesAttendGeom& g, hipStream_t st) {
  if (g.one_launch) {
    WAVE_LAUNCH("pages_attend", (pages_short_kernel<T, D>), p.a.B * p.a.Hkv, SHORT_THREADS, 0, st, p);
    return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
  }
  WAVE_LAUNCH("pages_attend", (pages_rows_kernel<T, D>), p.a.Hkv * g.pieces, 256, 0, st, p);
  if (hipGetLastError() != hipSuccess) return WAVE_ERR_HIP;
  return launch_attend_join(p.a, D, st);
}

}  // namespace

PagesAttendGeom pages_attend_geometry(const wave_pages& p, int Hq) {
  PagesAttendGeom g{};
  const long long room = (long long)p.max_pages * p.page + p.page - 1;
  // One launch where a wave has few steps to do and there are about as many units as CUs, so that its workgroups of eight waves fill
  // them: up to two steps for up to 512 units, four from 128, eight from 256 on.  (In pieces and in one launch, bf16, d = 128, us: one
  // sequence of 500 rows on eight KV heads 10.8 and 8.0; 32 of 160 .. 500 14.7 and 10.0, of 300 .. 1000 18.6 and 14.0, of 700 .. 2000 27.0
  // and 22.3; 64 of 700 .. 2000 42.0 and 39.3.  8 of 1000 11.4 and 11.6, 16 of 2000 16.6 and 18.3, 256 of 500 54 and 61.)  With many
  // sequences every piece's workgroup would read all their lengths.  The rule goes by the table's room, since the lengths are the
  // device's: in a table of 1024 pages the same short sequences are cut into pieces (3 of up to 200 6.6 and 10.1, one of 500 8.0 and 10.3, 32
  // of 160 .. 500 10.1 and 14.6, of 300 .. 1000 14.8 and 19.2).
  const long long steps = (room + SHORT_WAVES * 32 - 1) / (SHORT_WAVES * 32), units = (long long)p.B * p.Hkv;
  g.one_launch = steps <= 1 || (steps <= 2 && (units <= 512 || p.B > 512)) ||
                 (units <= 512 && ((steps <= 4 && units >= 128) || (steps <= 8 && units >= 256)));
  // Two pieces a CU, and one where they are short.  Three for many sequences that can still be cut alike, since each then has few:
  // 64 sequences of 700 .. 4351 rows on four KV heads that begin with the same 640 38.4 us, with three 34.4; 32 of 2000 .. 8000 on eight
  // 64.2 and 62.7.  (64 on eight, in proportion, 66.3 and 69.9; 8 of 3001 .. 65536 95 and 97.6; four or six a CU, in turns,
  // 95 and 102; one of 32000 with one and a half 21.6 for 19.1.)
  const auto pieces = [&](int per_cu) { return per_cu * 256 / p.Hkv > 1 ? per_cu * 256 / p.Hkv : 1; };
  g.target = pieces(p.B >= 32 && cuts_fit(p.B, pieces(3)) ? 3 : 2);
  g.few = pieces(1);
  const long long most = (long long)p.B * ((room + 127) / 128), cut = (long long)g.target + (cuts_fit(p.B, g.target) ? 0 : p.B);
  g.pieces = (int)(cut < most ? cut : most);
  size_t o = 0;
  g.off_info = o;  o = align_up(o + sizeof(int32_t) * 2 * (size_t)p.B);
  g.off_ml = o;    o = align_up(o + sizeof(float) * 2 * (size_t)Hq * g.pieces);
  g.off_acc = o;   o = align_up(o + sizeof(float) * p.d * (size_t)Hq * g.pieces);
  g.total = o;
  return g;
}

wave_status launch_pages_attend(const void* q, int Hq, const wave_pages& c, float* out, float* lse, void* ws, hipStream_t st) {
  const PagesAttendGeom g = pages_attend_geometry(c, Hq);
  char* w = static_cast<char*>(ws);
  PagesAttendArgs p{};
  AttendArgs& a = p.a;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(c.k_tail);
  a.v = static_cast<const char*>(c.v_tail);
  a.lengths = c.lengths;
  a.out = out;
  a.lse = lse;
  a.info = reinterpret_cast<int2*>(w + g.off_info);
  a.ml = reinterpret_cast<float2*>(w + g.off_ml);
  a.acc = reinterpret_cast<float*>(w + g.off_acc);
  a.pml = a.ml;  // (there is no prefix)
  a.pacc = a.acc;
  a.B = c.B;
  a.Hq = Hq;
  a.Hkv = c.Hkv;
  a.G = Hq / c.Hkv;
  a.capacity = c.max_pages * c.page + c.page - 1;
  a.target = g.target;
  a.few = g.few;
  a.pieces = g.pieces;
  a.scale = kLog2e / sqrtf((float)c.d);
  p.k_codes = reinterpret_cast<const char*>(c.k_codes);
  p.v_codes = reinterpret_cast<const char*>(c.v_codes);
  p.k_scales = c.k_scales;
  p.v_scales = c.v_scales;
  p.table = c.table;
  p.n_pages = c.n_pages;
  p.max_pages = c.max_pages;
  p.page = c.page;
  p.shift = c.page == 32 ? 5 : c.page == 64 ? 6 : 7;
  if (c.dtype == WAVE_BF16) return c.d == 128 ? pages_attend_td<bf16_t, 128>(p, g, st) : pages_attend_td<bf16_t, 64>(p, g, st);
  return c.d == 128 ? pages_attend_td<float, 128>(p, g, st) : pages_attend_td<float, 64>(p, g, st);
}

}  // namespace wave
