// Rotary positions and the rows of the plain cache: appending new tokens, evicting the least attended ones.
#include "wave_common.h"

namespace wave {

namespace {

// ----------------------------------------------------------------------------
// Rotary positions.  A work item is two 16-byte chunks of a row that hold EPC whole pairs (channels i .. and
// i + rot / 2 .. for halves, two neighbouring chunks for neighbours) or, behind the rotated channels, two chunks
// that are copied.  A thread keeps the sines and cosines of its item of one token and goes through the heads with
// them: they cost about forty instructions a pair (the angle in fp64), the turn itself six.
// ----------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&f)[Elem<T>::EPC]);
template <>
__device__ __forceinline__ uint4 pack<float>(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 pack<bf16_t>(const float (&f)[8]) {
  typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];  // nearest even
  return __builtin_bit_cast(uint4, v);
}

template <typename T, int D>
struct Turn {
  static constexpr int EPC = Elem<T>::EPC;
  static constexpr int ITEMS = D / (2 * EPC);  // work items of a row
  float c[EPC], s[EPC];
  int one, two;  // the item's chunks
  bool turns;

  __device__ __forceinline__ void place(const RotaryArgs& r, int item) {
    const int rotated = r.rot / (2 * EPC);
    turns = item < rotated;
    const bool halves = turns && r.pairing == WAVE_ROTARY_HALVES;
    one = halves ? item : 2 * item;
    two = halves ? item + rotated : 2 * item + 1;
  }
  // position(axis) of the item's token; a circle is `1` in turns, so the nearest whole number of circles comes off
  // without error
  template <typename F>
  __device__ __forceinline__ void angles(const RotaryArgs& r, int item, F&& position) {
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
      if (turns) {
        const int i = item * EPC + e;
        const double t = (double)position(r.axis[i]) * r.turns[i];
        sincospif((float)(2.0 * (t - rint(t))), &s[e], &c[e]);
      }
    }
  }
  __device__ __forceinline__ void apply(const RotaryArgs& r, uint4& a, uint4& b) const {
    if (!turns) return;
    float x[EPC], y[EPC];
    unpack<T>(a, x);
    unpack<T>(b, y);
    if (r.pairing == WAVE_ROTARY_HALVES) {
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const float u = x[e] * c[e] - y[e] * s[e], v = x[e] * s[e] + y[e] * c[e];
        x[e] = u;
        y[e] = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPC; e += 2) {
        const int p = e / 2, h = EPC / 2 + p;  // pairs of the first and of the second chunk
        const float u = x[e] * c[p] - x[e + 1] * s[p], v = x[e] * s[p] + x[e + 1] * c[p];
        const float w = y[e] * c[h] - y[e + 1] * s[h], z = y[e] * s[h] + y[e + 1] * c[h];
        x[e] = u;
        x[e + 1] = v;
        y[e] = w;
        y[e + 1] = z;
      }
    }
    a = pack<T>(x);
    b = pack<T>(y);
  }
};

// The threads of a workgroup: ITEMS a row, then `lanes` heads side by side, then the tokens.  A prompt takes one lane
// (a wave then reads whole neighbouring rows of one head), a decode step as many as there are.
struct TurnShape {
  int lane_shift;   // log2 of the heads side by side
  int tokens;       // tokens of a workgroup
  int head_groups;  // workgroups that share the heads of a tile of tokens
};
template <int ITEMS>
TurnShape turn_shape(int n, int B, int heads) {
  TurnShape t{0, 256 / ITEMS, 1};
  while (t.tokens > 1 && t.tokens / 2 >= n) {
    t.tokens /= 2;
    ++t.lane_shift;
  }
  // A workgroup's chain of heads is split while the launch leaves most CUs without work.
  const long long tiles = (long long)B * ((n + t.tokens - 1) / t.tokens);
  while (tiles * t.head_groups < 1024 && (heads >> t.lane_shift) > 4 * t.head_groups) t.head_groups *= 2;
  return t;
}

constexpr int TURN_BATCH = 4;  // heads whose loads are in flight together

template <typename T, int D>
__global__ __launch_bounds__(256) void rotary_kernel(const char* x, const int32_t* __restrict__ coords,
                                                     const RotaryArgs rot, int B, int H, int N, TurnShape sh,
                                                     int tiles, char* y) {
  typedef Turn<T, D> Tu;
  constexpr size_t ROW = D * sizeof(T);
  const unsigned block = workgroup_number();
  const int group = block % sh.head_groups, bt = block / sh.head_groups;
  const int b = bt / tiles, tile = bt % tiles;
  const int item = threadIdx.x % Tu::ITEMS, lane = (threadIdx.x / Tu::ITEMS) & ((1 << sh.lane_shift) - 1);
  const int n = tile * sh.tokens + (int)(threadIdx.x / Tu::ITEMS >> sh.lane_shift);
  if (b >= B || n >= N) return;
  Tu t;
  t.place(rot, item);
  const int step = sh.head_groups << sh.lane_shift;
  uint4 u[TURN_BATCH], v[TURN_BATCH];
  auto load = [&](int h0) {
#pragma unroll
    for (int k = 0; k < TURN_BATCH; ++k) {
      const int h = min(h0 + k * step, H - 1);
      const char* row = x + ((size_t)((size_t)b * H + h) * N + n) * ROW;
      u[k] = load16(row + t.one * 16);
      v[k] = load16(row + t.two * 16);
    }
  };
  // the first rows are on their way while the sines are formed
  int h0 = (group << sh.lane_shift) + lane;
  load(h0);
  t.angles(rot, item, [&](int axis) { return coords[((size_t)axis * B + b) * N + n]; });
  for (; h0 < H;) {
#pragma unroll
    for (int k = 0; k < TURN_BATCH; ++k)
      if (h0 + k * step < H) {
        char* row = y + ((size_t)((size_t)b * H + h0 + k * step) * N + n) * ROW;
        t.apply(rot, u[k], v[k]);
        store16(row + t.one * 16, u[k]);
        store16(row + t.two * 16, v[k]);
      }
    h0 += TURN_BATCH * step;
    if (h0 < H) load(h0);
  }
}

// ----------------------------------------------------------------------------
// Append.  The heads of a token are its q, k and v heads in this order.
// ----------------------------------------------------------------------------
struct AppendArgs {
  const char *q, *k_new, *v_new;
  char *q_out, *k, *v;
  int32_t* positions;
  float* weights;
  const int32_t *lengths, *tokens, *counts, *coords;
  int32_t *lengths_out, *tokens_out;
  int B, Hq, Hkv, n, capacity;
};
struct Share {
  int length, count, fit, first;  // rows before, tokens given, tokens that fit, number of the first token
};
__device__ __forceinline__ Share append_share(const AppendArgs& a, int b) {
  Share s;
  s.length = min(max(a.lengths[b], 0), a.capacity);
  s.count = a.counts ? min(max(a.counts[b], 0), a.n) : a.n;
  s.fit = min(s.count, a.capacity - s.length);
  s.first = a.tokens ? a.tokens[b] : 0;
  return s;
}

template <typename T, int D, bool ROT>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a, const RotaryArgs rot, TurnShape sh, int tiles,
                                                     bool advance) {
  typedef Turn<T, D> Tu;
  constexpr size_t ROW = D * sizeof(T);
  const unsigned block = workgroup_number();
  const int group = block % sh.head_groups, bt = block / sh.head_groups;
  const int b = bt / tiles, tile = bt % tiles;
  if (b >= a.B) return;
  const int item = threadIdx.x % Tu::ITEMS, lane = (threadIdx.x / Tu::ITEMS) & ((1 << sh.lane_shift) - 1);
  const int n = tile * sh.tokens + (int)(threadIdx.x / Tu::ITEMS >> sh.lane_shift);
  const Share s = append_share(a, b);
  const int slots = a.Hq + 2 * a.Hkv, row = s.length + n;
  if (n < s.count) {
    Tu t;
    if (ROT) {
      t.place(rot, item);
    } else {
      t.turns = false;
      t.one = 2 * item;
      t.two = 2 * item + 1;
    }
    const int step = sh.head_groups << sh.lane_shift;
    uint4 u[TURN_BATCH], v[TURN_BATCH];
    char* to[TURN_BATCH];
    auto load = [&](int h0) {
#pragma unroll
      for (int i = 0; i < TURN_BATCH; ++i) {
        const int h = min(h0 + i * step, slots - 1);
        const bool is_q = h < a.Hq, is_k = h < a.Hq + a.Hkv;
        const int heads = is_q ? a.Hq : a.Hkv, head = is_q ? h : h - a.Hq - (is_k ? 0 : a.Hkv);
        const size_t unit = (size_t)b * heads + head, at = (unit * a.n + n) * ROW;
        const char* from = (is_q ? a.q : is_k ? a.k_new : a.v_new) + at;
        u[i] = load16(from + t.one * 16);
        v[i] = load16(from + t.two * 16);
        to[i] = is_q ? a.q_out + at : (is_k ? a.k : a.v) + (unit * a.capacity + row) * ROW;
        if (h0 + i * step >= slots || (!is_q && n >= s.fit)) to[i] = nullptr;
      }
    };
    int h0 = (group << sh.lane_shift) + lane;
    load(h0);
    if (ROT) t.angles(rot, item, [&](int axis) { return a.coords ? a.coords[((size_t)axis * a.B + b) * a.n + n] : s.first + n; });
    for (; h0 < slots;) {
#pragma unroll
      for (int i = 0; i < TURN_BATCH; ++i)
        if (to[i]) {
          if (ROT && h0 + i * step < a.Hq + a.Hkv) t.apply(rot, u[i], v[i]);
          store16(to[i] + t.one * 16, u[i]);
          store16(to[i] + t.two * 16, v[i]);
        }
      h0 += TURN_BATCH * step;
      if (h0 < slots) load(h0);
    }
  }
  // positions and weights: the tile's tokens of all units, by the workgroup of the first heads
  if (group == 0 && (a.positions || a.weights)) {
    const int first = tile * sh.tokens, mine = min(sh.tokens, s.fit - first);
    for (int i = threadIdx.x; i < mine * a.Hkv; i += 256) {
      const int h = i / mine, j = first + i % mine;
      const size_t at = ((size_t)b * a.Hkv + h) * a.capacity + s.length + j;
      if (a.positions) a.positions[at] = s.first + j;
      if (a.weights) a.weights[at] = 0.f;
    }
  }
  // The numbers: by the first workgroup of a sequence, if no other one may still be reading them.
  if (advance && group == 0 && tile == 0) {
    __syncthreads();
    if (threadIdx.x == 0) {
      a.lengths_out[b] = s.length + s.fit;
      if (a.tokens_out) a.tokens_out[b] = s.first + s.fit;
    }
  }
}
__global__ __launch_bounds__(256) void advance_kernel(const AppendArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.B) return;
  const Share s = append_share(a, b);
  a.lengths_out[b] = s.length + s.fit;
  if (a.tokens_out) a.tokens_out[b] = s.first + s.fit;
}

// ----------------------------------------------------------------------------
// Eviction.  The n_keep-th largest key of a unit comes from three histograms (11, 11 and 10 bits, LDS atomics: integers, so
// the order of the counting does not show); then holes (rows below n_keep that leave) and movers (rows from n_keep on that
// stay) are listed in ascending order; there are as many of one as of the other.  evict_move_kernel copies the rows.
// Short caches: one workgroup per unit with the keys in registers.  Long ones (more than 16384 rows): slices of 8192 rows
// with a launch for each histogram, since one workgroup would be alone with the unit's atomics (120K rows of 16 units: one
// workgroup each 330 us).
// ----------------------------------------------------------------------------
struct EvictArgs {
  const int32_t *positions, *lengths, *tokens;
  const float* weights;
  int32_t *to_positions, *to_lengths, *to_tokens;
  float* to_weights;
  const char *k, *v;
  char *to_k, *to_v;
  // per unit: moved and kept rows; the lists of in-place moves; where K and V are written apart (else NULL) the old row of
  // every new one, -1 - i for the i-th mover's place
  int32_t *count, *hole, *mover, *source;
  uint32_t *hist_a, *hist_b;               // [units][slices][2048]
  int4* state;                             // [units] bits of the threshold so far, how many rows with them are kept
  int32_t* above;                          // [units][slices] rows of a slice above the threshold's bits so far
  int Hkv, capacity, to_capacity, n_keep, n_sink, n_local, moves;
  int slices, keep_slices;                 // slices of a unit; those of the rows below n_keep come first
};

// Order of the rows as integers: what has to stay above every weight, what is no number below.
__device__ __forceinline__ uint32_t evict_key(float w, int position, int n_sink, long long local) {
  if (position < n_sink || position >= local) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 counts as 0
  return (u >> 31) ? ~u : (u | 0x80000000u);
}

constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / 64, EVICT_BUCKETS = 2048;
constexpr int SLICE_PER = 8, SLICE_ROWS = SLICE_PER * EVICT_THREADS;
__device__ __forceinline__ constexpr int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ constexpr int digit_bits(int pass) { return pass == 2 ? 10 : 11; }

struct EvictUnit {
  int unit, b, len, keep;
  long long local;
  const int32_t* pos;
  const float* wts;
};
__device__ __forceinline__ EvictUnit evict_unit(const EvictArgs& a, int unit) {
  EvictUnit u;
  u.unit = unit;
  u.b = unit / a.Hkv;
  u.len = min(max(a.lengths[u.b], 0), a.capacity);
  u.keep = min(u.len, a.n_keep);
  u.local = (long long)a.tokens[u.b] - a.n_local;
  u.pos = a.positions + (size_t)unit * a.capacity;
  u.wts = a.weights + (size_t)unit * a.capacity;
  return u;
}
// Weights and positions of the rows r0 + i * 1024 + tid, of the last one below r1 where that is behind it; asked for before the
// histograms are, and made into keys after.
template <int PER>
struct EvictRows {
  float w[PER];
  int p[PER];
  __device__ __forceinline__ void load(const EvictUnit& u, int r0, int r1) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = max(min(r0 + i * EVICT_THREADS + (int)threadIdx.x, r1 - 1), 0);
      w[i] = u.wts[j];
      p[i] = u.pos[j];
    }
  }
  __device__ __forceinline__ void keys(const EvictArgs& a, const EvictUnit& u, uint32_t (&key)[PER]) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = evict_key(w[i], p[i], a.n_sink, u.local);
  }
};

struct EvictShared {
  uint32_t hist[EVICT_BUCKETS];
  int wave_total[EVICT_WAVES];
  int table[16 * EVICT_WAVES];
  int bucket, above;
};
// Counts the keys' digit `pass` where the digits before are `prefix`.
template <int PER>
__device__ __forceinline__ void evict_count(EvictShared& sh, const uint32_t (&key)[PER], int r0, int r1, int pass, uint32_t prefix) {
  for (int i = threadIdx.x; i < EVICT_BUCKETS; i += EVICT_THREADS) sh.hist[i] = 0;
  __syncthreads();
  const int shift = digit_shift(pass), bits = digit_bits(pass);
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (r0 + i * EVICT_THREADS + (int)threadIdx.x < r1 && (pass == 0 || key[i] >> (shift + bits) == prefix))
      atomicAdd(&sh.hist[(key[i] >> shift) & ((1 << bits) - 1)], 1u);
  __syncthreads();
}
// Given the counts c0, c1 of this thread's buckets 2047 - 2 tid and 2046 - 2 tid: the bucket in which the count from the
// top reaches `need`, and the count above it.  (The answer's place is written again only behind a barrier of what follows.)
__device__ __forceinline__ int2 evict_bucket(EvictShared& sh, int c0, int c1, int need) {
  const int tid = threadIdx.x, wave = tid >> 6, top = EVICT_BUCKETS - 1 - 2 * tid;
  const int incl = wave_incl_scan(c0 + c1);
  if ((tid & 63) == 63) sh.wave_total[wave] = incl;
  __syncthreads();
  const int lane = tid & 63, before = incl - c0 - c1 + wave_sum_i(lane < wave ? sh.wave_total[lane & (EVICT_WAVES - 1)] : 0);
  if (before < need && before + c0 >= need) {
    sh.bucket = top;
    sh.above = before;
  } else if (before + c0 < need && before + c0 + c1 >= need) {
    sh.bucket = top - 1;
    sh.above = before + c0;
  }
  __syncthreads();
  return make_int2(sh.bucket, sh.above);
}
// Exclusive sums, over (i, wave) in this order, of one number each wave has for every i; all threads call it.
template <int PER>
__device__ __forceinline__ int evict_scan(EvictShared& sh, const int (&mine)[PER], int (&before)[PER]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  constexpr int ALL = PER * EVICT_WAVES, EACH = (ALL + 63) / 64;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (lane == 0) sh.table[i * EVICT_WAVES + wave] = mine[i];
  __syncthreads();
  if (wave == 0) {
    int x[EACH], sum = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      x[e] = lane * EACH + e < ALL ? sh.table[lane * EACH + e] : 0;
      sum += x[e];
    }
    int run = wave_incl_scan(sum);
    if (lane == 63) sh.above = run;
    run -= sum;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      if (lane * EACH + e < ALL) sh.table[lane * EACH + e] = run;
      run += x[e];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) before[i] = sh.table[i * EVICT_WAVES + wave];
  const int total = sh.above;
  __syncthreads();
  return total;
}
// Lists the holes and movers among the rows r0 + i * 1024 + tid below r1.  need: how many rows with the threshold's key are
// kept, equal_before: how many of them lie before r0; hole_before, mover_before: what the lists hold from rows before r0.
// Returns holes | movers << 16 of these rows.
template <int PER>
__device__ __forceinline__ int evict_list(EvictShared& sh, const EvictArgs& a, const EvictUnit& u, const uint32_t (&key)[PER], int r0,
                                          int r1, uint32_t threshold, int need, int equal_before, int hole_before,
                                          int mover_before) {
  const int tid = threadIdx.x, lane = tid & 63;
  const uint64_t below = (1ull << lane) - 1;
  int mine[PER], before[PER];
  uint64_t eq[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    eq[i] = __ballot(r0 + i * EVICT_THREADS + tid < r1 && key[i] == threshold);
    mine[i] = __popcll(eq[i]);
  }
  evict_scan<PER>(sh, mine, before);
  uint64_t hb[PER], mb[PER];
  uint32_t kept_bits = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = r0 + i * EVICT_THREADS + tid;
    const int rank = equal_before + before[i] + __popcll(eq[i] & below);
    const bool kept = j < r1 && (key[i] > threshold || (key[i] == threshold && rank < need));
    if (kept) kept_bits |= 1u << i;
    hb[i] = __ballot(j < u.keep && !kept && j < r1);
    mb[i] = __ballot(j >= u.keep && kept);
    mine[i] = __popcll(hb[i]) | (__popcll(mb[i]) << 16);
  }
  const int total = evict_scan<PER>(sh, mine, before);
  int32_t* holes = a.hole + (size_t)u.unit * a.moves;
  int32_t* movers = a.mover + (size_t)u.unit * a.moves;
  int32_t* source = a.source ? a.source + (size_t)u.unit * a.n_keep : nullptr;
  int32_t* to_pos = a.to_positions + (size_t)u.unit * a.to_capacity;
  float* to_wts = a.to_weights + (size_t)u.unit * a.to_capacity;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = r0 + i * EVICT_THREADS + tid;
    const bool kept = (kept_bits >> i) & 1u;
    if (j < r1 && j < u.keep && !kept) {
      const int at = hole_before + (before[i] & 0xffff) + __popcll(hb[i] & below);
      if (source)
        source[j] = -1 - at;
      else
        holes[at] = j;
    }
    if (j >= u.keep && kept) movers[mover_before + (before[i] >> 16) + __popcll(mb[i] & below)] = j;
    if (kept && j < u.keep) {
      if (source) {
        source[j] = j;
      } else {
        if (to_pos != u.pos) to_pos[j] = u.pos[j];
        if (to_wts != u.wts) to_wts[j] = u.wts[j];
      }
    }
  }
  return total;
}

template <int PER>
__global__ __launch_bounds__(EVICT_THREADS) void evict_select_kernel(const EvictArgs a) {
  __shared__ EvictShared sh;
  const int tid = threadIdx.x;
  const EvictUnit u = evict_unit(a, blockIdx.x);
  if (u.len == 0 || (u.len <= a.n_keep && !a.source && a.to_positions == a.positions && a.to_weights == a.weights)) {
    if (tid == 0) {  // nothing to do
      a.count[2 * u.unit] = 0;
      a.count[2 * u.unit + 1] = u.keep;
    }
    return;
  }
  uint32_t key[PER];
  EvictRows<PER> rows;
  rows.load(u, 0, u.len);
  rows.keys(a, u, key);
  uint32_t threshold = 0;
  int need = u.len;  // nothing leaves: every key is at least 0
  if (u.len > a.n_keep) {
    need = u.keep;
    threshold = 0xffffffffu;
    if (need > 0) {
      threshold = 0;
      for (int pass = 0; pass < 3; ++pass) {
        evict_count<PER>(sh, key, 0, u.len, pass, threshold);
        const int top = EVICT_BUCKETS - 1 - 2 * tid;
        const int2 at = evict_bucket(sh, (int)sh.hist[top], (int)sh.hist[top - 1], need);
        threshold = (threshold << digit_bits(pass)) | (uint32_t)at.x;
        need -= at.y;
      }
    }
  }
  const int total = evict_list<PER>(sh, a, u, key, 0, u.len, threshold, need, 0, 0, 0);
  if (tid == 0) {
    a.count[2 * u.unit] = total & 0xffff;
    a.count[2 * u.unit + 1] = u.keep;
  }
}

// Rows of slice s: those below the budget and those from it on are cut on their own, so that a slice has holes or movers.
__device__ __forceinline__ int2 slice_rows(const EvictArgs& a, const EvictUnit& u, int s) {
  const bool low = s < a.keep_slices;
  const int from = low ? 0 : u.keep, to = low ? u.keep : u.len;
  const int r0 = min((long long)from + (long long)(low ? s : s - a.keep_slices) * SLICE_ROWS, (long long)to);
  return make_int2(r0, min(r0 + SLICE_ROWS, to));
}
__device__ __forceinline__ int2 slices_bucket(EvictShared& sh, const EvictArgs& a, const uint32_t* hist, int need) {
  const int top = EVICT_BUCKETS - 1 - 2 * (int)threadIdx.x;
  int c0 = 0, c1 = 0;
  for (int s0 = 0; s0 < a.slices; s0 += 8) {
    uint2 c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      c[k] = *reinterpret_cast<const uint2*>(hist + (size_t)min(s0 + k, a.slices - 1) * EVICT_BUCKETS + top - 1);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      c0 += s0 + k < a.slices ? (int)c[k].y : 0;
      c1 += s0 + k < a.slices ? (int)c[k].x : 0;
    }
  }
  return evict_bucket(sh, c0, c1, need);
}

// Histogram number PASS of a slice; the threshold's digit before comes from the histograms of all slices of the unit.
template <int PASS>
__global__ __launch_bounds__(EVICT_THREADS) void evict_slice_kernel(const EvictArgs a) {
  __shared__ EvictShared sh;
  const int unit = blockIdx.x / a.slices, s = blockIdx.x % a.slices, tid = threadIdx.x;
  const EvictUnit u = evict_unit(a, unit);
  if (u.len <= a.n_keep || u.keep == 0) return;
  const int2 r = slice_rows(a, u, s);
  EvictRows<SLICE_PER> rows;
  rows.load(u, r.x, r.y);
  uint32_t key[SLICE_PER], prefix = 0;
  if (PASS == 0) rows.keys(a, u, key);
  const size_t at = (size_t)unit * a.slices;
  if (PASS > 0) {
    const int4 st = PASS == 1 ? make_int4(0, u.keep, 0, 0) : a.state[2 * unit + PASS - 2];
    const int2 found = slices_bucket(sh, a, (PASS == 1 ? a.hist_a : a.hist_b) + at * EVICT_BUCKETS, st.y);
    const uint32_t old = (uint32_t)st.x;
    prefix = (old << digit_bits(PASS - 1)) | (uint32_t)found.x;
    rows.keys(a, u, key);
    if (s == 0 && tid == 0) a.state[2 * unit + PASS - 1] = make_int4((int)prefix, st.y - found.y, 0, 0);
    // this slice's rows that are above by their digit before
    int above = 0;
#pragma unroll
    for (int i = 0; i < SLICE_PER; ++i) {
      const uint32_t upper = key[i] >> digit_shift(PASS - 1);
      const bool row = r.x + i * EVICT_THREADS + tid < r.y;
      above += __popcll(__ballot(row && (PASS == 1 || upper >> digit_bits(PASS - 1) == old) && upper > prefix));
    }
    if ((tid & 63) == 0) sh.table[tid >> 6] = above;
    __syncthreads();
    if (tid == 0) {
      int sum = PASS == 1 ? 0 : a.above[at + s];
      for (int w = 0; w < EVICT_WAVES; ++w) sum += sh.table[w];
      a.above[at + s] = sum;
    }
  }
  evict_count<SLICE_PER>(sh, key, r.x, r.y, PASS, prefix);
  uint32_t* out = (PASS == 1 ? a.hist_b : a.hist_a) + (at + s) * EVICT_BUCKETS;
  for (int i = tid; i < EVICT_BUCKETS; i += EVICT_THREADS) out[i] = sh.hist[i];
}

// (64 registers: two workgroups a CU.  64 sequences x 4 units of 30000 rows 56 -> 47 us; one workgroup a CU or less 1 us more.)
__global__ __launch_bounds__(EVICT_THREADS, 8) void evict_emit_kernel(const EvictArgs a) {
  __shared__ EvictShared sh;
  const int unit = blockIdx.x / a.slices, s = blockIdx.x % a.slices, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const EvictUnit u = evict_unit(a, unit);
  const int2 r = slice_rows(a, u, s);
  EvictRows<SLICE_PER> rows;
  rows.load(u, r.x, r.y);
  const bool all = u.len <= a.n_keep, none = u.keep == 0;
  const size_t at = (size_t)unit * a.slices;
  uint32_t threshold = all ? 0u : 0xffffffffu;
  int need = all ? u.len : 0, equal_before = 0, hole_before = 0, mover_before = 0, holes = 0;
  if (!all && !none) {
    const int4 st = a.state[2 * unit + 1];
    const uint32_t* hist = a.hist_a + at * EVICT_BUCKETS;
    const int2 found = slices_bucket(sh, a, hist, st.y);
    threshold = ((uint32_t)st.x << digit_bits(2)) | (uint32_t)found.x;
    need = st.y - found.y;
    // Sixteen slices at a time: their rows above and at the threshold, a wave each; then, a lane each, what lies before this
    // slice.
    int seen_equal = 0, kept_low = 0, kept_high_before = 0, kept_low_before = 0;
    for (int s0 = 0; s0 < a.slices; s0 += EVICT_WAVES) {
      int above = 0;
      uint4 c[4];  // 1024 buckets
#pragma unroll
      for (int k = 0; k < 4; ++k)
        c[k] = load16(hist + (size_t)min(s0 + wave, a.slices - 1) * EVICT_BUCKETS + (k * 64 + lane) * 4);
      const int before = a.above[at + min(s0 + wave, a.slices - 1)];
      const int same = (int)hist[(size_t)min(s0 + wave, a.slices - 1) * EVICT_BUCKETS + found.x];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = (k * 64 + lane) * 4;
        above += (i > found.x ? (int)c[k].x : 0) + (i + 1 > found.x ? (int)c[k].y : 0) + (i + 2 > found.x ? (int)c[k].z : 0) +
                 (i + 3 > found.x ? (int)c[k].w : 0);
      }
      above = wave_sum_i(above);
      if (lane == 0) {
        sh.table[2 * wave] = s0 + wave < a.slices ? above + before : 0;
        sh.table[2 * wave + 1] = s0 + wave < a.slices ? same : 0;
      }
      __syncthreads();
      const int x = s0 + lane, equal = lane < EVICT_WAVES ? sh.table[2 * lane + 1] : 0;
      const int seen = seen_equal + wave_incl_scan(equal);
      const int kept = lane < EVICT_WAVES ? sh.table[2 * lane] + min(max(need - (seen - equal), 0), equal) : 0;
      const bool low = x < a.keep_slices;
      if (s >= s0 && s < s0 + EVICT_WAVES) equal_before = __builtin_amdgcn_readlane(seen - equal, s - s0);
      kept_low += wave_sum_i(low ? kept : 0);
      kept_low_before += wave_sum_i(low && x < s ? kept : 0);
      kept_high_before += wave_sum_i(!low && x < s ? kept : 0);
      seen_equal = __builtin_amdgcn_readlane(seen, 63);
      __syncthreads();
    }
    hole_before = s < a.keep_slices ? r.x - kept_low_before : 0;
    mover_before = kept_high_before;
    holes = u.keep - kept_low;
  }
  if (s == 0 && tid == 0) {
    a.count[2 * unit] = holes;
    a.count[2 * unit + 1] = u.keep;
  }
  if (r.x < r.y) {
    uint32_t key[SLICE_PER];
    rows.keys(a, u, key);
    evict_list<SLICE_PER>(sh, a, u, key, r.x, r.y, threshold, need, equal_before, hole_before, mover_before);
  }
}

// In place: move i of the lists.  Apart: row i of the new cache.  ROW / 16 lanes carry a row of K and of V, one row a thread
// (283 MB of scattered rows: 50 us, 63 us with four in flight a thread and a quarter of the workgroups).
template <int ROW>
constexpr int kMoveRows = 256 / (ROW / 16);
template <int ROW>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a, int chunks) {
  constexpr int LPR = ROW / 16;
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks, b = unit / a.Hkv;
  const int moved = a.count[2 * unit], keep = a.count[2 * unit + 1];
  if (chunk == 0 && unit % a.Hkv == 0 && threadIdx.x == 0) {
    a.to_lengths[b] = keep;
    a.to_tokens[b] = a.tokens[b];
  }
  const int i = chunk * kMoveRows<ROW> + (int)threadIdx.x / LPR, lane = threadIdx.x % LPR;
  if (i >= (a.source ? keep : moved)) return;
  const int32_t* movers = a.mover + (size_t)unit * a.moves;
  int src, dst;
  if (a.source) {
    dst = i;
    src = a.source[(size_t)unit * a.n_keep + i];
    if (src < 0) src = movers[-1 - src];
  } else {
    dst = a.hole[(size_t)unit * a.moves + i];
    src = movers[i];
  }
  const size_t from = (size_t)unit * a.capacity + src, to = (size_t)unit * a.to_capacity + dst;
  const uint4 k = load16_stream(a.k + from * ROW + lane * 16), v = load16_stream(a.v + from * ROW + lane * 16);
  store16(a.to_k + to * ROW + lane * 16, k);
  store16(a.to_v + to * ROW + lane * 16, v);
  if (lane == 0) {
    a.to_positions[to] = a.positions[from];
    a.to_weights[to] = a.weights[from];
  }
}

template <typename T, int D>
wave_status rotary_td(const void* x, const int32_t* coords, const RotaryArgs& rot, int B, int H, int N, void* y,
                      hipStream_t st) {
  const TurnShape sh = turn_shape<Turn<T, D>::ITEMS>(N, B, H);
  const int tiles = (N + sh.tokens - 1) / sh.tokens;
  const dim3 grid = grid_rows((long long)B * tiles * sh.head_groups);
  WAVE_LAUNCH("rotary", (rotary_kernel<T, D>), grid, 256, 0, st, static_cast<const char*>(x), coords, rot, B, H,
              N, sh, tiles, static_cast<char*>(y));
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

template <typename T, int D>
wave_status append_td(const AppendArgs& a, const RotaryArgs* rot, hipStream_t st) {
  const TurnShape sh = turn_shape<Turn<T, D>::ITEMS>(a.n, a.B, a.Hq + 2 * a.Hkv);
  const int tiles = (a.n + sh.tokens - 1) / sh.tokens;
  const dim3 grid = grid_rows((long long)a.B * tiles * sh.head_groups);
  // Numbers that go into the arrays that they come from wait for the readers: a workgroup that is alone with its
  // sequence knows, otherwise a launch of its own writes them.
  const bool in_place = a.lengths_out == a.lengths || (a.tokens_out && a.tokens_out == a.tokens);
  const bool advance = !in_place || tiles * sh.head_groups == 1;
  if (rot)
    WAVE_LAUNCH("append", (append_kernel<T, D, true>), grid, 256, 0, st, a, *rot, sh, tiles, advance);
  else
    WAVE_LAUNCH("append", (append_kernel<T, D, false>), grid, 256, 0, st, a, RotaryArgs{}, sh, tiles, advance);
  if (!advance) WAVE_LAUNCH("advance", advance_kernel, (a.B + 255) / 256, 256, 0, st, a);
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

}  // namespace

wave_status launch_rotary(const void* x, const int32_t* coords, const RotaryArgs& rot, int dtype, int B, int H, int N,
                          int d, void* y, hipStream_t st) {
  if (dtype == WAVE_BF16)
    return d == 128 ? rotary_td<bf16_t, 128>(x, coords, rot, B, H, N, y, st)
                    : rotary_td<bf16_t, 64>(x, coords, rot, B, H, N, y, st);
  return d == 128 ? rotary_td<float, 128>(x, coords, rot, B, H, N, y, st)
                  : rotary_td<float, 64>(x, coords, rot, B, H, N, y, st);
}

wave_status launch_cache_append(const wave_cache& c, const void* k_new, const void* v_new, const void* q, int Hq,
                                int n_new, const int32_t* counts, const RotaryArgs* rot, const int32_t* coords,
                                void* q_out, int32_t* lengths_out, int32_t* tokens_out, hipStream_t st) {
  AppendArgs a{};
  a.q = static_cast<const char*>(q);
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.q_out = static_cast<char*>(q_out);
  a.k = static_cast<char*>(c.k);
  a.v = static_cast<char*>(c.v);
  a.positions = c.positions;
  a.weights = c.weights;
  a.lengths = c.lengths;
  a.tokens = c.tokens;
  a.counts = counts;
  a.coords = coords;
  a.lengths_out = lengths_out;
  a.tokens_out = tokens_out;
  a.B = c.B;
  a.Hq = Hq;
  a.Hkv = c.Hkv;
  a.n = n_new;
  a.capacity = c.capacity;
  if (c.dtype == WAVE_BF16) return c.d == 128 ? append_td<bf16_t, 128>(a, rot, st) : append_td<bf16_t, 64>(a, rot, st);
  return c.d == 128 ? append_td<float, 128>(a, rot, st) : append_td<float, 64>(a, rot, st);
}

CacheEvictGeom cache_evict_geometry(const wave_cache& c, int n_keep) {
  CacheEvictGeom g{};
  const size_t units = (size_t)c.B * c.Hkv;
  const int kept = n_keep < c.capacity ? n_keep : c.capacity, rest = c.capacity - kept;
  g.moves = kept < rest ? kept : rest;
  if (c.capacity > 16 * EVICT_THREADS) {
    g.keep_slices = (int)(((long long)kept + SLICE_ROWS - 1) / SLICE_ROWS);
    g.slices = g.keep_slices + (int)(((long long)rest + SLICE_ROWS - 1) / SLICE_ROWS);
  }
  const size_t list = align_up(units * g.moves * sizeof(int32_t));
  const size_t hist = align_up(units * g.slices * EVICT_BUCKETS * sizeof(uint32_t));
  size_t o = 0;
  g.off_count = o;   o = align_up(o + units * 2 * sizeof(int32_t));
  g.off_hole = o;    o += list;
  g.off_mover = o;   o += list;
  g.off_source = o;  o = align_up(o + units * kept * sizeof(int32_t));
  g.off_hist_a = o;  o += hist;
  g.off_hist_b = o;  o += hist;
  g.off_state = o;   o = align_up(o + (g.slices ? units * 2 * sizeof(int4) : 0));
  g.off_above = o;   o = align_up(o + units * g.slices * sizeof(int32_t));
  g.total = o;
  return g;
}

template <int ROW>
static void launch_evict_move(const EvictArgs& a, int units, int rows, hipStream_t st) {
  const int chunks = rows > 0 ? (rows + kMoveRows<ROW> - 1) / kMoveRows<ROW> : 1;  // (one writes the lengths)
  WAVE_LAUNCH("evict_move", evict_move_kernel<ROW>, units * chunks, 256, 0, st, a, chunks);
}

template <int PER>
static void launch_evict_select(const EvictArgs& a, int units, hipStream_t st) {
  WAVE_LAUNCH("evict_select", evict_select_kernel<PER>, units, EVICT_THREADS, 0, st, a);
}

wave_status launch_cache_evict(const wave_cache& from, const wave_cache& to, int n_keep, int n_sink, int n_local,
                               void* ws, hipStream_t st) {
  const CacheEvictGeom g = cache_evict_geometry(from, n_keep);
  char* w = static_cast<char*>(ws);
  EvictArgs a{};
  a.positions = from.positions;
  a.lengths = from.lengths;
  a.tokens = from.tokens;
  a.weights = from.weights;
  a.to_positions = to.positions;
  a.to_lengths = to.lengths;
  a.to_tokens = to.tokens;
  a.to_weights = to.weights;
  a.k = static_cast<const char*>(from.k);
  a.v = static_cast<const char*>(from.v);
  a.to_k = static_cast<char*>(to.k);
  a.to_v = static_cast<char*>(to.v);
  a.count = reinterpret_cast<int32_t*>(w + g.off_count);
  a.hole = reinterpret_cast<int32_t*>(w + g.off_hole);
  a.mover = reinterpret_cast<int32_t*>(w + g.off_mover);
  a.source = to.k == from.k ? nullptr : reinterpret_cast<int32_t*>(w + g.off_source);
  a.hist_a = reinterpret_cast<uint32_t*>(w + g.off_hist_a);
  a.hist_b = reinterpret_cast<uint32_t*>(w + g.off_hist_b);
  a.state = reinterpret_cast<int4*>(w + g.off_state);
  a.above = reinterpret_cast<int32_t*>(w + g.off_above);
  a.Hkv = from.Hkv;
  a.capacity = from.capacity;
  a.to_capacity = to.capacity;
  a.n_keep = n_keep < from.capacity ? n_keep : from.capacity;
  a.n_sink = n_sink;
  a.n_local = n_local;
  a.moves = g.moves;
  a.slices = g.slices;
  a.keep_slices = g.keep_slices;
  const int units = from.B * from.Hkv, rows = a.source ? a.n_keep : g.moves;
  const int row_bytes = from.d * (from.dtype == WAVE_BF16 ? 2 : 4), move_rows = 4096 / row_bytes;
  if ((long long)units * ((long long)rows / move_rows + 1) >= (1ll << 24) || (long long)units * g.slices >= (1ll << 22))
    return WAVE_ERR_SHAPE;
  if (g.slices > 0) {
    const int grid = units * g.slices;
    WAVE_LAUNCH("evict_slice", evict_slice_kernel<0>, grid, EVICT_THREADS, 0, st, a);
    WAVE_LAUNCH("evict_slice", evict_slice_kernel<1>, grid, EVICT_THREADS, 0, st, a);
    WAVE_LAUNCH("evict_slice", evict_slice_kernel<2>, grid, EVICT_THREADS, 0, st, a);
    WAVE_LAUNCH("evict_emit", evict_emit_kernel, grid, EVICT_THREADS, 0, st, a);
  } else {
    // As many keys a thread as the room needs, to the row of threads: one more costs 0.2 .. 1 us (128 units, selection and moves:
    // 900 of 1000 rows 8.0 us with one, 8.5 with two; 4100 rows 11.7 with five, 12.2 with six, 12.9 with eight; 8900 rows 16.0
    // with nine, 20.2 with sixteen).
    switch ((from.capacity + EVICT_THREADS - 1) / EVICT_THREADS) {
#define WAVE_PER(n) \
  case n: launch_evict_select<n>(a, units, st); break;
      WAVE_PER(1) WAVE_PER(2) WAVE_PER(3) WAVE_PER(4) WAVE_PER(5) WAVE_PER(6) WAVE_PER(7) WAVE_PER(8)
      WAVE_PER(9) WAVE_PER(10) WAVE_PER(11) WAVE_PER(12) WAVE_PER(13) WAVE_PER(14) WAVE_PER(15) WAVE_PER(16)
#undef WAVE_PER
    }
  }
  switch (row_bytes) {
    case 128: launch_evict_move<128>(a, units, rows, st); break;
    case 256: launch_evict_move<256>(a, units, rows, st); break;
    default: launch_evict_move<512>(a, units, rows, st); break;
  }
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

}  // namespace wave
