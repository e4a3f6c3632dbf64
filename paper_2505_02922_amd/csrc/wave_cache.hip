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

  // position(axis) of the item's token; a circle is `1` in turns, so the nearest whole number of circles comes off
  // without error
  template <typename F>
  __device__ __forceinline__ void init(const RotaryArgs& r, int item, F&& position) {
    const int rotated = r.rot / (2 * EPC);
    turns = item < rotated;
    const bool halves = turns && r.pairing == WAVE_ROTARY_HALVES;
    one = halves ? item : 2 * item;
    two = halves ? item + rotated : 2 * item + 1;
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
  const int group = blockIdx.x % sh.head_groups, bt = blockIdx.x / sh.head_groups;
  const int b = bt / tiles, tile = bt % tiles;
  const int item = threadIdx.x % Tu::ITEMS, lane = (threadIdx.x / Tu::ITEMS) & ((1 << sh.lane_shift) - 1);
  const int n = tile * sh.tokens + (int)(threadIdx.x / Tu::ITEMS >> sh.lane_shift);
  if (n >= N) return;
  Tu t;
  t.init(rot, item, [&](int axis) { return coords[((size_t)axis * B + b) * N + n]; });
  const int step = sh.head_groups << sh.lane_shift;
  for (int h0 = (group << sh.lane_shift) + lane; h0 < H; h0 += TURN_BATCH * step) {
    uint4 u[TURN_BATCH], v[TURN_BATCH];
#pragma unroll
    for (int k = 0; k < TURN_BATCH; ++k) {
      const int h = min(h0 + k * step, H - 1);
      const char* row = x + ((size_t)((size_t)b * H + h) * N + n) * ROW;
      u[k] = load16(row + t.one * 16);
      v[k] = load16(row + t.two * 16);
    }
#pragma unroll
    for (int k = 0; k < TURN_BATCH; ++k)
      if (h0 + k * step < H) {
        char* row = y + ((size_t)((size_t)b * H + h0 + k * step) * N + n) * ROW;
        t.apply(rot, u[k], v[k]);
        store16(row + t.one * 16, u[k]);
        store16(row + t.two * 16, v[k]);
      }
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
  const int group = blockIdx.x % sh.head_groups, bt = blockIdx.x / sh.head_groups;
  const int b = bt / tiles, tile = bt % tiles;
  const int item = threadIdx.x % Tu::ITEMS, lane = (threadIdx.x / Tu::ITEMS) & ((1 << sh.lane_shift) - 1);
  const int n = tile * sh.tokens + (int)(threadIdx.x / Tu::ITEMS >> sh.lane_shift);
  const Share s = append_share(a, b);
  const int slots = a.Hq + 2 * a.Hkv, row = s.length + n;
  if (n < s.count) {
    Tu t;
    if (ROT) {
      t.init(rot, item, [&](int axis) { return a.coords ? a.coords[((size_t)axis * a.B + b) * a.n + n] : s.first + n; });
    } else {
      t.turns = false;
      t.one = 2 * item;
      t.two = 2 * item + 1;
    }
    const int step = sh.head_groups << sh.lane_shift;
    for (int h0 = (group << sh.lane_shift) + lane; h0 < slots; h0 += TURN_BATCH * step) {
      uint4 u[TURN_BATCH], v[TURN_BATCH];
      char* to[TURN_BATCH];
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
#pragma unroll
      for (int i = 0; i < TURN_BATCH; ++i)
        if (to[i]) {
          if (ROT && h0 + i * step < a.Hq + a.Hkv) t.apply(rot, u[i], v[i]);
          store16(to[i] + t.one * 16, u[i]);
          store16(to[i] + t.two * 16, v[i]);
        }
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
// Eviction.  evict_select_kernel: one workgroup per unit finds the n_keep-th largest key by three histogram sweeps
// (11, 11 and 10 bits), then lists, in ascending order, the holes (rows below n_keep that leave) and the movers (rows
// from n_keep on that stay); there are as many of one as of the other.  evict_move_kernel copies K and V rows.
// ----------------------------------------------------------------------------
struct EvictArgs {
  const int32_t *positions, *lengths, *tokens;
  const float* weights;
  int32_t *to_positions, *to_lengths, *to_tokens;
  float* to_weights;
  const char *k, *v;
  char *to_k, *to_v;
  int32_t *count, *hole, *mover, *source;  // source: NULL where K and V stay in place
  int Hkv, capacity, to_capacity, n_keep, n_sink, n_local, moves;
};

// Order of the rows as integers: what has to stay above every weight, what is no number below.
__device__ __forceinline__ uint32_t evict_key(float w, int position, int n_sink, long long local) {
  if (position < n_sink || position >= local) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 counts as 0
  return ((u >> 31) ? ~u : (u | 0x80000000u)) ;
}

constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / 64;

__global__ __launch_bounds__(EVICT_THREADS) void evict_select_kernel(const EvictArgs a) {
  __shared__ uint32_t hist[2048];
  __shared__ int wave_total[EVICT_WAVES][2];
  __shared__ uint32_t bucket_at;
  __shared__ int above_at;
  const int unit = blockIdx.x, b = unit / a.Hkv, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int len = min(max(a.lengths[b], 0), a.capacity);
  const long long local = (long long)a.tokens[b] - a.n_local;
  const int32_t* pos = a.positions + (size_t)unit * a.capacity;
  const float* wts = a.weights + (size_t)unit * a.capacity;
  int32_t* to_pos = a.to_positions + (size_t)unit * a.to_capacity;
  float* to_wts = a.to_weights + (size_t)unit * a.to_capacity;
  int32_t* source = a.source ? a.source + (size_t)unit * a.n_keep : nullptr;
  const bool copy_pos = to_pos != pos, copy_wts = to_wts != wts;
  const int keep = min(len, a.n_keep);
  if (tid == 0) {
    a.count[2 * unit] = 0;
    a.count[2 * unit + 1] = keep;
  }
  if (len <= a.n_keep) {
    for (int j = tid; j < len; j += EVICT_THREADS) {
      if (copy_pos) to_pos[j] = pos[j];
      if (copy_wts) to_wts[j] = wts[j];
      if (source) source[j] = j;
    }
    return;
  }
  if (keep == 0) return;
  auto key_of = [&](int j) { return evict_key(wts[j], pos[j], a.n_sink, local); };
  // the keep-th largest key: its upper bits one histogram at a time
  uint32_t prefix = 0;
  int need = keep;  // how many of the rows that share the prefix are kept
  const int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = shifts[pass], buckets = 1 << widths[pass];
    for (int i = tid; i < 2048; i += EVICT_THREADS) hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < len; j += EVICT_THREADS) {
      const uint32_t key = key_of(j);
      if (pass == 0 || (key >> (shift + widths[pass])) == prefix) atomicAdd(&hist[(key >> shift) & (buckets - 1)], 1u);
    }
    __syncthreads();
    // thread t has the buckets 2 t and 2 t + 1, counted from the top
    const int top = 2047 - 2 * tid;
    const int c0 = (int)hist[top], c1 = (int)hist[top - 1];
    const int incl = wave_incl_scan(c0 + c1);
    if (lane == 63) wave_total[wave][0] = incl;
    __syncthreads();
    int before = incl - c0 - c1;
    for (int w = 0; w < wave; ++w) before += wave_total[w][0];
    if (before < need && before + c0 >= need) {
      bucket_at = (uint32_t)top;
      above_at = before;
    } else if (before + c0 < need && before + c0 + c1 >= need) {
      bucket_at = (uint32_t)top - 1;
      above_at = before + c0;
    }
    __syncthreads();
    prefix = pass == 0 ? bucket_at : (prefix << widths[pass]) | bucket_at;
    need -= above_at;
    __syncthreads();
  }
  const uint32_t threshold = prefix;  // `need` of the rows with this key are kept, the lowest ones
  int32_t* holes = a.hole + (size_t)unit * a.moves;
  int32_t* movers = a.mover + (size_t)unit * a.moves;
  int equal_before = 0, listed = 0;  // rows with the threshold's key so far; holes, and from row n_keep on movers
  int n_holes = 0;
  for (int j0 = 0; j0 < len; j0 += EVICT_THREADS) {
    const int j = j0 + tid;
    const uint32_t key = j < len ? key_of(j) : 0u;
    const bool equal = j < len && key == threshold;
    const uint64_t eq = __ballot(equal), below = (1ull << lane) - 1;
    if (lane == 0) wave_total[wave][0] = __popcll(eq);
    __syncthreads();
    int rank = equal_before + __popcll(eq & below);
    int eq_all = 0;
    for (int w = 0; w < EVICT_WAVES; ++w) {
      if (w < wave) rank += wave_total[w][0];
      eq_all += wave_total[w][0];
    }
    equal_before += eq_all;
    const bool kept = j < len && (key > threshold || (equal && rank < need));
    const bool hole = j < keep && !kept, mover = j >= keep && kept;
    const uint64_t hb = __ballot(hole), mb = __ballot(mover);
    if (lane == 0) wave_total[wave][1] = __popcll(hb) | (__popcll(mb) << 16);
    __syncthreads();
    int hole_at = n_holes + __popcll(hb & below), mover_at = listed + __popcll(mb & below), all = 0;
    for (int w = 0; w < EVICT_WAVES; ++w) {
      if (w < wave) {
        hole_at += wave_total[w][1] & 0xffff;
        mover_at += wave_total[w][1] >> 16;
      }
      all += wave_total[w][1];
    }
    n_holes += all & 0xffff;
    listed += all >> 16;
    if (hole) holes[hole_at] = j;
    if (mover) movers[mover_at] = j;
    if (kept && j < keep) {
      if (copy_pos) to_pos[j] = pos[j];
      if (copy_wts) to_wts[j] = wts[j];
      if (source) source[j] = j;
    }
  }
  __syncthreads();  // the lists are complete and no key is read any more
  for (int i = tid; i < n_holes; i += EVICT_THREADS) {
    const int h = holes[i], m = movers[i];
    to_pos[h] = pos[m];
    to_wts[h] = wts[m];
    if (source) source[h] = m;
  }
  if (tid == 0) a.count[2 * unit] = n_holes;
}

constexpr int MOVE_ROWS = 64;  // rows of K and of V of one workgroup

// In place: pair i of the lists.  Apart: row i of the new cache.  D * es / 16 lanes carry a row, four rows of each of K
// and V in flight a thread.
template <int ROW>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a, int chunks) {
  constexpr int LPR = ROW / 16, GROUPS = 256 / LPR;
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks, b = unit / a.Hkv;
  const int moved = a.count[2 * unit], keep = a.count[2 * unit + 1];
  if (chunk == 0 && unit % a.Hkv == 0 && threadIdx.x == 0) {
    a.to_lengths[b] = keep;
    a.to_tokens[b] = a.tokens[b];
  }
  const int total = a.source ? keep : moved;
  const int lane = threadIdx.x % LPR, end = min(total, (chunk + 1) * MOVE_ROWS);
  constexpr int U = 4;
  for (int i0 = chunk * MOVE_ROWS + (int)threadIdx.x / LPR; i0 < end; i0 += U * GROUPS) {
    uint4 kk[U], vv[U];
    int dst[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * GROUPS, end - 1);
      const int src = a.source ? a.source[(size_t)unit * a.n_keep + i] : a.mover[(size_t)unit * a.moves + i];
      dst[u] = a.source ? i : a.hole[(size_t)unit * a.moves + i];
      const size_t at = ((size_t)unit * a.capacity + src) * ROW + lane * 16;
      kk[u] = load16_stream(a.k + at);
      vv[u] = load16_stream(a.v + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * GROUPS < end) {
        const size_t at = ((size_t)unit * a.to_capacity + dst[u]) * ROW + lane * 16;
        store16(a.to_k + at, kk[u]);
        store16(a.to_v + at, vv[u]);
      }
  }
}

template <typename T, int D>
wave_status rotary_td(const void* x, const int32_t* coords, const RotaryArgs& rot, int B, int H, int N, void* y,
                      hipStream_t st) {
  const TurnShape sh = turn_shape<Turn<T, D>::ITEMS>(N, B, H);
  const int tiles = (N + sh.tokens - 1) / sh.tokens;
  const long long grid = (long long)B * tiles * sh.head_groups;
  if (grid >= (1ll << 24)) return WAVE_ERR_SHAPE;
  WAVE_LAUNCH("rotary", (rotary_kernel<T, D>), (unsigned)grid, 256, 0, st, static_cast<const char*>(x), coords, rot, B, H,
              N, sh, tiles, static_cast<char*>(y));
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

template <typename T, int D>
wave_status append_td(const AppendArgs& a, const RotaryArgs* rot, hipStream_t st) {
  const TurnShape sh = turn_shape<Turn<T, D>::ITEMS>(a.n, a.B, a.Hq + 2 * a.Hkv);
  const int tiles = (a.n + sh.tokens - 1) / sh.tokens;
  const long long grid = (long long)a.B * tiles * sh.head_groups;
  if (grid >= (1ll << 24)) return WAVE_ERR_SHAPE;
  // Numbers that go into the arrays that they come from wait for the readers: a workgroup that is alone with its
  // sequence knows, otherwise a launch of its own writes them.
  const bool in_place = a.lengths_out == a.lengths || (a.tokens_out && a.tokens_out == a.tokens);
  const bool advance = !in_place || tiles * sh.head_groups == 1;
  if (rot)
    WAVE_LAUNCH("append", (append_kernel<T, D, true>), (unsigned)grid, 256, 0, st, a, *rot, sh, tiles, advance);
  else
    WAVE_LAUNCH("append", (append_kernel<T, D, false>), (unsigned)grid, 256, 0, st, a, RotaryArgs{}, sh, tiles, advance);
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
  g.moves = n_keep < c.capacity ? (n_keep < c.capacity - n_keep ? n_keep : c.capacity - n_keep) : 0;
  const size_t list = align_up(units * g.moves * sizeof(int32_t));
  const size_t kept = n_keep < c.capacity ? n_keep : c.capacity;
  size_t o = 0;
  g.off_count = o;   o = align_up(o + units * 2 * sizeof(int32_t));
  g.off_hole = o;    o += list;
  g.off_mover = o;   o += list;
  g.off_source = o;  o = align_up(o + units * kept * sizeof(int32_t));
  g.total = o;
  return g;
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
  a.Hkv = from.Hkv;
  a.capacity = from.capacity;
  a.to_capacity = to.capacity;
  a.n_keep = n_keep < from.capacity ? n_keep : from.capacity;
  a.n_sink = n_sink;
  a.n_local = n_local;
  a.moves = g.moves;
  const int units = from.B * from.Hkv, rows = a.source ? a.n_keep : g.moves;
  const int chunks = rows > 0 ? (rows + MOVE_ROWS - 1) / MOVE_ROWS : 1;
  if ((long long)units * chunks >= (1ll << 24)) return WAVE_ERR_SHAPE;
  WAVE_LAUNCH("evict_select", evict_select_kernel, units, EVICT_THREADS, 0, st, a);
  switch (from.d * (from.dtype == WAVE_BF16 ? 2 : 4)) {
    case 128: WAVE_LAUNCH("evict_move", evict_move_kernel<128>, units * chunks, 256, 0, st, a, chunks); break;
    case 256: WAVE_LAUNCH("evict_move", evict_move_kernel<256>, units * chunks, 256, 0, st, a, chunks); break;
    default: WAVE_LAUNCH("evict_move", evict_move_kernel<512>, units * chunks, 256, 0, st, a, chunks); break;
  }
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

}  // namespace wave
