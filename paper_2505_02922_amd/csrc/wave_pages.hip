// Norms with rotary positions, and the rows of the paged cache: appending new tokens, reading rows back, sharing pages.
#include "wave_rotary.h"

namespace wave {

namespace {

// ----------------------------------------------------------------------------
// Norms with rotary positions.  A work item is an item of a turn (wave_rotary.h): two 16-byte chunks of a row.  The lanes of a row
// add up its squares with DPP.  A workgroup forms the sines of its rows once, a pair of channels a thread, and leaves them in LDS:
// in registers they took eight copies of their code in every thread, which a decode step fetches from memory before it runs
// (one token of 64 sequences: 5.4 us so, 4.2 now), and eight lanes' work for each of a token's heads.
// Every fused multiply-add is written out: a row has the same bits whichever kernel, and whichever form of it, norms and turns it.
// ----------------------------------------------------------------------------
template <int LANES>
__device__ __forceinline__ float item_sum(float x) {
  static_assert(LANES == 4 || LANES == 8 || LANES == 16, "lanes of a row");
  x += dpp<DPP_XOR1>(x);
  x += dpp<DPP_XOR2>(x);
  if (LANES >= 8) x += dpp<DPP_HALF_MIRROR>(x);
  if (LANES >= 16) x += dpp<DPP_MIRROR>(x);
  return x;
}

// 1 / sqrt(x): the instruction's, which is off by a last place, and one step of Newton's iteration, unless that is infinite or zero.
__device__ __forceinline__ float inverse_root(float x) {
  const float r = rsqrtf(x), better = fmaf(0.5f * r, fmaf(-x * r, r, 1.f), r);
  return better == better ? better : r;
}

constexpr int THREADS = 256;

template <typename T, int D>
struct RowItem {
  static constexpr int EPC = Elem<T>::EPC, ITEMS = D / (2 * EPC), PAIRS = D / 2;
  struct Sines { float c[EPC], s[EPC]; };
  struct Weight {
    uint4 a, b;
    bool any;
  };
  int item, one, two;  // its chunks
  bool turns, halves;

  __device__ __forceinline__ void place(const RotaryArgs& r, bool rotates, int at) {
    const int rotated = rotates ? r.rot / (2 * EPC) : 0;
    item = at;
    turns = item < rotated;
    halves = turns && r.pairing == WAVE_ROTARY_HALVES;
    one = halves ? item : 2 * item;
    two = halves ? item + rotated : 2 * item + 1;
  }
  __device__ __forceinline__ Weight weight(const char* w) const {
    Weight r;
    r.any = w != nullptr;
    if (r.any) {
      r.a = load16(w + one * 16);
      r.b = load16(w + two * 16);
    }
    return r;
  }
  static __device__ __forceinline__ void pair(float& x, float& y, float c, float s) {
    const float u = fmaf(x, c, -(y * s));
    y = fmaf(x, s, y * c);
    x = u;
  }
  // All lanes of the row together.  (x * (1 / norm)) * w in fp32, then the turn, then one rounding.
  __device__ __forceinline__ void apply(const Weight& w, const Sines& t, float eps, uint4& a, uint4& b) const {
    if (!w.any && !turns) return;
    float x[EPC], y[EPC];
    unpack<T>(a, x);
    unpack<T>(b, y);
    if (w.any) {
      float sum_x = 0.f, sum_y = 0.f;
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        sum_x = fmaf(x[e], x[e], sum_x);
        sum_y = fmaf(y[e], y[e], sum_y);
      }
      const float f = inverse_root(fmaf(item_sum<ITEMS>(sum_x + sum_y), 1.f / D, eps));
      float u[EPC], v[EPC];
      unpack<T>(w.a, u);
      unpack<T>(w.b, v);
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        x[e] = x[e] * f * u[e];
        y[e] = y[e] * f * v[e];
      }
    }
    if (turns && halves) {
#pragma unroll
      for (int e = 0; e < EPC; ++e) pair(x[e], y[e], t.c[e], t.s[e]);
    } else if (turns) {  // pairs of the first and of the second chunk
#pragma unroll
      for (int e = 0; e < EPC; e += 2) {
        pair(x[e], x[e + 1], t.c[e / 2], t.s[e / 2]);
        pair(y[e], y[e + 1], t.c[EPC / 2 + e / 2], t.s[EPC / 2 + e / 2]);
      }
    }
    a = pack<T>(x);
    b = pack<T>(y);
  }
};

// Cosine (x) and sine (y) of `turns` circles, off by less than 0.88 of a last place (0.873 the most of 2 * 10^8 angles around an eighth of
// a circle, where both are furthest off; 0.84 of 3 * 10^7 anywhere): the angle is cut to an eighth of a circle in fp64, where whole and quarter circles come off without error, and its series (x^9 and x^10 in the last terms, the next ones
// are below 2^-28 of the sums) take it as two floats.  (A function of one float is off by pi u for the rounding of its argument, and
// by its own last places: four times as many rows would then be rounded to bf16 the other way.)
__device__ __forceinline__ float2 cosine_and_sine(double turns) {
  const double part = turns - rint(turns), quarters = rint(part * 4.0), angle = fma(quarters, -0.25, part) * 6.283185307179586477;
  const float x = (float)angle, rest = (float)(angle - (double)x), z = x * x, z_rest = fmaf(x, x, -z);
  const float sine_terms = z * fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
  const float sine = x + fmaf(x, sine_terms, rest);
  const float near = fmaf(z, -0.5f, 1.f), lost = fmaf(z, -0.5f, 1.f - near);  // 1 - z / 2 and what its rounding left
  const float cosine_terms = fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f);
  const float cosine = near + fmaf(z * z, cosine_terms, fmaf(x, -rest, fmaf(z_rest, -0.5f, lost)));
  const int q = (int)quarters;
  const float c = q & 1 ? sine : cosine, s = q & 1 ? cosine : sine;
  return make_float2((q + 1) & 2 ? -c : c, q & 2 ? -s : s);
}

// Cosines and sines of ROWS rows in LDS, a row's [two pairs of an item][item], so that the items of a row read neighbouring 16
// bytes.
template <typename T, int D, int ROWS>
struct SineTable {
  typedef RowItem<T, D> Item;
  static constexpr int PAIRS = Item::PAIRS, EPC = Item::EPC, ITEMS = Item::ITEMS, SIDE = THREADS / PAIRS;
  float4 pairs[ROWS][PAIRS / 2];
  int position[WAVE_ROTARY_MAX_AXES][ROWS];
  // Rows r0 .. r1 - 1; at(axis, row).  All threads together; the table is whole behind the call.
  template <typename F>
  __device__ __forceinline__ void fill(const RotaryArgs& rot, int r0, int r1, F&& at) {
    static_assert(ROWS <= THREADS, "");
    const int mine = threadIdx.x % ROWS;
    if (mine >= r0 && mine < r1)
      for (int axis = threadIdx.x / ROWS; axis < rot.n_axes; axis += THREADS / ROWS) position[axis][mine] = at(axis, mine);
    const int i = threadIdx.x % PAIRS, item = i / EPC, e = i % EPC;
    const bool any = i < rot.rot / 2;
    const int axis = any ? rot.axis[i] : 0;
    const double per = any ? rot.turns[i] : 0.0;
    __syncthreads();
    if (any) {
#pragma unroll 1
      for (int r = r0 + threadIdx.x / PAIRS; r < r1; r += SIDE) {
        reinterpret_cast<float2*>(&pairs[r][(e >> 1) * ITEMS + item])[e & 1] = cosine_and_sine((double)position[axis][r] * per);
      }
    }
    __syncthreads();
  }
  __device__ __forceinline__ void get(int row, int item, typename Item::Sines& t) const {
#pragma unroll
    for (int k = 0; k < EPC / 2; ++k) {
      const float4 x = pairs[row][k * ITEMS + item];
      t.c[2 * k] = x.x;
      t.s[2 * k] = x.y;
      t.c[2 * k + 1] = x.z;
      t.s[2 * k + 1] = x.w;
    }
  }
};

__device__ __forceinline__ const char* row_of(const HeadRows& r, int b, int h, int n) {
  return r.data + (b * r.b + h * r.h + n * r.n);
}

// Outputs of more than the eight L2s hold (32 MB) pass by the caches, as every input does, which is read once (40 heads of 32762 tokens,
// 671 MB: 135 us, 144 otherwise; 126 and 135 from dense rows; 5 TB/s, what a copy reaches).
constexpr size_t PAST_BYTES = size_t(32) << 20;

// The heads of a token are its q, k and v heads in this order; v's are only handed on.  count(): tokens that there are;
// position(axis, n); out(h, n): where a head's row goes (NULL: nowhere).
template <typename T, int D, int ROWS, typename Count, typename Position, typename Out>
__device__ __forceinline__ void norm_heads(const NormArgs& a, const HeadRows& values, int Hv, const RotaryArgs& rot, const TurnShape& sh,
                                           int b, int tile, int group, SineTable<T, D, ROWS>& table, Count&& count, Position&& position,
                                           Out&& out) {
  typedef RowItem<T, D> Item;
  const int item = threadIdx.x % Item::ITEMS, lane = (threadIdx.x / Item::ITEMS) & ((1 << sh.lane_shift) - 1);
  const int row = (int)(threadIdx.x / Item::ITEMS >> sh.lane_shift), first = tile * sh.tokens, n = first + row;
  Item t;
  t.place(rot, a.turns, item);
  const int row_n = min(n, a.N - 1), heads = a.Hq + a.Hk, slots = heads + Hv, step = sh.head_groups << sh.lane_shift;
  uint4 u[TURN_BATCH], v[TURN_BATCH];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < TURN_BATCH; ++i) {
      const int h = min(h0 + i * step, slots - 1);
      const char* at = h < a.Hq ? row_of(a.q, b, h, row_n) : h < heads ? row_of(a.k, b, h - a.Hq, row_n) : row_of(values, b, h - heads, row_n);
      u[i] = load16_stream(at + t.one * 16);
      v[i] = load16_stream(at + t.two * 16);
    }
  };
  // the first rows are on their way while the count is read and the sines are formed
  int h0 = (group << sh.lane_shift) + lane;
  load(h0);
  const typename Item::Weight wq = t.weight(a.q_weight), wk = t.weight(a.k_weight);
  const int given = count();
  typename Item::Sines sines;
  if (a.turns) {
    table.fill(rot, 0, min(sh.tokens, given - first), [&](int axis, int r) { return position(axis, first + r); });
    if (t.turns) table.get(row, item, sines);
  }
  if (n >= given) return;
  for (; h0 < slots;) {
#pragma unroll
    for (int i = 0; i < TURN_BATCH; ++i) {
      const int h = h0 + i * step;
      if (h < slots) {
        typename Item::Weight w = wk;
        if (h < a.Hq) w = wq;
        if (h < heads) t.apply(w, sines, a.eps, u[i], v[i]);
        char* to = out(h, n);
        if (!to) continue;
        if (a.past) {
          store16_stream(to + t.one * 16, u[i]);
          store16_stream(to + t.two * 16, v[i]);
        } else {
          store16(to + t.one * 16, u[i]);
          store16(to + t.two * 16, v[i]);
        }
      }
    }
    h0 += TURN_BATCH * step;
    if (h0 < slots) load(h0);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void norm_rotary_kernel(const NormArgs a, const RotaryArgs rot, TurnShape sh, int tiles) {
  constexpr size_t ROW = D * sizeof(T);
  __shared__ SineTable<T, D, THREADS / RowItem<T, D>::ITEMS> table;
  const unsigned block = workgroup_number();
  const int group = block % sh.head_groups, bt = block / sh.head_groups;
  const int b = bt / tiles, tile = bt % tiles;
  if (b >= a.B) return;
  norm_heads<T, D>(
      a, HeadRows{}, 0, rot, sh, b, tile, group, table, [&]() { return a.N; },
      [&](int axis, int n) { return a.coords[((size_t)axis * a.B + b) * a.N + n]; },
      [&](int h, int n) {
        return h < a.Hq ? a.q_out + (((size_t)b * a.Hq + h) * a.N + n) * ROW : a.k_out + (((size_t)b * a.Hk + h - a.Hq) * a.N + n) * ROW;
      });
}

template <typename T, int D>
wave_status norm_rotary_td(NormArgs a, const RotaryArgs& rot, hipStream_t st) {
  constexpr int ITEMS = RowItem<T, D>::ITEMS;
  a.past = (size_t)a.B * (a.Hq + a.Hk) * a.N * D * sizeof(T) > PAST_BYTES;
  const TurnShape sh = turn_shape<ITEMS>(a.N, a.B, a.Hq + a.Hk);
  const int tiles = (a.N + sh.tokens - 1) / sh.tokens;
  WAVE_LAUNCH("norm_rotary", (norm_rotary_kernel<T, D>), grid_rows((long long)a.B * tiles * sh.head_groups), 256, 0, st, a, rot, sh,
              tiles);
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

// ----------------------------------------------------------------------------
// The paged cache
// ----------------------------------------------------------------------------
__host__ __device__ inline int page_shift(int page) { return page == 32 ? 5 : page == 64 ? 6 : 7; }
__host__ __device__ inline int pages_room(const wave_pages& p) { return p.max_pages * p.page + p.page - 1; }
__device__ __forceinline__ int pages_length(const wave_pages& p, int b) { return min(max(p.lengths[b], 0), pages_room(p)); }
__device__ __forceinline__ int page_entry(const wave_pages& p, int b, int i) {
  return min(max(p.table[(size_t)b * p.max_pages + i], 0), p.n_pages - 1);
}

// A workgroup copies `chunks` times 16 bytes.
__device__ __forceinline__ void copy_chunks(const char* x, char* y, int chunks) {
  constexpr int BATCH = 4;
  for (int i = threadIdx.x; i < chunks; i += THREADS * BATCH) {
    uint4 u[BATCH];
#pragma unroll
    for (int e = 0; e < BATCH; ++e) u[e] = load16(x + (size_t)min(i + e * THREADS, chunks - 1) * 16);
#pragma unroll
    for (int e = 0; e < BATCH; ++e)
      if (i + e * THREADS < chunks) store16(y + (size_t)(i + e * THREADS) * 16, u[e]);
  }
}

// Append, first launch (but see OwnToken): one workgroup finds how many tokens of each sequence fit and which pages they take.  A sequence's
// share depends on what those before it take, and the free pages are found by going through references in ascending order,
// so the pages are the same in every run.  It is a chain of loads and scans behind barriers: 4.1 us for 64 sequences and a pool of
// 2600 pages (5.1 with sixteen loads and ballots a thread instead of four wide loads and one scan), and about 1.5 us more for every 16384
// pages in front of the last one wanted: with all but the last eight taken 3.9 us for 2600, 5.0 for 32768, 13.3 for 100000, 98 for a million.
struct PagesPlan {
  int4* sequence;   // [B] rows before, rows after, its first one among the taken pages, tokens given
  int32_t* taken;   // [n_pages] the taken pages in ascending order
  int32_t* last;    // [1] the last one (-1: none)
};
PagesPlan pages_plan(const wave_pages& p, void* ws) {
  char* w = static_cast<char*>(ws);
  PagesPlan r;
  r.last = reinterpret_cast<int32_t*>(w);
  r.sequence = reinterpret_cast<int4*>(w + 256);
  r.taken = reinterpret_cast<int32_t*>(w + 256 + align_up(sizeof(int4) * (size_t)p.B));
  return r;
}

constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64, PLAN_PER = 16, PLAN_ROUND = PLAN_PER * PLAN_THREADS;
constexpr int PLAN_MANY = (1 << 30) - 1;  // sums stop here: more pages than there can be
__device__ __forceinline__ int sum_to_many(int a, int b) { return min(a + b, PLAN_MANY); }
// What the threads before this one have, and all of them together, starting from `sum`; `sum` is then the whole.  Two barriers.
__device__ __forceinline__ int plan_scan(int x, int& sum, int (&part)[PLAN_WAVES]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan(x, 0, sum_to_many), below = __shfl_up(incl, 1);
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int before = sum;
#pragma unroll
  for (int w = 0; w < PLAN_WAVES; ++w) {
    if (w == wave) before = sum;
    sum = sum_to_many(sum, part[w]);
  }
  __syncthreads();
  return sum_to_many(before, lane ? below : 0);
}

// The references of PER pages side by side; pages that there are not count as taken.
template <int PER>
struct PageReferences {
  typedef __attribute__((ext_vector_type(4), aligned(4))) int int4_of_ints;
  int4_of_ints ref[PER / 4];
  __device__ __forceinline__ void load(const wave_pages& p, int first) {
    if (first + PER <= p.n_pages) {
#pragma unroll
      for (int i = 0; i < PER / 4; ++i) ref[i] = *reinterpret_cast<const int4_of_ints*>(p.references + first + i * 4);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = p.references[min(first + i, p.n_pages - 1)];
        ref[i / 4][i % 4] = first + i < p.n_pages ? r : 1;
      }
    }
  }
  __device__ __forceinline__ uint32_t free() const {  // a bit each
    uint32_t f = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) f |= (uint32_t)(ref[i / 4][i % 4] <= 0) << i;
    return f;
  }
};

__global__ __launch_bounds__(PLAN_THREADS) void pages_plan_kernel(const wave_pages from, const wave_pages to, const int32_t* counts, int n,
                                                                 const PagesPlan plan, bool apart) {
  __shared__ int part[PLAN_WAVES];
  const int tid = threadIdx.x, shift = page_shift(from.page);
  PageReferences<PLAN_PER> refs;
  refs.load(from, tid * PLAN_PER);
  int wanted = 0;  // pages wanted by the sequences so far
  int4 mine = make_int4(0, 0, 0, 0);
  for (int b0 = 0; b0 < from.B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    int length = 0, count = 0, need = 0;
    if (b < from.B) {
      length = pages_length(from, b);
      count = counts ? min(max(counts[b], 0), n) : n;
      const int fit = min(count, pages_room(from) - length);
      need = ((length + fit) >> shift) - (length >> shift);
    }
    // (where the sums stop, there is no page anyway)
    mine = make_int4(length, need, plan_scan(need, wanted, part), count);
    if (b0 + PLAN_THREADS < from.B) plan.sequence[b] = mine;  // (the last round's stay where they are)
  }
  int found = 0;
  if (tid == 0) plan.last[0] = -1;
  for (int r0 = 0; r0 < from.n_pages && found < wanted; r0 += PLAN_ROUND) {
    uint32_t free = refs.free();
    const int first = r0 + tid * PLAN_PER;
    if (r0 + PLAN_ROUND < from.n_pages) refs.load(from, first + PLAN_ROUND);
    int rank = plan_scan(__popc(free), found, part);
    for (; free && rank < wanted; free &= free - 1, ++rank) {
      const int page = first + __ffs(free) - 1;
      plan.taken[rank] = page;
      if (!apart) to.references[page] = 1;
      if (rank == wanted - 1) plan.last[0] = page;
    }
  }
  if (found < wanted && tid == 0) plan.last[0] = from.n_pages;  // every free page is taken
  for (int b = tid; b < from.B; b += PLAN_THREADS) {
    int4 s = mine;
    if (b - tid + PLAN_THREADS < from.B) s = plan.sequence[b];
    const int whole = s.x >> shift, got = min(max(found - s.z, 0), s.y);
    int end = s.x + min(s.w, pages_room(from) - s.x);
    if (got < s.y) end = ((whole + got + 1) << shift) - 1;
    s.y = end;
    plan.sequence[b] = s;
    to.lengths[b] = end;
  }
}

// Append, second launch.
//   pages   a workgroup has some heads' keys or values of one page of a sequence: rows that were in the tail, new rows, or both.
//           If the page is complete they are rounded to 8 bits (a thread keeps its 16 channels of every row between the maximum and
//           the codes), otherwise they are the new tail
//   tokens  queries, as in norm_rotary_kernel; and where one token is appended, its key and value rows too, straight into the tail
//           unless they complete a page: then the pages' workgroups have little to do but in the one sequence of `page` that does
//   lists   table and references of a state with arrays of its own
// Four prompts of up to 8191 tokens, 32 and 8 heads, d = 128: 118 us, 553 MB, 4.7 TB/s (132 before the next head's rows were asked for
// while this one's are rounded, and outputs passed by the caches).  One token of 64 sequences of 28 and 4 heads in place 4.8 us, 6.0 where one
// of them completes a page.
struct AppendGrid {
  unsigned reference_blocks;           // without a plan
  unsigned page_blocks, token_blocks;  // the others are lists
  int units, head_groups;              // pages that a sequence's new tokens may touch; workgroups that share a page's heads
  TurnShape sh;
  int tiles;
};

// code of x in a page whose values are x / inv
__device__ __forceinline__ int code_of(float x, float inv) {
  const float r = fminf(fmaxf(rintf(x * inv), -127.f), 127.f);  // (x * inv may be 127 and a little)
  return (int)r;
}

template <typename T, int D, int PAGE>
struct PageRows {
  typedef RowItem<T, D> Item;
  static constexpr int EPC = Item::EPC, ITEMS = Item::ITEMS, SIDE = THREADS / ITEMS;  // rows side by side
  static constexpr int PASSES = PAGE > SIDE ? PAGE / SIDE : 1, TOKENS = PAGE > SIDE ? PAGE : SIDE;
  static constexpr size_t ROW = D * sizeof(T);
  static constexpr bool AHEAD = PASSES <= 2;  // (more would take too many registers)
  typedef SineTable<T, D, TOKENS> Table;

  // Part u of sequence b's new state, heads first .. in steps of `step`; find(): the page that it goes to if it is complete; where
  // that is not SURE, negative if there is none, and then nothing is done.
  template <bool SURE, typename F>
  static __device__ __forceinline__ bool run(const wave_pages& from, const wave_pages& to, const PagesAppendArgs& a, const RotaryArgs& rot,
                                             const int4 s, int b, int u, bool keys, int first, int step, Table& table,
                                             uint32_t (*top)[4], F&& find) {
    const int tid = threadIdx.x, row0 = tid / ITEMS;
    const int whole = s.x / PAGE, start = (whole + u) * PAGE, end = s.y;
    const bool complete = start + PAGE <= end;
    const char* tail = static_cast<const char*>(keys ? from.k_tail : from.v_tail);
    char* to_tail = static_cast<char*>(keys ? to.k_tail : to.v_tail);
    const HeadRows& rows = keys ? a.k_new : a.v_new;
    Item t;
    t.place(rot, keys && a.rows.turns, tid % ITEMS);
    uint4 x[PASSES], y[PASSES];  // this head's rows
    // A lane's rows; lanes behind the page's last one have that one again.
    auto row = [&](int i) { return min(row0 + i * SIDE, PAGE - 1); };
    // (a load under a condition of the lanes would be waited for where it is; rows that are not there load the last one)
    auto load = [&](int h, uint4 (&u)[PASSES], uint4 (&v)[PASSES]) {
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int at = min(start + row(i), end - 1);
        const char* p = at < s.x ? tail + (((size_t)b * from.Hkv + h) * PAGE + (at - start)) * ROW : row_of(rows, b, h, at - s.x);
        u[i] = load16_stream(p + t.one * 16);
        v[i] = load16_stream(p + t.two * 16);
      }
    };
    load(first, x, y);
    const typename Item::Weight w = t.weight(keys ? a.rows.k_weight : nullptr);
    const int r0 = max(s.x - start, 0), r1 = min(end - start, PAGE);  // the new rows
    if (keys && a.rows.turns && r0 < r1)
      table.fill(rot, r0, r1, [&](int axis, int r) {
        return a.rows.coords ? a.rows.coords[((size_t)axis * from.B + b) * a.n + start + r - s.x] : start + r;
      });
    const int page = complete ? find() : 0;
    if (!SURE && page < 0) return false;
    if (complete && keys && first == 0 && tid == 0) to.table[(size_t)b * to.max_pages + whole + u] = page;
    int turn = 0;
    for (int h = first; h < from.Hkv; h += step, turn ^= 1) {
      // the next head's rows are on their way
      uint4 next_x[PASSES], next_y[PASSES];
      const bool more = h + step < from.Hkv;
      if (AHEAD && more) load(h + step, next_x, next_y);
      auto advance = [&]() {
        if (!more) return;
        if (AHEAD) {
#pragma unroll
          for (int i = 0; i < PASSES; ++i) {
            x[i] = next_x[i];
            y[i] = next_y[i];
          }
        } else {
          load(h + step, x, y);
        }
      };
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        if (row(i) >= r0 && row(i) < r1) {
          typename Item::Sines sines;
          if (t.turns) table.get(row(i), t.item, sines);
          t.apply(w, sines, a.rows.eps, x[i], y[i]);
        }
      }
      if (!complete) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          const int r = row0 + i * SIDE, at = start + r;
          if (r < PAGE && at < end && (a.apart || at >= s.x)) {
            char* p = to_tail + (((size_t)b * from.Hkv + h) * PAGE + r) * ROW;
            store16(p + t.one * 16, x[i]);
            store16(p + t.two * 16, y[i]);
          }
        }
        advance();
        continue;
      }
      // magnitudes order like integers, what is no number above infinity
      uint32_t most = 0;
      float f[2 * EPC];
      auto values = [&](int i) {
        float lo[EPC], hi[EPC];
        unpack<T>(x[i], lo);
        unpack<T>(y[i], hi);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          f[e] = lo[e];
          f[EPC + e] = hi[e];
        }
      };
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        values(i);
#pragma unroll
        for (int e = 0; e < 2 * EPC; ++e) most = max(most, __float_as_uint(f[e]) & 0x7fffffffu);
      }
      most = wave_max_u(most);
      if ((tid & 63) == 0) top[turn][tid >> 6] = most;
      __syncthreads();
      most = max(max(top[turn][0], top[turn][1]), max(top[turn][2], top[turn][3]));
      // (below 2^-100, where 127 / max may be infinite, the page counts as zeros.  The definition has the quotient as a reciprocal and a
      // product, two roundings for 127 / max's one.  With the product that follows x * inv is off by up to 3 u of itself, 2.3e-5 at 127: a
      // code may fall otherwise where its value lies as near to a border, 1.5e-5 with the one quotient.  From 2^126 on 1 / max is
      // subnormal and off by up to 2^-22 of itself: 4.6e-5.)
      const bool number = most < 0x7f800000u, some = most >= 0x0d800000u;
      const float inv = number && some ? 1.f / __uint_as_float(most) * 127.f : 0.f;
      const float scale = !number ? __uint_as_float(0x7fc00000u) : some ? __uint_as_float(most) / 127.f : 0.f;
      const size_t unit = (size_t)page * from.Hkv + h;
      if (tid == 0) (keys ? to.k_scales : to.v_scales)[unit] = scale;
      int8_t* codes = (keys ? to.k_codes : to.v_codes) + unit * PAGE * D;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int r = row0 + i * SIDE;
        values(i);
        uint32_t word[EPC / 2];  // both chunks' codes, four a word
#pragma unroll
        for (int j = 0; j < EPC / 2; ++j) {
          uint32_t o = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) o |= (uint32_t)((inv == 0.f ? 0 : code_of(f[j * 4 + e], inv)) & 0xff) << (8 * e);
          word[j] = o;
        }
        if (r < PAGE) {
          int8_t* p = codes + (size_t)r * D;
          if constexpr (EPC == 8) {
            *reinterpret_cast<uint2*>(p + t.one * 8) = make_uint2(word[0], word[1]);
            *reinterpret_cast<uint2*>(p + t.two * 8) = make_uint2(word[2], word[3]);
          } else {
            *reinterpret_cast<uint32_t*>(p + t.one * 4) = word[0];
            *reinterpret_cast<uint32_t*>(p + t.two * 4) = word[1];
          }
        }
      }
      advance();
    }
    return true;
  }
};

// One token into a state of its own arrays: `from` stays as it is, so a workgroup can find by itself what the plan says.  Only one whose
// token completes a page has to look further than its sequence's length: at the other lengths, for how many before it do, and at
// references; the rows are on their way meanwhile.  In one launch (with a plan's, us; calls in a row, so the host's part too): 64
// sequences of 28 and 4 heads 10.7 (14.2), kernels 8.4 (4.0 + 6.2); 256 of them with 15.8K pages 16.1 (18.2), 16.1 (4.6 + 12.5); where
// all complete a page the kernels are even.  Beyond these numbers of sequences and pages the plan, which reads them once: the 64 sequences in
// a pool of 65536 pages, with the rows read back, 19.5 for 16.5.
// The functions below take all threads together.  Their loads stand side by side without conditions: behind one each would be waited
// for alone (12.5 -> 18.9 for 256 sequences).
constexpr int OWN_SEQUENCES = 4 * THREADS, OWN_PAGES = 64 * THREADS, OWN_REFERENCES = 4;
__device__ __forceinline__ int workgroup_sum(int x, int (&part)[THREADS / 64]) {
  x = wave_sum_i(x);
  __syncthreads();  // (what the call before this one left has been read)
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}
struct OwnToken {
  int length;
  bool given, fits, completes;
  __device__ __forceinline__ OwnToken(const wave_pages& p, int held, int count) {
    length = min(max(held, 0), pages_room(p));
    given = count > 0;
    fits = given && length < pages_room(p);
    completes = fits && ((length + 1) & (p.page - 1)) == 0;
  }
  __device__ __forceinline__ OwnToken(const wave_pages& p, const int32_t* counts, int b)
      : OwnToken(p, p.lengths[b], counts ? counts[b] : 1) {}
};
// how many sequences below `end` complete a page
__device__ __forceinline__ int own_wanted(const wave_pages& p, const int32_t* counts, int end, int (&part)[THREADS / 64]) {
  constexpr int PER = OWN_SEQUENCES / THREADS;
  int held[PER], count[PER], n = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) held[i] = p.lengths[min((int)threadIdx.x + i * THREADS, p.B - 1)];
#pragma unroll
  for (int i = 0; i < PER; ++i) count[i] = 1;
  if (counts) {
#pragma unroll
    for (int i = 0; i < PER; ++i) count[i] = counts[min((int)threadIdx.x + i * THREADS, p.B - 1)];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool completes = OwnToken(p, held[i], count[i]).completes;
    n += (int)threadIdx.x + i * THREADS < end ? completes : 0;
  }
  return workgroup_sum(n, part);
}
// Four pages' references and which of them are free (a bit each, none behind the pool), without a branch: the last ones are read from
// the pool's end on.
struct OwnReferences {
  PageReferences<4>::int4_of_ints ref;
  int moved;
  __device__ __forceinline__ void load(const wave_pages& p, int first) {
    const int at = min(first, p.n_pages - 4);
    ref = *reinterpret_cast<const PageReferences<4>::int4_of_ints*>(p.references + at);
    moved = min(first - at, 31);
  }
  __device__ __forceinline__ uint32_t free() const {
    uint32_t f = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) f |= (uint32_t)(ref[i] <= 0) << i;
    return f >> moved;
  }
};
struct OwnCounts {
  int sums[THREADS / 64], free[64], found;
};
// the page that sequence b, which completes one, takes (-1: none is free for it)
__device__ __forceinline__ int own_page(const wave_pages& p, const int32_t* counts, int b, OwnCounts& shared) {
  // Pieces of 256 pages, a piece each wave and round: how many are free in each, which one has the page, and then where it is there.
  constexpr int PER = OWN_REFERENCES, PIECE = 64 * PER, WAVES = THREADS / 64, ROUNDS = OWN_PAGES / PIECE / WAVES;
  static_assert(ROUNDS * WAVES == 64, "a lane each");
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  OwnReferences refs[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) refs[r].load(p, (r * WAVES + wave) * PIECE + lane * PER);
  const int rank = own_wanted(p, counts, b, shared.sums);
  uint64_t free = 0;  // this lane's, PER bits a round
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    int n = 0;
    const uint32_t mine = refs[r].free();
    free |= (uint64_t)mine << (PER * r);
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popcll(__ballot(mine >> i & 1));
    if (lane == 0) shared.free[r * WAVES + wave] = n;
  }
  __syncthreads();
  const int upto = wave_incl_scan(shared.free[lane]);
  const uint64_t behind = __ballot(upto > rank);
  if (!behind) return -1;
  const int piece = __ffsll((unsigned long long)behind) - 1;
  if (piece % WAVES == wave) {
    uint32_t mine = (uint32_t)(free >> (PER * (piece / WAVES))) & ((1u << PER) - 1);
    const int here = __popc(mine);
    int at = (piece ? __builtin_amdgcn_readlane(upto, piece - 1) : 0) + wave_incl_scan(here) - here;
    if (rank >= at && rank < at + here) {
      for (; at < rank; ++at) mine &= mine - 1;
      shared.found = piece * PIECE + lane * PER + __ffs(mine) - 1;
    }
  }
  __syncthreads();
  return shared.found;
}
// references of the pages that workgroup `block` has: those of the first `wanted` free ones become 1
__device__ __forceinline__ void own_references(const wave_pages& from, const wave_pages& to, const int32_t* counts, int block,
                                               OwnCounts& shared) {
  int(&part)[THREADS / 64] = shared.sums;
  constexpr int PER = OWN_REFERENCES;
  const int r0 = block * THREADS * PER, first = r0 + threadIdx.x * PER;
  PageReferences<PER> refs;
  refs.load(from, first);
  const uint32_t free = refs.free();
  int before = 0;  // free pages in front of the workgroup's
  OwnReferences others[OWN_PAGES / THREADS / PER];
#pragma unroll
  for (int i = 0; i < OWN_PAGES / THREADS / PER; ++i) others[i].load(from, (min(i, block) * THREADS + threadIdx.x) * PER);
#pragma unroll
  for (int i = 0; i < OWN_PAGES / THREADS / PER; ++i)
    before += i < block ? __popc(others[i].free()) : 0;
  const int wanted = own_wanted(from, counts, from.B, part);
  int rank = wanted;  // free pages in front of the thread's
  if (wanted > 0) {
    const int here = __popc(free), incl = wave_incl_scan(here), wave = threadIdx.x >> 6;
    rank = workgroup_sum(before, part) + incl - here;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave; ++w) rank += part[w];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (first + i < from.n_pages) {
      const bool is_free = free >> i & 1;
      to.references[first + i] = is_free && rank < wanted ? 1 : refs.ref[0][i];
      rank += is_free;
    }
}

// FINDS: without a plan
template <typename T, int D, int PAGE, bool FINDS>
__global__ __launch_bounds__(THREADS) void pages_append_kernel(const wave_pages from, const wave_pages to, const PagesAppendArgs a,
                                                               const RotaryArgs rot, const PagesPlan plan, const AppendGrid grid) {
  typedef PageRows<T, D, PAGE> Rows;
  __shared__ typename Rows::Table table;
  __shared__ uint32_t top[2][4];
  __shared__ OwnCounts own;
  unsigned block = workgroup_number();
  if constexpr (FINDS) {  // (first, as theirs is the longest chain)
    if (block < grid.reference_blocks) {
      own_references(from, to, a.counts, block, own);
      return;
    }
    block -= grid.reference_blocks;
  }
  if (block < grid.page_blocks) {
    const int group = block % grid.head_groups, keys = (block / grid.head_groups) & 1;
    const unsigned bu = block / grid.head_groups / 2;
    const int b = bu / grid.units;
    int u = bu % grid.units, parts = 1;
    int4 s;
    if constexpr (FINDS) {
      const OwnToken t(from, a.counts, b);
      s = make_int4(t.length, t.length + t.fits, 0, t.given);
    } else {
      s = plan.sequence[b];
    }
    const int rest = s.y / PAGE - s.x / PAGE;  // the unit whose rows are the tail
    auto copy_tail = [&]() {
      for (int h = group; h < from.Hkv; h += grid.head_groups) {
        const size_t at = ((size_t)b * from.Hkv + h) * PAGE * D * sizeof(T);
        copy_chunks(static_cast<const char*>(keys ? from.k_tail : from.v_tail) + at, static_cast<char*>(keys ? to.k_tail : to.v_tail) + at,
                    s.x % PAGE * (int)(D * sizeof(T) / 16));
      }
    };
    if (FINDS || a.n == 1) {
      // (a token that completes no page is written by its own workgroup: here only old rows go on)
      if (s.y == s.x || s.y % PAGE != 0) {
        if (FINDS || a.apart) copy_tail();
        return;
      }
    } else {
      // In place the rows that page 0 takes from the tail are where the new tail goes: the same workgroup does both.
      const bool both = !a.apart && rest > 0 && s.x % PAGE != 0 && s.y % PAGE != 0;
      if (u > rest || (u == rest && (both || s.y % PAGE == 0))) return;
      if (u == 0 && both) parts = 2;
    }
    if constexpr (FINDS) {
      const bool found = Rows::template run<false>(from, to, a, rot, s, b, 0, keys, group, grid.head_groups, table, top,
                                   [&]() { return own_page(from, a.counts, b, own); });
      if (!found) copy_tail();
      if (keys && group == 0 && threadIdx.x == 0) to.lengths[b] = found ? s.y : s.x;
    } else {
      for (int i = 0; i < parts; ++i) {
        if (i) {
          __syncthreads();  // everything that was in the tail has been read, the sines and the maxima too
          u = rest;
        }
        const int page = u < rest ? plan.taken[s.z + u] : 0;
        Rows::template run<true>(from, to, a, rot, s, b, u, keys, group, grid.head_groups, table, top, [page]() { return page; });
      }
    }
    return;
  }
  block -= grid.page_blocks;
  if (block < grid.token_blocks) {
    const int group = block % grid.sh.head_groups, bt = block / grid.sh.head_groups;
    const int b = bt / grid.tiles, tile = bt % grid.tiles;
    int4 s;
    norm_heads<T, D>(
        a.rows, a.v_new, FINDS || a.n == 1 ? from.Hkv : 0, rot, grid.sh, b, tile, group, table,
        [&]() {
          if constexpr (FINDS) {  // (a token that completes a page is the pages' workgroups' in any case)
            const OwnToken t(from, a.counts, b);
            s = make_int4(t.length, t.length + t.fits, 0, t.given);
          } else {
            s = plan.sequence[b];
          }
          return s.w;
        },
        [&](int axis, int n) { return a.rows.coords ? a.rows.coords[((size_t)axis * from.B + b) * a.n + n] : s.x + n; },
        [&](int h, int n) -> char* {
          constexpr size_t ROW = D * sizeof(T);
          if (h < a.rows.Hq) return a.rows.q_out + (((size_t)b * a.rows.Hq + h) * a.n + n) * ROW;
          if (s.y == s.x || s.y % PAGE == 0) return nullptr;  // no room, or part of a page
          h -= a.rows.Hq;
          const bool keys = h < from.Hkv;
          char* tail = static_cast<char*>(keys ? to.k_tail : to.v_tail);
          return tail + (((size_t)b * from.Hkv + (keys ? h : h - from.Hkv)) * PAGE + s.x % PAGE) * ROW;
        });
    return;
  }
  block -= grid.token_blocks;
  if (!a.apart) return;
  // one workgroup a sequence for the tables, the others for references
  if (block < (unsigned)from.B) {
    int whole;
    if constexpr (FINDS) {
      const OwnToken t(from, a.counts, block);
      whole = t.length / PAGE;
      if (!t.completes && threadIdx.x == 0) to.lengths[block] = t.length + t.fits;
    } else {
      whole = plan.sequence[block].x / PAGE;
    }
    const size_t at = (size_t)block * from.max_pages;
    for (int i = threadIdx.x; i < whole; i += 256) to.table[at + i] = from.table[at + i];
    return;
  }
  if constexpr (FINDS) return;
  const int last = plan.last[0];
  const long long i = (long long)(block - from.B) * 256 + threadIdx.x;
  if (i < from.n_pages) {
    const int r = from.references[i];
    to.references[i] = r <= 0 && i <= last ? 1 : r;
  }
}

template <typename T, int D, int PAGE>
wave_status pages_append_tdp(const wave_pages& from, const wave_pages& to, PagesAppendArgs a, const RotaryArgs& rot,
                             const PagesPlan& plan, hipStream_t st) {
  a.rows.past = a.n > 1 && (size_t)from.B * a.rows.Hq * a.n * D * sizeof(T) > PAST_BYTES;
  AppendGrid g{};
  const bool finds = a.n == 1 && a.apart && from.B <= OWN_SEQUENCES && from.n_pages >= 4 && from.n_pages <= OWN_PAGES;
  if (!finds) WAVE_LAUNCH("pages_plan", pages_plan_kernel, 1, PLAN_THREADS, 0, st, from, to, a.counts, a.n, plan, a.apart);
  g.units = a.n == 1 ? 1 : (int)(((long long)PAGE - 2 + a.n) / PAGE) + 1;
  // A page's heads are split while the launch leaves most CUs without work; together they share the sines.
  g.head_groups = 1;
  while ((long long)from.B * g.units * 2 * g.head_groups < 1024 && g.head_groups < from.Hkv) g.head_groups *= 2;
  if (g.head_groups > from.Hkv) g.head_groups = from.Hkv;
  long long blocks = (long long)from.B * g.units * 2 * g.head_groups;
  g.page_blocks = (unsigned)blocks;
  if (a.n == 1) {
    a.rows.k = a.k_new;
    a.rows.Hk = from.Hkv;
  }
  const int heads = a.rows.Hq + (a.n == 1 ? 2 * from.Hkv : 0);
  if (heads > 0) {
    g.sh = turn_shape<RowItem<T, D>::ITEMS>(a.n, from.B, heads);
    g.tiles = (a.n + g.sh.tokens - 1) / g.sh.tokens;
    g.token_blocks = (unsigned)((long long)from.B * g.tiles * g.sh.head_groups);
    blocks += g.token_blocks;
  }
  g.reference_blocks = finds ? (from.n_pages + THREADS * OWN_REFERENCES - 1) / (THREADS * OWN_REFERENCES) : 0;
  if (a.apart) blocks += from.B + (finds ? (long long)g.reference_blocks : ((long long)from.n_pages + 255) / 256);
  if (finds)
    WAVE_LAUNCH("pages_append", (pages_append_kernel<T, D, PAGE, true>), grid_rows(blocks), 256, 0, st, from, to, a, rot, plan, g);
  else
    WAVE_LAUNCH("pages_append", (pages_append_kernel<T, D, PAGE, false>), grid_rows(blocks), 256, 0, st, from, to, a, rot, plan, g);
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}
template <typename T, int D>
wave_status pages_append_td(const wave_pages& from, const wave_pages& to, const PagesAppendArgs& a, const RotaryArgs& rot,
                            const PagesPlan& plan, hipStream_t st) {
  return from.page == 32   ? pages_append_tdp<T, D, 32>(from, to, a, rot, plan, st)
         : from.page == 64 ? pages_append_tdp<T, D, 64>(from, to, a, rot, plan, st)
                           : pages_append_tdp<T, D, 128>(from, to, a, rot, plan, st);
}

// ----------------------------------------------------------------------------
// Reading back.  A wave has 32 rows that begin at a multiple of 32, so they are one page's, or the tail's: its page and scale
// are the wave's.  A lane turns what it loads into 16 bytes, neighbouring lanes into neighbouring ones: 141 us for 122877 tokens of
// eight heads, 755 MB, 5.3 TB/s, what a copy reaches (203 with 32 bytes a lane and a page's number, and its scale, for each lane).
// ----------------------------------------------------------------------------
struct ReadArgs {
  const int32_t* first;
  char *k_out, *v_out;
  int n, tiles;
};
constexpr int READ_CHUNK = 32, READ_TILE = 4 * READ_CHUNK;

template <typename T, int D>
__global__ __launch_bounds__(256) void pages_read_kernel(const wave_pages p, const ReadArgs a, int sides) {
  constexpr int EPC = Elem<T>::EPC, LANES = D / EPC, SIDE = 64 / LANES, STEPS = READ_CHUNK / SIDE;
  constexpr size_t ROW = D * sizeof(T);
  unsigned block = workgroup_number();
  const bool keys = sides == 2 ? (block & 1) == 0 : a.k_out != nullptr;
  block /= sides;
  const int tile = block % a.tiles;
  const unsigned unit = block / a.tiles;
  if (unit >= (unsigned)(p.B * p.Hkv)) return;
  const int b = unit / p.Hkv, h = unit % p.Hkv, shift = page_shift(p.page);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int length = pages_length(p, b), whole = length >> shift << shift;
  const long long first = a.first ? a.first[b] : 0;
  const long long at = (first & ~31ll) + (long long)tile * READ_TILE + wave * READ_CHUNK;  // the wave's first row
  const long long low = first > 0 ? first : 0, high = min(first + a.n, (long long)length);
  if (at + READ_CHUNK <= low || at >= high) return;
  const int c0 = (int)at, sub = lane / LANES, part = lane % LANES;
  char* out = (keys ? a.k_out : a.v_out) + ((size_t)unit * a.n + sub) * ROW + part * 16 + (at - first) * (long long)ROW;
  auto inside = [&](int i) { return c0 + i * SIDE + sub >= low && c0 + i * SIDE + sub < high; };
  if (c0 >= whole) {
    const char* from = static_cast<const char*>(keys ? p.k_tail : p.v_tail) + ((size_t)unit * p.page + (c0 - whole) + sub) * ROW + part * 16;
#pragma unroll 4
    for (int i = 0; i < STEPS; ++i)
      if (inside(i)) store16(out + (size_t)i * SIDE * ROW, load16(from + (size_t)i * SIDE * ROW));
    return;
  }
  const size_t held = (size_t)page_entry(p, b, c0 >> shift) * p.Hkv + h;
  const float scale = (keys ? p.k_scales : p.v_scales)[held];
  const int8_t* from = (keys ? p.k_codes : p.v_codes) + ((held << shift) + (c0 & (p.page - 1)) + sub) * D + part * EPC;
  uint32_t word[STEPS][EPC / 4];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    if constexpr (EPC == 8) {
      const uint2 u = load8_stream(from + i * SIDE * D);
      word[i][0] = u.x;
      word[i][1] = u.y;
    } else {
      word[i][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(from + i * SIDE * D));
    }
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    float f[EPC];
#pragma unroll
    for (int e = 0; e < EPC; ++e) f[e] = (float)(int8_t)(word[i][e / 4] >> (8 * (e & 3))) * scale;
    if (inside(i)) store16(out + (size_t)i * SIDE * ROW, pack<T>(f));
  }
}

template <typename T, int D>
wave_status pages_read_td(const wave_pages& p, ReadArgs a, hipStream_t st) {
  // (the first chunk begins up to 31 rows before the first row, which is the device's)
  a.tiles = (int)(((long long)a.n + (a.first ? READ_CHUNK - 1 : 0) + READ_TILE - 1) / READ_TILE);
  const int sides = (a.k_out ? 1 : 0) + (a.v_out ? 1 : 0);
  WAVE_LAUNCH("pages_read", (pages_read_kernel<T, D>), grid_rows((long long)p.B * p.Hkv * a.tiles * sides), 256, 0, st, p, a, sides);
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

// ----------------------------------------------------------------------------
// Reordering.  References change by atomic additions of whole numbers, whose order does not show.
// ----------------------------------------------------------------------------
__device__ __forceinline__ int parent_of(const wave_pages& from, const int32_t* parent, int b) {
  const int p = parent[b];
  return p >= 0 && p < from.B ? p : -1;
}

// to's references as from's: what the next launch adds to
__global__ __launch_bounds__(256) void pages_references_kernel(const int32_t* from, int32_t* to, int n) {
  const long long i = (long long)workgroup_number() * 256 + threadIdx.x;
  if (i < n) to[i] = from[i];
}

// Into arrays of its own.
//   counts  COUNT_PAGES pages' references: from's, and what changes, counted in LDS by going through the tables of those sequences
//           whose pages gain or lose.  Where these have more than COUNT_ENTRIES entries (or there are so many pages that they would be
//           read too often), references are copied by a launch before this one, and each sequence's workgroup adds to them.  (Us, in one
//           launch and in two: 8 sequences 5.7 and 8.9, 64 of 64 entries 7.0 and 8.5, 1000 of 4 7.3 and 8.9, two of 2000 6.7 and 8.9; 128
//           of 64, whose tails take as long, 11.1 and 9.1; 256 of 63 18.0 and 14.1.)  The host knows the table's entries, not those in
//           use: eight beams of six pages take 5.7 in a table of six entries a row, 8.4 in one of 1024
//   tables  a sequence of `to`: its table, its length.  A sequence that stays where it is changes no reference
//   leave   a sequence of `from`, where it takes its references away itself
//   tails   a head's keys or values of a sequence
constexpr int COUNT_PAGES = 1024, COUNT_SEQUENCES = 1024, COUNT_ENTRIES = 4096, COUNT_READS = 1 << 22;
struct CopyGrid {
  unsigned counts, leave;  // workgroups
  int row_bytes, lane_shift;
};

__device__ __forceinline__ void count_references(const wave_pages& from, const wave_pages& to, const int32_t* parent, int p0, int lane_shift) {
  // what a sequence of `from` adds to its pages' references: the sequences of `to` that come from it elsewhere, less itself if it leaves
  __shared__ int count[COUNT_PAGES], weight[COUNT_SEQUENCES], held[COUNT_SEQUENCES];
  const int pages = min(COUNT_PAGES, from.n_pages - p0), shift = page_shift(from.page);
  for (int i = threadIdx.x; i < pages; i += THREADS) count[i] = from.references[p0 + i];
  for (int s = threadIdx.x; s < from.B; s += THREADS) {
    weight[s] = s < to.B && parent[s] == s ? 0 : -1;
    held[s] = pages_length(from, s) >> shift;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < to.B; b += THREADS) {
    const int s = parent_of(from, parent, b);
    if (s >= 0 && s != b) atomicAdd(&weight[s], 1);
  }
  __syncthreads();
  // 2^lane_shift lanes a row of the table
  constexpr int BATCH = 8;
  const int lane = threadIdx.x & ((1 << lane_shift) - 1), rows = THREADS >> lane_shift;
  for (int s0 = threadIdx.x >> lane_shift; s0 < from.B; s0 += rows * BATCH) {
    int w[BATCH], end[BATCH], most = 0;
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int s = s0 + k * rows;
      w[k] = s < from.B ? weight[s] : 0;
      end[k] = w[k] ? held[s] : 0;
      most = max(most, end[k]);
    }
    for (int column = lane; column < most; column += 1 << lane_shift) {
      int page[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) page[k] = page_entry(from, min(s0 + k * rows, from.B - 1), column);
#pragma unroll
      for (int k = 0; k < BATCH; ++k)
        if (column < end[k] && page[k] >= p0 && page[k] < p0 + pages) atomicAdd(&count[page[k] - p0], w[k]);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < pages; i += THREADS) to.references[p0 + i] = count[i];
}

__global__ __launch_bounds__(256) void pages_copy_kernel(const wave_pages from, const wave_pages to, const int32_t* parent, const CopyGrid grid) {
  unsigned block = workgroup_number();
  const int shift = page_shift(from.page);
  if (block < grid.counts) {
    count_references(from, to, parent, block * COUNT_PAGES, grid.lane_shift);
    return;
  }
  block -= grid.counts;
  if (block < (unsigned)to.B) {
    const int b = block, s = parent_of(from, parent, b);
    const int length = s < 0 ? 0 : pages_length(from, s), whole = length >> shift;
    if (threadIdx.x == 0) to.lengths[b] = length;
    for (int i = threadIdx.x; i < whole; i += 256) {
      const int entry = from.table[(size_t)s * from.max_pages + i];
      to.table[(size_t)b * to.max_pages + i] = entry;
      if (grid.counts == 0 && s != b) atomicAdd(&to.references[min(max(entry, 0), from.n_pages - 1)], 1);
    }
    return;
  }
  block -= to.B;
  if (block < grid.leave) {
    const int b = block;
    if (b < to.B && parent[b] == b) return;
    const int whole = pages_length(from, b) >> shift;
    for (int i = threadIdx.x; i < whole; i += 256) atomicSub(&to.references[page_entry(from, b, i)], 1);
    return;
  }
  block -= grid.leave;
  const bool keys = (block & 1) == 0;
  const unsigned unit = block / 2;
  const int b = unit / from.Hkv, h = unit % from.Hkv;
  if (b >= to.B) return;
  const int s = parent_of(from, parent, b);
  if (s < 0) return;
  const int chunks = (pages_length(from, s) & (from.page - 1)) * (grid.row_bytes / 16);
  const size_t page_bytes = (size_t)from.page * grid.row_bytes;
  const char* x = static_cast<const char*>(keys ? from.k_tail : from.v_tail) + ((size_t)s * from.Hkv + h) * page_bytes;
  char* y = static_cast<char*>(keys ? to.k_tail : to.v_tail) + unit * page_bytes;
  copy_chunks(x, y, chunks);
}

// In place: those that leave.
__global__ __launch_bounds__(256) void pages_leave_kernel(const wave_pages p, const int32_t* parent) {
  const unsigned b = workgroup_number();
  if (b >= (unsigned)p.B || parent[b] == (int)b) return;
  const int whole = pages_length(p, b) >> page_shift(p.page);
  __syncthreads();
  if (threadIdx.x == 0) p.lengths[b] = 0;
  for (int i = threadIdx.x; i < whole; i += 256) atomicSub(&p.references[page_entry(p, b, i)], 1);
}

}  // namespace

wave_status launch_norm_rotary(const NormArgs& a, const RotaryArgs& rot, int dtype, int d, hipStream_t st) {
  if (dtype == WAVE_BF16) return d == 128 ? norm_rotary_td<bf16_t, 128>(a, rot, st) : norm_rotary_td<bf16_t, 64>(a, rot, st);
  return d == 128 ? norm_rotary_td<float, 128>(a, rot, st) : norm_rotary_td<float, 64>(a, rot, st);
}

size_t pages_append_workspace(const wave_pages& p) {
  return align_up(256 + align_up(sizeof(int4) * (size_t)p.B) + sizeof(int32_t) * (size_t)p.n_pages);
}

wave_status launch_pages_append(const wave_pages& from, const wave_pages& to, PagesAppendArgs a, const RotaryArgs& rot,
                                void* ws, hipStream_t st) {
  const PagesPlan plan = pages_plan(from, ws);
  if (from.dtype == WAVE_BF16)
    return from.d == 128 ? pages_append_td<bf16_t, 128>(from, to, a, rot, plan, st) : pages_append_td<bf16_t, 64>(from, to, a, rot, plan, st);
  return from.d == 128 ? pages_append_td<float, 128>(from, to, a, rot, plan, st) : pages_append_td<float, 64>(from, to, a, rot, plan, st);
}

wave_status launch_pages_read(const wave_pages& p, const int32_t* first, int n, void* k_out, void* v_out, hipStream_t st) {
  ReadArgs a{};
  a.first = first;
  a.n = n;
  a.k_out = static_cast<char*>(k_out);
  a.v_out = static_cast<char*>(v_out);
  if (p.dtype == WAVE_BF16) return p.d == 128 ? pages_read_td<bf16_t, 128>(p, a, st) : pages_read_td<bf16_t, 64>(p, a, st);
  return p.d == 128 ? pages_read_td<float, 128>(p, a, st) : pages_read_td<float, 64>(p, a, st);
}

wave_status launch_pages_reorder(const wave_pages& from, const wave_pages& to, const int32_t* parent, hipStream_t st) {
  if (to.lengths == from.lengths) {
    WAVE_LAUNCH("pages_leave", pages_leave_kernel, grid_rows(from.B), 256, 0, st, from, parent);
  } else {
    CopyGrid g{};
    g.row_bytes = from.d * (from.dtype == WAVE_BF16 ? 2 : 4);
    const long long entries = (long long)from.B * from.max_pages, blocks = ((long long)from.n_pages + COUNT_PAGES - 1) / COUNT_PAGES;
    if (from.B <= COUNT_SEQUENCES && to.B <= 4 * COUNT_SEQUENCES && entries <= COUNT_ENTRIES && entries * blocks <= COUNT_READS) {
      g.counts = (unsigned)blocks;
      while (g.lane_shift < 8 && 1 << g.lane_shift < from.max_pages) ++g.lane_shift;
    } else {
      g.leave = from.B;
      WAVE_LAUNCH("pages_references", pages_references_kernel, grid_rows(((long long)from.n_pages + 255) / 256), 256, 0, st,
                  from.references, to.references, from.n_pages);
    }
    WAVE_LAUNCH("pages_copy", pages_copy_kernel, grid_rows(g.counts + to.B + (long long)g.leave + (long long)to.B * to.Hkv * 2), 256, 0, st,
                from, to, parent, g);
  }
  return hipGetLastError() == hipSuccess ? WAVE_OK : WAVE_ERR_HIP;
}

}  // namespace wave
