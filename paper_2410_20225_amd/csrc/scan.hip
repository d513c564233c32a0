// The gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) x_t, a = sigmoid(f), along the rows of sequences that lie one after
// another, its gradients, and one row of many sequences on a table of states.
//   With s_t the gradient that reaches h_t:  s_t = dh_t + a_(t+1) s_(t+1)  (a sequence's last row: + dh_last),
//   dx = s (1 - a),   df = s (h_(t-1) - x) a (1 - a),   dh0 = a_1 s_1.
#include <algorithm>

#include "rows.h"

namespace tdf {
namespace {

using namespace rows;

// a = sigmoid(f) = 1 / (1 + E) and keep = 1 - a = a E with E = exp(-f): both have a small relative error wherever f lies.  E ends at
// 2^126, so that a E is 1 there.  bf16: the hardware's exponential and reciprocal as they are, a few 2^-24 off, and E up to |f| 2^-24
// more, since the exponential's argument is rounded.  fp32: the argument with the bits that its product loses, and a Newton step for the reciprocal.
template <int DT> __device__ __forceinline__ void gate(float f, float& a, float& keep) {
  constexpr float LOG2E = 1.44269504088896340736f, LOW = 1.92596299112661746887e-8f;   // log2(e) and what that leaves of it
  if constexpr (DT == TDF_BF16) {
    const float e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(f * -LOG2E, 126.0f));
    a = __builtin_amdgcn_rcpf(1.0f + e);
    keep = a * e;
  } else {
    const float p = __builtin_elementwise_minimum(f * -LOG2E, 126.0f);
    const float rest = fmaf(f, -LOW, fmaf(f, -LOG2E, -p));
    float e = __builtin_amdgcn_exp2f(p);
    if (fabsf(f) < 80.0f) e = fmaf(e, rest * 0.693147180559945309f, e);   // (beyond, p is the bound or e is nothing beside 1)
    const float d = 1.0f + e, r = __builtin_amdgcn_rcpf(d);
    a = fmaf(fmaf(-d, r, 1.0f), r, r);
    keep = a * e;
  }
}

struct ScanArgs {
  int64_t n_rows, n_cols, n_seqs;
  const void* f;
  int64_t ld_f;
  const void* x;
  int64_t ld_x;
  const int64_t* offsets;
  const float* h0;
  void* h;
  int64_t ld_h;
  float* h_last;
  // gradients
  const void* dh;
  int64_t ld_dh;
  const float* dh_last;
  void* df;
  int64_t ld_df;
  void* dx;
  int64_t ld_dx;
  float* dh0;
  // tiles
  int64_t n_tiles, n_blocks;     // of rows and of columns
  int64_t n_more;                // workgroups for sequences without a row, THREADS each
  uint64_t *sums, *group_sums, *super;   // [.. x n_cols], see Sum
  uint32_t* tickets;             // a counter for each block of columns, TICKET_APART from each other
  uint64_t* marks;               // [n_rows / 128 x 4]: rows where sequences begin and where they end, a bit a row
  int32_t *starts, *ends;        // [n_rows]: which, for those rows
};

constexpr int RUN = 16;          // tiles of a group, groups of a super-group
constexpr int THREADS = 256;
constexpr int TICKET_APART = 32;  // counters: a line each

// A tile is COLS columns and PARTS x L rows: 16 lanes beside each other take four columns each (of bf16 they read 128 bytes of a row), and
// each of the PARTS parts of the workgroup L rows one after the other, whose elements are all in flight together.  L is eight; four for the
// gradients in fp32, whose elements would take all registers.
constexpr int VEC = 4, LANES = 16, COLS = LANES * VEC, PARTS = THREADS / LANES;
constexpr int WAVES = THREADS / 64;                      // of a workgroup
constexpr int length(int dt, bool back) { return dt == TDF_F32 && back ? 4 : 8; }
constexpr int rows_of(int dt, bool back) { return PARTS * length(dt, back); }
constexpr int MOST_ROWS_OF = 128, LEAST_ROWS_OF = 64;    // of a tile

// The rows of a matrix that a tile reads or writes: `n` rows from `row` on.  LOOSE false: through a buffer descriptor that ends with
// them, so that offsets are 32 bits and rows and columns beyond the matrix read as zeros and are not written; the host has seen to it that a
// tile's rows span less than 2 GiB, that four columns are aligned together and that their number is a multiple of four.  LOOSE: anything.
template <int DT, bool LOOSE> struct Window {
  typedef typename TypeOf<DT>::type T;
  typedef T Pack __attribute__((ext_vector_type(VEC)));
  typedef unsigned int Words __attribute__((ext_vector_type(VEC * sizeof(T) / 4)));
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t step;                 // bytes from a row to the next
  __device__ __forceinline__ Window(const void* p, int64_t ld, int64_t row, int64_t n, int64_t n_cols) {
    step = (uint32_t)(ld * sizeof(T));
    rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)const_cast<void*>(p) + row * ld * (int64_t)sizeof(T), 0, (int)((n - 1) * step + n_cols * sizeof(T)), 0x00027000);
  }
  // (beyond 2^31 stays beyond with any row of the tile added)
  __device__ __forceinline__ uint32_t place(int row, int64_t c, int cols) const { return cols ? row * step + (uint32_t)c * (uint32_t)sizeof(T) : 0x80000000u; }
  __device__ __forceinline__ Pack load(uint32_t place, int i) const {
    if constexpr (sizeof(Pack) == 8) return __builtin_bit_cast(Pack, __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)(place + i * step), 0, 0));
    else return __builtin_bit_cast(Pack, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(place + i * step), 0, 0));
  }
  __device__ __forceinline__ void store(uint32_t place, int i, const float* x) const {
    Pack p;
#pragma unroll
    for (int v = 0; v < VEC; ++v) p[v] = (T)x[v];
    if constexpr (sizeof(Pack) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(Words, p), rsrc, (int)(place + i * step), 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(Words, p), rsrc, (int)(place + i * step), 0, 0);
  }
};
template <int DT> struct Window<DT, true> {
  typedef typename TypeOf<DT>::type T;
  typedef T Pack __attribute__((ext_vector_type(VEC)));
  struct __attribute__((packed, aligned(sizeof(T)))) Any {
    Pack p;
  };
  T* p;
  int64_t ld, n;
  struct Place {
    int row, cols;
    T* p;
  };
  __device__ __forceinline__ Window(const void* q, int64_t ld_, int64_t row, int64_t n_, int64_t) : p((T*)const_cast<void*>(q) + row * ld_), ld(ld_), n(n_) {}
  __device__ __forceinline__ Place place(int row, int64_t c, int cols) const { return Place{row, cols, p + row * ld + c}; }
  __device__ __forceinline__ Pack load(Place at, int i) const {
    Pack r;
#pragma unroll
    for (int v = 0; v < VEC; ++v) r[v] = (T)0.0f;
    if (at.row + i < 0 || at.row + i >= n) return r;
    if (at.cols == VEC) return ((const Any*)(at.p + i * ld))->p;
#pragma unroll
    for (int v = 0; v < VEC - 1; ++v)
      if (v < at.cols) r[v] = at.p[i * ld + v];
    return r;
  }
  __device__ __forceinline__ void store(Place at, int i, const float* x) const {
    if (at.row + i < 0 || at.row + i >= n) return;
    if (at.cols == VEC) {
      Any a;
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.p[v] = (T)x[v];
      *(Any*)(at.p + i * ld) = a;
      return;
    }
#pragma unroll
    for (int v = 0; v < VEC - 1; ++v)
      if (v < at.cols) at.p[i * ld + v] = (T)x[v];
  }
};

// For MARK rows: which sequence begins there and which ends, -1: none.
constexpr int MARK = 128;
__device__ inline void mark_rows(const ScanArgs& a, int64_t t0, int32_t* starts, int32_t* ends) {
  const int tid = threadIdx.x;
  if (tid < MARK) starts[tid] = ends[tid] = -1;
  if (!a.offsets) {
    __syncthreads();
    if (tid == 0) {
      if (t0 == 0) starts[0] = 0;
      if (a.n_rows - 1 - t0 < MARK) ends[a.n_rows - 1 - t0] = 0;
    }
    __syncthreads();
    return;
  }
  // how many offsets lie below t0: as many as there are threads at a time, evenly spaced
  int64_t lo = 0, n = a.n_seqs + 1;
  while (n > 0) {
    const int64_t stride = (n + THREADS - 1) / THREADS, at = (tid + 1) * stride - 1;
    const int64_t c = __syncthreads_count(at < n && a.offsets[lo + at] < t0);
    lo += c * stride;
    if (stride == 1) break;
    n = min(stride, n - c * stride);
  }
  for (int64_t s0 = max(lo - 1, (int64_t)0); s0 < a.n_seqs; s0 += THREADS) {
    const int64_t s = s0 + tid;
    bool more = false;
    if (s < a.n_seqs) {
      const int64_t first = a.offsets[s], end = a.offsets[s + 1];
      if (first < end) {
        if (first >= t0 && first < t0 + MARK) starts[first - t0] = (int32_t)s;
        if (end > t0 && end <= t0 + MARK) ends[end - 1 - t0] = (int32_t)s;
      }
      more = first < t0 + MARK;
    }
    if (__syncthreads_count(more) < THREADS) break;
  }
  __syncthreads();
}

// Where sequences begin and end in a thread's L rows from `row` on (t0: the tile's first): bit i for its i-th, and which.  In a chain from
// what k_scan_mark left, through the scalar cache, with no wait for the rows' elements, which are on their way; else from shared memory.
template <int L, bool CHAINED> struct Marks {
  uint32_t first, last;
  const int32_t *starts, *ends;
  __device__ __forceinline__ void of_chain(const ScanArgs& a, int64_t t0, int row) {
    typedef const __attribute__((address_space(4))) uint64_t* Scalar;
    const Scalar m = (Scalar)(a.marks + (t0 / MARK) * 4);
    uint64_t f, l;
    if constexpr (PARTS * L == MARK) {
      const uint64_t f0 = m[0], f1 = m[1], l0 = m[2], l1 = m[3];
      f = row < 64 ? f0 : f1;
      l = row < 64 ? l0 : l1;
    } else {
      static_assert(PARTS * L == 64, "a word a tile");
      const int half = (int)(t0 / 64 % 2);
      f = m[half];
      l = m[2 + half];
    }
    first = (uint32_t)(f >> (row & 63)) & ((1u << L) - 1);
    last = (uint32_t)(l >> (row & 63)) & ((1u << L) - 1);
    starts = a.starts + t0 + row;
    ends = a.ends + t0 + row;
  }
  __device__ __forceinline__ void of_shared(int row, const int32_t* sh_starts, const int32_t* sh_ends) {
    starts = sh_starts + row;
    ends = sh_ends + row;
    first = last = 0;
#pragma unroll
    for (int i = 0; i < L; ++i) first |= (uint32_t)(starts[i] >= 0) << i, last |= (uint32_t)(ends[i] >= 0) << i;
  }
};

// Sequences without a row hand their state on: workgroups of their own, THREADS sequences each.
__device__ inline void hand_on(const ScanArgs& a, int64_t block, const float* from, float* to) {
  const int lane = threadIdx.x & 63;
  const int64_t s = block * THREADS + threadIdx.x, s0 = s - lane;
  bool empty = false;
  if (s < a.n_seqs) empty = a.offsets ? a.offsets[s] >= a.offsets[s + 1] : a.n_rows == 0;
  for (uint64_t left = __ballot(empty); left; left &= left - 1) {
    const int64_t at = (s0 + __builtin_ctzll(left)) * a.n_cols;
    for (int64_t c = lane; c < a.n_cols; c += 64) to[at + c] = from ? from[at + c] : 0.0f;
  }
}

// What rows make of the state that enters them: A state + B, or B whatever enters (a sequence begins among them).  As a word of memory
// that one workgroup writes once and others wait for: all ones until then; A is at most one, and 2 stands for the second kind.
// Word and wait are one 64-bit access at device scope, so nothing else has to be made visible with it.
struct Sum {
  float a, b;
  __device__ __forceinline__ bool cut() const { return a == 2.0f; }
  __device__ __forceinline__ float of(float state) const { return cut() ? b : fmaf(a, state, b); }
  // this after `first`
  __device__ __forceinline__ Sum after(Sum first) const {
    Sum r;
    r.a = cut() || first.cut() ? 2.0f : a * first.a;
    r.b = of(first.b);
    return r;
  }
};
constexpr uint64_t UNWRITTEN = ~0ull;
__device__ __forceinline__ void publish(uint64_t* w, Sum s) {
  uint64_t x = (uint64_t)__float_as_uint(s.b) << 32 | __float_as_uint(s.a);
  if (x == UNWRITTEN) x = 0x7FC000007FC00000ull;   // (two NaNs are two NaNs)
  __hip_atomic_store(w, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Waits for N words, `apart` from each other, the first `n` of them.  Whoever writes them took an earlier ticket and is on its way, so the
// wait ends; the bound (ten seconds of the 100 MHz clock) is for the case that this is wrong, and then the results are NaN.
template <int N> __device__ __forceinline__ void await(const uint64_t* w, int64_t apart, int n, Sum* s) {
  uint64_t x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = 0;
  long long t0 = 0;
  for (uint32_t k = 1;; ++k) {
    bool there = true;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) x[i] = __hip_atomic_load(w + i * apart, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int i = 0; i < N; ++i) there = there && x[i] != UNWRITTEN;
    if (there) break;
    __builtin_amdgcn_s_sleep(1);
    if (k % 256 == 0) {
      if (t0 == 0) t0 = wall_clock64();
      if (wall_clock64() - t0 > 1000000000ll) break;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = Sum{__uint_as_float((uint32_t)x[i]), __uint_as_float((uint32_t)(x[i] >> 32))};
}

// A tile's parts and what came before it, in shared memory.
template <bool CHAINED> struct Chain {
  Sum part[PARTS][COLS];                // the parts' sums, in the order of the recurrence
  float enter[PARTS][COLS];             // the states that enter the parts
  Sum before[CHAINED ? RUN : 1][COLS];  // sums of tiles or groups before this one
  uint32_t ticket;
};

// Lane j < p: whether a sequence begins (BACK: ends) in the j-th of the p tiles that are before tile i in its group of 16.
template <int ROWS, bool BACK> __device__ __forceinline__ uint64_t cuts_before(const ScanArgs& a, int64_t i) {
  const int p = (int)((uint64_t)i % RUN), lane = threadIdx.x & 63;
  if (lane >= p) return 0;
  const int64_t at = i - p + lane, t0 = (BACK ? a.n_tiles - 1 - at : at) * ROWS;
  const uint64_t* m = a.marks + t0 / MARK * 4 + (BACK ? 2 : 0);
  if constexpr (ROWS == MARK) return m[0] | m[1];
  else return m[t0 / 64 % 2];
}

// The parts' sums have been written.  The first wave, a lane a column, joins them in order, and hands every part the state that enters it.
// A chain: tile i of it (counted in the order of the recurrence) publishes its sum; the last one of 16 that of
// the group, the last one of 16 groups the state after them.  A tile joins at most 15 sums of its group, 15 of the groups before and one
// state, each waited for at most once (a wave waits for four), and always in the same order, so results do not depend on who
// comes when.  `cuts`: of cuts_before; what is before the last tile of the group with a cut does not matter and is not waited for.
template <bool CHAINED> __device__ __forceinline__ void enter(const ScanArgs& a, Chain<CHAINED>& chain, int64_t i, int64_t block, uint64_t cuts) {
  constexpr int EACH = RUN / WAVES;
  static_assert(COLS == 64 && EACH * WAVES == RUN, "a lane a column");
  const int p = (int)((uint64_t)i % RUN), q = (int)((uint64_t)i / RUN % RUN), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = block * COLS + lane;
  const bool mine = c < a.n_cols, last = i + 1 == a.n_tiles;
  Sum own{1.0f, 0.0f};
  float state = 0;
  if constexpr (CHAINED) {
    if (wave == 0) {
      for (int g = 0; g < PARTS; ++g) own = chain.part[g][lane].after(own);
      if (mine && !last) publish(a.sums + i * a.n_cols + c, own);
    }
    const uint64_t cut = __ballot(cuts != 0);
    const int from = cut ? 63 - __builtin_clzll(cut) : 0;
    const bool alone = cut || i < RUN;            // nothing before the group matters
    Sum s[EACH];
    const int j0 = (WAVES - 1 - wave) * EACH;     // (the first wave, which was busy, has one sum less to wait for)
    const int j1 = max(j0, from);
    int n = mine ? min(p, j0 + EACH) - j1 : 0;
    await<EACH>(a.sums + (i - p + j1) * a.n_cols + c, a.n_cols, n, s);
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (j < n) chain.before[j1 + j][lane] = s[j];
    __syncthreads();
    Sum group{1.0f, 0.0f};                        // what is before the tile in its group
    if (wave == 0) {
      for (int j = from; j < p; ++j) group = chain.before[j][lane].after(group);
      if (p == RUN - 1 && mine && !last) publish(a.group_sums + i / RUN * a.n_cols + c, own.after(group));
    }
    if (!alone) {
      __syncthreads();
      n = mine ? min(q - j0, EACH) : 0;
      await<EACH>(a.group_sums + (i / RUN - q + j0) * a.n_cols + c, a.n_cols, n, s);
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        if (j < n) chain.before[j0 + j][lane] = s[j];
      if (wave == 0 && mine && i >= RUN * RUN) {
        await<1>(a.super + (i / (RUN * RUN) - 1) * a.n_cols + c, 0, 1, s);
        state = s[0].b;
      }
      __syncthreads();
      if (wave == 0)
        for (int j = 0; j < q; ++j) state = chain.before[j][lane].of(state);
    }
    state = group.of(state);
    if (wave == 0 && p == RUN - 1 && q == RUN - 1 && mine && !last) publish(a.super + i / (RUN * RUN) * a.n_cols + c, Sum{2.0f, own.of(state)});
  }
  if (wave == 0) {
    for (int g = 0; g < PARTS; ++g) {
      chain.enter[g][lane] = state;
      state = chain.part[g][lane].of(state);
    }
  }
  __syncthreads();
}

// A block of columns is a chain of its own, with a counter of its own (one counter for all gives 60 tickets a microsecond at most, which
// is 3 TB/s).  Tickets are taken in order, so whoever holds a chain's first one that is not done waits for nobody.
__device__ __forceinline__ uint32_t draw(const ScanArgs& a, int64_t block) {
  return threadIdx.x == 0 ? __hip_atomic_fetch_add(a.tickets + block * TICKET_APART, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
}
__device__ __forceinline__ int64_t take(Chain<true>& chain, uint32_t drawn) {
  if (threadIdx.x == 0) chain.ticket = drawn;
  __syncthreads();
  return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)chain.ticket);
}

// Up to VEC values of a state's row in memory.
typedef float State __attribute__((ext_vector_type(VEC)));
template <bool LOOSE> __device__ __forceinline__ void load_state(const float* p, float* x, int cols) {
  if constexpr (LOOSE) {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (v < cols) x[v] = p[v];
  } else if (cols) {
    const State s = *(const State*)p;
#pragma unroll
    for (int v = 0; v < VEC; ++v) x[v] = s[v];
  }
}
template <bool LOOSE> __device__ __forceinline__ void store_state(float* p, const float* x, int cols) {
  if constexpr (LOOSE) {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (v < cols) p[v] = x[v];
  } else if (cols) {
    State s;
#pragma unroll
    for (int v = 0; v < VEC; ++v) s[v] = x[v];
    *(State*)p = s;
  }
}

// A thread's part of tile k of the rows: its elements, and the two passes over them, one for what the rows make of any state, and when
// the state that enters is known one for their results.  The gates are computed in both: kept, they would take twice the elements'
// registers, and what hides the waits is how many tiles a compute unit has at a time.
template <int DT, bool LOOSE, bool BACK, bool CHAINED> struct Tile {
  static constexpr int L = length(DT, BACK), ROWS = PARTS * L;
  typedef Window<DT, LOOSE> W;
  typedef typename W::Pack Pack;
  const ScanArgs& a;
  int64_t k, t0, n, c0;
  int at, cols, part;              // its columns, `cols` of them inside the matrix, and which of the parts it is
  Pack f[L], x[L], dh[BACK ? L : 1], h[BACK ? L : 1];
  Marks<L, CHAINED> m;

  __device__ __forceinline__ Tile(const ScanArgs& args, int64_t tile, int64_t block) : a(args), k(tile) {
    t0 = k * ROWS;
    n = min(a.n_rows - t0, (int64_t)ROWS);
    part = threadIdx.x / LANES;
    at = threadIdx.x % LANES * VEC;
    c0 = block * COLS + at;
    cols = (int)min(max(a.n_cols - c0, (int64_t)0), (int64_t)VEC);
    const W wf(a.f, a.ld_f, t0, n, a.n_cols), wx(a.x, a.ld_x, t0, n, a.n_cols);
    const auto pf = wf.place(part * L, c0, cols);
    const auto px = wx.place(part * L, c0, cols);
    if constexpr (BACK) {
      const int shift = t0 > 0;       // (of the first tile there is no row before the first)
      const W wdh(a.dh, a.ld_dh, t0, n, a.n_cols), wh(a.h, a.ld_h, t0 - shift, n, a.n_cols);
      const auto pdh = wdh.place(part * L, c0, a.dh ? cols : 0);
      const auto ph = wh.place(part * L - 1 + shift, c0, cols);
#pragma unroll
      for (int i = 0; i < L; ++i) f[i] = wf.load(pf, i), dh[i] = wdh.load(pdh, i);
#pragma unroll
      for (int i = 0; i < L; ++i) x[i] = wx.load(px, i), h[i] = wh.load(ph, i);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) f[i] = wf.load(pf, i), x[i] = wx.load(px, i);
    }
  }

  // For the compiler, other values than before: what follows from them is computed again instead of kept.
  static __device__ __forceinline__ void renew(Pack& p) {
    typedef unsigned int Words __attribute__((ext_vector_type(sizeof(p) / 4)));
    Words w = __builtin_bit_cast(Words, p);
    asm volatile("" : "+v"(w));
    p = __builtin_bit_cast(Pack, w);
  }

  // The state that a sequence begins with at row i, or the gradient that it ends with; others go on with s.
  __device__ __forceinline__ void cut(int i, float* s) const {
    if ((BACK ? m.last : m.first) >> i & 1) {
      const float* init = BACK ? a.dh_last : a.h0;
#pragma unroll
      for (int v = 0; v < VEC; ++v) s[v] = 0;
      if (init) load_state<LOOSE>(init + (BACK ? m.ends : m.starts)[i] * a.n_cols + c0, s, cols);
    }
  }

  __device__ __forceinline__ void sums(Chain<CHAINED>& chain) {
    Sum sum[VEC];
    float s[VEC] = {};
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum[v].a = 1.0f;
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int i = BACK ? L - 1 - j : j;
      cut(i, s);
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float al, keep;
        gate<DT>((float)f[i][v], al, keep);
        if constexpr (BACK) s[v] = al * (s[v] + (float)dh[i][v]);   // what travels is a_t s_t, the gradient that reaches the state before row t
        else s[v] = fmaf(al, s[v], keep * (float)x[i][v]);
        sum[v].a *= al;
      }
    }
    const bool any = (BACK ? m.last : m.first) != 0;
#pragma unroll
    for (int v = 0; v < VEC; ++v) chain.part[BACK ? PARTS - 1 - part : part][at + v] = Sum{any ? 2.0f : sum[v].a, s[v]};
  }

  __device__ __forceinline__ void results(const Chain<CHAINED>& chain, int64_t valid, int64_t end) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      renew(f[i]);
      if constexpr (BACK) renew(dh[i]);
      else renew(x[i]);
    }
    float s[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) s[v] = chain.enter[BACK ? PARTS - 1 - part : part][at + v];
    if constexpr (!BACK) {
      const W wh(a.h, a.ld_h, t0, n, a.n_cols);
      const auto ph = wh.place(part * L, c0, cols);
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const int64_t r = t0 + part * L + i;
        cut(i, s);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          float al, keep;
          gate<DT>((float)f[i][v], al, keep);
          s[v] = fmaf(al, s[v], keep * (float)x[i][v]);
        }
        if (r >= valid && r < end) wh.store(ph, i, s);
        if ((m.last >> i & 1) && a.h_last) store_state<LOOSE>(a.h_last + m.ends[i] * a.n_cols + c0, s, cols);
      }
    } else {
      const W wdf(a.df, a.ld_df, t0, n, a.n_cols), wdx(a.dx, a.ld_dx, t0, n, a.n_cols);
      const auto pdf = wdf.place(part * L, c0, cols);
      const auto pdx = wdx.place(part * L, c0, cols);
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        const int64_t r = t0 + part * L + i;
        const bool begins = m.first >> i & 1;
        float prior[VEC], df[VEC], dx[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) prior[v] = (float)h[i][v];
        if (begins) {
#pragma unroll
          for (int v = 0; v < VEC; ++v) prior[v] = 0;
          if (a.h0) load_state<LOOSE>(a.h0 + m.starts[i] * a.n_cols + c0, prior, cols);
        }
        cut(i, s);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          float al, keep;
          gate<DT>((float)f[i][v], al, keep);
          s[v] += (float)dh[i][v];
          dx[v] = s[v] * keep;
          s[v] *= al;
          df[v] = dx[v] * al * (prior[v] - (float)x[i][v]);
        }
        if (r >= valid && r < end) wdx.store(pdx, i, dx), wdf.store(pdf, i, df);
        if (begins && a.dh0) store_state<LOOSE>(a.dh0 + m.starts[i] * a.n_cols + c0, s, cols);
      }
    }
  }
};

// Workgroups that a compute unit is to have room for, and the registers of a wave that this leaves.  Rows at whole four elements need no
// more than these (79 of 80 for results in bf16, 104 to 112 of 128 in the others).  Rows at any element keep scalars in vector registers (20 to 32 in three of
// four kernels), and results in bf16 five vector registers in scratch, 16 bytes a lane; fewer workgroups for these have not been measured.
constexpr int wgs_wanted(int dt, bool back) { return dt == TDF_BF16 ? (back ? 4 : 6) : (back ? 4 : 4); }

// Several tiles of rows: every workgroup takes one ticket.  What bounds it is how long tiles are under way, waits for those before them among
// that, and the gates: 65,536 x 512 in bf16, one sequence, 55 us (3.7 TB/s; a large copy 5.0 to 5.4) and 69 with the launch before it, the vector
// units busy for half of it; 266,000 x 256, 4,096 sequences, 102 and 110; gradients of 65,536 x 1,024, two sequences, 195 and 198.
// (Workgroups that stay and take one after the other wait for their stores before the next tile's elements, which counts more than what it takes to begin: 78 us against 72 for 65,536 x 512 in bf16.)
template <int DT, bool LOOSE, bool BACK>
__global__ void __launch_bounds__(THREADS, wgs_wanted(DT, BACK)) k_scan_chain(ScanArgs a) {
  __shared__ Chain<true> chain;
  typedef const __attribute__((address_space(4))) int64_t* Scalar;
  typedef Tile<DT, LOOSE, BACK, true> T;
  const int64_t block = blockIdx.x % (uint32_t)a.n_blocks, turn = take(chain, draw(a, block));
  const uint64_t cuts = cuts_before<T::ROWS, BACK>(a, turn);
  T tile(a, BACK ? a.n_tiles - 1 - turn : turn, block);
  tile.m.of_chain(a, tile.t0, tile.part * T::L);
  const int64_t valid = a.offsets ? ((Scalar)a.offsets)[0] : 0, end = a.offsets ? ((Scalar)a.offsets)[a.n_seqs] : a.n_rows;
  tile.sums(chain);
  __syncthreads();
  enter(a, chain, turn, block, cuts);
  tile.results(chain, valid, end);
}

// One tile of rows, or none.
template <int DT, bool LOOSE, bool BACK>
__global__ void __launch_bounds__(THREADS) k_scan_tile(ScanArgs a) {
  __shared__ int32_t starts[MARK], ends[MARK];
  __shared__ Chain<false> chain;
  if ((int64_t)blockIdx.x >= a.n_tiles * a.n_blocks) {
    hand_on(a, blockIdx.x - a.n_tiles * a.n_blocks, BACK ? a.dh_last : a.h0, BACK ? a.dh0 : a.h_last);
    return;
  }
  Tile<DT, LOOSE, BACK, false> tile(a, 0, blockIdx.x);
  mark_rows(a, 0, starts, ends);
  tile.m.of_shared(tile.part * tile.L, starts, ends);
  tile.sums(chain);
  __syncthreads();
  enter(a, chain, 0, blockIdx.x, 0);
  tile.results(chain, a.offsets ? a.offsets[0] : 0, a.offsets ? a.offsets[a.n_seqs] : a.n_rows);
}

// Before a chain: the rows' marks, words that nobody has written yet, no ticket taken, and sequences without a row.
__global__ void __launch_bounds__(THREADS) k_scan_mark(ScanArgs a, int64_t words, const float* from, float* to) {
  __shared__ int32_t starts[MARK], ends[MARK];
  if ((int64_t)blockIdx.x < a.n_more) {
    hand_on(a, blockIdx.x, from, to);
    return;
  }
  const int64_t wg = blockIdx.x - a.n_more, wgs = gridDim.x - a.n_more;
  for (int64_t i = wg * THREADS + threadIdx.x; i < words; i += wgs * THREADS) a.sums[i] = UNWRITTEN;
  for (int64_t i = wg * THREADS + threadIdx.x; i < a.n_blocks; i += wgs * THREADS) a.tickets[i * TICKET_APART] = 0;
  for (int64_t k = wg; k * MARK < a.n_rows; k += wgs) {
    mark_rows(a, k * MARK, starts, ends);
    const int tid = threadIdx.x;
    if (tid < MARK) {
      const int32_t s = starts[tid], e = ends[tid];
      const uint64_t first = __ballot(s >= 0), last = __ballot(e >= 0);
      if ((tid & 63) == 0) a.marks[k * 4 + (tid >> 6)] = first, a.marks[k * 4 + 2 + (tid >> 6)] = last;
      if (s >= 0) a.starts[k * MARK + tid] = s;
      if (e >= 0) a.ends[k * MARK + tid] = e;
    }
    __syncthreads();
  }
}

struct StepArgs {
  int64_t n_rows, n_cols, n_states;
  const void* f;
  int64_t ld_f;
  const void* x;
  int64_t ld_x;
  const int32_t* slot;
  float* state;
  void* h;
  int64_t ld_h;
};

// A thread an element.  256 x 512: 2.7 us, the launch; 4,096 x 4,096 in fp32 51 us, 6.6 TB/s.
template <int DT>
__global__ void __launch_bounds__(256) k_scan_step(StepArgs a) {
  typedef typename TypeOf<DT>::type T;
  const int64_t blocks = (a.n_cols + 255) / 256, r = blockIdx.x / blocks, c = blockIdx.x % blocks * 256 + threadIdx.x;
  if (c >= a.n_cols) return;
  const int64_t s = a.slot ? a.slot[r] : r;
  float h = 0;
  if (s >= 0 && s < a.n_states) {
    float al, keep;
    gate<DT>((float)((const T*)a.f)[r * a.ld_f + c], al, keep);
    h = fmaf(al, a.state[s * a.n_cols + c], keep * (float)((const T*)a.x)[r * a.ld_x + c]);
    a.state[s * a.n_cols + c] = h;
  }
  if (a.h) ((T*)a.h)[r * a.ld_h + c] = (T)h;
}

constexpr int64_t MOST_ROWS = 1ll << 40, MOST_COLS = 1ll << 24;
constexpr int64_t MOST_SEQS = 1 << 30, MOST_TILES = (3ll << 22) - 1;   // (their workgroups together: less than 2^32 threads)

bool bad_sizes(int64_t n_rows, int64_t n_cols) { return n_rows < 0 || n_rows > MOST_ROWS || n_cols < 1 || n_cols > MOST_COLS; }

int64_t parts_of(int64_t n, int64_t of) { return (n + of - 1) / of; }

// Four elements of its rows can be read at a time, and a tile's rows span less than 2 GiB (Window).
bool fits(const void* p, int64_t ld, size_t size) { return aligned(p, ld, size, 4 * size) && ld < (1ll << 31) / MOST_ROWS_OF / (int64_t)size; }

// Words of the sums of tiles, groups and super-groups.
int64_t words_of(int64_t n_tiles, int64_t n_cols) { return (n_tiles + n_tiles / RUN + n_tiles / (RUN * RUN)) * n_cols; }

// In bytes: the tickets, the words, the marks and the rows' sequences.
struct ScanSpace {
  size_t words, marks, starts, ends, total;
  ScanSpace(int64_t n_rows, int64_t n_cols) {
    const size_t tiles = (size_t)parts_of(n_rows, LEAST_ROWS_OF), marked = (size_t)parts_of(n_rows, MARK);
    words = ((size_t)parts_of(n_cols, COLS) * TICKET_APART * sizeof(uint32_t) + 255) / 256 * 256;
    marks = words + (size_t)words_of(tiles, n_cols) * sizeof(uint64_t);
    starts = marks + marked * 4 * sizeof(uint64_t);
    ends = starts + marked * MARK * sizeof(int32_t);
    total = n_rows <= LEAST_ROWS_OF ? 0 : ends + marked * MARK * sizeof(int32_t);
  }
};

template <int DT, bool LOOSE, bool BACK> void launch_scan(ScanArgs a, int cus, hipStream_t s) {
  const float* from = BACK ? a.dh_last : a.h0;
  float* to = BACK ? a.dh0 : a.h_last;
  a.n_tiles = parts_of(a.n_rows, rows_of(DT, BACK));
  a.n_blocks = parts_of(a.n_cols, COLS);
  a.n_more = to ? (a.n_seqs + THREADS - 1) / THREADS : 0;
  const int64_t tiles = a.n_tiles * a.n_blocks;
  if (a.n_tiles <= 1) {
    if (tiles + a.n_more) k_scan_tile<DT, LOOSE, BACK><<<(unsigned)(tiles + a.n_more), THREADS, 0, s>>>(a);
    return;
  }
  a.group_sums = a.sums + a.n_tiles * a.n_cols;
  a.super = a.group_sums + a.n_tiles / RUN * a.n_cols;
  const int64_t words = words_of(a.n_tiles, a.n_cols);
  const int64_t wgs = std::min<int64_t>(std::max(a.n_tiles, (words + 4 * THREADS - 1) / (4 * THREADS)), 16 * cus);
  k_scan_mark<<<(unsigned)(a.n_more + wgs), THREADS, 0, s>>>(a, words, from, to);
  k_scan_chain<DT, LOOSE, BACK><<<(unsigned)tiles, THREADS, 0, s>>>(a);
}

// `wide`: as Window wants the rows of all matrices.
tdf_status launch_scan(const char* who, ScanArgs& a, int32_t dtype, bool wide, bool backward, void* workspace, hipStream_t s) {
  int device = 0, cus = 0;
  if (hipGetDevice(&device) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) {
    set_error(std::string(who) + ": no device");
    return TDF_ERR_DEVICE;
  }
  char* const w = (char*)workspace;
  const ScanSpace at(a.n_rows, a.n_cols);
  a.tickets = (uint32_t*)w;
  a.sums = (uint64_t*)(w + at.words);
  a.marks = (uint64_t*)(w + at.marks);
  a.starts = (int32_t*)(w + at.starts);
  a.ends = (int32_t*)(w + at.ends);
  const bool bf16 = dtype == TDF_BF16;
  if (backward) {
    if (wide) bf16 ? launch_scan<TDF_BF16, false, true>(a, cus, s) : launch_scan<TDF_F32, false, true>(a, cus, s);
    else bf16 ? launch_scan<TDF_BF16, true, true>(a, cus, s) : launch_scan<TDF_F32, true, true>(a, cus, s);
  } else {
    if (wide) bf16 ? launch_scan<TDF_BF16, false, false>(a, cus, s) : launch_scan<TDF_F32, false, false>(a, cus, s);
    else bf16 ? launch_scan<TDF_BF16, true, false>(a, cus, s) : launch_scan<TDF_F32, true, false>(a, cus, s);
  }
  return launched(who);
}

tdf_status check_scan(const char* who, const tdf_scan* in, const void* workspace, size_t workspace_bytes) {
  if (!in) return refuse(who, "in is NULL");
  if (!known_type(in->dtype)) return refuse(who, "bad dtype");
  if (bad_sizes(in->n_rows, in->n_cols)) return refuse(who, "n_rows or n_cols out of range");
  if (in->n_seqs < 1 || in->n_seqs > MOST_SEQS) return refuse(who, "n_seqs out of range");
  if (parts_of(in->n_rows, LEAST_ROWS_OF) > MOST_TILES / parts_of(in->n_cols, COLS)) return refuse(who, "n_rows or n_cols out of range");
  if (!in->offsets && in->n_seqs != 1) return refuse(who, "several sequences need offsets");
  if ((uintptr_t)in->offsets % 8 || bad_floats(in->h0)) return refuse(who, "offsets or h0 is not aligned");
  const size_t size = element_size(in->dtype);
  if (in->n_rows) {
    if (const char* bad = bad_matrix(in->f, in->ld_f, in->n_rows, in->n_cols, size)) return refuse(who, bad);
    if (const char* bad = bad_matrix(in->x, in->ld_x, in->n_rows, in->n_cols, size)) return refuse(who, bad);
  }
  size_t need = 0;
  tdf_gated_scan_workspace_size(in->n_rows, in->n_cols, &need);
  if (need && (!workspace || workspace_bytes < need || (uintptr_t)workspace % 256)) {
    set_error(std::string(who) + ": workspace too small or misaligned");
    return TDF_ERR_WORKSPACE;
  }
  return TDF_OK;
}

}  // namespace
}  // namespace tdf

using namespace tdf;

extern "C" tdf_status tdf_gated_scan_workspace_size(int64_t n_rows, int64_t n_cols, size_t* bytes) {
  const char* who = "tdf_gated_scan_workspace_size";
  if (!bytes) return refuse(who, "bytes is NULL");
  if (bad_sizes(n_rows, n_cols)) return refuse(who, "a size is out of range");
  *bytes = ScanSpace(n_rows, n_cols).total;
  return TDF_OK;
}

extern "C" tdf_status tdf_gated_scan(const tdf_scan* in, void* h, int64_t ld_h, float* h_last, void* workspace, size_t workspace_bytes,
                                     void* hip_stream) {
  const char* who = "tdf_gated_scan";
  const tdf_status st = check_scan(who, in, workspace, workspace_bytes);
  if (st != TDF_OK) return st;
  if (const char* bad = in->n_rows ? bad_matrix(h, ld_h, in->n_rows, in->n_cols, element_size(in->dtype)) : nullptr) return refuse(who, bad);
  if (bad_floats(h_last)) return refuse(who, "h_last is not aligned");
  if (in->n_rows && (h == in->f || h == in->x)) return refuse(who, "h overlaps an input");
  // (a tile reads h0 again when another may have written h_last)
  if (overlap(in->h0, h_last, in->n_seqs * in->n_cols)) return refuse(who, "h_last overlaps h0");
  ScanArgs a{in->n_rows, in->n_cols, in->n_seqs, in->f, in->ld_f, in->x, in->ld_x, in->offsets, in->h0, h, ld_h, h_last};
  const size_t size = element_size(in->dtype);
  const bool wide = in->n_cols % 4 == 0 && fits(in->f, in->ld_f, size) && fits(in->x, in->ld_x, size) && fits(h, ld_h, size) &&
                    ((uintptr_t)in->h0 | (uintptr_t)h_last) % 16 == 0;
  return launch_scan(who, a, in->dtype, wide, false, workspace, (hipStream_t)hip_stream);
}

extern "C" tdf_status tdf_gated_scan_grad(const tdf_scan* in, const tdf_scan_grads* g, void* workspace, size_t workspace_bytes,
                                          void* hip_stream) {
  const char* who = "tdf_gated_scan_grad";
  const tdf_status st = check_scan(who, in, workspace, workspace_bytes);
  if (st != TDF_OK) return st;
  if (!g) return refuse(who, "grads is NULL");
  const size_t size = element_size(in->dtype);
  if (in->n_rows) {
    if (const char* bad = bad_matrix(g->h, g->ld_h, in->n_rows, in->n_cols, size)) return refuse(who, bad);
    if (const char* bad = g->dh ? bad_matrix(g->dh, g->ld_dh, in->n_rows, in->n_cols, size) : nullptr) return refuse(who, bad);
    if (const char* bad = bad_matrix(g->df, g->ld_df, in->n_rows, in->n_cols, size)) return refuse(who, bad);
    if (const char* bad = bad_matrix(g->dx, g->ld_dx, in->n_rows, in->n_cols, size)) return refuse(who, bad);
    for (const void* out : {(const void*)g->df, (const void*)g->dx})
      if (out == in->f || out == in->x || out == g->h || out == g->dh) return refuse(who, "a gradient overlaps an input");
    if (g->df == g->dx) return refuse(who, "df overlaps dx");
  }
  if (bad_floats(g->dh_last) || bad_floats(g->dh0)) return refuse(who, "dh_last or dh0 is not aligned");
  if (overlap(g->dh_last, g->dh0, in->n_seqs * in->n_cols)) return refuse(who, "dh0 overlaps dh_last");
  if (overlap(in->h0, g->dh0, in->n_seqs * in->n_cols)) return refuse(who, "dh0 overlaps h0");
  // (without dh its window is one row at NULL, all of whose places lie beyond its end)
  ScanArgs a{in->n_rows, in->n_cols, in->n_seqs, in->f, in->ld_f, in->x, in->ld_x, in->offsets, in->h0, const_cast<void*>(g->h), g->ld_h, nullptr,
             g->dh, g->dh ? g->ld_dh : 0, g->dh_last, g->df, g->ld_df, g->dx, g->ld_dx, g->dh0};
  const bool wide = in->n_cols % 4 == 0 && fits(in->f, in->ld_f, size) && fits(in->x, in->ld_x, size) && fits(g->h, g->ld_h, size) &&
                    (!g->dh || fits(g->dh, g->ld_dh, size)) && fits(g->df, g->ld_df, size) && fits(g->dx, g->ld_dx, size) &&
                    ((uintptr_t)in->h0 | (uintptr_t)g->dh_last | (uintptr_t)g->dh0) % 16 == 0;
  return launch_scan(who, a, in->dtype, wide, true, workspace, (hipStream_t)hip_stream);
}

extern "C" tdf_status tdf_gated_scan_step(const tdf_scan_step* in, void* hip_stream) {
  const char* who = "tdf_gated_scan_step";
  if (!in) return refuse(who, "in is NULL");
  if (!known_type(in->dtype)) return refuse(who, "bad dtype");
  if (bad_sizes(in->n_rows, in->n_cols)) return refuse(who, "n_rows or n_cols out of range");
  if (in->n_states < 0 || in->n_states > MOST_ROWS) return refuse(who, "n_states out of range");
  if (!in->slot && in->n_states < in->n_rows) return refuse(who, "fewer states than rows");
  if ((uintptr_t)in->slot % 4 || bad_floats(in->state)) return refuse(who, "slot or state is not aligned");
  if (in->n_rows == 0) return TDF_OK;
  if (in->n_states && !in->state) return refuse(who, "state is NULL");
  const size_t size = element_size(in->dtype);
  if (const char* bad = bad_matrix(in->f, in->ld_f, in->n_rows, in->n_cols, size)) return refuse(who, bad);
  if (const char* bad = bad_matrix(in->x, in->ld_x, in->n_rows, in->n_cols, size)) return refuse(who, bad);
  if (const char* bad = in->h ? bad_matrix(in->h, in->ld_h, in->n_rows, in->n_cols, size) : nullptr) return refuse(who, bad);
  if (in->h && (in->h == in->f || in->h == in->x || in->h == in->state)) return refuse(who, "h overlaps an input");
  const int64_t wide = (in->n_cols + 255) / 256;
  in_runs(in->n_rows, MOST_WORKGROUPS / wide, [&](int64_t r, int64_t n) {
    const StepArgs a{n, in->n_cols, in->n_states, (const char*)in->f + r * in->ld_f * size, in->ld_f, (const char*)in->x + r * in->ld_x * size, in->ld_x,
                     in->slot ? in->slot + r : nullptr, in->slot ? in->state : in->state + r * in->n_cols, in->h ? (char*)in->h + r * in->ld_h * size : nullptr, in->ld_h};
    const unsigned grid = (unsigned)(n * wide);
    if (in->dtype == TDF_BF16) k_scan_step<TDF_BF16><<<grid, 256, 0, (hipStream_t)hip_stream>>>(a);
    else k_scan_step<TDF_F32><<<grid, 256, 0, (hipStream_t)hip_stream>>>(a);
  });
  return launched(who);
}
