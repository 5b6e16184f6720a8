// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: out[t] = s W[tok t]; a copy of rows, bound by memory (or by one memory latency for a few tokens).
//
// Gradient: dW[v] = s sum_{t: tok t = v} dY[t].  The (token, place) pairs are sorted by token, stably, so that every row's sum is
// taken in the order of places without atomics on floats: the result does not change from call to call.  A token's run may be
// anything from one place to all of them (text holds its most frequent token in some ten percent of the places), so the sorted
// list is cut into pieces of equal length: a group of threads sums up one piece, stores runs that lie inside it, and leaves the
// float32 sums of runs that cross its ends (two at most) for a second launch, which adds them in order.  Rows that no token
// names are set to zero by further workgroups of the same launch, which look them up in the sorted list: the dense gradient is written
// once.  Up to 512 places (a few sequences' ends, a probe) nothing is sorted: every workgroup finds the places of its token itself.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "chm_elements.h"
#include "chm_overlap.h"

namespace {

using namespace chm_elements;

constexpr int NT = 256;
typedef float f4 __attribute__((ext_vector_type(4)));
constexpr int SMALL = 512;               // places the unsorted kernel takes
constexpr int RANGES_MAX = 16384, RANGE_ROWS = 512 * 512 - 1;      // places and rows the sort by ranges of keys takes
constexpr int BINS = 512, DIGIT = 9;
constexpr int SORT_GROUPS = 64;
constexpr int ZERO_ROWS = 32;            // rows that a workgroup sets to zero at a time where no token names them
// A grid has fewer than 2^32 threads: workgroups that set rows to zero go on to further ones beyond 2^25 rows, a lookup is a launch for every 2^24 places
constexpr int64_t ZERO_GROUPS_MAX = 1 << 20, LOOKUP_PLACES = 1 << 24;

struct Tokens {
  const void *p;
  int32_t bits;
  uint32_t rows;
};
// the token of place i as a key: `rows` for one outside the table, behind all others
__device__ __forceinline__ uint32_t key_of(const Tokens &t, int64_t i) {
  if (t.bits == 32) {
    const uint32_t v = ((const CHM_GLOBAL uint32_t *)t.p)[i];
    return v < t.rows ? v : t.rows;
  }
  const uint64_t v = ((const CHM_GLOBAL uint64_t *)t.p)[i];
  return v < t.rows ? (uint32_t)v : t.rows;
}
// the keys of the places first, first + 64, ...; ~0, behind everything, from place n on.  All loads are issued before any is used.
template <int N>
__device__ __forceinline__ void keys_of(const Tokens &t, int first, int n, uint32_t *key) {
  if (t.bits == 32) {
    uint32_t v[N];
#pragma unroll
    for (int r = 0; r < N; ++r) v[r] = ((const CHM_GLOBAL uint32_t *)t.p)[first + r * 64 < n ? first + r * 64 : n - 1];
#pragma unroll
    for (int r = 0; r < N; ++r) key[r] = first + r * 64 >= n ? ~0u : v[r] < t.rows ? v[r] : t.rows;
  } else {
    uint64_t v[N];
#pragma unroll
    for (int r = 0; r < N; ++r) v[r] = ((const CHM_GLOBAL uint64_t *)t.p)[first + r * 64 < n ? first + r * 64 : n - 1];
#pragma unroll
    for (int r = 0; r < N; ++r) key[r] = first + r * 64 >= n ? ~0u : v[r] < t.rows ? (uint32_t)v[r] : t.rows;
  }
}

// ---------------------------------------------------------------------------------------------- rows in pieces of 16 bytes
// `count` (<= N) values of a row as float32; the rest 0
template <int DT>
__device__ __forceinline__ void row_load(const char *p, int count, float *v) {
  typedef Lane<DT> L;
  if (count >= L::N) {
    L::up(load16(p), v);
  } else {
#pragma unroll
    for (int e = 0; e < L::N; ++e) v[e] = e < count ? L::one(p + e * L::SIZE) : 0.f;
  }
}
template <int DT, int N, int PAST>
__device__ __forceinline__ void row_store(char *p, int count, const float *v) {
  typedef Lane<DT> L;
  if (count >= N) {
#pragma unroll
    for (int i = 0; i < N / L::N; ++i) {
      if (PAST) store16_past(p + i * 16, L::down(v + i * L::N));
      else store16(p + i * 16, L::down(v + i * L::N));
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < count) L::put(p + e * L::SIZE, v[e]);
  }
}
template <int DT, int N>
__device__ __forceinline__ void row_add(char *p, int count, float *v) {
  typedef Lane<DT> L;
  if (count >= N) {
#pragma unroll
    for (int i = 0; i < N / L::N; ++i) {
      float old[L::N];
      L::up(load16(p + i * 16), old);
#pragma unroll
      for (int e = 0; e < L::N; ++e) v[i * L::N + e] += old[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < count) v[e] += L::one(p + e * L::SIZE);
  }
}

// ---------------------------------------------------------------------------------------------- lookup
struct Lookup {
  Tokens tokens;
  const char *table;
  char *out;
  int64_t n, ld_table, ld_out;           // rows in bytes
  int32_t width, across;                 // threads along a row
  float scale;
};

template <int DT, int ROWS>
__global__ void __launch_bounds__(NT) k_lookup(Lookup c) {
  typedef Lane<DT> L;
  const int x = threadIdx.x % c.across, y = threadIdx.x / c.across, down = NT / c.across;
  const int col = (blockIdx.y * c.across + x) * L::N, left = c.width - col;
  if (left <= 0) return;
  const int64_t first = (int64_t)blockIdx.x * down * ROWS + y;
  float v[ROWS][8];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t t = first + (int64_t)r * down;
    const uint32_t key = t < c.n ? key_of(c.tokens, t) : c.tokens.rows;
    if (key < c.tokens.rows) {
      row_load<DT>(c.table + key * c.ld_table + (int64_t)col * L::SIZE, left, v[r]);
    } else {
#pragma unroll
      for (int e = 0; e < L::N; ++e) v[r][e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < L::N; ++e) v[r][e] = key < c.tokens.rows ? v[r][e] * c.scale : 0.f;
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t t = first + (int64_t)r * down;
    if (t < c.n) row_store<DT, L::N, (ROWS > 1)>(c.out + t * c.ld_out + (int64_t)col * L::SIZE, left, v[r]);
  }
}

// ---------------------------------------------------------------------------------------------- sort
// Stable sort by digits of at most 9 bits.  Lanes of a wavefront that hold the same digit find each other by ballots; a
// wavefront's items keep their order, wavefronts take consecutive items.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((d >> b) & 1);
    m &= (d >> b) & 1 ? set : ~set;
  }
  return m;
}

// n <= 16,384 and at most 512 x 512 rows: every workgroup takes 512 neighbouring keys.  It looks at all tokens: those below its keys give
// the place where its own begin, its own are counted by key and wavefront, and then put where they belong, in order.  Nothing is written
// in between, and one launch sorts; all workgroups read the same 64 or 128 KiB from the cache.
__global__ void __launch_bounds__(1024) k_sort_ranges(Tokens tokens, int n, uint32_t *keys, uint32_t *places, uint8_t *named) {
  __shared__ __attribute__((aligned(16))) uint32_t counts[BINS * 16];           // [key][wavefront]
  __shared__ uint32_t totals[16], belows[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t base = blockIdx.x * BINS;
  const int rounds = (n + 1023) / 1024, first = wave * rounds * 64 + lane, end = (wave + 1) * rounds * 64;
  for (int i = threadIdx.x; i < BINS * 16 / 4; i += 1024) ((Words *)counts)[i] = Words{0, 0, 0, 0};
  uint32_t key[16];
  keys_of<16>(tokens, first, n < end ? n : end, key);
  __syncthreads();
  uint32_t below = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (r >= rounds) continue;
    below += __popcll(__ballot(key[r] < base));
    if (key[r] - base < BINS) atomicAdd(&counts[(key[r] - base) * 16 + wave], 1u);
  }
  if (lane == 0) belows[wave] = below;
  __syncthreads();
  // exclusive sums over (key, wavefront), 8 entries a thread, behind all smaller keys
  uint32_t c[8], sum = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) { c[e] = counts[threadIdx.x * 8 + e]; sum += c[e]; }
  const uint32_t both = sum + __shfl_xor(sum, 1);
  if (!(threadIdx.x & 1) && base + threadIdx.x / 2 < tokens.rows) named[base + threadIdx.x / 2] = both != 0;
  uint32_t incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) totals[wave] = incl;
  __syncthreads();
  uint32_t at = incl - sum;
  for (int w = 0; w < 16; ++w) at += belows[w] + (w < wave ? totals[w] : 0u);
#pragma unroll
  for (int e = 0; e < 8; ++e) { counts[threadIdx.x * 8 + e] = at; at += c[e]; }
  __syncthreads();
  volatile uint32_t *mine = counts + wave;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (r >= rounds) continue;
    const bool in = key[r] - base < BINS;
    const uint64_t ins = __ballot(in);
    if (!ins) continue;
    const uint32_t d = in ? key[r] - base : 0;
    uint64_t m = 0;
    if (__popcll(ins) > 8) {
      m = same_digit(d, DIGIT) & ins;
    } else {                                // few lanes: key by key
      for (uint64_t left = ins; left;) {
        const uint32_t one = __builtin_amdgcn_readlane(d, __ffsll((unsigned long long)left) - 1);
        const uint64_t same = __ballot(in && d == one);
        if (d == one) m = same;
        left &= ~same;
      }
    }
    if (in) {
      const uint32_t to = mine[d * 16];
      const uint32_t p = to + __popcll(m & ((1ull << lane) - 1));
      keys[p] = key[r];
      places[p] = first + r * 64;
      if ((m >> lane) == 1) mine[d * 16] = to + __popcll(m);        // the group's last lane; the wavefront's reads are behind it
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Many workgroups: per pass, the digits of every workgroup's stretch are counted, then its pairs are moved
struct SortPass {
  Tokens tokens;                          // first pass: keys come from here, places are the indices
  const uint32_t *keys_in, *places_in;    // null in the first pass
  uint32_t *keys, *places, *counts;       // counts: [workgroup][BINS]
  uint8_t *named;                         // first pass: which rows are named by a token
  int64_t n;
  int32_t stretch, shift, digit;          // stretch: items of a workgroup, a multiple of 512
};
constexpr int SORT_NT = 512;

__device__ __forceinline__ uint32_t pass_key(const SortPass &c, int64_t i) { return c.keys_in ? c.keys_in[i] : key_of(c.tokens, i); }

__global__ void __launch_bounds__(SORT_NT) k_sort_count(SortPass c) {
  __shared__ uint32_t counts[BINS];
  counts[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * c.stretch, last = first + c.stretch < c.n ? first + c.stretch : c.n;
  const uint32_t mask = (1u << c.digit) - 1;
  if (!c.keys_in)
    for (int64_t i = (int64_t)blockIdx.x * SORT_NT + threadIdx.x; i < c.tokens.rows; i += (int64_t)gridDim.x * SORT_NT) c.named[i] = 0;
  for (int64_t i = first + threadIdx.x; i < last; i += SORT_NT) atomicAdd(&counts[(pass_key(c, i) >> c.shift) & mask], 1u);
  __syncthreads();
  c.counts[(int64_t)blockIdx.x * BINS + threadIdx.x] = counts[threadIdx.x];
}

__global__ void __launch_bounds__(SORT_NT) k_sort_move(SortPass c) {
  constexpr int WAVES = SORT_NT / 64;
  __shared__ uint32_t counts[BINS * WAVES];
  __shared__ uint32_t totals[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t mask = (1u << c.digit) - 1;
  const int64_t first = (int64_t)blockIdx.x * c.stretch + (int64_t)wave * (c.stretch / WAVES);
  const int64_t end = first + c.stretch / WAVES, last = end < c.n ? end : c.n;
  for (int i = threadIdx.x; i < BINS * WAVES; i += SORT_NT) counts[i] = 0;
  __syncthreads();
  for (int64_t i = first + lane; i < last; i += 64) atomicAdd(&counts[((pass_key(c, i) >> c.shift) & mask) * WAVES + wave], 1u);
  // where this workgroup's items of digit threadIdx.x start: all smaller digits, and this one in the workgroups before
  uint32_t all = 0, before = 0;
#pragma unroll 16
  for (uint32_t g = 0; g < gridDim.x; ++g) {
    const uint32_t v = c.counts[(int64_t)g * BINS + threadIdx.x];
    if (g < blockIdx.x) before += v;
    all += v;
  }
  uint32_t incl = all;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) totals[wave] = incl;
  __syncthreads();
  uint32_t at = incl - all + before;
  for (int w = 0; w < wave; ++w) at += totals[w];
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const uint32_t v = counts[threadIdx.x * WAVES + w];
    counts[threadIdx.x * WAVES + w] = at;
    at += v;
  }
  __syncthreads();
  volatile uint32_t *mine = counts + wave;
  for (int64_t i0 = first; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool in = i < last;
    const uint32_t key = in ? pass_key(c, i) : 0;
    const uint32_t place = in ? (c.places_in ? c.places_in[i] : (uint32_t)i) : 0;
    const uint32_t d = (key >> c.shift) & mask;
    const uint64_t m = same_digit(d, c.digit) & __ballot(in);
    const uint32_t base = mine[d * WAVES];
    __builtin_amdgcn_wave_barrier();
    if (in) {
      if ((m >> lane) == 1) mine[d * WAVES] = base + __popcll(m);
      const uint32_t to = base + __popcll(m & ((1ull << lane) - 1));
      c.keys[to] = key;
      c.places[to] = place;
      if (!c.keys_in && key < c.tokens.rows) c.named[key] = 1;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------------------------------------- sums over runs
struct Gather {
  Tokens tokens;
  const uint32_t *keys, *places;         // sorted
  const uint8_t *named;                  // [rows]: some token names the row
  const char *dy;
  char *grad;
  float *part;                           // [pieces][2][width rounded up to 8]
  int64_t n, ld_dy, ld_grad;             // rows in bytes
  int32_t width, across, zero_across, piece, pieces;
  int32_t piece_groups;                  // workgroups (along x) that take pieces; the ones behind set rows to zero
  int32_t accumulate;
  float scale;
};

template <int GT, int N>
__device__ __forceinline__ void finish_row(const Gather &c, uint32_t key, int col, int left, float *v) {
  char *p = c.grad + key * c.ld_grad + (int64_t)col * Lane<GT>::SIZE;
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] *= c.scale;
  if (c.accumulate) row_add<GT, N>(p, left, v);
  row_store<GT, N, 1>(p, left, v);
}

__device__ __forceinline__ int64_t part_row(const Gather &c, int64_t piece, int slot) {
  return (piece * 2 + slot) * ((c.width + 7) & ~7);
}

// rows [first, first + ZERO_ROWS) without a token, of which `named` knows
template <int GT>
__device__ __forceinline__ void zero_rows(const Gather &c, int64_t first, const uint8_t *named) {
  constexpr int N = Lane<GT>::N;
  const float zero[N] = {};
  // a power of two of threads along a row, as many rows at a time as that leaves
  const int x = threadIdx.x & (c.zero_across - 1), down = NT / c.zero_across;
  for (int r = threadIdx.x / c.zero_across; r < ZERO_ROWS; r += down) {
    if (named[r]) continue;
    char *row = c.grad + (first + r) * c.ld_grad;
    for (int col = x * N; col < c.width; col += c.zero_across * N) row_store<GT, N, 1>(row + (int64_t)col * Lane<GT>::SIZE, c.width - col, zero);
  }
}

template <int DT, int GT>
__global__ void __launch_bounds__(NT) k_runs(Gather c) {
  typedef Lane<DT> L;
  constexpr int N = L::N, AT_ONCE = 8;
  __shared__ uint32_t lk[2048], lp[2048];        // NT / across pieces of at most 64 places, across >= 8
  if ((int)blockIdx.x >= c.piece_groups) {
    if (blockIdx.y) return;
    __shared__ uint8_t named[ZERO_ROWS];
    const int64_t step = (int64_t)(gridDim.x - c.piece_groups) * ZERO_ROWS;
    for (int64_t first = (int64_t)(blockIdx.x - c.piece_groups) * ZERO_ROWS; first < c.tokens.rows; first += step) {
      if (threadIdx.x < ZERO_ROWS) named[threadIdx.x] = first + threadIdx.x < c.tokens.rows ? c.named[first + threadIdx.x] : 1;
      __syncthreads();
      zero_rows<GT>(c, first, named);
      __syncthreads();
    }
    return;
  }
  const int x = threadIdx.x % c.across, y = threadIdx.x / c.across, down = NT / c.across;
  const int64_t group_first = (int64_t)blockIdx.x * down * c.piece;
  for (int i = threadIdx.x; i < down * c.piece; i += NT)
    if (group_first + i < c.n) { lk[i] = c.keys[group_first + i]; lp[i] = c.places[group_first + i]; }
  __syncthreads();
  const int64_t piece = (int64_t)blockIdx.x * down + y, lo = piece * c.piece;
  const int col = (blockIdx.y * c.across + x) * N, left = c.width - col;
  if (piece >= c.pieces || left <= 0) return;
  const int count = c.n - lo < c.piece ? (int)(c.n - lo) : c.piece;
  const uint32_t *k = lk + y * c.piece, *p = lp + y * c.piece;
  const uint32_t before = lo > 0 ? c.keys[lo - 1] : ~0u, behind = lo + count < c.n ? c.keys[lo + count] : ~0u;
  const char *dy = c.dy + (int64_t)col * L::SIZE;
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  bool started = k[0] != before;
  for (int i0 = 0; i0 < count; i0 += AT_ONCE) {
    float v[AT_ONCE][N];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u < count ? i0 + u : count - 1;
      if (k[i] < c.tokens.rows) row_load<DT>(dy + p[i] * c.ld_dy, left, v[u]);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u;
      if (i >= count || k[i] >= c.tokens.rows) break;
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += v[u][e];
      const uint32_t next = i + 1 < count ? k[i + 1] : behind;
      if (next == k[i] && i + 1 < count) continue;
      if (next != k[i] && started) {
        finish_row<GT, N>(c, k[i], col, left, sum);
      } else {
        float *to = c.part + part_row(c, piece, started) + col;
#pragma unroll
        for (int e = 0; e < N; e += 4) *(Words *)(to + e) = Lane<CHM_F32>::down(sum + e);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] = 0.f;
      started = true;
    }
  }
}

// Runs that cross pieces: the piece in which one starts adds up what the others have left, in order.  A workgroup takes 256 columns of
// JOIN_PIECES pieces, its four wavefronts a quarter of every run each, so that the most frequent token's run (some ten percent of the places)
// is no chain of additions as long as its pieces.
constexpr int JOIN_PIECES = 2;
template <int GT>
__global__ void __launch_bounds__(NT) k_join(Gather c) {
  constexpr int N = 4, AT_ONCE = 8;
  __shared__ f4 sums[NT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = (blockIdx.y * 64 + lane) * N, left = c.width - col;
  // pieces of this workgroup in which a run starts that goes on behind them
  uint32_t key = 0;
  bool starts = false;
  const int64_t piece = (int64_t)blockIdx.x * JOIN_PIECES + lane;
  if (lane < JOIN_PIECES && piece + 1 < c.pieces) {
    const int64_t lo = piece * c.piece, hi = lo + c.piece;
    key = c.keys[hi - 1];
    starts = key < c.tokens.rows && key == c.keys[hi] && !(c.keys[lo] == key && lo > 0 && c.keys[lo - 1] == key);
  }
  uint64_t todo = __ballot(starts);
  while (todo) {
    const int l = __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    const uint32_t k = __builtin_amdgcn_readlane(key, l);
    const int64_t p = (int64_t)blockIdx.x * JOIN_PIECES + l;
    int64_t last = p;                       // the last piece that begins with the key
    for (bool more = true; more;) {
      const int64_t q = last + 1 + lane;
      const uint64_t same = __ballot(q < c.pieces && c.keys[q < c.pieces ? q * c.piece : 0] == k);
      more = same == ~0ull;
      last += more ? 64 : __ffsll((unsigned long long)~same) - 1;
    }
    // parts: slot 1 of piece p, slot 0 of p + 1 .. last
    const int count = (int)(last - p) + 1, from = count * wave / 4, to = count * (wave + 1) / 4;
    f4 sum = {0.f, 0.f, 0.f, 0.f};
    if (left > 0)
      for (int i0 = from; i0 < to; i0 += AT_ONCE) {
        f4 v[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
          const int i = i0 + u < to ? i0 + u : to - 1;
          v[u] = *(const CHM_GLOBAL f4 *)(c.part + part_row(c, p + i, i == 0) + col);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
          if (i0 + u < to) sum += v[u];
      }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (wave == 0 && left > 0) {
      sum = sums[lane] + sums[64 + lane] + sums[128 + lane] + sums[192 + lane];
      float v[N] = {sum[0], sum[1], sum[2], sum[3]};
      char *to_row = c.grad + k * c.ld_grad + (int64_t)col * Lane<GT>::SIZE;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (e >= left) break;
        v[e] *= c.scale;
        if (c.accumulate) v[e] += Lane<GT>::one(to_row + e * Lane<GT>::SIZE);
        Lane<GT>::put(to_row + e * Lane<GT>::SIZE, v[e]);
      }
    }
    __syncthreads();
  }
}

// n <= SMALL: workgroup (t, columns) sums up the places of the token at t if t is its first; the ones behind set rows to zero
template <int DT, int GT>
__global__ void __launch_bounds__(NT) k_few(Gather c) {
  typedef Lane<DT> L;
  constexpr int N = L::N, AT_ONCE = 8, EACH = SMALL / NT, WAVES = NT / 64;
  const int n = (int)c.n;
  uint32_t own[EACH];                       // tokens threadIdx.x, threadIdx.x + NT, ...
#pragma unroll
  for (int i = 0; i < EACH; ++i) own[i] = (int)threadIdx.x + i * NT < n ? key_of(c.tokens, threadIdx.x + i * NT) : ~0u;
  if ((int)blockIdx.x >= n) {
    if (blockIdx.y) return;
    __shared__ uint8_t named[ZERO_ROWS];
    const int64_t step = (int64_t)(gridDim.x - n) * ZERO_ROWS;
    for (int64_t first = (int64_t)(blockIdx.x - n) * ZERO_ROWS; first < c.tokens.rows; first += step) {
      if (threadIdx.x < ZERO_ROWS) named[threadIdx.x] = first + threadIdx.x >= c.tokens.rows;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (own[i] < c.tokens.rows && own[i] >= first && own[i] < first + ZERO_ROWS) named[own[i] - first] = 1;
      __syncthreads();
      zero_rows<GT>(c, first, named);
      __syncthreads();
    }
    return;
  }
  __shared__ uint16_t list[SMALL];
  __shared__ int counts[EACH * WAVES];
  const uint32_t key = key_of(c.tokens, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t m[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    m[i] = __ballot(own[i] == key);
    if (lane == 0) counts[i * WAVES + wave] = __popcll(m[i]);
  }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    int at = __popcll(m[i] & ((1ull << lane) - 1));
    for (int w = 0; w < i * WAVES + wave; ++w) at += counts[w];
    if (own[i] == key) list[at] = (uint16_t)(threadIdx.x + i * NT);
  }
  for (int w = 0; w < EACH * WAVES; ++w) total += counts[w];
  __syncthreads();
  if (key >= c.tokens.rows || list[0] != blockIdx.x) return;
  const int col = (blockIdx.y * NT + threadIdx.x) * N, left = c.width - col;
  if (left <= 0) return;
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  for (int i0 = 0; i0 < total; i0 += AT_ONCE) {
    float v[AT_ONCE][N];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
      if (i0 + u < total) row_load<DT>(c.dy + list[i0 + u] * c.ld_dy + (int64_t)col * L::SIZE, left, v[u]);
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (i0 + u >= total) break;
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += v[u][e];
    }
  }
  finish_row<GT, N>(c, key, col, left, sum);
}

// ---------------------------------------------------------------------------------------------- host side
int size_of(int dtype) { return dtype == CHM_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == CHM_F32 || dtype == CHM_BF16 || dtype == CHM_F16; }

// threads along a row of `groups` 16-byte groups: a power of two from 8 to 256
int across_of(int64_t groups) {
  int a = 8;
  while (a < NT && a < groups) a <<= 1;
  return a;
}

// at most that many threads
int zero_across_of(int64_t groups) {
  int a = 8;
  while (a < NT && a * 2 <= groups) a <<= 1;
  return a;
}

// places of a piece: about 512 pieces and more, 8 to 64 places each
int piece_of(int64_t n) {
  int p = 8;
  while (p < 64 && n / p > 512) p <<= 1;
  return p;
}

struct Scratch { uint64_t keys[2], places[2], counts, named, part, bytes; };

bool by_ranges(int64_t n, int64_t rows) { return n <= RANGES_MAX && rows <= RANGE_ROWS; }

Scratch scratch_of(int64_t n, int64_t rows, int64_t width) {
  Scratch s{};
  if (n <= SMALL) return s;
  uint64_t at = 0;
  const auto take = [&](uint64_t bytes) { const uint64_t o = at; at += (bytes + 255) & ~255ull; return o; };
  for (int i = 0; i < 2; ++i) { s.keys[i] = take(n * 4); s.places[i] = take(n * 4); }
  s.counts = take((uint64_t)SORT_GROUPS * BINS * 4);
  s.named = take(rows);
  const int64_t pieces = (n + piece_of(n) - 1) / piece_of(n);
  s.part = take((uint64_t)pieces * 2 * ((width + 7) & ~7ll) * 4);
  s.bytes = at;
  return s;
}

// workgroups that set the rows without a token to zero
int64_t zero_groups(const Gather &c) {
  const int64_t g = ((int64_t)c.tokens.rows + ZERO_ROWS - 1) / ZERO_ROWS;
  return c.accumulate ? 0 : g < ZERO_GROUPS_MAX ? g : ZERO_GROUPS_MAX;
}

template <int DT, int GT>
bool launch_few(Gather c, hipStream_t st) {
  c.zero_across = zero_across_of(c.width / Lane<GT>::N);
  const int64_t zero = zero_groups(c);
  const int cols = (c.width + NT * Lane<DT>::N - 1) / (NT * Lane<DT>::N);
  if (c.n + zero) hipLaunchKernelGGL((k_few<DT, GT>), dim3((uint32_t)(c.n + zero), cols), dim3(NT), 0, st, c);
  return hipGetLastError() == hipSuccess;
}

template <int DT, int GT>
bool launch_runs(Gather c, hipStream_t st) {
  const int64_t groups = (c.width + Lane<DT>::N - 1) / Lane<DT>::N;
  c.across = across_of(groups);
  c.zero_across = zero_across_of(c.width / Lane<GT>::N);
  const int down = NT / c.across;
  c.piece_groups = (c.pieces + down - 1) / down;
  const int64_t zero = zero_groups(c);
  hipLaunchKernelGGL((k_runs<DT, GT>), dim3((uint32_t)(c.piece_groups + zero), (uint32_t)((groups + c.across - 1) / c.across)), dim3(NT), 0, st, c);
  hipLaunchKernelGGL((k_join<GT>), dim3((uint32_t)((c.pieces + JOIN_PIECES - 1) / JOIN_PIECES), (uint32_t)((c.width + 255) / 256)), dim3(NT), 0, st, c);
  return hipGetLastError() == hipSuccess;
}

template <int DT>
bool launch_lookup(Lookup c, hipStream_t st) {
  const int64_t groups = (c.width + Lane<DT>::N - 1) / Lane<DT>::N;
  c.across = across_of(groups);
  const uint32_t cols = (uint32_t)((groups + c.across - 1) / c.across);
  const int down = NT / c.across;
  for (int64_t left = c.n; left > 0; left -= LOOKUP_PLACES) {
    c.n = left < LOOKUP_PLACES ? left : LOOKUP_PLACES;
    if (c.n >= 4096) hipLaunchKernelGGL((k_lookup<DT, 2>), dim3((uint32_t)((c.n + 2 * down - 1) / (2 * down)), cols), dim3(NT), 0, st, c);
    else hipLaunchKernelGGL((k_lookup<DT, 1>), dim3((uint32_t)((c.n + down - 1) / down), cols), dim3(NT), 0, st, c);
    c.tokens.p = (const char *)c.tokens.p + LOOKUP_PLACES * (c.tokens.bits / 8);
    c.out += LOOKUP_PLACES * c.ld_out;
  }
  return hipGetLastError() == hipSuccess;
}

bool aligned(const void *p, int64_t to) { return (uintptr_t)p % to == 0; }

using chm_overlap::Rows;
using chm_overlap::stretch;
Rows rows_of(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size) { return Rows{p, rows, cols * size, ld * size}; }

}  // namespace

extern "C" int chm_embedding_lookup(int32_t dtype, int32_t index_bits, const void *tokens, int64_t n, const void *table,
                                    int64_t ld_table, int64_t rows, int64_t width, float scale, void *out, int64_t ld_out,
                                    void *hip_stream) {
  if (!known(dtype) || (index_bits != 32 && index_bits != 64) || n < 0 || n > INT32_MAX || rows < 0 || rows > INT32_MAX || width < 1 ||
      width > (1 << 24) || ld_table < width || ld_out < width || ld_table > INT32_MAX || ld_out > INT32_MAX)
    return CHM_ERR_ARG;
  const int size = size_of(dtype);
  if (!aligned(tokens, index_bits / 8) || !aligned(table, size) || !aligned(out, size)) return CHM_ERR_ARG;
  if (n == 0) return CHM_OK;
  if (!tokens || !out || (rows > 0 && !table)) return CHM_ERR_ARG;
  const Rows result[] = {rows_of(out, n, width, ld_out, size)}, inputs[] = {rows_of(table, rows, width, ld_table, size), stretch(tokens, n * (index_bits / 8))};
  if (chm_overlap::clash(result, inputs)) return CHM_ERR_ARG;
  Lookup c{};
  c.tokens = Tokens{tokens, index_bits, (uint32_t)rows};
  c.table = (const char *)table;
  c.out = (char *)out;
  c.n = n;
  c.ld_table = ld_table * size;
  c.ld_out = ld_out * size;
  c.width = (int32_t)width;
  c.scale = scale;
  hipStream_t st = (hipStream_t)hip_stream;
  const bool ok = dtype == CHM_F32 ? launch_lookup<CHM_F32>(c, st) : dtype == CHM_BF16 ? launch_lookup<CHM_BF16>(c, st) : launch_lookup<CHM_F16>(c, st);
  return ok ? CHM_OK : CHM_ERR_HIP;
}

extern "C" int chm_embedding_gradient_scratch(int64_t n, int64_t rows, int64_t width, uint64_t *bytes) {
  if (!bytes || n < 0 || n > INT32_MAX || rows < 0 || rows > INT32_MAX || width < 1 || width > (1 << 24)) return CHM_ERR_ARG;
  *bytes = scratch_of(n, rows, width).bytes;
  return CHM_OK;
}

extern "C" int chm_embedding_gradient(int32_t dtype, int32_t grad_dtype, int32_t index_bits, const void *tokens, int64_t n, const void *dy,
                                      int64_t ld_dy, int64_t rows, int64_t width, float scale, void *grad, int64_t ld_grad,
                                      int32_t accumulate, void *scratch, uint64_t scratch_bytes, void *hip_stream) {
  if (!known(dtype) || (grad_dtype != dtype && grad_dtype != CHM_F32) || (index_bits != 32 && index_bits != 64) || n < 0 || n > INT32_MAX ||
      rows < 0 || rows > INT32_MAX || width < 1 || width > (1 << 24) || ld_dy < width || ld_grad < width || ld_dy > INT32_MAX ||
      ld_grad > INT32_MAX)
    return CHM_ERR_ARG;
  if (!aligned(tokens, index_bits / 8) || !aligned(dy, size_of(dtype)) || !aligned(grad, size_of(grad_dtype)) || !aligned(scratch, 16))
    return CHM_ERR_ARG;
  if (rows == 0) return CHM_OK;
  if (!grad || (n > 0 && (!tokens || !dy))) return CHM_ERR_ARG;
  const Scratch s = scratch_of(n, rows, width);
  if (s.bytes && !scratch) return CHM_ERR_ARG;
  if (scratch_bytes < s.bytes) return CHM_ERR_LIMIT;
  const Rows results[] = {rows_of(grad, rows, width, ld_grad, size_of(grad_dtype)), stretch(scratch, (int64_t)s.bytes)},
             inputs[] = {rows_of(dy, n, width, ld_dy, size_of(dtype)), stretch(tokens, n * (index_bits / 8))};
  if (chm_overlap::clash(results, inputs)) return CHM_ERR_ARG;
  hipStream_t st = (hipStream_t)hip_stream;
  char *mem = (char *)scratch;
  Gather c{};
  c.tokens = Tokens{tokens, index_bits, (uint32_t)rows};
  c.dy = (const char *)dy;
  c.grad = (char *)grad;
  c.n = n;
  c.ld_dy = ld_dy * size_of(dtype);
  c.ld_grad = ld_grad * size_of(grad_dtype);
  c.width = (int32_t)width;
  c.accumulate = accumulate != 0;
  c.scale = scale;
  if (n > SMALL) {
    int bits = 0;
    while (bits < 32 && (uint64_t)rows >> bits) ++bits;                  // keys 0 .. rows
    const int passes = (bits + DIGIT - 1) / DIGIT, digit = (bits + passes - 1) / passes;
    uint32_t *keys = (uint32_t *)(mem + s.keys[0]), *places = (uint32_t *)(mem + s.places[0]);
    if (by_ranges(n, rows)) {
      hipLaunchKernelGGL(k_sort_ranges, dim3((uint32_t)(rows / BINS + 1)), dim3(1024), 0, st, c.tokens, (int)n, keys, places, (uint8_t *)(mem + s.named));
    } else {
      SortPass p{};
      p.tokens = c.tokens;
      p.counts = (uint32_t *)(mem + s.counts);
      p.named = (uint8_t *)(mem + s.named);
      p.n = n;
      int64_t stretch = (n + SORT_GROUPS - 1) / SORT_GROUPS;
      if (stretch < 1024) stretch = 1024;
      stretch = (stretch + 511) & ~511ll;
      p.stretch = (int32_t)stretch;
      p.digit = digit;
      const uint32_t groups = (uint32_t)((n + stretch - 1) / stretch);
      for (int pass = 0; pass < passes; ++pass) {
        const int to = (passes - 1 - pass) & 1;                          // the last pass ends in the first set
        p.keys_in = pass ? (uint32_t *)(mem + s.keys[to ^ 1]) : nullptr;
        p.places_in = pass ? (uint32_t *)(mem + s.places[to ^ 1]) : nullptr;
        p.keys = (uint32_t *)(mem + s.keys[to]);
        p.places = (uint32_t *)(mem + s.places[to]);
        p.shift = pass * digit;
        hipLaunchKernelGGL(k_sort_count, dim3(groups), dim3(SORT_NT), 0, st, p);
        hipLaunchKernelGGL(k_sort_move, dim3(groups), dim3(SORT_NT), 0, st, p);
      }
    }
    c.keys = keys;
    c.places = places;
    c.named = (const uint8_t *)(mem + s.named);
    c.part = (float *)(mem + s.part);
    c.piece = piece_of(n);
    c.pieces = (int32_t)((n + c.piece - 1) / c.piece);
  }
  const bool few = n <= SMALL;
  bool ok;
  if (dtype == CHM_F32) ok = few ? launch_few<CHM_F32, CHM_F32>(c, st) : launch_runs<CHM_F32, CHM_F32>(c, st);
  else if (dtype == CHM_BF16 && grad_dtype == CHM_F32) ok = few ? launch_few<CHM_BF16, CHM_F32>(c, st) : launch_runs<CHM_BF16, CHM_F32>(c, st);
  else if (dtype == CHM_BF16) ok = few ? launch_few<CHM_BF16, CHM_BF16>(c, st) : launch_runs<CHM_BF16, CHM_BF16>(c, st);
  else if (grad_dtype == CHM_F32) ok = few ? launch_few<CHM_F16, CHM_F32>(c, st) : launch_runs<CHM_F16, CHM_F32>(c, st);
  else ok = few ? launch_few<CHM_F16, CHM_F16>(c, st) : launch_runs<CHM_F16, CHM_F16>(c, st);
  return ok ? CHM_OK : CHM_ERR_HIP;
}
