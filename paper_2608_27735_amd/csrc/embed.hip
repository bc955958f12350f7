// embed.hip -- rows of a table by index, scaled, and the table's gradient by sorted
// indexes.
//
// y[i] = scale table[index[i]]; dtable[r] = scale times the sum of dy[i] over the i whose
// index is r, in the order of i. An index outside the table gives a row of zeros and has
// no gradient.
//
// The sort: positions by index, equal ones in order (stable, least digit first), with
// counts of every digit by parts of kSortPart keys, their prefix sums, and a scatter whose
// ranks come from ballots: three launches for each digit of up to kSortBits bits, and no
// atomics on memory; of few positions all pairs compared in one launch. ranges[r] is where row r's positions begin and end in that order.
//
// The gradient: rows of up to kRun positions are added up by the lanes that write them;
// of longer ones (a feature that thousands share, a frequent token) every chunk of kRun
// positions in order gives a partial sum in fp32, and a workgroup for each such row adds
// these. Either way the order of the sums is fixed by the indexes alone.
//
// Lookup of 1M x 64 from 100,000 rows in bf16: 39 us; of its 145 MB the table's rows come
// about nine times from behind the L2s, which hold a third of it (115 MB read, 128
// written). Gradient of the same in fp32: sums 57 us (285 MB, 5.0 TB/s), and 54 for the sort
// in seven launches, of which the scatters are 12 and 10 and the others 4 to 8, near what a
// launch takes. 8,192 positions of 2,048 in bf16 into 32,000 rows: 32 us (the gradient's 131 MB
// written), the sort 16 to 17 in two launches (13 with the indexes in a cache).
#include <algorithm>

#include "sides.h"

namespace abcd {
namespace {

constexpr int kSortItems = 8, kSortPart = kBlock * kSortItems, kSortBits = 10;
constexpr int kRun = 64;
constexpr int kRowTurns = 4;  // rows that a wave looks at together where most are empty (32 us for 44)

// ------------------------------------------------------------------ lookup

struct EmbedArgs {
  const void* table;
  const void* index;
  void* y;
  int64_t ldt, ldy, n, m;
  int d, lanes;  // lanes: threads along a row, a power of two up to kBlock
  int tf32;
  float scale;
};

template <typename T, typename I, bool kWhole>
__global__ __launch_bounds__(kBlock) void embed_kernel(EmbedArgs a) {
  constexpr int N = kPer16<T>, kAhead = 4;
  const int t = threadIdx.x & (a.lanes - 1), rows = kBlock / a.lanes;
  const int64_t step = (int64_t)gridDim.x * rows;
  for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / a.lanes; row < a.n; row += kAhead * step) {
    int64_t from[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t r = row + u * step;
      const int64_t i = r < a.n ? (int64_t)static_cast<const I*>(a.index)[r] : -1;
      from[u] = i >= 0 && i < a.m ? i : -1;
    }
    for (int c = t * N; c < a.d; c += a.lanes * N) {
      Floats<N> v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        v[u] = 0.0f;
        if (from[u] >= 0) v[u] = load_param<T, N, kWhole>(a.table, from[u] * a.ldt + c, a.d - c, a.tf32);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t r = row + u * step;
        if (r < a.n) store_vec<T, N, kWhole>(static_cast<T*>(a.y) + r * a.ldy + c, v[u] * a.scale, a.d - c);
      }
    }
  }
}

// -------------------------------------------------------------------- sort

struct SortArgs {
  const void* index;
  const uint32_t *keys_in, *vals_in;
  uint32_t *keys_out, *vals_out;
  uint32_t* counts;  // [digit][part]: how many; from the scan on, how many before
  uint32_t* totals;  // [digit]
  int2* ranges;
  int64_t n;
  int32_t m;
  int parts, shift, bits;
};

// Key i: its row, those outside the table behind all rows.
template <typename I>
__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int64_t i) {
  if (a.keys_in) return a.keys_in[i];
  const int64_t k = (int64_t)static_cast<const I*>(a.index)[i];
  return (uint32_t)(k >= 0 && k < a.m ? k : a.m);
}

// Counts of a part's digits; with the first digit, rows without positions are marked too.
template <typename I>
__global__ __launch_bounds__(kBlock) void embed_count_kernel(SortArgs a) {
  __shared__ uint32_t count[1 << kSortBits];
  const int digits = 1 << a.bits;
  if (!a.keys_in)
    for (int64_t r = (int64_t)blockIdx.x * kBlock + threadIdx.x; r < a.m; r += (int64_t)gridDim.x * kBlock)
      a.ranges[r] = make_int2(0, 0);
  if ((int)blockIdx.x >= a.parts) return;
  for (int i = threadIdx.x; i < digits; i += kBlock) count[i] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortPart + threadIdx.x;
  uint32_t key[kSortItems];
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) key[k] = first + k * kBlock < a.n ? sort_key<I>(a, first + k * kBlock) : 0u;
#pragma unroll
  for (int k = 0; k < kSortItems; ++k)
    if (first + k * kBlock < a.n) atomicAdd(&count[(key[k] >> a.shift) & (digits - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < digits; i += kBlock) a.counts[(int64_t)i * a.parts + blockIdx.x] = count[i];
}

// Sum over the lanes before this one; total: over all.
__device__ __forceinline__ uint32_t wave_before(uint32_t v, uint32_t& total) {
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t u = (uint32_t)__shfl_up((int)s, d, 64);
    if ((int)(threadIdx.x & 63) >= d) s += u;
  }
  total = (uint32_t)__shfl((int)s, 63, 64);
  return s - v;
}

// A wave for each digit: its counts become the counts before each part.
__global__ __launch_bounds__(kWave) void embed_scan_kernel(SortArgs a) {
  constexpr int kAhead = 4;
  uint32_t* const c = a.counts + (int64_t)blockIdx.x * a.parts;
  uint32_t before = 0;
  for (int p = 0; p < a.parts; p += kAhead * kWave) {
    uint32_t own[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = p + u * kWave + (int)threadIdx.x;
      own[u] = i < a.parts ? c[i] : 0;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = p + u * kWave + (int)threadIdx.x;
      uint32_t all;
      const uint32_t at = wave_before(own[u], all);
      if (i < a.parts) c[i] = before + at;
      before += all;
    }
  }
  if (threadIdx.x == 0) a.totals[blockIdx.x] = before;
}

// Lanes of the wave whose digit of up to kBits bits equals this one's, among those `in`.
template <int kBits>
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool in) {
  constexpr int kAndEqual = 0x90;  // a & ~(b ^ c)
  const uint64_t there = __ballot(in);
  uint32_t lo = (uint32_t)there, hi = (uint32_t)(there >> 32);
#pragma unroll
  for (int b = 0; b < kBits; ++b) {
    const uint32_t m = (uint32_t)((int32_t)(d << (31 - b)) >> 31);
    const uint64_t set = __ballot(m != 0);
    lo = __builtin_amdgcn_bitop3_b32(lo, (uint32_t)set, m, kAndEqual);
    hi = __builtin_amdgcn_bitop3_b32(hi, (uint32_t)(set >> 32), m, kAndEqual);
  }
  return (uint64_t)hi << 32 | lo;
}

// Every wave ranks its quarter of the part in order, 64 keys at a time: lanes with the
// same digit find each other by ballots. The part is then ordered in LDS, so that keys of a
// digit leave next to each other (1M keys: 12 us; straight from the registers, each key to a
// line of its own, 19).
template <typename I>
__global__ __launch_bounds__(kBlock) void embed_scatter_kernel(SortArgs a) {
  constexpr int kWaves = kBlock / kWave, kTurns = kSortPart / kBlock, kPer = (1 << kSortBits) / kBlock;
  __shared__ uint32_t at[kWaves][1 << kSortBits];  // by wave: counts, then places in the part
  __shared__ uint32_t to[1 << kSortBits];          // of a digit: where its first key goes, less its place in the part
  __shared__ uint32_t keys[kSortPart], vals[kSortPart];
  __shared__ uint32_t sums[2][kWaves];
  const int digits = 1 << a.bits, w = threadIdx.x / kWave, l = threadIdx.x % kWave;
  // parts whose keys end up next to each other are one XCD's, whose L2 joins their lines
  const int part = xcd_order(blockIdx.x, a.parts);
  const int64_t first = (int64_t)part * kSortPart + w * (kSortPart / kWaves) + l;
  uint32_t key[kTurns], val[kTurns], place[kTurns], total[kPer], before_part[kPer];
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int64_t i = first + k * kWave;
    key[k] = i < a.n ? sort_key<I>(a, i) : 0u;
    val[k] = a.vals_in && i < a.n ? a.vals_in[i] : (uint32_t)i;
  }
  const int per = max(digits / kBlock, 1), digit = (int)threadIdx.x * per;  // a thread's digits
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const bool there = k < per && digit + k < digits;
    total[k] = there ? a.totals[digit + k] : 0u;
    before_part[k] = there ? a.counts[(int64_t)(digit + k) * a.parts + part] : 0u;
  }
  for (int i = threadIdx.x; i < kWaves << kSortBits; i += kBlock) (&at[0][0])[i] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const bool in = first + k * kWave < a.n;
    const uint32_t d = (key[k] >> a.shift) & (uint32_t)(digits - 1);
    const uint64_t same = same_digit<kSortBits>(d, in);
    uint32_t start = 0;
    const int leader = in ? __ffsll((unsigned long long)same) - 1 : l;
    if (in && l == leader) start = atomicAdd(&at[w][d], (uint32_t)__popcll(same));
    place[k] = (uint32_t)__shfl((int)start, leader, 64) + (uint32_t)__popcll(same & ((1ull << l) - 1ull));
  }
  __syncthreads();
  // a digit's keys go behind all smaller digits and the parts before this one; in the part
  // behind its smaller digits, wave by wave
  uint32_t sum = 0, own = 0, all;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    sum += total[k];
    if (k < per && digit + k < digits)
      for (int v = 0; v < kWaves; ++v) own += at[v][digit + k];
  }
  uint32_t before = wave_before(sum, all);
  if (l == 0) sums[0][w] = all;
  uint32_t here = wave_before(own, all);
  if (l == 0) sums[1][w] = all;
  __syncthreads();
  for (int v = 0; v < w; ++v) {
    before += sums[0][v];
    here += sums[1][v];
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (k < per && digit + k < digits) {
      to[digit + k] = before + before_part[k] - here;
      for (int v = 0; v < kWaves; ++v) {
        const uint32_t c = at[v][digit + k];
        at[v][digit + k] = here;
        here += c;
      }
    }
    before += total[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    if (first + k * kWave >= a.n) continue;
    const uint32_t slot = at[w][(key[k] >> a.shift) & (uint32_t)(digits - 1)] + place[k];
    keys[slot] = key[k];
    vals[slot] = val[k];
  }
  __syncthreads();
  const int64_t left = a.n - (int64_t)part * kSortPart;
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int slot = k * kBlock + (int)threadIdx.x;
    if (slot >= left) continue;
    const uint32_t v = keys[slot], place_of = to[(v >> a.shift) & (uint32_t)(digits - 1)] + (uint32_t)slot;
    a.keys_out[place_of] = v;
    a.vals_out[place_of] = vals[slot];
  }
}

// Few positions: place of key i is the number of keys below it and of equal ones before it. A
// workgroup has kRankKeys keys, one a lane and twice in each wave, and half a wave compares them
// with a part of all keys, read from LDS: a subtraction whose borrow is counted and whose zeros
// are the equal ones. Keys with no equal one before or behind them begin or end their row
// (embed_count's workgroups have marked all rows as empty).
//
// Five instructions for two comparisons bound it: both launches take 6.3 us for 1,000 positions,
// 12.8 for 8,192 (one workgroup that sorts digits of 8 bits in LDS 9.5 and 22, of 1M rows 12.4 and
// 34; ballots counted by the scalar unit 7.9 and 22), and by the launches for many 8,193 take 16 with
// 1,000 rows, 27 with 32,000 and 39 with 1M.
constexpr int kRankKeys = 32, kRankWaves = 16, kRankMost = 8192;
template <typename I, int kTurns>
__global__ __launch_bounds__(kRankWaves* kWave) void embed_rank_kernel(SortArgs a) {
  constexpr int kPart = kTurns * kRankKeys;  // keys of half a wave
  constexpr uint32_t kNone = 0xffffffffu;    // neither below nor equal to any
  __shared__ __align__(16) uint32_t keys[kRankWaves * 2 * kPart];
  __shared__ int places[kRankWaves][kRankKeys], alike[kRankWaves][kRankKeys];
  const int n = (int)a.n, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l = threadIdx.x % kWave;
  const int first = blockIdx.x * kRankKeys, mine = first + l % kRankKeys;
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {  // a wave's own part
    const int i = w * 2 * kPart + k * kWave + l;
    keys[i] = i < n ? sort_key<I>(a, i) : kNone;
  }
  const uint32_t own = mine < n ? sort_key<I>(a, mine) : kNone;
  __syncthreads();
  const int begin = w * 2 * kPart + l / kRankKeys * kPart;  // of the half wave's part
  int place = 0, equal = 0;  // equal: bit 0 before it, bit 1 behind it
  // count keys from `from` on, which lie all in front or all behind; in front the order is turned
  // round by `flip`, what is below then being above
  auto compare = [&](int from, auto count, auto front, uint32_t flip) {
    const uint32_t o = own ^ flip;
    uint32_t least = kNone;
    int below = 0;
#pragma unroll 4
    for (int t = 0; t < decltype(count)::value; t += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(keys + from + t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t other = e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
        uint32_t d;  // (own - other is ~other - ~own)
        below += decltype(front)::value ? __builtin_usub_overflow(own, other, &d) : __builtin_usub_overflow(other ^ flip, o, &d);
        least = min(least, d);
      }
    }
    place += flip ? decltype(count)::value - below : below;
    if (least == 0) equal |= flip ? 1 : 2;
  };
  if (first >= (w + 1) * 2 * kPart) {
    compare(begin, std::integral_constant<int, kPart>{}, std::true_type{}, ~0u);
  } else if (first < w * 2 * kPart) {
    compare(begin, std::integral_constant<int, kPart>{}, std::false_type{}, 0u);
  } else {
    for (int from = begin; from < begin + kPart; from += kRankKeys) {
      if (from != first) {
        compare(from, std::integral_constant<int, kRankKeys>{}, std::false_type{}, from < first ? ~0u : 0u);
        continue;
      }
      for (int t = 0; t < kRankKeys; ++t) {
        const uint32_t other = keys[from + t];
        place += other < own || (other == own && from + t < mine);
        if (other == own && from + t != mine) equal |= from + t < mine ? 1 : 2;
      }
    }
  }
  place += __shfl_xor(place, kRankKeys, kWave);
  equal |= __shfl_xor(equal, kRankKeys, kWave);
  if (l < kRankKeys) {
    places[w][l] = place;
    alike[w][l] = equal;
  }
  __syncthreads();
  if ((int)threadIdx.x >= kRankKeys || mine >= n) return;
  place = equal = 0;
#pragma unroll
  for (int v = 0; v < kRankWaves; ++v) {
    place += places[v][l];
    equal |= alike[v][l];
  }
  a.keys_out[place] = own;
  a.vals_out[place] = (uint32_t)mine;
  if (own >= (uint32_t)a.m) return;
  if (!(equal & 1)) a.ranges[own].x = place;
  if (!(equal & 2)) a.ranges[own].y = place + 1;
}

__global__ __launch_bounds__(kBlock) void embed_ranges_kernel(SortArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= a.n) return;
  const uint32_t k = a.keys_in[i];
  if (k >= (uint32_t)a.m) return;
  if (i == 0 || a.keys_in[i - 1] != k) a.ranges[k].x = (int)i;
  if (i == a.n - 1 || a.keys_in[i + 1] != k) a.ranges[k].y = (int)(i + 1);
}

// ---------------------------------------------------------------- gradient

struct EmbedBwdArgs {
  const void* dy;
  const int32_t* order;
  const int32_t* rows;  // of the sorted positions
  const int2* ranges;
  void* dtable;
  float* part;       // [chunk][2][pitch]: of the long row that reaches into a chunk, and of the one that begins there
  int64_t lddy, ldt, n, m, pitch;
  int d, lanes, row_blocks, turns;  // turns: rows of the table that a group of lanes takes
  int wf32;
  float scale;
};

template <typename T, int N, bool kWhole>
__device__ __forceinline__ void put_row(const EmbedBwdArgs& a, int64_t r, int c, Floats<N> v) {
  v *= a.scale;
  if (a.wf32)
    store_vec<float, N, kWhole>(static_cast<float*>(a.dtable) + r * a.ldt + c, v, a.d - c);
  else
    store_vec<T, N, kWhole>(static_cast<T*>(a.dtable) + r * a.ldt + c, v, a.d - c);
}

// Where a row's positions are. What the caller has kept of the sort is not checked on the
// host: whatever it holds, no access leaves the arrays.
__device__ __forceinline__ int2 range_of(const EmbedBwdArgs& a, int64_t r) {
  const int2 at = a.ranges[r];
  return make_int2(max(at.x, 0), max(min(at.y, (int)a.n), 0));
}

// The sum of columns c.. of dy over positions [from, to) of the order.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ Floats<N> sum_run(const EmbedBwdArgs& a, int from, int to, int c) {
  constexpr int kAhead = 8;
  Floats<N> s = 0.0f;
  for (int p = from; p < to; p += kAhead) {
    typename Frag<T>::type v[kAhead];
    int64_t at[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) at[u] = a.order[p + u < to ? p + u : from];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int left = p + u < to && (uint64_t)at[u] < (uint64_t)a.n ? a.d - c : 0;
      v[u] = load_frag<T, kWhole>(static_cast<const T*>(a.dy) + at[u] * a.lddy + c, left,
                                  room_of(a.n, at[u], a.lddy, left));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      s += __builtin_convertvector((first_of<T, kWhole>(v[u], a.d - c)), Floats<N>);
  }
  return s;
}

// Workgroups below row_blocks: rows of the table with up to kRun positions. The others:
// chunks of the order, of which they take what belongs to longer rows. blockIdx.y: blocks
// of kBlock vectors of columns at most.
template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void embed_bwd_kernel(EmbedBwdArgs a) {
  constexpr int N = kPer16<T>;
  const int rows = kBlock / a.lanes, c = ((int)blockIdx.y * a.lanes + (threadIdx.x & (a.lanes - 1))) * N;
  if (c >= a.d) return;
  if ((int)blockIdx.x < a.row_blocks) {
    const int64_t step = (int64_t)a.row_blocks * rows * a.turns;
    for (int64_t r = (int64_t)blockIdx.x * rows * a.turns + threadIdx.x / a.lanes; r < a.m; r += step) {
      if (a.turns == 1) {
        const int2 at = range_of(a, r);
        if (at.y - at.x <= kRun) put_row<T, N, kWhole>(a, r, c, sum_run<T, N, kWhole>(a, at.x, at.y, c));
        continue;
      }
      int2 at[kRowTurns];
#pragma unroll
      for (int k = 0; k < kRowTurns; ++k) at[k] = r + k * rows < a.m ? range_of(a, r + k * rows) : make_int2(0, kRun + 1);
#pragma unroll
      for (int k = 0; k < kRowTurns; ++k)
        if (at[k].y - at[k].x <= kRun)
          put_row<T, N, kWhole>(a, r + k * rows, c, sum_run<T, N, kWhole>(a, at[k].x, at[k].y, c));
    }
    return;
  }
  const int64_t chunk = (int64_t)((int)blockIdx.x - a.row_blocks) * rows + threadIdx.x / a.lanes, begin = chunk * kRun;
  if (begin >= a.n) return;
  const int64_t end = begin + kRun < a.n ? begin + kRun : a.n;
  // a row of more than kRun positions that has any here has the first or the last one
  const int first_row = a.rows[begin], last_row = a.rows[end - 1];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int r = k == 0 ? first_row : last_row;
    if ((uint32_t)r >= (uint32_t)a.m || (k == 1 && last_row == first_row)) continue;
    const int2 at = range_of(a, r);
    if (at.y - at.x <= kRun) continue;
    const int which = at.x >= begin ? 1 : 0;
    const Floats<N> s = sum_run<T, N, kWhole>(a, max(at.x, (int)begin), min(at.y, (int)end), c);
    store_vec<float, N, true>(a.part + (chunk * 2 + which) * a.pitch + c, s, N);
  }
}

constexpr int kJoinWaves = 16;

// Rows of more than kRun positions that begin in one of 64 chunks: 64 columns a workgroup,
// the chunks that a row reaches dealt to its waves.
template <typename T>
__global__ __launch_bounds__(kJoinWaves* kWave) void embed_join_kernel(EmbedBwdArgs a) {
  __shared__ float red[kJoinWaves][kWave];
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave, c = (int)blockIdx.y * kWave + l;
  // a row that begins in a chunk and goes on behind it has the chunk's last position
  const int64_t chunk = (int64_t)blockIdx.x * kWave + l, behind = (chunk + 1) * kRun;
  int row = a.m, end = 0;
  bool begins = false;
  if (behind < a.n) {
    row = a.rows[behind - 1];
    if ((uint32_t)row < (uint32_t)a.m) {
      const int2 at = range_of(a, row);
      end = at.y;
      begins = at.y - at.x > kRun && at.x >= chunk * kRun;
    }
  }
  for (uint64_t left = __ballot(begins); left; left &= left - 1) {
    const int own = __ffsll((unsigned long long)left) - 1;
    const int r = __shfl(row, own, 64);
    const int64_t first = (int64_t)blockIdx.x * kWave + own, last = (__shfl(end, own, 64) - 1) / kRun;
    float s = 0.0f;
    if (c < a.d) {
      if (w == 0) s = a.part[(first * 2 + 1) * a.pitch + c];
      int64_t k = first + 1 + w;
      for (; k + 7 * kJoinWaves <= last; k += 8 * kJoinWaves) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = a.part[(k + u * kJoinWaves) * 2 * a.pitch + c];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
      }
      for (; k <= last; k += kJoinWaves) s += a.part[k * 2 * a.pitch + c];
    }
    red[w][l] = s;
    __syncthreads();
    if (w == 0 && c < a.d) {
      for (int v = 1; v < kJoinWaves; ++v) s += red[v][l];
      put_row<T, 1, true>(a, r, c, Floats<1>(s));
    }
    __syncthreads();
  }
}

// Up to a wave's lanes of positions, without a sort: every wave has all indexes, and finds by a
// ballot those that name one of the rows it writes. The table's bytes or the launch bound it: 4
// positions of 24,402 x 40 in fp16 9.1 us a call (with a sort 26), 64 of 1M x 64 in bf16 19.5 (41),
// 64 that all name one of 16 rows of 2,048 15.4.
struct EmbedFewArgs {
  const void* dy;
  const void* index;
  void* dtable;
  int64_t lddy, ldt, n, m;
  int d, lanes, wf32;
  float scale;
};
template <typename T, typename I, bool kWhole>
__global__ __launch_bounds__(kBlock) void embed_bwd_few_kernel(EmbedFewArgs a) {
  constexpr int N = kPer16<T>, kAhead = 8;
  const int l = threadIdx.x % kWave, t = l & (a.lanes - 1), rows = kWave / a.lanes;
  const int c = ((int)blockIdx.y * a.lanes + t) * N;
  const int64_t index = l < a.n ? (int64_t)static_cast<const I*>(a.index)[l] : -1;
  const int64_t step = (int64_t)gridDim.x * (kBlock / kWave) * rows;
  for (int64_t r0 = ((int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave) * rows; r0 < a.m; r0 += step) {
    const int64_t row = r0 + l / a.lanes;
    Floats<N> s = 0.0f;
    uint64_t left = __ballot(index >= r0 && index < r0 + rows);
    while (left) {
      Floats<N> v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {  // positions in their order
        const int p = left ? __ffsll((unsigned long long)left) - 1 : 0;
        const bool mine = left && r0 + (__shfl((int)(index - r0), p, kWave)) == row;
        left &= left - 1;
        v[u] = 0.0f;
        if (mine && c < a.d) v[u] = load_vec<T, N, kWhole>(static_cast<const T*>(a.dy) + p * a.lddy + c, a.d - c);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) s += v[u];
    }
    if (row >= a.m || c >= a.d) continue;
    s *= a.scale;
    if (a.wf32)
      store_vec<float, N, kWhole>(static_cast<float*>(a.dtable) + row * a.ldt + c, s, a.d - c);
    else
      store_vec<T, N, kWhole>(static_cast<T*>(a.dtable) + row * a.ldt + c, s, a.d - c);
  }
}

// --------------------------------------------------------------- launching

int bits_of(int64_t v) {
  int b = 1;
  while (v >> b) ++b;
  return b;
}

struct SortScratch {
  uint32_t *keys, *vals, *counts, *totals;
  size_t bytes;
  int passes, bits;
  int64_t parts;
};
SortScratch sort_layout(int64_t n, int64_t m, void* workspace) {
  SortScratch s{};
  const int bits = bits_of(m);
  s.passes = (bits + kSortBits - 1) / kSortBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.parts = (n + kSortPart - 1) / kSortPart;
  Pieces p{static_cast<char*>(workspace)};
  s.keys = static_cast<uint32_t*>(p.take(n * sizeof(uint32_t)));
  s.vals = static_cast<uint32_t*>(p.take(n * sizeof(uint32_t)));
  s.counts = static_cast<uint32_t*>(p.take(((size_t)s.parts << s.bits) * sizeof(uint32_t)));
  s.totals = static_cast<uint32_t*>(p.take(sizeof(uint32_t) << s.bits));
  s.bytes = p.used;
  return s;
}

int64_t embed_chunks(int64_t n) { return (n + kRun - 1) / kRun; }
int64_t embed_pitch(int64_t d) { return (d + 7) & ~int64_t(7); }

// Calls f with a value of the index type.
template <typename F>
int32_t with_index(int32_t bits, F f) {
  return bits == 64 ? f(int64_t(0)) : f(int32_t(0));
}

// Threads along a row of nvec vectors.
int embed_lanes(int nvec) {
  int l = 1;
  while (l < kWave && l < nvec) l *= 2;
  return l;
}

}  // namespace

int32_t launch_embed(int32_t dtype, int64_t n, int64_t m, int64_t d, int32_t tdtype, const void* table, int64_t ldt,
                     int32_t index_bits, const void* index, float scale, void* y, int64_t ldy, hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  EmbedArgs a{table, index, y, ldt, ldy, n, m, (int)d, 0, tdtype == ABCD_F32 && dtype != ABCD_F32, scale};
  return with_type(dtype, [&](auto z) -> int32_t {
    return with_index(index_bits, [&](auto zi) -> int32_t {
      typedef decltype(z) T;
      typedef decltype(zi) I;
      a.lanes = embed_lanes((int)((d + kPer16<T> - 1) / kPer16<T>));
      const int64_t rows = kBlock / a.lanes, blocks = std::min<int64_t>((n + 4 * rows - 1) / (4 * rows), 1 << 20);
      if (d % kPer16<T> == 0)
        ABCD_LAUNCH("embed", (embed_kernel<T, I, true>), blocks, kBlock, 0, stream, a);
      else
        ABCD_LAUNCH("embed", (embed_kernel<T, I, false>), blocks, kBlock, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    });
  });
}

size_t embed_sort_workspace_bytes(int64_t n, int64_t m) { return std::max<size_t>(256, sort_layout(n, m, nullptr).bytes); }

int32_t launch_embed_sort(int64_t n, int64_t m, int32_t index_bits, const void* index, int32_t* order, int32_t* rows,
                          int32_t* ranges, void* workspace, hipStream_t stream) {
  const SortScratch s = sort_layout(n, m, workspace);
  SortArgs a{};
  a.index = index;
  a.counts = s.counts;
  a.totals = s.totals;
  a.ranges = reinterpret_cast<int2*>(ranges);
  a.n = n;
  a.m = (int32_t)m;
  a.parts = (int)s.parts;
  a.bits = s.bits;
  return with_index(index_bits, [&](auto zi) -> int32_t {
    typedef decltype(zi) I;
    if (n <= kRankMost) {
      const int64_t zero = std::min<int64_t>((m + kBlock - 1) / kBlock, 2048);
      a.parts = 0;  // all that this does is mark the rows
      ABCD_LAUNCH("embed_count", (embed_count_kernel<I>), zero, kBlock, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      if (n == 0) return ABCD_OK;
      a.keys_out = reinterpret_cast<uint32_t*>(rows);
      a.vals_out = reinterpret_cast<uint32_t*>(order);
      const int64_t grid = (n + kRankKeys - 1) / kRankKeys;
      auto rank = [&](auto turns) {
        ABCD_LAUNCH("embed_rank", (embed_rank_kernel<I, decltype(turns)::value>), grid, kRankWaves * kWave, 0, stream, a);
      };
      constexpr int kTurn = kRankWaves * kWave;  // keys
      static_assert(8 * kTurn == kRankMost);
      if (n <= kTurn)
        rank(std::integral_constant<int, 1>{});
      else if (n <= 2 * kTurn)
        rank(std::integral_constant<int, 2>{});
      else if (n <= 4 * kTurn)
        rank(std::integral_constant<int, 4>{});
      else
        rank(std::integral_constant<int, 8>{});
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    }
    for (int pass = 0; pass < s.passes; ++pass) {
      // two places take turns so that the last pass writes the result
      const bool own = (s.passes - 1 - pass) & 1;
      a.shift = pass * s.bits;
      a.keys_in = pass == 0 ? nullptr : a.keys_out;
      a.vals_in = pass == 0 ? nullptr : a.vals_out;
      a.keys_out = own ? s.keys : reinterpret_cast<uint32_t*>(rows);
      a.vals_out = own ? s.vals : reinterpret_cast<uint32_t*>(order);
      const int64_t zero = pass == 0 ? std::min<int64_t>((m + kBlock - 1) / kBlock, 2048) : 0;
      ABCD_LAUNCH("embed_count", (embed_count_kernel<I>), std::max<int64_t>(s.parts, zero), kBlock, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      ABCD_LAUNCH("embed_scan", embed_scan_kernel, 1 << s.bits, kWave, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      ABCD_LAUNCH("embed_scatter", (embed_scatter_kernel<I>), s.parts, kBlock, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      if (pass == s.passes - 1) {
        a.keys_in = a.keys_out;
        ABCD_LAUNCH("embed_ranges", embed_ranges_kernel, (n + kBlock - 1) / kBlock, kBlock, 0, stream, a);
        ABCD_HIP(hipGetLastError());
      }
    }
    return ABCD_OK;
  });
}

size_t embed_bwd_workspace_bytes(int64_t n, int64_t d) {
  Pieces p{nullptr};
  p.take((size_t)embed_chunks(n) * 2 * embed_pitch(d) * sizeof(float));
  return std::max<size_t>(256, p.used);
}

int32_t launch_embed_bwd(int32_t dtype, int64_t n, int64_t m, int64_t d, const void* dy, int64_t lddy,
                         const int32_t* order, const int32_t* rows_of, const int32_t* ranges, float scale, int32_t wdtype, void* dtable, int64_t ldt, void* workspace, hipStream_t stream) {
  if (m == 0) return ABCD_OK;
  Pieces p{static_cast<char*>(workspace)};
  const int64_t pitch = embed_pitch(d), chunks = embed_chunks(n);
  float* const part = static_cast<float*>(p.take((size_t)chunks * 2 * pitch * sizeof(float)));
  EmbedBwdArgs a{dy, order, rows_of, reinterpret_cast<const int2*>(ranges), dtable, part, lddy, ldt, n, m, pitch,
                 (int)d, 0, 0, 1, wdtype == ABCD_F32 && dtype != ABCD_F32, scale};
  return with_type(dtype, [&](auto z) -> int32_t {
    typedef decltype(z) T;
    const int nvec = (int)((d + kPer16<T> - 1) / kPer16<T>);
    a.lanes = embed_lanes(nvec);
    const int64_t rows = kBlock / a.lanes;
    // where most rows are empty, and long, a wave looks at several of them at once (bf16, sums alone,
    // one row at a time against four: 8,192 of 32,000 x 2,048 47 against 36 us, x 512 17.1 against 15.1,
    // but x 256 11.4 against 12.4; 100,000 of 32,000 x 2,048 125 against 131. Short rows of a large
    // table would gain too, 20,000 of 1M x 64 41 against 31, which this rule leaves out)
    a.turns = n < m && nvec >= kWave ? kRowTurns : 1;
    a.row_blocks = (int)std::min<int64_t>((m + rows * a.turns - 1) / (rows * a.turns), 1 << 18);
    const int64_t blocks = a.row_blocks + (chunks + rows - 1) / rows;
    const dim3 grid(blocks, (nvec + a.lanes - 1) / a.lanes);
    if (d % kPer16<T> == 0)
      ABCD_LAUNCH("embed_bwd", (embed_bwd_kernel<T, true>), grid, kBlock, 0, stream, a);
    else
      ABCD_LAUNCH("embed_bwd", (embed_bwd_kernel<T, false>), grid, kBlock, 0, stream, a);
    ABCD_HIP(hipGetLastError());
    if (n > kRun) {
      const dim3 joins((chunks + kWave - 1) / kWave, (d + kWave - 1) / kWave);
      ABCD_LAUNCH("embed_join", (embed_join_kernel<T>), joins, kJoinWaves * kWave, 0, stream, a);
      ABCD_HIP(hipGetLastError());
    }
    return ABCD_OK;
  });
}

int32_t launch_embed_bwd_few(int32_t dtype, int64_t n, int64_t m, int64_t d, const void* dy, int64_t lddy,
                             int32_t index_bits, const void* index, float scale, int32_t wdtype, void* dtable, int64_t ldt,
                             hipStream_t stream) {
  EmbedFewArgs a{dy, index, dtable, lddy, ldt, n, m, (int)d, 0, wdtype == ABCD_F32 && dtype != ABCD_F32, scale};
  return with_type(dtype, [&](auto z) -> int32_t {
    return with_index(index_bits, [&](auto zi) -> int32_t {
      typedef decltype(z) T;
      typedef decltype(zi) I;
      const int nvec = (int)((d + kPer16<T> - 1) / kPer16<T>);
      a.lanes = embed_lanes(nvec);
      const int64_t rows = kBlock / a.lanes;
      const dim3 grid(std::min<int64_t>((m + rows - 1) / rows, 1 << 14), (nvec + a.lanes - 1) / a.lanes);
      if (d % kPer16<T> == 0)
        ABCD_LAUNCH("embed_bwd_few", (embed_bwd_few_kernel<T, I, true>), grid, kBlock, 0, stream, a);
      else
        ABCD_LAUNCH("embed_bwd_few", (embed_bwd_few_kernel<T, I, false>), grid, kBlock, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    });
  });
}

}  // namespace abcd
