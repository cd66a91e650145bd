// Embedding rows of a list of tokens, scaled, and their table's gradient, for
// gfx950 (MI355X).
//
// Forward: out[i] = scale * E[ids[i]].  LPR lanes cover a row in pieces of V
// elements, with four rows a lane in flight (two: 3 % slower, eight: no faster).
// The bound is HBM: distinct rows read, token rows written, past the caches, so
// that these are left to the rows that come again (2.1 M tokens of 128 over 1 M
// rows: bf16 100 us, 6.2 TB/s, through the caches 169; bf16 to fp32 173, 6.7
// TB/s, rather than 298).
//
// Backward: dE[v] = scale * sum_{i: ids[i] = v} dout[i].  Tokens are sorted by
// id (least significant digit first, stable, so equal ids stay in token order).
// A workgroup then sums a span of sorted tokens: a group of LPR lanes adds the
// rows of a chunk, eight in flight, and writes each row of the gradient that
// begins and ends in it; rows cut by chunk borders are joined in LDS, those cut
// by span borders by a second kernel.  Every sum has a fixed order and there
// are no float atomics, so the result does not depend on timing.  The rows
// without tokens are zeroed by workgroups of the sort's later launches, which
// leave the memory idle otherwise, from marks that its first pass sets (all rows
// zeroed beside the sort, the touched ones to be written again by the sums: 379
// us for 2.1 M tokens of 128 bf16 over 1 M rows).  The bound is HBM: dout read,
// the gradient written, both past the caches (the sums of that case: 194 us
// through them, 157 past them, 4.5 TB/s).
#include "elem.h"
#include "seq_internal.h"
#include "wave_scan.h"

#include <algorithm>

namespace dpi {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsInFlight = 4;

// ------------------------------------------------------------------ forward
template <typename TIN, typename TOUT, int V>
__global__ __launch_bounds__(kThreads) void embed_kernel(const EmbedArgs a, int lpr_log) {
  const int lpr = 1 << lpr_log, groups = kThreads >> lpr_log;
  const int g = threadIdx.x >> lpr_log, k = threadIdx.x & (lpr - 1);
  const int64_t first = (int64_t)blockIdx.x * groups * kRowsInFlight + g;
  const int col = ((int)blockIdx.y * lpr + k) * V;
  const TIN* __restrict__ table = static_cast<const TIN*>(a.table);
  TOUT* __restrict__ out = static_cast<TOUT*>(a.out);
  const bool mine = col < a.dim;
  Elems<TIN, V> e[kRowsInFlight];
  bool held[kRowsInFlight];
#pragma unroll
  for (int u = 0; u < kRowsInFlight; ++u) {
    const int64_t i = first + (int64_t)u * groups;
    const int32_t id = i < a.tokens ? a.ids[i] : a.padding_id;
    const bool pad = i >= a.tokens || (a.padding_id >= 0 && id == a.padding_id);
    const bool inside = id >= 0 && (int64_t)id < a.num_rows;
    if (!pad && !inside && a.status && k == 0 && blockIdx.y == 0) atomicOr(a.status, DPI_DEVSTAT_BAD_ID);
    held[u] = !pad && inside && mine;
    if (held[u]) e[u] = load_elems<true, TIN, V>(table + (int64_t)id * a.dim + col, V);
  }
#pragma unroll
  for (int u = 0; u < kRowsInFlight; ++u) {
    const int64_t i = first + (int64_t)u * groups;
    if (i >= a.tokens || !mine) continue;
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = held[u] ? a.scale * e[u][j] : 0.f;
    store_once<TOUT, V>(out + i * a.out_stride + col, v);
  }
}

// --------------------------------------------------------------------- sort
__device__ __forceinline__ uint32_t key_of(const EmbedGradArgs& a, int64_t i, bool report) {
  const int32_t id = a.ids[i];
  const bool pad = a.padding_id >= 0 && id == a.padding_id;
  const bool inside = id >= 0 && (int64_t)id < a.num_rows;
  if (report && !pad && !inside && a.status) atomicOr(a.status, DPI_DEVSTAT_BAD_ID);
  return pad || !inside ? (uint32_t)a.num_rows : (uint32_t)id;   // num_rows: after every row, in no row's sum
}

// One row of `units` units, by the lanes of a group.
template <typename U>
__device__ __forceinline__ void zero_row(void* row, int units, int lane, int lanes) {
  for (int i = lane; i < units; i += lanes) __builtin_nontemporal_store(U{}, static_cast<U*>(row) + i);
}

// Share `share` of a.zero_shares of the gradient's rows set to zero by `blocks` workgroups, of which this is `block`;
// MARKED: but those with tokens.
template <bool MARKED>
__device__ __forceinline__ void zero_rows(const EmbedGradArgs& a, int share, int64_t block, int64_t blocks) {
  typedef int quad __attribute__((ext_vector_type(4)));
  const int64_t row_bytes = (int64_t)a.dim * (a.grad_dtype == DPI_F32 ? 4 : 2);
  const uint32_t odd = (uint32_t)(reinterpret_cast<uintptr_t>(a.grad) | (uintptr_t)row_bytes);
  const int unit = odd & 15 ? (odd & 3 ? 2 : 4) : 16, units = (int)(row_bytes / unit);
  int lanes_log = 0;
  while (lanes_log < 6 && (1 << lanes_log) < units) ++lanes_log;
  const int lanes = 1 << lanes_log, lane = threadIdx.x & (lanes - 1);
  const int64_t groups = blockDim.x >> lanes_log, end = a.num_rows * (share + 1) / a.zero_shares;
  const int64_t step = blocks * groups;
  for (int64_t r = a.num_rows * share / a.zero_shares + block * groups + (threadIdx.x >> lanes_log); r < end; r += 4 * step) {
    bool held[4];   // four rows' marks in flight
#pragma unroll
    for (int u = 0; u < 4; ++u) held[u] = r + u * step >= end || (MARKED && a.touched[r + u * step]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (held[u]) continue;
      char* row = static_cast<char*>(a.grad) + (r + u * step) * row_bytes;
      if (unit == 16)
        zero_row<quad>(row, units, lane, lanes);
      else if (unit == 4)
        zero_row<int>(row, units, lane, lanes);
      else
        zero_row<int16_t>(row, units, lane, lanes);
    }
  }
}

// What the workgroups beside the sort's own do in launch `step` of a pass (count, scan if there is one, scatter): clear the
// marks in the first launch; the first pass's scatter sets them; every later launch zeroes a share of the rows, with the
// marks once they are set.  A sort of one pass, of few rows, zeroes them all in the first launch.
__device__ __forceinline__ void beside_sort(const EmbedGradArgs& a, int pass, int step, int64_t block, int64_t blocks) {
  if (a.passes == 1) {
    if (step == 0) zero_rows<false>(a, 0, block, blocks);
  } else if (pass > 0) {
    zero_rows<true>(a, a.launches * pass + step - 1, block, blocks);
  } else if (step > 0) {
    zero_rows<false>(a, step - 1, block, blocks);
  } else {
    for (int64_t i = block * blockDim.x + threadIdx.x; i < (a.num_rows + 15) / 16; i += blocks * blockDim.x)
      reinterpret_cast<int4*>(a.touched)[i] = int4{0, 0, 0, 0};
  }
}

// A tile of the sort: workgroups go to the 8 XCDs in turn, and the tiles of an XCD are neighbours, so that the few items
// that each of them has of a digit, which lie side by side in the output, fill cache lines of one L2.
__device__ __forceinline__ int64_t tile_of(const EmbedGradArgs& a) {
  const int64_t per = (a.tiles + 7) >> 3, x = blockIdx.x & 7, i = blockIdx.x >> 3;
  const int64_t whole = a.tiles & 7;   // XCDs with `per` tiles when they do not divide evenly
  return whole == 0 || x < whole ? x * per + i : whole * per + (x - whole) * (per - 1) + i;
}

// Exclusive prefix over the workgroup of one value a thread; *total: their sum.  sums: a word a wave, free to use.
template <int THREADS>
__device__ __forceinline__ uint32_t block_prefix(uint32_t x, uint32_t* sums, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t incl = wave_incl_scan32(x, lane);
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  *total = all;
  return before + incl - x;
}

// A wave's item of each lane to its place among the wave's items of the same digit: where the digit's next one goes,
// counted on.  Lanes that are not live have no place.
__device__ __forceinline__ uint32_t place_of_digit(uint32_t digit, bool live, int bits, int lane, uint32_t* next) {
  uint64_t same = __ballot(live);   // lanes with this lane's digit
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((digit >> b) & 1);
    same &= (digit >> b) & 1 ? set : ~set;
  }
  const int rank = __popcll(same & ((1ull << lane) - 1));
  const uint32_t at = live ? next[digit] + rank : 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // every lane has read before one counts on
  if (live && rank == 0) next[digit] += (uint32_t)__popcll(same);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return at;
}

// A pass of the sort is three launches: a tile's counts of the digits, their prefixes over the tiles, and the items to their
// places.  2.1 M tokens: 8, 18 and 28 us in the passes whose workgroups zero nothing, 110,593: 3.3, 4.5 and 7, bound by the
// latency of a few dependent accesses each.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const EmbedGradArgs a, int pass) {
  __shared__ uint32_t count[1 << kSortMaxBits];
  if (blockIdx.x >= a.tiles) {
    beside_sort(a, pass, 0, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    return;
  }
  const int bins = 1 << a.bits, shift = pass * a.bits;
  const int64_t tile = tile_of(a), base = tile * kSortThreads * ITEMS;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  const uint2* __restrict__ pairs = a.pairs[(pass + 1) & 1];
  uint32_t key[ITEMS];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int64_t i = base + u * kSortThreads + threadIdx.x;
    key[u] = i < a.tokens ? (pass == 0 ? key_of(a, i, true) : pairs[i].x) : 0;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < ITEMS; ++u)
    if (base + u * kSortThreads + threadIdx.x < a.tokens) atomicAdd(&count[(key[u] >> shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) a.hist[(tile << a.bits) + b] = count[b];
}

// The tiles' counts of 64 digits to their exclusive prefixes over the tiles, and the digits' totals: a lane a digit, the
// 16 waves a range of tiles each.
constexpr int kSortScanWaves = 16;

__global__ __launch_bounds__(64 * kSortScanWaves) void sort_scan_kernel(const EmbedGradArgs a, int pass) {
  __shared__ uint32_t sums[kSortScanWaves][64];
  const int bins = 1 << a.bits, groups = (bins + 63) / 64;
  if ((int)blockIdx.x >= groups) {
    beside_sort(a, pass, 1, blockIdx.x - groups, gridDim.x - groups);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = blockIdx.x * 64 + lane;
  const int64_t per = (a.tiles + kSortScanWaves - 1) / kSortScanWaves;
  const int64_t begin = min(wave * per, a.tiles), end = min(begin + per, a.tiles);
  const auto walk = [&](auto use) {   // eight tiles' counts in flight
    for (int64_t t0 = begin; t0 < end; t0 += 8) {
      uint32_t c[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) c[u] = b < bins ? a.hist[(min(t0 + u, end - 1) << a.bits) + b] : 0;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (t0 + u < end) use(t0 + u, c[u]);
    }
  };
  uint32_t sum = 0;
  walk([&](int64_t, uint32_t c) { sum += c; });
  sums[wave][lane] = sum;
  __syncthreads();
  uint32_t at = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kSortScanWaves; ++w) {
    if (w < wave) at += sums[w][lane];
    all += sums[w][lane];
  }
  if (b >= bins) return;
  walk([&](int64_t t, uint32_t c) {
    a.hist[(t << a.bits) + b] = at;
    at += c;
  });
  if (wave == 0) a.total[b] = all;
}

// The same for a tile by its own workgroup, where the tiles' counts are few (sort_scans): `before`, the counts of the tiles
// before it, and `total`, of all of them, of the thread's 4 neighbouring digits.  Up to 8 parts of the tiles are read at
// once, a thread 4 digits of each, and added up in `parts`, 8 words a thread.
__device__ __forceinline__ void sum_tiles(const EmbedGradArgs& a, int64_t tile, uint32_t* parts, uint32_t* before,
                                          uint32_t* total) {
  typedef uint32_t quad __attribute__((ext_vector_type(4)));
  const int quads = 1 << (a.bits - 2), many = min(kSortThreads / quads, 8);
  const int q = threadIdx.x & (quads - 1), part = threadIdx.x >> (a.bits - 2);
  const quad* __restrict__ hist = reinterpret_cast<const quad*>(a.hist);
  quad low{0, 0, 0, 0}, all{0, 0, 0, 0};
  if (part < many) {
    const int tiles = (int)a.tiles, per = (tiles + many - 1) / many, end = min((part + 1) * per, tiles);
    for (int t0 = part * per; t0 < end; t0 += 16) {
      quad c[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) c[u] = hist[min(t0 + u, end - 1) * quads + q];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        if (t0 + u >= end) continue;
        all += c[u];
        if (t0 + u < tile) low += c[u];
      }
    }
    reinterpret_cast<quad*>(parts)[2 * threadIdx.x] = low;
    reinterpret_cast<quad*>(parts)[2 * threadIdx.x + 1] = all;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) before[j] = total[j] = 0;
  if ((int)threadIdx.x < quads) {
    for (int i = 0; i < many; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        before[j] += parts[(i * quads + threadIdx.x) * 8 + j];
        total[j] += parts[(i * quads + threadIdx.x) * 8 + 4 + j];
      }
    }
  }
  __syncthreads();   // `parts` is free again
}

// SCANNED: a launch before this one made the tiles' prefixes.
template <int ITEMS, bool SCANNED>
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const EmbedGradArgs a, int pass) {
  constexpr int kWaves = kSortThreads / 64, kEach = (1 << kSortMaxBits) / kSortThreads;
  static_assert(kEach == 4 && kWaves * (1 << kSortMaxBits) >= 8 * kSortThreads, "what sum_tiles takes");
  __shared__ __align__(16) uint32_t next[kWaves][1 << kSortMaxBits];
  __shared__ uint32_t sums[kWaves];
  if (blockIdx.x >= a.tiles) {
    beside_sort(a, pass, a.launches - 1, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    return;
  }
  const int bins = 1 << a.bits, shift = pass * a.bits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t tile = tile_of(a), base = (tile * kWaves + wave) * 64 * ITEMS;   // a wave's items are consecutive
  uint2 item[ITEMS];
  const uint2* __restrict__ pairs = a.pairs[(pass + 1) & 1];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int64_t i = base + u * 64 + lane;
    item[u] = uint2{0, 0};
    if (i < a.tokens) item[u] = pass == 0 ? uint2{key_of(a, i, false), (uint32_t)i} : pairs[i];
  }
  // kEach neighbouring digits a thread: where they start, and this tile's part of them
  uint32_t total[kEach], mine[kEach], sum = 0;
  if constexpr (!SCANNED) sum_tiles(a, tile, next[0], mine, total);
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int b = threadIdx.x * kEach + j;
    if constexpr (SCANNED) {
      total[j] = b < bins ? a.total[b] : 0;
      mine[j] = b < bins ? a.hist[(tile << a.bits) + b] : 0;
    }
    sum += total[j];
  }
  for (int b = threadIdx.x; b < bins; b += kSortThreads) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) next[w][b] = 0;
  }
  uint32_t all;
  uint32_t start = block_prefix<kSortThreads>(sum, sums, &all);   // its barrier also ends the clearing
#pragma unroll
  for (int u = 0; u < ITEMS; ++u)
    if (base + u * 64 + lane < a.tokens) atomicAdd(&next[wave][(item[u].x >> shift) & (bins - 1)], 1u);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int b = threadIdx.x * kEach + j;
    if (b < bins) {
      uint32_t at = start + mine[j];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = next[w][b];
        next[w][b] = at;
        at += c;
      }
    }
    start += total[j];
  }
  __syncthreads();
  uint2* __restrict__ out = a.pairs[pass & 1];
  const bool mark = pass == 0 && a.passes > 1;
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const bool live = base + u * 64 + lane < a.tokens;
    const uint32_t at = place_of_digit((item[u].x >> shift) & (bins - 1), live, a.bits, lane, next[wave]);
    if (live) out[at] = item[u];
    if (live && mark && item[u].x < (uint32_t)a.num_rows) a.touched[item[u].x] = 1;   // the same by whoever writes it
  }
}

// A short list, sorted by one workgroup in LDS (4,096 tokens and two digits: 14 us, most of it barriers and LDS accesses one
// after the other); the others zero the gradient.
__global__ __launch_bounds__(kSortOneThreads) void sort_one_kernel(const EmbedGradArgs a) {
  constexpr int kWaves = kSortOneThreads / 64, kTile = kSortOneThreads * kSortOneItems;
  constexpr int kEach = (1 << kSortMaxBits) / kSortOneThreads;
  static_assert(kEach == 1, "a thread a digit");
  __shared__ uint32_t next[kWaves][1 << kSortMaxBits];
  __shared__ uint32_t lkey[kTile], ltok[kTile];
  __shared__ uint32_t sums[kWaves];
  if (blockIdx.x > 0) {
    zero_rows<false>(a, 0, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  const int bins = 1 << a.bits, n = (int)a.tokens;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, base = wave * 64 * kSortOneItems;
  uint32_t key[kSortOneItems], tok[kSortOneItems];
#pragma unroll
  for (int u = 0; u < kSortOneItems; ++u) {
    const int i = base + u * 64 + lane;
    key[u] = i < n ? key_of(a, i, true) : 0;
    tok[u] = (uint32_t)i;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    if ((int)threadIdx.x < bins) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) next[w][threadIdx.x] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortOneItems; ++u)
      if (base + u * 64 + lane < n) atomicAdd(&next[wave][(key[u] >> shift) & (bins - 1)], 1u);
    __syncthreads();
    uint32_t sum = 0;
    if ((int)threadIdx.x < bins) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = next[w][threadIdx.x];
        next[w][threadIdx.x] = sum;
        sum += c;
      }
    }
    uint32_t all;
    const uint32_t start = block_prefix<kSortOneThreads>(sum, sums, &all);
    if ((int)threadIdx.x < bins) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) next[w][threadIdx.x] += start;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortOneItems; ++u) {
      const bool live = base + u * 64 + lane < n;
      const uint32_t at = place_of_digit((key[u] >> shift) & (bins - 1), live, a.bits, lane, next[wave]);
      if (live) {
        lkey[at] = key[u];
        ltok[at] = tok[u];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortOneItems; ++u) {
      const int i = base + u * 64 + lane;
      if (i < n) {
        key[u] = lkey[i];
        tok[u] = ltok[i];
      }
    }
  }
  uint2* __restrict__ out = a.pairs[(a.passes + 1) & 1];
#pragma unroll
  for (int u = 0; u < kSortOneItems; ++u) {
    const int i = base + u * 64 + lane;
    if (i < n) out[i] = uint2{key[u], tok[u]};
  }
}

// ---------------------------------------------------------------------- sum
template <int V>
__device__ __forceinline__ void write_row(const EmbedGradArgs& a, uint32_t row, int col, const float* acc) {
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = a.scale * acc[j];
  const int64_t at = (int64_t)row * a.dim + col;
  if (a.grad_dtype == DPI_F32)
    store_once<float, V>(static_cast<float*>(a.grad) + at, v);
  else if (a.grad_dtype == DPI_F16)
    store_once<f16_t, V>(static_cast<f16_t*>(a.grad) + at, v);
  else
    store_once<bf16_t, V>(static_cast<bf16_t*>(a.grad) + at, v);
}

// How a launch covers the sorted tokens: groups of 2^lpr_log lanes take `chunk` of them each, a workgroup's a span.
struct SumShape {
  int32_t lpr_log, chunk;
  int64_t span, spans;
};

// The sums: 2.1 M tokens of 128 bf16 over 1 M rows, 154 us, 4.5 TB/s of scattered rows of 256 bytes; 110,593 tokens of 64
// fp16 over 200,000 rows, 12 us.  An element a lane where rows are not aligned: the whole gradient 575 us rather than 293,
// and 58 rather than 52.
//
// Where a chunk's first row comes from and its last goes to.
constexpr uint32_t kRowCut = 1;       // the first row began before the chunk: its part is the chunk's `head`
constexpr uint32_t kRowGoesOn = 2;    // the last row, begun in the chunk, goes on after it: its part is the `tail`
constexpr uint32_t kRowThrough = 4;   // one row, begun before the chunk, goes on after it: its part is the `head`

template <typename TIN, int V>
__global__ __launch_bounds__(kSumThreads) void embed_sum_kernel(const EmbedGradArgs a, const SumShape sh) {
  __shared__ float head[kSumThreads * V], tail[kSumThreads * V];   // a thread's own V at [V * thread]
  __shared__ uint32_t state[kSumThreads];                          // of each group
  const int lpr = 1 << sh.lpr_log, groups = kSumThreads >> sh.lpr_log, g = threadIdx.x >> sh.lpr_log;
  const int col = ((int)blockIdx.y * lpr + ((int)threadIdx.x & (lpr - 1))) * V;
  const uint2* __restrict__ pairs = a.pairs[(a.passes + 1) & 1];
  const TIN* __restrict__ dout = static_cast<const TIN*>(a.dout);
  const uint32_t none = (uint32_t)a.num_rows;
  const int64_t begin = (int64_t)blockIdx.x * sh.span + g * sh.chunk, end = min(begin + sh.chunk, a.tokens);
  const bool mine = col < a.dim;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  uint32_t how = 0, row = none, last_row = none;
  if (begin < end) {
    row = pairs[begin].x;
    bool cut = row != none && begin > 0 && pairs[begin - 1].x == row;
    if (cut) how |= kRowCut;
    for (int64_t i0 = begin; i0 < end && row != none; i0 += 8) {
      uint32_t key[9], tok[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint2 item = pairs[min(i0 + u, a.tokens - 1)];
        key[u] = item.x;
        tok[u] = item.y;
      }
      key[8] = i0 + 8 < a.tokens ? pairs[i0 + 8].x : none;
      Elems<TIN, V> e[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (mine && i0 + u < end && key[u] != none) e[u] = load_once<TIN, V>(dout + (int64_t)tok[u] * a.dout_stride + col);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int64_t i = i0 + u;
        if (i >= end || key[u] == none) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += e[u][j];
        const bool goes_on = i + 1 < a.tokens && key[u + 1] == key[u];
        row = key[u];
        if (goes_on && i + 1 < end) continue;
        if (cut) {
#pragma unroll
          for (int j = 0; j < V; ++j) head[threadIdx.x * V + j] = acc[j];
          if (goes_on) how |= kRowThrough;
        } else if (goes_on) {
#pragma unroll
          for (int j = 0; j < V; ++j) tail[threadIdx.x * V + j] = acc[j];
          how |= kRowGoesOn;
        } else if (mine) {
          write_row<V>(a, row, col, acc);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        last_row = row;
        cut = false;
        row = i + 1 < a.tokens ? key[u + 1] : none;
      }
    }
  }
  if ((threadIdx.x & (lpr - 1)) == 0) state[g] = how;
  __syncthreads();
  if (!mine) return;
  // a row that begins in this chunk and goes on: the chunks after it, while it goes through them
  const bool first = g == 0 && (how & kRowCut);   // ... and one that began before the span
  // acc and the heads of the chunks from k on, eight in flight; whether the row is still open after the last
  const auto add_heads = [&](int k) {
    for (;; k += 8) {
      uint32_t how_k[8];
      float h[8][V];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int ku = min(k + u, groups - 1);
        how_k[u] = state[ku];
#pragma unroll
        for (int j = 0; j < V; ++j) h[u][j] = head[((int)(threadIdx.x & (lpr - 1)) + (ku << sh.lpr_log)) * V + j];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (k + u >= groups) return true;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += h[u][j];
        if (!(how_k[u] & kRowThrough)) return false;
      }
    }
  };
  if (first) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    add_heads(0);
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.dim + col;
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = acc[j];
  }
  if (how & kRowGoesOn) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = tail[threadIdx.x * V + j];
    if (add_heads(g + 1)) {   // on into the next span
      float* part = a.part + ((int64_t)blockIdx.x * 2 + 1) * a.dim + col;
#pragma unroll
      for (int j = 0; j < V; ++j) part[j] = acc[j];
    } else {
      write_row<V>(a, last_row, col, acc);
    }
  }
}

// The rows cut by span borders.  A wave for the span in which one begins adds the parts of up to 7 spans after it, its
// groups of lanes taking turns; a row that goes on further is the whole workgroup's.  (A workgroup for every span took 28
// us for 4,096 spans: each waits for memory a few times, and they did not all fit at once.)
constexpr int kJoinWaves = kSumThreads / 64, kJoinNear = 8;

template <int V>
__global__ __launch_bounds__(kSumThreads) void embed_join_kernel(const EmbedGradArgs a, const SumShape sh) {
  __shared__ float sum[kSumThreads * V];
  __shared__ int64_t far[kJoinWaves];   // the waves' spans whose row goes far, or -1
  const uint2* __restrict__ pairs = a.pairs[(a.passes + 1) & 1];
  const uint32_t none = (uint32_t)a.num_rows;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lpr = 1 << sh.lpr_log, col = ((int)blockIdx.y * lpr + (lane & (lpr - 1))) * V;
  const bool mine = col < a.dim;
  // how many of `window` spans from k0 on begin with the row, a lane each
  const auto follow = [&](uint32_t row, int64_t k0, int window, uint32_t start) {
    const uint64_t same = __ballot(k0 + lane < sh.spans && lane < window && start == row);
    return ~same ? __builtin_ctzll(~same) : 64;
  };
  const auto start_of = [&](int64_t k0, int window) { return pairs[min(k0 + min(lane, window - 1), sh.spans - 1) * sh.span].x; };
  const auto part_of = [&](int64_t k, int which, bool use, float* v) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = use && mine ? a.part[(k * 2 + which) * a.dim + col + j] : 0.f;
  };
  {
    const int64_t span = (int64_t)blockIdx.x * kJoinWaves + wave;
    int64_t goes_far = -1;
    if (span + 1 < sh.spans) {
      const int64_t begin = span * sh.span, end = begin + sh.span;
      const uint32_t row = pairs[end - 1].x, first_row = pairs[begin].x, before = pairs[max(begin - 1, (int64_t)0)].x;
      const bool goes_on = row != none && pairs[end].x == row;
      if (goes_on && !(begin > 0 && first_row == row && before == row)) {   // a row that begins in this span
        const int many = follow(row, span + 1, kJoinNear, start_of(span + 1, kJoinNear));
        if (many == kJoinNear) {
          goes_far = span;
        } else {
          const int groups = 64 >> sh.lpr_log, g = lane >> sh.lpr_log;
          float acc[V], v[V];
          part_of(span, 1, g == 0, acc);
          for (int i = g; i < many; i += groups) {
            part_of(span + 1 + i, 0, true, v);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += v[j];
          }
          for (int d = lpr; d < 64; d <<= 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += __shfl_xor(acc[j], d, 64);
          }
          if (g == 0 && mine) write_row<V>(a, row, col, acc);
        }
      }
    }
    if (lane == 0) far[wave] = goes_far;
  }
  __syncthreads();
  for (int w = 0; w < kJoinWaves; ++w) {
    const int64_t span = far[w];
    if (span < 0) continue;
    const int groups = kSumThreads >> sh.lpr_log, g = threadIdx.x >> sh.lpr_log;
    const uint32_t row = pairs[(span + 1) * sh.span - 1].x;
    float acc[V];
    part_of(span, 1, g == 0, acc);
    int64_t k0 = span + 1;
    int many = follow(row, k0, 64, start_of(k0, 64));
    for (;;) {   // 64 spans at a time, four of a group's in flight, and the next ones' starts
      const bool more = many == 64;
      const uint32_t start = more ? start_of(k0 + 64, 64) : 0;
      for (int i0 = g; i0 < many; i0 += 4 * groups) {
        float v[4][V];
#pragma unroll
        for (int u = 0; u < 4; ++u) part_of(k0 + i0 + u * groups, 0, i0 + u * groups < many, v[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] += v[u][j];
        }
      }
      if (!more) break;
      k0 += 64;
      many = follow(row, k0, 64, start);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sum[threadIdx.x * V + j] = acc[j];
    __syncthreads();
    if (g == 0 && mine) {
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] = 0.f;
      for (int k = 0; k < groups; ++k) {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += sum[(threadIdx.x + (k << sh.lpr_log)) * V + j];
      }
      write_row<V>(a, row, col, acc);
    }
    __syncthreads();
  }
}

int lanes_log(int32_t dim, int v) {
  int l = 0;
  while (l < 6 && (int64_t)v << l < dim) ++l;
  return l;
}

// Chunks of kSumMaxChunk tokens, shorter ones where that leaves fewer than a thousand workgroups, longer ones where it
// takes more than a launch has.
SumShape sum_shape(int64_t tokens, int lpr_log) {
  SumShape sh{};
  sh.lpr_log = lpr_log;
  const int64_t groups = kSumThreads >> lpr_log;
  sh.chunk = kSumMaxChunk;
  while (sh.chunk > 8 && tokens < 1024 * groups * sh.chunk) sh.chunk /= 2;
  while (tokens > kMostGroups * groups * sh.chunk) sh.chunk *= 2;
  sh.span = groups * sh.chunk;
  sh.spans = (tokens + sh.span - 1) / sh.span;
  return sh;
}

// The most spans that a call can have, whatever pieces its rows allow.
int64_t part_spans(int64_t tokens, int32_t dim) {
  int64_t most = 0;
  for (int v = 1; v <= 8; v *= 2) most = std::max(most, sum_shape(tokens, lanes_log(dim, v)).spans);
  return most;
}

template <typename TIN, typename TOUT, int V>
hipError_t run_forward(const EmbedArgs& a, hipStream_t s) {
  const int l = lanes_log(a.dim, V);
  const int64_t rows = (int64_t)(kThreads >> l) * kRowsInFlight;
  const unsigned columns = (unsigned)((a.dim + (V << l) - 1) / (V << l));
  for (int64_t t = 0; t < a.tokens; t += kMostGroups * rows) {
    EmbedArgs part = a;
    part.ids = a.ids + t;
    part.out = static_cast<TOUT*>(a.out) + t * a.out_stride;
    part.tokens = std::min(a.tokens - t, kMostGroups * rows);
    embed_kernel<TIN, TOUT, V><<<dim3((unsigned)((part.tokens + rows - 1) / rows), columns), kThreads, 0, s>>>(part, l);
  }
  return hipGetLastError();
}

template <typename TIN, typename TOUT>
hipError_t forward_by_piece(const EmbedArgs& a, hipStream_t s) {
  // One access of at most 16 bytes a lane on either side: stores past the caches want whole lines at once (2.1 M tokens of
  // 128 bf16 to fp32: 445 us with two stores a lane, 173 with one).  An element a lane where rows are not aligned: with the
  // same tokens, 528 us through the caches where pieces took 321.
  constexpr bool kBoth16 = sizeof(TIN) == 2 && sizeof(TOUT) == 2;
  int v = kBoth16 ? 8 : 4;
  const auto fits = [&](int w) {
    const uintptr_t in = std::min<size_t>(16, w * sizeof(TIN)) - 1, out = std::min<size_t>(16, w * sizeof(TOUT)) - 1;
    return a.dim % w == 0 && (reinterpret_cast<uintptr_t>(a.table) & in) == 0 && (a.dim * sizeof(TIN) & in) == 0 &&
           (reinterpret_cast<uintptr_t>(a.out) & out) == 0 && (a.out_stride * sizeof(TOUT) & out) == 0;
  };
  while (v > 1 && !fits(v)) v >>= 1;
  switch (v) {
    case 8: if constexpr (kBoth16) return run_forward<TIN, TOUT, 8>(a, s);
    case 4: return run_forward<TIN, TOUT, 4>(a, s);
    case 2: return run_forward<TIN, TOUT, 2>(a, s);
    default: return run_forward<TIN, TOUT, 1>(a, s);
  }
}

template <typename TIN>
hipError_t forward_by_out(const EmbedArgs& a, hipStream_t s) {
  if (a.out_dtype == DPI_F32) return forward_by_piece<TIN, float>(a, s);
  if (a.out_dtype == DPI_F16) return forward_by_piece<TIN, f16_t>(a, s);
  return forward_by_piece<TIN, bf16_t>(a, s);
}

template <typename TIN, int V>
hipError_t run_sums(const EmbedGradArgs& a, hipStream_t s) {
  const SumShape sh = sum_shape(a.tokens, lanes_log(a.dim, V));
  const unsigned columns = (unsigned)((a.dim + (V << sh.lpr_log) - 1) / (V << sh.lpr_log));
  embed_sum_kernel<TIN, V><<<dim3((unsigned)sh.spans, columns), kSumThreads, 0, s>>>(a, sh);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sh.spans == 1) return e;
  embed_join_kernel<V><<<dim3((unsigned)((sh.spans - 1 + kJoinWaves - 1) / kJoinWaves), columns), kSumThreads, 0, s>>>(a, sh);
  return hipGetLastError();
}

template <typename TIN>
hipError_t sums_by_piece(const EmbedGradArgs& a, hipStream_t s) {
  const size_t eg = elem_size(a.grad_dtype);
  int v = sizeof(TIN) == 2 ? 8 : 4;
  const auto fits = [&](int w) {
    const uintptr_t in = std::min<size_t>(16, w * sizeof(TIN)) - 1, out = std::min<size_t>(16, w * eg) - 1;
    return a.dim % w == 0 && (reinterpret_cast<uintptr_t>(a.dout) & in) == 0 && (a.dout_stride * sizeof(TIN) & in) == 0 &&
           (reinterpret_cast<uintptr_t>(a.grad) & out) == 0 && (a.dim * eg & out) == 0;
  };
  // Narrow rows still take 4 lanes: with one lane a row, a workgroup's 256 chunks are a long span, of which few lists have
  // many, and the rows that go through all of them a long way to join (105,209 tokens of 8 fp16 over 513 rows:
  // the sums take 27 us with a lane a row, 11.4 with four).
  while (v > 1 && (!fits(v) || a.dim < 4 * v)) v >>= 1;
  switch (v) {
    case 8: if constexpr (sizeof(TIN) == 2) return run_sums<TIN, 8>(a, s);
    case 4: return run_sums<TIN, 4>(a, s);
    case 2: return run_sums<TIN, 2>(a, s);
    default: return run_sums<TIN, 1>(a, s);
  }
}

}  // namespace

EmbedGradLayout embed_grad_layout(int64_t num_rows, int32_t dim, int64_t tokens) {
  EmbedGradLayout L{};
  int key_bits = 1;
  while (key_bits < 32 && (num_rows >> key_bits) != 0) ++key_bits;   // keys are 0 .. num_rows
  L.passes = (key_bits + kSortMaxBits - 1) / kSortMaxBits;
  L.bits = (key_bits + L.passes - 1) / L.passes;
  // Few items a thread make many workgroups, many items long runs of a digit.  Few / many, us, 1 M rows of 64 bf16: 78 / 100
  // for 131,072 tokens, 100 / 115 for 524,288, 141 / 136 for 1,048,576, 229 / 195 for 2,097,152.  One workgroup alone: 64
  // tokens over 500 rows in 12 us rather than 20, 4,096 in 20 rather than 26.
  const int64_t tile = kSortThreads * (tokens <= kSortFewTokens ? kSortFewItems : kSortManyItems);
  L.tiles = tokens <= kSortOneThreads * kSortOneItems ? 1 : (tokens + tile - 1) / tile;
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~size_t(255);
    return at;
  };
  for (int k = 0; k < 2; ++k) L.pairs[k] = take((size_t)tokens * 8);
  L.touched = take((size_t)num_rows);
  L.hist = take(((size_t)L.tiles << L.bits) * 4);
  L.total = take((size_t(1) << L.bits) * 4);
  L.part = take((size_t)part_spans(tokens, dim) * 2 * (size_t)dim * 4);
  L.bytes = std::max<size_t>(off, 256);
  return L;
}

// Whether the tiles' prefixes take a launch of their own.  Without one each workgroup reads the counts of all tiles, which
// costs less than a launch while they are few.  Whole gradients of 64 fp16, us, with / without: 5,000 tokens over 200,000
// rows (2,560 counts) 40 / 35, 20,000 (10,240) 42 / 37, 50,000 (25,088) 43 / 40.5, 110,593 (55,808) 44 / 47.5; 30,000 over
// 1 M rows (30,720) 55 / 51; 600,000 of 8 over 15 rows (9,376 counts of 586 tiles) 46 / 44.
static bool sort_scans(const EmbedGradArgs& a) {
  return a.tiles << a.bits > kSortScanCounts || a.bits < 2 || a.tokens > kSortFewTokens;
}

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s) {
  if (a.tokens == 0) return hipSuccess;
  if (a.table_dtype == DPI_F32) return forward_by_out<float>(a, s);
  if (a.table_dtype == DPI_F16) return forward_by_out<f16_t>(a, s);
  return forward_by_out<bf16_t>(a, s);
}

hipError_t launch_embed_grad(const EmbedGradArgs& args, hipStream_t s) {
  EmbedGradArgs a = args;
  const int64_t bytes = a.num_rows * a.dim * elem_size(a.grad_dtype);
  // A workgroup that zeroes has some 16 KB of it.  Those beside the one that sorts alone are at most a CU's each, which its
  // LDS has no room for two of: 25.6 MB beside 64 tokens take 31 us in 1,564 workgroups, 18 in 255.
  const auto zero_blocks = [&](int shares) { return std::min<int64_t>((bytes / shares + 16383) / 16384, 4096); };
  hipError_t e = hipSuccess;
  if (a.tokens == 0 && bytes == 0) return e;
  if (a.tiles == 1 || a.tokens == 0) {
    a.zero_shares = 1;
    sort_one_kernel<<<dim3((unsigned)(1 + std::min<int64_t>(zero_blocks(1), 255))), kSortOneThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (a.tokens == 0) return e;
  } else {
    const bool few = a.tokens <= kSortFewTokens, scans = sort_scans(a);
    a.launches = scans ? 3 : 2;
    a.zero_shares = a.passes == 1 ? 1 : a.launches * a.passes - 1;
    const int64_t zero = zero_blocks(a.zero_shares);
    const dim3 tiles((unsigned)(a.tiles + zero)), scan((unsigned)(((1 << a.bits) + 63) / 64 + (zero + 3) / 4));
    for (int p = 0; p < a.passes && e == hipSuccess; ++p) {
      if (few)
        sort_count_kernel<kSortFewItems><<<tiles, kSortThreads, 0, s>>>(a, p);
      else
        sort_count_kernel<kSortManyItems><<<tiles, kSortThreads, 0, s>>>(a, p);
      if (scans) sort_scan_kernel<<<scan, 64 * kSortScanWaves, 0, s>>>(a, p);
      if (!scans)
        sort_scatter_kernel<kSortFewItems, false><<<tiles, kSortThreads, 0, s>>>(a, p);
      else if (few)
        sort_scatter_kernel<kSortFewItems, true><<<tiles, kSortThreads, 0, s>>>(a, p);
      else
        sort_scatter_kernel<kSortManyItems, true><<<tiles, kSortThreads, 0, s>>>(a, p);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  if (a.dout_dtype == DPI_F32) return sums_by_piece<float>(a, s);
  if (a.dout_dtype == DPI_F16) return sums_by_piece<f16_t>(a, s);
  return sums_by_piece<bf16_t>(a, s);
}

}  // namespace dpi
