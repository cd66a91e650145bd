// Embedding rows of a list of tokens, scaled, and their table's gradient, for
// gfx950 (MI355X).
//
// Forward: out[i] = scale * E[ids[i]].  LPR lanes cover a row in pieces of V
// elements.  The bound is HBM: distinct rows read, token rows written.
//
// Backward: dE[v] = scale * sum_{i: ids[i] = v} dout[i].  Tokens are sorted by
// id (least significant digit first, stable, so equal ids stay in token order).
// A workgroup then sums a span of sorted tokens: a group of LPR lanes adds the
// rows of a chunk, eight in flight, and writes each row of the gradient that
// begins and ends in it; rows cut by chunk borders are joined in LDS, those cut
// by span borders by a second kernel.  Every sum has a fixed order and there
// are no float atomics, so the result does not depend on timing.  The rows
// without tokens are zeroed by workgroups of the sort's launches, which leave
// the memory idle otherwise.  The bound is HBM: dout read, the gradient written.
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
    store_elems<true, TOUT, V>(out + i * a.out_stride + col, v, V);
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

// Share `share` of a.launches of the gradient set to zero by `blocks` workgroups, of which this is `block`.
__device__ __forceinline__ void zero_share(const EmbedGradArgs& a, int share, int64_t block, int64_t blocks) {
  typedef int quad __attribute__((ext_vector_type(4)));
  const int64_t bytes = a.num_rows * a.dim * (a.grad_dtype == DPI_F32 ? 4 : 2);
  const int64_t step = blocks * blockDim.x, me = block * blockDim.x + threadIdx.x;
  const int64_t quads = (reinterpret_cast<uintptr_t>(a.grad) & 15) == 0 ? bytes / 16 : 0;
  const int64_t end = quads * (share + 1) / a.launches;
  for (int64_t i = quads * share / a.launches + me; i < end; i += step) static_cast<quad*>(a.grad)[i] = quad{0, 0, 0, 0};
  if (share == 0)   // what 16-byte stores cannot reach
    for (int64_t i = quads * 8 + me; i < bytes / 2; i += step) static_cast<uint16_t*>(a.grad)[i] = 0;
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

template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const EmbedGradArgs a, int pass) {
  __shared__ uint32_t count[1 << kSortMaxBits];
  if (blockIdx.x >= a.tiles) {
    zero_share(a, 3 * pass, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    return;
  }
  const int bins = 1 << a.bits, shift = pass * a.bits;
  const int64_t base = (int64_t)blockIdx.x * kSortThreads * ITEMS;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  const uint32_t* __restrict__ keys = a.keys[(pass + 1) & 1];
  uint32_t key[ITEMS];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int64_t i = base + u * kSortThreads + threadIdx.x;
    key[u] = i < a.tokens ? (pass == 0 ? key_of(a, i, true) : keys[i]) : 0;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < ITEMS; ++u)
    if (base + u * kSortThreads + threadIdx.x < a.tokens) atomicAdd(&count[(key[u] >> shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) a.hist[((int64_t)blockIdx.x << a.bits) + b] = count[b];
}

// The tiles' counts of 64 digits to their exclusive prefixes over the tiles, and the digits' totals: a lane a digit, the
// 16 waves a range of tiles each.
constexpr int kSortScanWaves = 16;

__global__ __launch_bounds__(64 * kSortScanWaves) void sort_scan_kernel(const EmbedGradArgs a, int pass) {
  __shared__ uint32_t sums[kSortScanWaves][64];
  const int bins = 1 << a.bits, groups = (bins + 63) / 64;
  if ((int)blockIdx.x >= groups) {
    zero_share(a, 3 * pass + 1, blockIdx.x - groups, gridDim.x - groups);
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

template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const EmbedGradArgs a, int pass) {
  constexpr int kWaves = kSortThreads / 64, kEach = (1 << kSortMaxBits) / kSortThreads;
  __shared__ uint32_t next[kWaves][1 << kSortMaxBits];
  __shared__ uint32_t sums[kWaves];
  if (blockIdx.x >= a.tiles) {
    zero_share(a, 3 * pass + 2, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    return;
  }
  const int bins = 1 << a.bits, shift = pass * a.bits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t base = ((int64_t)blockIdx.x * kWaves + wave) * 64 * ITEMS;   // a wave's items are consecutive
  uint32_t key[ITEMS], tok[ITEMS];
  const uint32_t* __restrict__ keys = a.keys[(pass + 1) & 1];
  const uint32_t* __restrict__ toks = a.toks[(pass + 1) & 1];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int64_t i = base + u * 64 + lane;
    key[u] = tok[u] = 0;
    if (i < a.tokens) {
      key[u] = pass == 0 ? key_of(a, i, false) : keys[i];
      tok[u] = pass == 0 ? (uint32_t)i : toks[i];
    }
  }
  // kEach neighbouring digits a thread: where they start, and this tile's part of them
  uint32_t total[kEach], mine[kEach], sum = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int b = threadIdx.x * kEach + j;
    total[j] = b < bins ? a.total[b] : 0;
    mine[j] = b < bins ? a.hist[((int64_t)blockIdx.x << a.bits) + b] : 0;
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
    if (base + u * 64 + lane < a.tokens) atomicAdd(&next[wave][(key[u] >> shift) & (bins - 1)], 1u);
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
  uint32_t* __restrict__ keys_out = a.keys[pass & 1];
  uint32_t* __restrict__ toks_out = a.toks[pass & 1];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const bool live = base + u * 64 + lane < a.tokens;
    const uint32_t at = place_of_digit((key[u] >> shift) & (bins - 1), live, a.bits, lane, next[wave]);
    if (live) {
      keys_out[at] = key[u];
      toks_out[at] = tok[u];
    }
  }
}

// A short list, sorted by one workgroup in LDS; the others zero the gradient.
__global__ __launch_bounds__(kSortOneThreads) void sort_one_kernel(const EmbedGradArgs a) {
  constexpr int kWaves = kSortOneThreads / 64, kTile = kSortOneThreads * kSortOneItems;
  constexpr int kEach = (1 << kSortMaxBits) / kSortOneThreads;
  static_assert(kEach == 1, "a thread a digit");
  __shared__ uint32_t next[kWaves][1 << kSortMaxBits];
  __shared__ uint32_t lkey[kTile], ltok[kTile];
  __shared__ uint32_t sums[kWaves];
  if (blockIdx.x > 0) {
    zero_share(a, 0, blockIdx.x - 1, gridDim.x - 1);
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
  uint32_t* __restrict__ keys_out = a.keys[(a.passes + 1) & 1];
  uint32_t* __restrict__ toks_out = a.toks[(a.passes + 1) & 1];
#pragma unroll
  for (int u = 0; u < kSortOneItems; ++u) {
    const int i = base + u * 64 + lane;
    if (i < n) {
      keys_out[i] = key[u];
      toks_out[i] = tok[u];
    }
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
    store_elems<true, float, V>(static_cast<float*>(a.grad) + at, v, V);
  else if (a.grad_dtype == DPI_F16)
    store_elems<true, f16_t, V>(static_cast<f16_t*>(a.grad) + at, v, V);
  else
    store_elems<true, bf16_t, V>(static_cast<bf16_t*>(a.grad) + at, v, V);
}

// How a launch covers the sorted tokens: groups of 2^lpr_log lanes take `chunk` of them each, a workgroup's a span.
struct SumShape {
  int32_t lpr_log, chunk;
  int64_t span, spans;
};

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
  const uint32_t* __restrict__ keys = a.keys[(a.passes + 1) & 1];
  const uint32_t* __restrict__ toks = a.toks[(a.passes + 1) & 1];
  const TIN* __restrict__ dout = static_cast<const TIN*>(a.dout);
  const uint32_t none = (uint32_t)a.num_rows;
  const int64_t begin = (int64_t)blockIdx.x * sh.span + g * sh.chunk, end = min(begin + sh.chunk, a.tokens);
  const bool mine = col < a.dim;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  uint32_t how = 0, row = none, last_row = none;
  if (begin < end) {
    row = keys[begin];
    bool cut = row != none && begin > 0 && keys[begin - 1] == row;
    if (cut) how |= kRowCut;
    for (int64_t i0 = begin; i0 < end && row != none; i0 += 8) {
      uint32_t key[9], tok[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        tok[u] = toks[min(i0 + u, a.tokens - 1)];
        key[u] = keys[min(i0 + u, a.tokens - 1)];
      }
      key[8] = i0 + 8 < a.tokens ? keys[i0 + 8] : none;
      Elems<TIN, V> e[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (mine && i0 + u < end && key[u] != none) e[u] = load_elems<true, TIN, V>(dout + (int64_t)tok[u] * a.dout_stride + col, V);
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
  if (first) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = head[threadIdx.x * V + j];
    for (int k = 0; k + 1 < groups && (state[k] & kRowThrough); ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += head[(threadIdx.x + ((k + 1) << sh.lpr_log)) * V + j];
    }
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.dim + col;
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = acc[j];
  }
  if (how & kRowGoesOn) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = tail[threadIdx.x * V + j];
    bool open = true;
    for (int k = g + 1; k < groups && open; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += head[(threadIdx.x + ((k - g) << sh.lpr_log)) * V + j];
      open = (state[k] & kRowThrough) != 0;
    }
    if (open) {   // on into the next span
      float* part = a.part + ((int64_t)blockIdx.x * 2 + 1) * a.dim + col;
#pragma unroll
      for (int j = 0; j < V; ++j) part[j] = acc[j];
    } else {
      write_row<V>(a, last_row, col, acc);
    }
  }
}

// The rows cut by span borders: a workgroup for the span in which one begins, its groups of lanes taking turns at the
// spans after it.
template <int V>
__global__ __launch_bounds__(kSumThreads) void embed_join_kernel(const EmbedGradArgs a, const SumShape sh) {
  __shared__ float sum[kSumThreads * V];
  const uint32_t* __restrict__ keys = a.keys[(a.passes + 1) & 1];
  const uint32_t none = (uint32_t)a.num_rows;
  const int64_t span = blockIdx.x, begin = span * sh.span, end = begin + sh.span;   // one more span follows
  const uint32_t row = keys[end - 1];
  if (row == none || keys[end] != row) return;                               // nothing goes on after this span
  if (begin > 0 && keys[begin] == row && keys[begin - 1] == row) return;     // it began before this span
  const int lpr = 1 << sh.lpr_log, groups = kSumThreads >> sh.lpr_log, g = threadIdx.x >> sh.lpr_log;
  const int col = ((int)blockIdx.y * lpr + ((int)threadIdx.x & (lpr - 1))) * V;
  const bool mine = col < a.dim;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  for (int64_t k = span + 1 + g; k < sh.spans && keys[k * sh.span] == row; k += groups) {
    if (!mine) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += a.part[k * 2 * a.dim + col + j];
  }
#pragma unroll
  for (int j = 0; j < V; ++j) sum[threadIdx.x * V + j] = acc[j];
  __syncthreads();
  if (g != 0 || !mine) return;
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = a.part[(span * 2 + 1) * a.dim + col + j];
  for (int k = 0; k < groups; ++k) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += sum[(threadIdx.x + (k << sh.lpr_log)) * V + j];
  }
  write_row<V>(a, row, col, acc);
}

int lanes_log(int32_t dim, int v) {
  int l = 0;
  while (l < 6 && (int64_t)v << l < dim) ++l;
  return l;
}

// Chunks of at most kSumMaxChunk tokens, shorter ones where that leaves fewer than a thousand workgroups.
SumShape sum_shape(int64_t tokens, int lpr_log) {
  SumShape sh{};
  sh.lpr_log = lpr_log;
  const int64_t groups = kSumThreads >> lpr_log;
  sh.chunk = kSumMaxChunk;
  while (sh.chunk > 8 && tokens < 1024 * groups * sh.chunk) sh.chunk /= 2;
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
  const dim3 grid((unsigned)((a.tokens + rows - 1) / rows), (unsigned)((a.dim + (V << l) - 1) / (V << l)));
  embed_kernel<TIN, TOUT, V><<<grid, kThreads, 0, s>>>(a, l);
  return hipGetLastError();
}

template <typename TIN, typename TOUT>
hipError_t forward_by_piece(const EmbedArgs& a, hipStream_t s) {
  int v = sizeof(TIN) == 2 ? 8 : 4;
  const auto fits = [&](int w) {
    const uintptr_t in = std::min<size_t>(16, w * sizeof(TIN)) - 1, out = std::min<size_t>(16, w * sizeof(TOUT)) - 1;
    return a.dim % w == 0 && (reinterpret_cast<uintptr_t>(a.table) & in) == 0 && (a.dim * sizeof(TIN) & in) == 0 &&
           (reinterpret_cast<uintptr_t>(a.out) & out) == 0 && (a.out_stride * sizeof(TOUT) & out) == 0;
  };
  while (v > 1 && !fits(v)) v >>= 1;
  switch (v) {
    case 8: if constexpr (sizeof(TIN) == 2) return run_forward<TIN, TOUT, 8>(a, s);
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
  embed_join_kernel<V><<<dim3((unsigned)sh.spans - 1, columns), kSumThreads, 0, s>>>(a, sh);
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
  while (v > 1 && !fits(v)) v >>= 1;
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
  const int64_t tile = kSortThreads * (tokens <= kSortFewTokens ? kSortFewItems : kSortManyItems);
  L.tiles = tokens <= kSortOneThreads * kSortOneItems ? 1 : (tokens + tile - 1) / tile;
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~size_t(255);
    return at;
  };
  for (int k = 0; k < 2; ++k) L.keys[k] = take((size_t)tokens * 4);
  for (int k = 0; k < 2; ++k) L.toks[k] = take((size_t)tokens * 4);
  L.hist = take(((size_t)L.tiles << L.bits) * 4);
  L.total = take((size_t(1) << L.bits) * 4);
  L.part = take((size_t)part_spans(tokens, dim) * 2 * (size_t)dim * 4);
  L.bytes = std::max<size_t>(off, 256);
  return L;
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
  // a workgroup that zeroes has some 64 KB of it
  const auto zero_blocks = [&](int shares) { return std::min<int64_t>((bytes / shares + 65535) / 65536, 8192); };
  hipError_t e = hipSuccess;
  if (a.tiles == 1 || a.tokens == 0) {
    a.launches = 1;
    sort_one_kernel<<<dim3((unsigned)(1 + zero_blocks(1))), kSortOneThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (a.tokens == 0) return e;
  } else {
    a.launches = 3 * a.passes;
    const int64_t zero = zero_blocks(a.launches);
    const dim3 tiles((unsigned)(a.tiles + zero)), scan((unsigned)(((1 << a.bits) + 63) / 64 + zero));
    const bool few = a.tokens <= kSortFewTokens;
    for (int p = 0; p < a.passes && e == hipSuccess; ++p) {
      if (few)
        sort_count_kernel<kSortFewItems><<<tiles, kSortThreads, 0, s>>>(a, p);
      else
        sort_count_kernel<kSortManyItems><<<tiles, kSortThreads, 0, s>>>(a, p);
      sort_scan_kernel<<<scan, 64 * kSortScanWaves, 0, s>>>(a, p);
      if (few)
        sort_scatter_kernel<kSortFewItems><<<tiles, kSortThreads, 0, s>>>(a, p);
      else
        sort_scatter_kernel<kSortManyItems><<<tiles, kSortThreads, 0, s>>>(a, p);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  if (a.dout_dtype == DPI_F32) return sums_by_piece<float>(a, s);
  if (a.dout_dtype == DPI_F16) return sums_by_piece<f16_t>(a, s);
  return sums_by_piece<bf16_t>(a, s);
}

}  // namespace dpi
