// Embedding rows of a list of tokens, scaled, and their table's gradient, for
// gfx950 (MI355X).
//
// Forward: out[i] = scale * E[ids[i]].  LPR lanes cover a row in pieces of V
// elements.  The bound is HBM: distinct rows read, token rows written.
//
// Backward: dE[v] = scale * sum_{i: ids[i] = v} dout[i].  Tokens are sorted by
// id (least significant digit first, stable, so equal ids stay in token order);
// a group of lanes then adds the rows of kSumChunk sorted tokens and writes
// each row of the gradient that begins and ends among them.  A row cut by
// chunk borders leaves a part per chunk, and a second kernel adds those in
// order: no float atomics, so the sums do not depend on timing.
#include "elem.h"
#include "seq_internal.h"

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

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const EmbedGradArgs a, int pass) {
  __shared__ uint32_t count[1 << kSortMaxBits];
  const int bins = 1 << a.bits, shift = pass * a.bits;
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  __syncthreads();
  const uint32_t* __restrict__ keys = a.keys[(pass + 1) & 1];
#pragma unroll
  for (int u = 0; u < kSortItems; ++u) {
    const int64_t i = base + u * kSortThreads + threadIdx.x;
    if (i < a.tokens) {
      const uint32_t key = pass == 0 ? key_of(a, i, true) : keys[i];
      atomicAdd(&count[(key >> shift) & (bins - 1)], 1u);
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) a.hist[(int64_t)b * gridDim.x + blockIdx.x] = count[b];
}

// A wave per digit: its counts over the tiles to their exclusive prefixes, and the digit's total.
__global__ __launch_bounds__(64) void sort_scan_kernel(const EmbedGradArgs a, int64_t tiles) {
  uint32_t* h = a.hist + (int64_t)blockIdx.x * tiles;
  uint32_t sum = 0;
  for (int64_t i0 = 0; i0 < tiles; i0 += 64) {
    const int64_t i = i0 + threadIdx.x;
    const uint32_t c = i < tiles ? h[i] : 0;
    uint32_t x = c;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = (uint32_t)__shfl_up((int)x, d, 64);
      if ((int)threadIdx.x >= d) x += y;
    }
    if (i < tiles) h[i] = sum + x - c;
    sum += (uint32_t)__shfl((int)x, 63, 64);
  }
  if (threadIdx.x == 0) a.total[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const EmbedGradArgs a, int pass) {
  constexpr int kWaves = kSortThreads / 64;
  __shared__ uint32_t next[kWaves][1 << kSortMaxBits];
  __shared__ uint32_t start[1 << kSortMaxBits];
  const int bins = 1 << a.bits, shift = pass * a.bits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t base = (int64_t)blockIdx.x * kSortTile + wave * 64 * kSortItems;   // a wave's items are consecutive
  for (int b = threadIdx.x; b < kWaves * bins; b += kSortThreads) next[b / bins][b % bins] = 0;
  // the digits' starts: an exclusive scan of their totals by the first wave
  if (wave == 0) {
    uint32_t sum = 0;
    for (int b0 = 0; b0 < bins; b0 += 64) {
      const uint32_t c = b0 + lane < bins ? a.total[b0 + lane] : 0;
      uint32_t x = c;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)x, d, 64);
        if (lane >= d) x += y;
      }
      if (b0 + lane < bins) start[b0 + lane] = sum + x - c;
      sum += (uint32_t)__shfl((int)x, 63, 64);
    }
  }
  uint32_t key[kSortItems], tok[kSortItems];
  const uint32_t* __restrict__ keys = a.keys[(pass + 1) & 1];
  const uint32_t* __restrict__ toks = a.toks[(pass + 1) & 1];
#pragma unroll
  for (int u = 0; u < kSortItems; ++u) {
    const int64_t i = base + u * 64 + lane;
    key[u] = tok[u] = 0;
    if (i < a.tokens) {
      key[u] = pass == 0 ? key_of(a, i, false) : keys[i];
      tok[u] = pass == 0 ? (uint32_t)i : toks[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kSortItems; ++u)
    if (base + u * 64 + lane < a.tokens) atomicAdd(&next[wave][(key[u] >> shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) {
    uint32_t at = start[b] + a.hist[(int64_t)b * gridDim.x + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = next[w][b];
      next[w][b] = at;
      at += c;
    }
  }
  __syncthreads();
  uint32_t* __restrict__ keys_out = a.keys[pass & 1];
  uint32_t* __restrict__ toks_out = a.toks[pass & 1];
#pragma unroll
  for (int u = 0; u < kSortItems; ++u) {
    const bool live = base + u * 64 + lane < a.tokens;
    const uint32_t digit = (key[u] >> shift) & (bins - 1);
    // lanes with this lane's digit
    uint64_t same = __ballot(live);
    for (int b = 0; b < a.bits; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1);
      same &= (digit >> b) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (live) {
      const uint32_t at = next[wave][digit] + rank;
      keys_out[at] = key[u];
      toks_out[at] = tok[u];
    }
    __builtin_amdgcn_wave_barrier();
    if (live && rank == 0) next[wave][digit] += (uint32_t)__popcll(same);
    __builtin_amdgcn_wave_barrier();
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

template <typename TIN, int V>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(const EmbedGradArgs a, int lpr_log, int64_t chunks) {
  const int lpr = 1 << lpr_log;
  const int64_t chunk = (int64_t)blockIdx.x * (kThreads >> lpr_log) + (threadIdx.x >> lpr_log);
  const int col = ((int)blockIdx.y * lpr + ((int)threadIdx.x & (lpr - 1))) * V;
  if (chunk >= chunks || col >= a.dim) return;
  const uint32_t* __restrict__ keys = a.keys[(a.passes + 1) & 1];
  const uint32_t* __restrict__ toks = a.toks[(a.passes + 1) & 1];
  const TIN* __restrict__ dout = static_cast<const TIN*>(a.dout);
  const uint32_t none = (uint32_t)a.num_rows;
  const int64_t begin = chunk * kSumChunk, end = min(begin + kSumChunk, a.tokens);
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  uint32_t row = keys[begin];
  bool cut = begin > 0 && keys[begin - 1] == row;   // the row began before this chunk
  for (int64_t i = begin; i < end && row != none; ++i) {
    const Elems<TIN, V> e = load_elems<true, TIN, V>(dout + (int64_t)toks[i] * a.dout_stride + col, V);
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += e[j];
    const uint32_t after = i + 1 < a.tokens ? keys[i + 1] : none;
    if (after == row && i + 1 < end) continue;
    if (cut || after == row) {   // a part of the row: its first piece is a chunk's second, every other a chunk's first
      float* part = a.part + (chunk * 2 + (cut ? 0 : 1)) * a.dim + col;
#pragma unroll
      for (int j = 0; j < V; ++j) part[j] = acc[j];
    } else {
      write_row<V>(a, row, col, acc);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    row = after;
    cut = false;
  }
}

// The rows cut by chunk borders: a group of lanes for the chunk in which one begins.
template <int V>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(const EmbedGradArgs a, int lpr_log, int64_t chunks) {
  const int lpr = 1 << lpr_log;
  const int64_t chunk = (int64_t)blockIdx.x * (kThreads >> lpr_log) + (threadIdx.x >> lpr_log);
  const int col = ((int)blockIdx.y * lpr + ((int)threadIdx.x & (lpr - 1))) * V;
  if (chunk >= chunks || col >= a.dim) return;
  const uint32_t* __restrict__ keys = a.keys[(a.passes + 1) & 1];
  const uint32_t none = (uint32_t)a.num_rows;
  const int64_t begin = chunk * kSumChunk, end = begin + kSumChunk;
  if (end >= a.tokens) return;
  const uint32_t row = keys[end - 1];
  if (row == none || keys[end] != row) return;                                    // nothing goes on after this chunk
  if (begin > 0 && keys[begin] == row && keys[begin - 1] == row) return;          // it began before this chunk
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = a.part[(chunk * 2 + 1) * a.dim + col + j];
  for (int64_t c = chunk + 1; c < chunks && keys[c * kSumChunk] == row; ++c) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += a.part[c * 2 * a.dim + col + j];
  }
  write_row<V>(a, row, col, acc);
}

__global__ __launch_bounds__(kThreads) void fill_zero_kernel(void* p, int64_t bytes) {
  typedef int quad __attribute__((ext_vector_type(4)));
  const int64_t step = (int64_t)gridDim.x * kThreads, me = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t quads = (reinterpret_cast<uintptr_t>(p) & 15) == 0 ? bytes / 16 : 0;
  for (int64_t i = me; i < quads; i += step) static_cast<quad*>(p)[i] = quad{0, 0, 0, 0};
  for (int64_t i = quads * 8 + me; i < bytes / 2; i += step) static_cast<uint16_t*>(p)[i] = 0;
}


int lanes_log(int32_t dim, int v) {
  int l = 0;
  while (l < 6 && (int64_t)v << l < dim) ++l;
  return l;
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
  const int l = lanes_log(a.dim, V);
  const int64_t chunks = (a.tokens + kSumChunk - 1) / kSumChunk, groups = kThreads >> l;
  const dim3 grid((unsigned)((chunks + groups - 1) / groups), (unsigned)((a.dim + (V << l) - 1) / (V << l)));
  embed_sum_kernel<TIN, V><<<grid, kThreads, 0, s>>>(a, l, chunks);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  embed_join_kernel<V><<<grid, kThreads, 0, s>>>(a, l, chunks);
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
  L.tiles = (tokens + kSortTile - 1) / kSortTile;
  L.chunks = (tokens + kSumChunk - 1) / kSumChunk;
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
  L.part = take((size_t)L.chunks * 2 * (size_t)dim * 4);
  L.bytes = std::max<size_t>(off, 256);
  return L;
}

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s) {
  if (a.tokens == 0) return hipSuccess;
  if (a.table_dtype == DPI_F32) return forward_by_out<float>(a, s);
  if (a.table_dtype == DPI_F16) return forward_by_out<f16_t>(a, s);
  return forward_by_out<bf16_t>(a, s);
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, hipStream_t s) {
  const int64_t bytes = a.num_rows * a.dim * elem_size(a.grad_dtype);
  hipError_t e = hipSuccess;
  if (bytes > 0) {
    const int64_t blocks = std::min<int64_t>((bytes / 16 + kThreads) / kThreads, 8192);
    fill_zero_kernel<<<dim3((unsigned)blocks), kThreads, 0, s>>>(a.grad, bytes);
    e = hipGetLastError();
  }
  if (a.tokens == 0) return e;
  const int64_t tiles = (a.tokens + kSortTile - 1) / kSortTile;
  for (int p = 0; p < a.passes && e == hipSuccess; ++p) {
    sort_count_kernel<<<dim3((unsigned)tiles), kSortThreads, 0, s>>>(a, p);
    sort_scan_kernel<<<dim3(1u << a.bits), 64, 0, s>>>(a, tiles);
    sort_scatter_kernel<<<dim3((unsigned)tiles), kSortThreads, 0, s>>>(a, p);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  if (a.dout_dtype == DPI_F32) return sums_by_piece<float>(a, s);
  if (a.dout_dtype == DPI_F16) return sums_by_piece<f16_t>(a, s);
  return sums_by_piece<bf16_t>(a, s);
}

}  // namespace dpi
