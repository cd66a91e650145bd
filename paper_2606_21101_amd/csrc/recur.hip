// Gated linear recurrence over packed sequences, forward, backward and one
// token at a time, for gfx950 (MI355X).
//
//   a_t = sigmoid(gate_t),   h_t = a_t h_{t-1} + (1 - a_t) x_t   per channel.
//
// A step is the map h -> A h + S; maps compose: (A2, S2) after (A1, S1) is
// (A2 A1, A2 S1 + S2).  The token axis is cut into blocks of G * K tokens: a
// thread composes K tokens of V channels in registers, lanes that hold later
// tokens of the same channels join their maps by shuffles, waves by LDS, and
// each thread then walks its K tokens again from the state that enters them.
// A sequence's first token is a map that forgets the state: its A is marked by
// a set sign bit (a's are never negative), so that an infinite state of one
// sequence is not multiplied into the next.
//
// A workgroup takes the sequences that begin in its range of tokens and walks
// their blocks one after the other, so no state passes between workgroups.
// The backward pass runs c_t = a_t (dh_t + c_{t+1}) the same way from the end,
// c_t being the gradient of h_{t-1}, and computes the states again in fp32 from
// the state that entered each block, which the forward pass saved.  The bound
// is HBM: 3 arrays forward, 5 backward.
#include "elem.h"
#include "seq_internal.h"

#include <algorithm>

namespace dpi {
namespace {

constexpr int V = kGlrV, K = kGlrK, kThreads = kGlrThreads, kWaves = kThreads / 64;
constexpr int kMaxGroups = kThreads;              // one lane covers a row
constexpr int kMaxTokens = kMaxGroups * K;        // of a block

// a = sigmoid(g) and 1 - a, each with a small relative error wherever it lies (no 1 - a of an a near 1).
__device__ __forceinline__ void gate_of(float g, float& a, float& keep) {
  const float e = __expf(-fabsf(g));
  const float r = __builtin_amdgcn_rcpf(1.f + e);
  const float s = e * r;
  a = g >= 0.f ? r : s;
  keep = g >= 0.f ? s : r;
  if (g != g) a = keep = g;
}

__device__ __forceinline__ bool forgets(float a) { return __float_as_int(a) < 0; }

// (A, S) after (A0, S0), into (A, S).
__device__ __forceinline__ void after(float& A, float& S, float A0, float S0) {
  if (!forgets(A)) {
    S = fmaf(A, S0, S);
    A = A * A0;   // A >= 0: A0's mark goes through
  }
}

// First sequence that ends after token t: the one that holds t when the offsets are sound; seqs for a t past the end.
__device__ __forceinline__ int32_t sequence_of(const GlrArgs& a, int64_t t) {
  if (t < 0) return -1;
  if (t >= a.tokens) return (int32_t)a.seqs;
  int64_t lo = 0, hi = a.seqs;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if ((int64_t)a.offsets[mid + 1] > t)
      hi = mid;
    else
      lo = mid + 1;
  }
  return (int32_t)lo;
}

// Tokens [lo, hi) of the sequences that begin in the workgroup's range, from two threads' searches.
__device__ __forceinline__ void owned_tokens(const GlrArgs& a, int64_t block_tokens, int64_t* shared, int64_t& lo,
                                             int64_t& hi) {
  if (threadIdx.x < 2) {
    const int64_t t = ((int64_t)blockIdx.x + threadIdx.x) * a.range_blocks * block_tokens;
    int64_t begin = min(t, a.tokens);
    if (t > 0 && t < a.tokens) {
      const int32_t s = sequence_of(a, t - 1);
      begin = s < a.seqs ? min(max((int64_t)a.offsets[s + 1], t), a.tokens) : a.tokens;
    }
    shared[threadIdx.x] = begin;
  }
  __syncthreads();
  lo = shared[0];
  hi = shared[1];
}

// Offsets of this workgroup's share of the sequences: malformed ones are reported, empty sequences' end states (their
// gradients, backward) copied from `from` (zeros without it) to `to`.
__device__ __forceinline__ void share_of_sequences(const GlrArgs& a, const float* from, float* to) {
  const int64_t per = (a.seqs + gridDim.x - 1) / gridDim.x;
  const int64_t begin = blockIdx.x * per, end = min(begin + per, a.seqs);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  bool bad = blockIdx.x == 0 && threadIdx.x == 0 && (a.offsets[0] != 0 || (int64_t)a.offsets[a.seqs] != a.tokens);
  for (int64_t s0 = begin + wave * 64; s0 < end; s0 += kWaves * 64) {
    const int64_t s = s0 + lane;
    bool empty = false;
    if (s < end) {
      const int32_t o0 = a.offsets[s], o1 = a.offsets[s + 1];
      bad |= o1 < o0;
      empty = o1 == o0;
    }
    if (!to) continue;
    for (uint64_t left = __ballot(empty); left; left &= left - 1) {
      const int64_t at = (s0 + __builtin_ctzll(left)) * a.dim;
      for (int c = blockIdx.y * 64 + lane; c < a.dim; c += gridDim.y * 64) to[at + c] = from ? from[at + c] : 0.f;
    }
  }
  if (bad && a.status) atomicOr(a.status, DPI_DEVSTAT_BAD_OFFSETS);
}

// What a thread knows of its place: lane c of LC covers channels [ch, ch + V), group g tokens [g K, g K + K) of a block.
struct Place {
  int lc, c, g, groups, ch, have;   // have: channels that exist, 0 for none
};

__device__ __forceinline__ Place place_of(const GlrArgs& a) {
  Place p;
  p.lc = 1 << a.lc_log;
  p.c = threadIdx.x & (p.lc - 1);
  p.g = threadIdx.x >> a.lc_log;
  p.groups = kThreads >> a.lc_log;
  p.ch = ((int)blockIdx.y * p.lc + p.c) * V;
  p.have = max(0, min(V, a.dim - p.ch));
  return p;
}

template <bool WIDE, typename T>
__device__ __forceinline__ Elems<T, V> row_part(const void* base, int64_t stride, int64_t t, const Place& p) {
  // a thread without channels reads the row's first ones
  const T* q = static_cast<const T*>(base) + t * stride + (p.have > 0 ? p.ch : 0);
  return load_elems<WIDE, T, V>(q, p.have > 0 ? p.have : 1);
}

// The state that enters the thread's tokens, from the groups before it.  (A, S): the thread's map, `in`: the state
// that enters the block, replaced by the one that leaves it.  UP: groups in order of time, else against it.
template <bool UP>
__device__ __forceinline__ void join_groups(const Place& p, const float* A, const float* S, float (*tot)[kWaves][64 * V],
                                            float* in, float* enter) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float a[V], s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) a[v] = A[v], s[v] = S[v];
  for (int d = p.lc; d < 64; d <<= 1) {
    const bool has = UP ? lane >= d : lane + d < 64;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float a0 = UP ? __shfl_up(a[v], d, 64) : __shfl_down(a[v], d, 64);
      const float s0 = UP ? __shfl_up(s[v], d, 64) : __shfl_down(s[v], d, 64);
      if (has) after(a[v], s[v], a0, s0);
    }
  }
  const bool last = UP ? lane >= 64 - p.lc : lane < p.lc;
  if (last) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      tot[0][wave][p.c * V + v] = a[v];
      tot[1][wave][p.c * V + v] = s[v];
    }
  }
  __syncthreads();
  const bool first = UP ? lane < p.lc : lane >= 64 - p.lc;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float h = in[v], mine = h;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int from = UP ? w : kWaves - 1 - w;
      if (from == wave) mine = h;
      const float wa = tot[0][from][p.c * V + v], ws = tot[1][from][p.c * V + v];
      h = forgets(wa) ? ws : fmaf(wa, h, ws);
    }
    const float a0 = UP ? __shfl_up(a[v], p.lc & 63, 64) : __shfl_down(a[v], p.lc & 63, 64);
    const float s0 = UP ? __shfl_up(s[v], p.lc & 63, 64) : __shfl_down(s[v], p.lc & 63, 64);
    enter[v] = first ? mine : (forgets(a0) ? s0 : fmaf(a0, mine, s0));
    in[v] = h;
  }
}

// seq[1 + i]: the sequence of token begin + i of a block, with one before and one after it.
__device__ __forceinline__ void block_sequences(const GlrArgs& a, int64_t begin, int tokens, int32_t* seq) {
  for (int i = threadIdx.x; i < tokens + 2; i += kThreads) seq[i] = sequence_of(a, begin + i - 1);
}

template <bool WIDE, typename T>
__global__ __launch_bounds__(kThreads) void glr_forward_kernel(const GlrArgs a) {
  __shared__ int32_t seq[kMaxTokens + 2];
  __shared__ float tot[2][2][kWaves][64 * V];
  __shared__ int64_t range[2];
  const Place p = place_of(a);
  const int block_tokens = p.groups * K;
  int64_t lo, hi;
  owned_tokens(a, block_tokens, range, lo, hi);
  share_of_sequences(a, a.h0, a.h_last);
  float state[V];
#pragma unroll
  for (int v = 0; v < V; ++v) state[v] = 0.f;
  int parity = 0;
  for (int64_t block = lo / block_tokens; block * block_tokens < hi; ++block, parity ^= 1) {
    const int64_t begin = block * block_tokens, mine = begin + p.g * K;
    Elems<T, V> x[K], g[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t t = min(max(mine + k, lo), hi - 1);
      x[k] = row_part<WIDE, T>(a.x, a.x_stride, t, p);
      g[k] = row_part<WIDE, T>(a.gate, a.gate_stride, t, p);
    }
    block_sequences(a, begin, block_tokens, seq);
    __syncthreads();
    if (a.entry && begin >= lo && p.g == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v < p.have) a.entry[block * a.dim + p.ch + v] = state[v];
    }
    float fa[K][V], fb[K][V], A[V], S[V];
    uint32_t starts = 0, ends = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.f, S[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool live = mine + k >= lo && mine + k < hi;
      const int i = p.g * K + k + 1;
      const int32_t s = seq[i];
      const bool start = live && seq[i - 1] != s;
      if (start) starts |= 1u << k;
      if (live && seq[i + 1] != s) ends |= 1u << k;
      const bool from_h0 = start && a.h0 && s < a.seqs;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float ga, keep;
        gate_of(g[k][v], ga, keep);
        float gb = keep > 0.f ? keep * x[k][v] : 0.f;   // a token that keeps the state whole has no say in it
        if (from_h0 && v < p.have) gb = fmaf(ga, a.h0[(int64_t)s * a.dim + p.ch + v], gb);
        fa[k][v] = live ? ga : 1.f;
        fb[k][v] = live ? gb : 0.f;
        if (start) {
          A[v] = -1.f;
          S[v] = fb[k][v];
        } else {
          A[v] *= fa[k][v];
          S[v] = fmaf(fa[k][v], S[v], fb[k][v]);
        }
      }
    }
    float h[V];
    join_groups<true>(p, A, S, tot[parity], state, h);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool live = mine + k >= lo && mine + k < hi;
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = starts >> k & 1 ? fb[k][v] : fmaf(fa[k][v], h[v], fb[k][v]);
      if (!live || p.have == 0) continue;
      store_elems<WIDE, T, V>(static_cast<T*>(a.h) + (mine + k) * a.h_stride + p.ch, h, p.have);
      if (a.h_last && (ends >> k & 1)) {
        const int32_t s = seq[p.g * K + k + 1];
        if (s < a.seqs) {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (v < p.have) a.h_last[(int64_t)s * a.dim + p.ch + v] = h[v];
        }
      }
    }
    __syncthreads();   // seq is read to here
  }
}

template <bool WIDE, typename T>
__global__ __launch_bounds__(kThreads) void glr_backward_kernel(const GlrArgs a) {
  __shared__ int32_t seq[kMaxTokens + 2];
  __shared__ float tot[2][2][kWaves][64 * V];
  __shared__ int64_t range[2];
  const Place p = place_of(a);
  const int block_tokens = p.groups * K;
  int64_t lo, hi;
  owned_tokens(a, block_tokens, range, lo, hi);
  share_of_sequences(a, a.dh_last, a.dh0);
  float grad[V];
#pragma unroll
  for (int v = 0; v < V; ++v) grad[v] = 0.f;
  if (lo >= hi) return;
  for (int64_t block = (hi - 1) / block_tokens; block >= lo / block_tokens; --block) {
    const int64_t begin = block * block_tokens, mine = begin + p.g * K;
    Elems<T, V> x[K], g[K], d[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t t = min(max(mine + k, lo), hi - 1);
      x[k] = row_part<WIDE, T>(a.x, a.x_stride, t, p);
      g[k] = row_part<WIDE, T>(a.gate, a.gate_stride, t, p);
      if (a.dh) d[k] = row_part<WIDE, T>(a.dh, a.dh_stride, t, p);
    }
    block_sequences(a, begin, block_tokens, seq);
    float state[V];   // enters the block, if its sequence began before it
#pragma unroll
    for (int v = 0; v < V; ++v) state[v] = begin > lo && v < p.have ? a.entry[block * a.dim + p.ch + v] : 0.f;
    __syncthreads();
    float fa[K][V], kp[K][V], A[V], S[V], RA[V], RS[V];
    uint32_t starts = 0, ends = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = RA[v] = 1.f, S[v] = RS[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool live = mine + k >= lo && mine + k < hi;
      const int i = p.g * K + k + 1;
      const int32_t s = seq[i];
      const bool start = live && seq[i - 1] != s;
      if (start) starts |= 1u << k;
      if (live && seq[i + 1] != s) ends |= 1u << k;
      const bool from_h0 = start && a.h0 && s < a.seqs;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float ga, keep;
        gate_of(g[k][v], ga, keep);
        fa[k][v] = live ? ga : 1.f;
        kp[k][v] = live ? keep : 0.f;
        const float b = kp[k][v] > 0.f ? keep * x[k][v] : 0.f;
        if (start) {
          A[v] = -1.f;
          S[v] = from_h0 && v < p.have ? fmaf(ga, a.h0[(int64_t)s * a.dim + p.ch + v], b) : b;
        } else {
          A[v] *= fa[k][v];
          S[v] = fmaf(fa[k][v], S[v], b);
        }
      }
    }
    float h[V];
    join_groups<true>(p, A, S, tot[0], state, h);
    // dg needs the state before each token, in order of time
    float hp[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int32_t s = seq[p.g * K + k + 1];
      const bool start = starts >> k & 1;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (start) h[v] = a.h0 && s < a.seqs && v < p.have ? a.h0[(int64_t)s * a.dim + p.ch + v] : 0.f;
        hp[k][v] = h[v];
        h[v] = fmaf(fa[k][v], h[v], kp[k][v] > 0.f ? kp[k][v] * x[k][v] : 0.f);
      }
    }
    // the gradients' maps, from the last token on
    float de[K][V];
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      const bool live = mine + k >= lo && mine + k < hi;
      const int32_t s = seq[p.g * K + k + 1];
      const bool end = ends >> k & 1;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float e = live && a.dh ? d[k][v] : 0.f;
        if (end && a.dh_last && s < a.seqs && v < p.have) e += a.dh_last[(int64_t)s * a.dim + p.ch + v];
        de[k][v] = e;
        if (end) {
          RA[v] = -fa[k][v];
          RS[v] = fa[k][v] * e;
        } else {
          RA[v] *= fa[k][v];
          RS[v] = fmaf(fa[k][v], RS[v], fa[k][v] * e);
        }
      }
    }
    float c[V];
    join_groups<false>(p, RA, RS, tot[1], grad, c);
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      const bool live = mine + k >= lo && mine + k < hi;
      float dx[V], dg[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float e = ends >> k & 1 ? de[k][v] : de[k][v] + c[v];
        dx[v] = kp[k][v] * e;
        dg[v] = kp[k][v] > 0.f ? fa[k][v] * kp[k][v] * (hp[k][v] - x[k][v]) * e : dx[v];
        if (live) c[v] = fa[k][v] * e;
      }
      if (!live || p.have == 0) continue;
      store_elems<WIDE, T, V>(static_cast<T*>(a.dx) + (mine + k) * a.dx_stride + p.ch, dx, p.have);
      store_elems<WIDE, T, V>(static_cast<T*>(a.dgate) + (mine + k) * a.dgate_stride + p.ch, dg, p.have);
      if (a.dh0 && (starts >> k & 1)) {
        const int32_t s = seq[p.g * K + k + 1];
        if (s < a.seqs) {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (v < p.have) a.dh0[(int64_t)s * a.dim + p.ch + v] = c[v];
        }
      }
    }
    __syncthreads();   // seq and the waves' maps are read to here
  }
}

template <bool WIDE, typename T>
__global__ __launch_bounds__(kThreads) void glr_step_kernel(const GlrStepArgs a) {
  const int pieces = (a.dim + V - 1) / V;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.batch * pieces) return;
  const int64_t b = i / pieces;
  const int ch = (int)(i % pieces) * V, have = min(V, a.dim - ch);
  const int64_t slot = a.slots ? a.slots[b] : b;
  const bool inside = slot >= 0 && slot < a.num_slots;
  float h[V];
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = 0.f;
  if (inside) {
    const Elems<T, V> x = load_elems<WIDE, T, V>(static_cast<const T*>(a.x) + b * a.x_stride + ch, have);
    const Elems<T, V> g = load_elems<WIDE, T, V>(static_cast<const T*>(a.gate) + b * a.gate_stride + ch, have);
    float* state = a.state + slot * a.dim + ch;
    const Elems<float, V> s = load_elems<WIDE, float, V>(state, have);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float ga, keep;
      gate_of(g[v], ga, keep);
      h[v] = fmaf(ga, s[v], keep > 0.f ? keep * x[v] : 0.f);
    }
    store_elems<WIDE, float, V>(state, h, have);
  } else if (ch == 0 && a.status) {
    atomicOr(a.status, DPI_DEVSTAT_BAD_ID);
  }
  store_elems<WIDE, T, V>(static_cast<T*>(a.h) + b * a.h_stride + ch, h, have);
}

template <typename T>
hipError_t run_pass(const GlrArgs& a, bool backward, hipStream_t s) {
  const GlrShape sh = glr_shape(a.tokens, a.dim);
  const int64_t ranges = std::max<int64_t>(1, (sh.blocks + a.range_blocks - 1) / a.range_blocks);
  const dim3 grid((unsigned)ranges, (unsigned)sh.channel_blocks);
  if (backward) {
    if (a.wide)
      glr_backward_kernel<true, T><<<grid, kThreads, 0, s>>>(a);
    else
      glr_backward_kernel<false, T><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (a.wide)
      glr_forward_kernel<true, T><<<grid, kThreads, 0, s>>>(a);
    else
      glr_forward_kernel<false, T><<<grid, kThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t run_by_dtype(const GlrArgs& a, bool backward, hipStream_t s) {
  if (a.seqs == 0) return hipSuccess;
  if (a.dtype == DPI_F32) return run_pass<float>(a, backward, s);
  if (a.dtype == DPI_F16) return run_pass<f16_t>(a, backward, s);
  return run_pass<bf16_t>(a, backward, s);
}

template <typename T>
hipError_t run_step(const GlrStepArgs& a, hipStream_t s) {
  const int64_t threads = a.batch * ((a.dim + V - 1) / V);
  const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
  if (a.wide)
    glr_step_kernel<true, T><<<grid, kThreads, 0, s>>>(a);
  else
    glr_step_kernel<false, T><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Lanes of a power of two cover up to 64 * V channels; the other lanes of a workgroup take later tokens.
GlrShape glr_shape(int64_t tokens, int32_t dim) {
  GlrShape sh{};
  while (sh.lc_log < 6 && (V << sh.lc_log) < dim) ++sh.lc_log;
  sh.block_tokens = (int64_t)(kThreads >> sh.lc_log) * K;
  sh.blocks = (tokens + sh.block_tokens - 1) / sh.block_tokens;
  sh.channel_blocks = (dim + (V << sh.lc_log) - 1) / (V << sh.lc_log);
  return sh;
}

hipError_t launch_glr_forward(const GlrArgs& a, hipStream_t s) { return run_by_dtype(a, false, s); }
hipError_t launch_glr_backward(const GlrArgs& a, hipStream_t s) { return run_by_dtype(a, true, s); }

hipError_t launch_glr_step(const GlrStepArgs& a, hipStream_t s) {
  if (a.batch == 0) return hipSuccess;
  if (a.dtype == DPI_F32) return run_step<float>(a, s);
  if (a.dtype == DPI_F16) return run_step<f16_t>(a, s);
  return run_step<bf16_t>(a, s);
}

}  // namespace dpi
