// Gated linear recurrence over packed sequences, forward, backward and one
// token at a time, for gfx950 (MI355X).
//
//   a_t = sigmoid(gate_t),   h_t = a_t h_{t-1} + (1 - a_t) x_t   per channel.
//
// A step is the map h -> A h + S; maps compose: (A2, S2) after (A1, S1) is
// (A2 A1, A2 S1 + S2).  A wave walks a range of tokens a block at a time: LC
// lanes cover the channels, V each, and the wave's 64 / LC groups of lanes take
// K tokens each.  A thread composes its K tokens in registers, groups join
// their maps by shuffles, and each thread walks its tokens again from the state
// that enters them.  Waves share nothing, so nothing waits for a barrier.
//
// A sequence's first token is the map with A = 0.  Products with such an A are
// legacy ones, where 0 times anything is 0: no infinity and no NaN of one
// sequence gets into the next.  So is (1 - a) x, where a token of gate +inf
// keeps the state whatever x it has.
//
// Work is split in one of two ways.  Whole: a wave takes the sequences that
// begin in its range of tokens, to their ends; one launch.  Cut: a wave takes
// its range's tokens only; a first launch composes each range's map, a second
// scans the maps, a third walks the ranges from the states that enter them.
//
// The backward pass runs c_t = a_t (dh_t + c_{t+1}) the same way from the end,
// c_t being the gradient of h_{t-1}, and computes the states again in fp32 from
// the state that entered each block, which the forward pass saved.  The bound
// is HBM: 3 arrays forward, 5 backward.
#include "elem.h"
#include "seq_internal.h"

#include <algorithm>
#include <cmath>

namespace dpi {
namespace {

constexpr int V = kGlrV, K = kGlrK, kThreads = kGlrThreads, kWaves = kThreads / 64;
constexpr int kMaxTokens = 64 * K;   // of a block: one lane covers a row

// Product in which 0 times anything is 0.
__device__ __forceinline__ float mul0(float a, float b) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// a = sigmoid(g) and 1 - a, each with a small relative error wherever it lies (no 1 - a of an a near 1); a is not below
// 2^-126, and a NaN stays one.
__device__ __forceinline__ void gate_of(float g, float& a, float& keep) {
  const float e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(g * -1.44269504f, 126.f));
  a = __builtin_amdgcn_rcpf(1.f + e);
  keep = e * a;
}

// First s in [0, seqs] with offsets[s + 1] > t, by the whole wave: the sequence that holds token t when the offsets are
// sound.
__device__ __forceinline__ int64_t sequence_of(const GlrArgs& a, int64_t t, int lane) {
  int64_t lo = 0, count = a.seqs;   // the answer lies in [lo, lo + count]
  while (count > 0) {
    const int64_t step = (count + 63) >> 6, at = lo + (lane + 1) * step - 1;   // 64 candidates, the last of each part
    const bool before = at < lo + count && (int64_t)a.offsets[at + 1] <= t;
    const int parts = __popcll(__ballot(before));
    lo += parts * step;
    count = min(step - 1, max(count - parts * step, (int64_t)0));
  }
  return __builtin_amdgcn_readfirstlane((int32_t)lo);
}

// A wave's tokens [lo, hi), and the sequence that holds the first (forwards) or the last of them (backwards).
struct Span {
  int64_t lo, hi, seq;
};

__device__ __forceinline__ int64_t clamped(int64_t x, int64_t lo, int64_t hi) { return min(max(x, lo), hi); }

// The same for the whole wave.
__device__ __forceinline__ int64_t offset_at(const GlrArgs& a, int64_t s) {
  return __builtin_amdgcn_readfirstlane(a.offsets[s]);
}

// Whole: from the first sequence start at or after the range's begin to the end of the last sequence begun before its
// end.
template <bool CUT, bool FORWARD>
__device__ __forceinline__ Span span_of(const GlrArgs& a, int64_t unit, int lane) {
  Span s;
  const int64_t t0 = min(unit * a.range, a.tokens), t1 = min(t0 + a.range, a.tokens);
  s.lo = t0;
  s.hi = t1;
  s.seq = 0;
  if (t0 >= t1) return s;
  if (CUT) {
    s.seq = sequence_of(a, FORWARD ? t0 : t1 - 1, lane);
    return s;
  }
  const int64_t first = t0 > 0 ? sequence_of(a, t0 - 1, lane) : -1;
  const int64_t last = sequence_of(a, t1 - 1, lane);
  if (t0 > 0) s.lo = first < a.seqs ? clamped(offset_at(a, first + 1), t0, a.tokens) : a.tokens;
  s.hi = last < a.seqs ? clamped(offset_at(a, last + 1), t1, a.tokens) : a.tokens;
  if (s.lo >= t1) s.hi = s.lo;   // no sequence begins in the range
  s.seq = FORWARD ? max(first, (int64_t)0) : last;
  return s;
}

// 64 neighbouring sequences, one a lane, and the marks of those that begin or end in a block of tokens.
struct Window {
  int64_t base;
  int32_t begin, end;   // of the lane's sequence; an empty one past the last

  __device__ __forceinline__ void load(const GlrArgs& a, int64_t b, int lane) {
    base = max(b, (int64_t)0);
    const int64_t s = base + lane;
    begin = s < a.seqs ? a.offsets[s] : INT32_MAX;
    end = s < a.seqs ? a.offsets[s + 1] : INT32_MAX;
  }
};

// starts / ends: the lane's K tokens of the block at `t0` that are a sequence's first / last; seq_of[i], end_of[i]: that
// sequence, where it is.  Only tokens of [lo, hi) are marked.
template <bool FORWARD>
__device__ __forceinline__ void marks_of(const GlrArgs& a, Window& w, int64_t t0, int tokens, int64_t lo, int64_t hi,
                                         int lane, int mine, int32_t* starts_at, int32_t* ends_at, uint32_t& starts,
                                         uint32_t& ends) {
  const int64_t t1 = t0 + tokens;
  starts = ends = 0;
  bool any = false;
  for (;;) {
    const bool full = w.end > w.begin;
    const bool b = full && w.begin >= max(t0, lo) && w.begin < min(t1, hi);
    const bool e = full && w.end > max(t0, lo) && w.end <= min(t1, hi);
    if (__ballot(b || e)) {
      if (!any) {
        any = true;
        for (int i = lane; i < tokens; i += 64) starts_at[i] = ends_at[i] = -1;
      }
      if (b) starts_at[w.begin - t0] = (int32_t)(w.base + lane);
      if (e) ends_at[w.end - 1 - t0] = (int32_t)(w.base + lane);
    }
    if (FORWARD) {
      const int32_t far = __builtin_amdgcn_readlane(w.end, 63);
      if ((int64_t)far > t1 || w.base + 64 >= a.seqs) break;
      w.load(a, w.base + 64, lane);
    } else {
      const int32_t far = __builtin_amdgcn_readfirstlane(w.begin);
      if ((int64_t)far <= t0 || w.base == 0) break;
      w.load(a, w.base - 63, lane);   // one again: its begin says whether to go on
    }
  }
  if (any) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (starts_at[mine + k] >= 0) starts |= 1u << k;
      if (ends_at[mine + k] >= 0) ends |= 1u << k;
    }
  }
}

// Malformed offsets of this workgroup's share of the sequences are reported; empty sequences' end states (their
// gradients, backward) are copied from `from` (zeros without it) to `to`.
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

// What a thread knows of its place: lane c of LC covers channels [ch, ch + V), its group tokens [mine, mine + K) of a
// block.
struct Place {
  int lane, wave, lc, c, mine, tokens, ch, have;   // have: channels that exist, 0 for none
};

__device__ __forceinline__ Place place_of(const GlrArgs& a) {
  Place p;
  p.lane = threadIdx.x & 63;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.lc = 1 << a.lc_log;
  p.c = p.lane & (p.lc - 1);
  p.mine = (p.lane >> a.lc_log) * K;
  p.tokens = (64 >> a.lc_log) * K;
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

__device__ __forceinline__ void put_channels(float* row, const Place& p, const float* v) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < p.have) row[p.ch + i] = v[i];
}

// x, gate (and dh) of a block's tokens; those outside [lo, hi) as tokens that keep the state (and have no gradient).
template <bool WIDE, typename T>
__device__ __forceinline__ void load_block(const GlrArgs& a, const Place& p, int64_t t0, int64_t lo, int64_t hi,
                                           Elems<T, V>* x, Elems<T, V>* g, Elems<T, V>* d) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t t = clamped(t0 + p.mine + k, lo, hi - 1);
    if (x) x[k] = row_part<WIDE, T>(a.x, a.x_stride, t, p);
    g[k] = row_part<WIDE, T>(a.gate, a.gate_stride, t, p);
    if (d) d[k] = row_part<WIDE, T>(a.dh, a.dh_stride, t, p);
  }
  if (t0 >= lo && t0 + p.tokens <= hi) return;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t t = t0 + p.mine + k;
    if (t >= lo && t < hi) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      g[k].raw[v] = (T)INFINITY;
      if (x) x[k].raw[v] = (T)0.f;
      if (d) d[k].raw[v] = (T)0.f;
    }
  }
}

// Groups' maps (A, S) to the state that enters the thread's tokens, `enter`; `state`, the one that enters the block,
// becomes the one that leaves it.  UP: groups in order of time, else against it.
template <bool UP>
__device__ __forceinline__ void join_groups(const Place& p, float* A, float* S, float* state, float* enter) {
  const bool first = UP ? p.lane < p.lc : p.lane >= 64 - p.lc;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (first) {   // from here on its map forgets what came before it
      S[v] = mul0(A[v], state[v]) + S[v];
      A[v] = 0.f;
    }
  }
  for (int d = p.lc; d < 64; d <<= 1) {
    const bool has = UP ? p.lane >= d : p.lane + d < 64;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float s0 = UP ? __shfl_up(S[v], d, 64) : __shfl_down(S[v], d, 64);
      const float a0 = UP ? __shfl_up(A[v], d, 64) : __shfl_down(A[v], d, 64);
      if (has) {
        S[v] = mul0(A[v], s0) + S[v];
        A[v] *= a0;
      }
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float s0 = UP ? __shfl_up(S[v], p.lc & 63, 64) : __shfl_down(S[v], p.lc & 63, 64);
    enter[v] = first ? state[v] : s0;
    state[v] = __shfl(S[v], UP ? 64 - p.lc + p.c : p.c, 64);
  }
}

// The maps of a thread's tokens, and their composition (A, S): a start's b takes h0 in, and its a becomes 0.
template <typename T>
__device__ __forceinline__ void compose(const GlrArgs& a, const Place& p, const Elems<T, V>* x, const Elems<T, V>* g,
                                        uint32_t starts, const int32_t* starts_at, float (*fa)[V], float (*fb)[V],
                                        float* A, float* S) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float keep;
      gate_of(g[k][v], fa[k][v], keep);
      fb[k][v] = mul0(keep, x[k][v]);
    }
    if (starts >> k & 1) {
      const float* h0 = a.h0 ? a.h0 + (int64_t)starts_at[p.mine + k] * a.dim + p.ch : nullptr;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (h0 && v < p.have) fb[k][v] = fmaf(fa[k][v], h0[v], fb[k][v]);
        fa[k][v] = 0.f;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      S[v] = k == 0 ? fb[k][v] : mul0(fa[k][v], S[v]) + fb[k][v];
      A[v] = k == 0 ? fa[k][v] : A[v] * fa[k][v];
    }
  }
}

template <bool CUT, bool WIDE, typename T>
__global__ __launch_bounds__(kThreads) void glr_forward_kernel(const GlrArgs a) {
  __shared__ int32_t marks[kWaves][2][kMaxTokens];
  const Place p = place_of(a);
  share_of_sequences(a, a.h0, a.h_last);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + p.wave;
  const Span s = span_of<CUT, true>(a, unit, p.lane);
  if (s.lo >= s.hi) return;
  int32_t *starts_at = marks[p.wave][0], *ends_at = marks[p.wave][1];
  Window w;
  w.load(a, s.seq, p.lane);
  float state[V];
#pragma unroll
  for (int v = 0; v < V; ++v) state[v] = CUT && v < p.have ? a.map_s[unit * a.dim + p.ch + v] : 0.f;
  for (int64_t block = s.lo / p.tokens; block * p.tokens < s.hi; ++block) {
    const int64_t t0 = block * p.tokens;
    Elems<T, V> x[K], g[K];
    load_block<WIDE, T>(a, p, t0, s.lo, s.hi, x, g, nullptr);
    uint32_t starts, ends;
    marks_of<true>(a, w, t0, p.tokens, s.lo, s.hi, p.lane, p.mine, starts_at, ends_at, starts, ends);
    if (a.entry && t0 >= s.lo && p.mine == 0) put_channels(a.entry + block * a.dim, p, state);
    float fa[K][V], fb[K][V], A[V], S[V], h[V];
    compose<T>(a, p, x, g, starts, starts_at, fa, fb, A, S);
    join_groups<true>(p, A, S, state, h);
    if (p.have == 0) continue;
    T* out = static_cast<T*>(a.h) + (t0 + p.mine) * a.h_stride + p.ch;
#pragma unroll
    for (int k = 0; k < K; ++k, out += a.h_stride) {
      const int64_t t = t0 + p.mine + k;
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = mul0(fa[k][v], h[v]) + fb[k][v];
      if (t >= s.lo && t < s.hi) store_elems<WIDE, T, V>(out, h, p.have);
      if ((ends >> k & 1) && a.h_last) put_channels(a.h_last + (int64_t)ends_at[p.mine + k] * a.dim, p, h);
    }
  }
}

template <bool CUT, bool WIDE, typename T>
__global__ __launch_bounds__(kThreads) void glr_backward_kernel(const GlrArgs a) {
  __shared__ int32_t marks[kWaves][2][kMaxTokens];
  const Place p = place_of(a);
  share_of_sequences(a, a.dh_last, a.dh0);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + p.wave;
  const Span s = span_of<CUT, false>(a, unit, p.lane);
  if (s.lo >= s.hi) return;
  int32_t *starts_at = marks[p.wave][0], *ends_at = marks[p.wave][1];
  Window w;
  w.load(a, s.seq - 62, p.lane);   // the span's last sequence, or one past it, is the window's last
  float grad[V];
#pragma unroll
  for (int v = 0; v < V; ++v) grad[v] = CUT && v < p.have ? a.map_s[unit * a.dim + p.ch + v] : 0.f;
  for (int64_t block = (s.hi - 1) / p.tokens; block >= s.lo / p.tokens; --block) {
    const int64_t t0 = block * p.tokens;
    Elems<T, V> x[K], g[K], d[K];
    load_block<WIDE, T>(a, p, t0, s.lo, s.hi, x, g, a.dh ? d : nullptr);
    float state[V];   // enters the block, if its sequence began before it
#pragma unroll
    for (int v = 0; v < V; ++v) state[v] = t0 >= s.lo && v < p.have ? a.entry[block * a.dim + p.ch + v] : 0.f;
    uint32_t starts, ends;
    marks_of<false>(a, w, t0, p.tokens, s.lo, s.hi, p.lane, p.mine, starts_at, ends_at, starts, ends);
    float fa[K][V], kp[K][V], hx[K][V], A[V], S[V], h[V];
    {
      float la[K][V], fb[K][V];
      compose<T>(a, p, x, g, starts, starts_at, la, fb, A, S);
      join_groups<true>(p, A, S, state, h);
      // the state before each token less its x, which dgate needs
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (starts >> k & 1) {
          const float* h0 = a.h0 ? a.h0 + (int64_t)starts_at[p.mine + k] * a.dim + p.ch : nullptr;
#pragma unroll
          for (int v = 0; v < V; ++v) h[v] = h0 && v < p.have ? h0[v] : 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          hx[k][v] = h[v] - x[k][v];
          h[v] = mul0(la[k][v], h[v]) + fb[k][v];
        }
      }
    }
    // the gradients' maps, from the last token on
    float RA[V], RS[V], de[K][V];
#pragma unroll
    for (int v = 0; v < V; ++v) RA[v] = 1.f, RS[v] = 0.f;
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        gate_of(g[k][v], fa[k][v], kp[k][v]);
        de[k][v] = a.dh ? d[k][v] : 0.f;
      }
      if (ends >> k & 1) {
        const float* last = a.dh_last ? a.dh_last + (int64_t)ends_at[p.mine + k] * a.dim + p.ch : nullptr;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (last && v < p.have) de[k][v] += last[v];
          RA[v] = RS[v] = 0.f;
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        RS[v] = fa[k][v] * (RS[v] + de[k][v]);
        RA[v] *= fa[k][v];
      }
    }
    float c[V];
    join_groups<false>(p, RA, RS, grad, c);
    if (p.have == 0) continue;
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      const int64_t t = t0 + p.mine + k;
      float dx[V], dg[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (ends >> k & 1) c[v] = 0.f;
        const float e = de[k][v] + c[v];
        c[v] = fa[k][v] * e;
        dx[v] = kp[k][v] * e;
        dg[v] = mul0(kp[k][v], hx[k][v]) * c[v];
      }
      if (t >= s.lo && t < s.hi) {
        store_elems<WIDE, T, V>(static_cast<T*>(a.dx) + t * a.dx_stride + p.ch, dx, p.have);
        store_elems<WIDE, T, V>(static_cast<T*>(a.dgate) + t * a.dgate_stride + p.ch, dg, p.have);
      }
      if ((starts >> k & 1) && a.dh0) put_channels(a.dh0 + (int64_t)starts_at[p.mine + k] * a.dim, p, c);
    }
  }
}

// Cut: the map of a range's tokens.  Only those after the last sequence start in it (backwards: before the first end)
// have a say, and none where a sequence ends (begins) with the range.
template <bool FORWARD, bool WIDE, typename T>
__global__ __launch_bounds__(kThreads) void glr_maps_kernel(const GlrArgs a) {
  __shared__ int32_t marks[kWaves][2][kMaxTokens];
  const Place p = place_of(a);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + p.wave;
  if (unit >= a.units) return;
  const int64_t lo = min(unit * a.range, a.tokens), hi = min(lo + a.range, a.tokens);
  const int64_t seq = sequence_of(a, FORWARD ? hi - 1 : lo, p.lane);
  const int64_t begin = seq < a.seqs ? offset_at(a, seq) : 0, end = seq < a.seqs ? offset_at(a, seq + 1) : hi;
  const int64_t from = FORWARD ? clamped(begin, lo, hi - 1) : lo, to = FORWARD ? hi : clamped(end, lo + 1, hi);
  float A[V], S[V], prod[V], state[V];
#pragma unroll
  for (int v = 0; v < V; ++v) prod[v] = 1.f, state[v] = 0.f;
  if (FORWARD ? end > hi : begin < lo) {   // the range's edge lies within the sequence
    int32_t *starts_at = marks[p.wave][0], *ends_at = marks[p.wave][1];
    Window w;
    w.load(a, FORWARD ? seq : seq - 62, p.lane);
    const int64_t b0 = from / p.tokens, b1 = (to - 1) / p.tokens;
    for (int64_t i = b0; i <= b1; ++i) {
      const int64_t t0 = (FORWARD ? i : b0 + b1 - i) * p.tokens;
      Elems<T, V> x[K], g[K], d[K];
      load_block<WIDE, T>(a, p, t0, from, to, FORWARD ? x : nullptr, g, !FORWARD && a.dh ? d : nullptr);
      uint32_t starts, ends;
      marks_of<FORWARD>(a, w, t0, p.tokens, from, to, p.lane, p.mine, starts_at, ends_at, starts, ends);
      float enter[V];
      if (FORWARD) {
        float fa[K][V], fb[K][V];
        compose<T>(a, p, x, g, starts, starts_at, fa, fb, A, S);
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = 1.f, S[v] = 0.f;
#pragma unroll
        for (int k = K - 1; k >= 0; --k) {
          const bool stop = ends >> k & 1;
          const float* last = stop && a.dh_last ? a.dh_last + (int64_t)ends_at[p.mine + k] * a.dim + p.ch : nullptr;
#pragma unroll
          for (int v = 0; v < V; ++v) {
            float ga, keep, e = a.dh ? d[k][v] : 0.f;
            gate_of(g[k][v], ga, keep);
            if (last && v < p.have) e += last[v];
            S[v] = ga * ((stop ? 0.f : S[v]) + e);
            A[v] = stop ? 0.f : A[v] * ga;
          }
        }
      }
      // the product over the block's groups
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float all = A[v];
        for (int dd = p.lc; dd < 64; dd <<= 1) all *= __shfl_xor(all, dd, 64);
        prod[v] *= all;
      }
      join_groups<FORWARD>(p, A, S, state, enter);
    }
  }
  if (p.mine == 0) {
    put_channels(a.map_a + unit * a.dim, p, prod);
    put_channels(a.map_s + unit * a.dim, p, state);
  }
}

// Cut: the ranges' maps to the states that enter them, in place of map_s.  A workgroup takes 16 channels; its 64 groups
// of threads take neighbouring ranges, compose them, join by LDS and walk them again.
constexpr int kScanThreadsGlr = 1024, kScanChannels = 16, kScanGroups = kScanThreadsGlr / kScanChannels;

template <bool FORWARD>
__global__ __launch_bounds__(kScanThreadsGlr) void glr_scan_kernel(const GlrArgs a) {
  __shared__ float la[kScanGroups][kScanChannels], ls[kScanGroups][kScanChannels];
  const int c = threadIdx.x % kScanChannels, g = threadIdx.x / kScanChannels;
  const int ch = (int)blockIdx.x * kScanChannels + c;
  const int64_t per = (a.units + kScanGroups - 1) / kScanGroups, begin = min(g * per, a.units), end = min(begin + per, a.units);
  const auto at = [&](int64_t i) { return (FORWARD ? i : a.units - 1 - i) * a.dim + ch; };
  // eight ranges' maps in flight
  const auto walk = [&](auto use) {
    for (int64_t i0 = begin; i0 < end; i0 += 8) {
      float ma[8], ms[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int64_t i = min(i0 + u, end - 1);
        ma[u] = a.map_a[at(i)];
        ms[u] = a.map_s[at(i)];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u < end) use(i0 + u, ma[u], ms[u]);
    }
  };
  float A = 1.f, S = 0.f, h = 0.f;
  if (ch < a.dim)
    walk([&](int64_t, float ma, float ms) {
      S = mul0(ma, S) + ms;
      A *= ma;
    });
  la[g][c] = A;
  ls[g][c] = S;
  __syncthreads();
  for (int i = 0; i < g; ++i) h = mul0(la[i][c], h) + ls[i][c];
  if (ch < a.dim)
    walk([&](int64_t i, float ma, float ms) {
      a.map_s[at(i)] = h;
      h = mul0(ma, h) + ms;
    });
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
      h[v] = fmaf(ga, s[v], mul0(keep, x[v]));
    }
    store_elems<WIDE, float, V>(state, h, have);
  } else if (ch == 0 && a.status) {
    atomicOr(a.status, DPI_DEVSTAT_BAD_ID);
  }
  store_elems<WIDE, T, V>(static_cast<T*>(a.h) + b * a.h_stride + ch, h, have);
}

template <bool WIDE, typename T>
hipError_t run_pass(const GlrArgs& a, bool backward, hipStream_t s) {
  const GlrShape sh = glr_shape(a.tokens, a.dim);
  const dim3 grid((unsigned)std::max<int64_t>(1, (a.units + kWaves - 1) / kWaves), (unsigned)sh.channel_blocks);
  if (!a.cut) {
    if (backward)
      glr_backward_kernel<false, WIDE, T><<<grid, kThreads, 0, s>>>(a);
    else
      glr_forward_kernel<false, WIDE, T><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  const dim3 scan((unsigned)((a.dim + kScanChannels - 1) / kScanChannels));
  if (backward) {
    glr_maps_kernel<false, WIDE, T><<<grid, kThreads, 0, s>>>(a);
    glr_scan_kernel<false><<<scan, kScanThreadsGlr, 0, s>>>(a);
    glr_backward_kernel<true, WIDE, T><<<grid, kThreads, 0, s>>>(a);
  } else {
    glr_maps_kernel<true, WIDE, T><<<grid, kThreads, 0, s>>>(a);
    glr_scan_kernel<true><<<scan, kScanThreadsGlr, 0, s>>>(a);
    glr_forward_kernel<true, WIDE, T><<<grid, kThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t run_wide(const GlrArgs& a, bool backward, hipStream_t s) {
  return a.wide ? run_pass<true, T>(a, backward, s) : run_pass<false, T>(a, backward, s);
}

hipError_t run_by_dtype(const GlrArgs& a, bool backward, hipStream_t s) {
  if (a.seqs == 0) return hipSuccess;
  if (a.dtype == DPI_F32) return run_wide<float>(a, backward, s);
  if (a.dtype == DPI_F16) return run_wide<f16_t>(a, backward, s);
  return run_wide<bf16_t>(a, backward, s);
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

// Lanes of a power of two cover up to 64 * V channels; a wave's other lanes take later tokens.
GlrShape glr_shape(int64_t tokens, int32_t dim) {
  GlrShape sh{};
  while (sh.lc_log < 6 && (V << sh.lc_log) < dim) ++sh.lc_log;
  sh.block_tokens = (int64_t)(64 >> sh.lc_log) * K;
  sh.blocks = (tokens + sh.block_tokens - 1) / sh.block_tokens;
  sh.channel_blocks = (dim + (V << sh.lc_log) - 1) / (V << sh.lc_log);
  return sh;
}

GlrSplit glr_split(int64_t tokens, int32_t dim, int64_t max_len) {
  const GlrShape sh = glr_shape(tokens, dim);
  GlrSplit sp{};
  const int64_t longest = max_len > 0 ? std::min(max_len, tokens) : tokens;
  sp.cut = longest > kGlrWholeBlocks * sh.block_tokens;
  const int64_t waves = kGlrWaves / sh.channel_blocks + 1;
  const int64_t blocks = std::min<int64_t>(std::max<int64_t>(1, (sh.blocks + waves - 1) / waves), kGlrRangeBlocks);
  sp.range = blocks * sh.block_tokens;
  sp.units = (tokens + sp.range - 1) / sp.range;
  return sp;
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
