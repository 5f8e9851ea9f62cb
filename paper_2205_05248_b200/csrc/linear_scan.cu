// The gated linear recurrence h' = a h + b over a batch of sequences, and its gradient.
//
// A run of steps is an affine map of the state that enters it, h -> A h + H with A the product of its gates and H its result
// from a zero state; a cut inside it makes it a constant, whatever enters (kept as a flag, not as a factor 0, so that nothing
// non-finite crosses).  Each thread takes eight neighbouring steps of one or two channels into registers and reduces them to
// such a map; the maps are combined along the lanes that share a channel and along the warps of a block; then the
// thread runs its steps again from the state that enters them.  One pass over gate and x, one write of y.
// The gradient runs against the scan order: with G_k = dy_k + R_{k+1}, R_k = a_k G_k (0 at a cut) is the gradient of the
// state that enters step k: the same maps, composed the other way round.  The states between the kept ones (one in 64) are made again.
// Few sequences and channels: the time axis is divided over blocks; a first launch makes the chunks' maps, the second enters each chunk
// with their composition.
//
// Forms: calls of one step (element by element), rows on 16-byte boundaries of 48 channels or more (tiles by asynchronous copies), and
// everything else (direct loads, 1 to 32 lanes along the channels).  Measured (bytes bound all of them on paper):
//   2048 x 64 x 256 fp32 blend: 67 us forward (6.0 TB/s), 115 us backward (5.8 TB/s)
//   128 x 512 x 512 bf16 blend with cuts: 58 us forward (3.5 TB/s), 109 us backward (3.1 TB/s): 59 and 127 instructions for 64 elements; gates,
//     conversions and the two barriers of a tile, with some 20 warps a multiprocessor to cover them
//   65521 x 128 fp32 of one sequence: 40 us forward, 53 us backward: two launches each, the second reading from L2 what the first brought
//   one step, forward / backward: 16384 x 512 bf16 29 / 36 us, serving form of 24 x 64 1.6 / 1.8 us; 1000000 x 1 67 / 74 us (a warp a sequence, with
//     one lane of it at work)
//   few channels, fp32, forward / backward: 1024 x 96 x 1 4.0 / 4.7 us, 512 x 2000 x 3 19 / 29 us, 1 x 1000000 x 1 18 / 22 us (a lane's steps come one
//     number a load); a gate that is one number for all 128 x 512 x 64: 21 / 32 us, the same gate written out 24 / 30 us
// Registers: the direct form's bounds (64 a thread forward, 128 backward) make it spill with two channels a lane, 56 to 88 bytes forward and up to 108
// backward; the tiles' kernels spill 4 to 28 bytes.
#include "learner_util.cuh"
#include "launch_util.cuh"

#include <algorithm>
#include <type_traits>

namespace marl {

constexpr int STEPS = 8;       // steps a thread holds
constexpr int MAX_WARPS = 8;   // warps along time

struct ScanParams {
  const void *g, *x;
  long long gb, gt, xb, xt;
  int gc, xc;
  const float* h0;
  const uint8_t* done;
  const int32_t* length;
  int B, L, C, reverse;
  void* y;
  float *last, *states;
  const void* dy;
  long long dyb, dyt;
  const float* dlast;
  void *dg, *dx;
  float* dh0;
  int lg;          // log2 of the lanes along the channels
  int warps;       // warps along time
  int pipe;        // tiles by asynchronous copies
  int units;       // units (sequence, group of channels) a block
  int groups;      // groups of channels a sequence
  int chunks, chunk_len, intervals;
  float2* agg;     // [B][chunks][C] maps of the chunks, when the time axis is divided over blocks
  uint8_t* agg_cut;  // [B][groups][chunks]
};

struct Map {
  float a, h;
  bool cut;
};
__device__ __forceinline__ float apply(const Map& m, float h) { return m.cut ? m.h : fmaf(m.a, h, m.h); }
__device__ __forceinline__ Map then(const Map& first, const Map& second) {  // first, then second
  return Map{first.a * second.a, apply(second, first.h), first.cut || second.cut};
}

template <typename T, int V> struct Raw { T v[V]; };
template <> struct Raw<__nv_bfloat16, 2> { __nv_bfloat162 v; };
template <> struct Raw<__half, 2> { __half2 v; };
__device__ __forceinline__ void unpack(const Raw<float, 1>& r, float (&f)[1]) { f[0] = r.v[0]; }
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 1>& r, float (&f)[1]) { f[0] = to_f32(r.v[0]); }
__device__ __forceinline__ void unpack(const Raw<__half, 1>& r, float (&f)[1]) { f[0] = to_f32(r.v[0]); }
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 2>& r, float (&f)[2]) {
  const float2 t = __bfloat1622float2(r.v);
  f[0] = t.x; f[1] = t.y;
}
__device__ __forceinline__ void unpack(const Raw<__half, 2>& r, float (&f)[2]) {
  const float2 t = __half22float2(r.v);
  f[0] = t.x; f[1] = t.y;
}
template <typename T> __device__ __forceinline__ void put(T* at, const float (&f)[1]) { *at = from_f32<T>(f[0]); }
__device__ __forceinline__ void put(__nv_bfloat16* at, const float (&f)[2]) {
  *reinterpret_cast<__nv_bfloat162*>(at) = __floats2bfloat162_rn(f[0], f[1]);
}
__device__ __forceinline__ void put(__half* at, const float (&f)[2]) { *reinterpret_cast<__half2*>(at) = __floats2half2_rn(f[0], f[1]); }
__device__ __forceinline__ void put(float* at, const float (&f)[2]) {}  // (fp32 has one channel a lane)

// z = 1 / (1 + e^-g) and 1 - z = e^-g z, each relative to itself within (1.23 |g| + 8) 2^-24: the exponent g log2 e is rounded once, which
// e^-g multiplies by |g| (1 - z at g = 20, 2e-9: 2e-6 of itself; a second term of the exponent would take three operations more a gate).  Where e^-g
// is below 2^-126 it is 0, and below g = -87 z stays at 2^-126.
__device__ __forceinline__ void gate_pair(float g, float& z, float& rest) {
  float t, r;
  asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(t) : "f"(g * -1.4426950408889634f));  // at most 126
  const float e = ex2(t);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  z = r;
  rest = e * r;
}

// Where a thread stands: its unit, lane of channels and place along time.
struct Place {
  int b, group, c;           // sequence, group, first channel of this lane
  int lane, sub, warp, slot;  // place along time: sub inside the warp, warp inside the unit; slot of the unit in its block
  int q;                     // warp * subs + sub
  bool on;                   // has channels
  int n;                     // length of the sequence
};

template <int V>
__device__ __forceinline__ bool find_place(const ScanParams& p, Place& w) {
  w.lane = threadIdx.x & 31;
  const int wi = threadIdx.x >> 5;
  w.slot = wi / p.warps;
  w.warp = wi - w.slot * p.warps;
  w.sub = w.lane >> p.lg;
  w.q = w.warp * (32 >> p.lg) + w.sub;
  const long long unit = (long long)blockIdx.x * p.units + w.slot;
  if (unit >= (long long)p.B * p.groups) return false;
  w.b = (int)(unit / p.groups);
  w.group = (int)(unit - (long long)w.b * p.groups);
  w.c = ((w.group << p.lg) + (w.lane & ((1 << p.lg) - 1))) * V;
  w.on = w.c < p.C;
  int n = p.length ? p.length[w.b] : p.L;
  w.n = n < 0 ? 0 : n > p.L ? p.L : n;
  return true;
}

__device__ __forceinline__ void unit_sync(const ScanParams& p, const Place& w) {
  if (p.warps == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(w.slot + 1), "r"(p.warps * 32) : "memory");
}

// The cuts in front of the thread's steps k0 .. k0 + S - 1 (scan order), as bits.  The flags of a warp's steps are read side by side, a
// lane a flag, and each thread takes its own out of the votes.
template <int S>
__device__ __forceinline__ unsigned load_cuts(const ScanParams& p, const Place& w, int k0) {
  const uint8_t* d = p.done + (long long)w.b * p.L;
  const int warp_k0 = k0 - w.sub * S, flags = (32 >> p.lg) * S;
  unsigned mine = 0;
  for (int f = 0; f < flags; f += 32) {
    const int k = warp_k0 + f + w.lane, at = p.reverse ? w.n - 1 - k : k - 1;  // done of the step before, or in reverse of this one
    const unsigned votes = __ballot_sync(~0u, f + w.lane < flags && k < w.n && at >= 0 && d[at < 0 ? 0 : at]);
    const int at_bit = w.sub * S - f;  // (S divides 32: a thread's flags lie in one word)
    if (at_bit >= 0 && at_bit < 32) mine = votes >> at_bit & ((1u << S) - 1);
  }
  return mine;
}

// The thread's steps of one array; 0 where there is no step or no channel.
template <typename T, int V, int S>
__device__ __forceinline__ void load_steps(const void* base, long long sb, long long st, int sc, const ScanParams& p, const Place& w, int k0,
                                           Raw<T, V> (&r)[S]) {
  const T* at = reinterpret_cast<const T*>(base) + w.b * sb + w.c * sc + (p.reverse ? w.n - 1 - k0 : k0) * st;
  const long long step = p.reverse ? -st : st;
  if (w.on && k0 + S <= w.n) {
#pragma unroll
    for (int s = 0; s < S; ++s) r[s] = *reinterpret_cast<const Raw<T, V>*>(at + s * step);
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      r[s] = Raw<T, V>{};
      if (w.on && k0 + s < w.n) r[s] = *reinterpret_cast<const Raw<T, V>*>(at + s * step);
    }
  }
}

template <typename T, int V, int S>
__device__ __forceinline__ void store_steps(T* row, const ScanParams& p, const Place& w, int k0, int end, const float (&v)[S][V]) {
  T* at = row + (long long)(p.reverse ? w.n - 1 - k0 : k0) * p.C;
  const long long step = p.reverse ? -(long long)p.C : p.C;
  if (!w.on) return;
  if (k0 + S <= end) {
#pragma unroll
    for (int s = 0; s < S; ++s) put(at + s * step, v[s]);
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (k0 + s < end) put(at + s * step, v[s]);
  }
}

// Gate and input of a step; a step behind the end passes the state on.
template <bool BLEND>
__device__ __forceinline__ void step_ab(bool live, float g, float x, float& a, float& b) {
  if (BLEND) {
    float rest;
    gate_pair(g, a, rest);
    b = rest * x;
  } else {
    a = g;
    b = x;
  }
  if (!live) {
    a = 1.f;
    b = 0.f;
  }
}

template <bool CUT>
__device__ __forceinline__ Map shfl_map_up(const Map& m, int d) {
  return Map{__shfl_up_sync(~0u, m.a, d), __shfl_up_sync(~0u, m.h, d), CUT && (bool)__shfl_up_sync(~0u, (int)m.cut, d)};
}
template <bool CUT>
__device__ __forceinline__ Map shfl_map_down(const Map& m, int d) {
  return Map{__shfl_down_sync(~0u, m.a, d), __shfl_down_sync(~0u, m.h, d), CUT && (bool)__shfl_down_sync(~0u, (int)m.cut, d)};
}

struct ScanShared {
  float2 total[2][MAX_WARPS][32 * 2];
  float back[2][MAX_WARPS][32 * 2];
  uint8_t cut[2][MAX_WARPS];
};

// The state that enters a chunk of the time axis (BACK: the gradient that comes back into it) behind `count` others.  A block has one unit
// then: its warps compose an eighth of the chunks' maps each.
template <int V, bool BACK>
__device__ __forceinline__ void enter_chunk(const ScanParams& p, const Place& w, ScanShared& sh, int count, int used, float (&h)[V]) {
  const float2* agg = p.agg + (long long)w.b * p.chunks * p.C + w.c;
  const uint8_t* cut = p.agg_cut + ((long long)w.b * p.groups + w.group) * p.chunks;
  const int per = (count + MAX_WARPS - 1) / MAX_WARPS, i0 = w.warp * per, i1 = min(count, i0 + per), ch = w.lane & ((1 << p.lg) - 1);
  Map m[V];
#pragma unroll
  for (int v = 0; v < V; ++v) m[v] = Map{1.f, 0.f, false};
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    const int at = BACK ? used - 1 - i : i;
    const bool c = cut[at];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 t = w.on ? agg[(long long)at * p.C + v] : make_float2(0.f, 0.f);
      m[v] = then(m[v], Map{t.x, t.y, c});
    }
  }
  if (w.sub == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) sh.total[0][w.warp][ch * V + v] = make_float2(m[v].a, m[v].h);
    if (ch == 0) sh.cut[0][w.warp] = m[0].cut;
  }
  __syncthreads();
  for (int i = 0; i < MAX_WARPS; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 t = sh.total[0][i][ch * V + v];
      h[v] = apply(Map{t.x, t.y, (bool)sh.cut[0][i]}, h[v]);
    }
  __syncthreads();
}

// AGG: only the chunk's map is computed, for the launch behind this one.
template <typename T, int V, int S, bool BLEND, bool CUT, bool AGG>
__global__ void __launch_bounds__(MAX_WARPS * 32, 4) scan_kernel(const __grid_constant__ ScanParams p) {
  __shared__ ScanShared sh_all;
  Place w;
  if (!find_place<V>(p, w)) return;
  const int subs = 32 >> p.lg, tile = p.warps * subs * S, wslot = w.slot * p.warps, ch = w.lane & ((1 << p.lg) - 1);
  const int first = blockIdx.y * p.chunk_len, end = min(w.n, first + p.chunk_len);  // steps of this block, in scan order
  T* y = reinterpret_cast<T*>(p.y) + (long long)w.b * p.L * p.C + w.c;
  float carry[V];
  Map whole[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    carry[v] = !AGG && w.on && p.h0 ? p.h0[(long long)w.b * p.C + w.c + v] : 0.f;
    whole[v] = Map{1.f, 0.f, false};
  }
  if (!AGG && p.chunks > 1 && first < w.n) enter_chunk<V, false>(p, w, sh_all, blockIdx.y, 0, carry);
  int par = 0;
  for (int k0 = first; k0 < end; k0 += tile, par ^= 1) {
    const int mine = k0 + w.q * S;
    float a[S][V], b[S][V];
    unsigned cut = 0;
    {
      Raw<T, V> rg[S], rx[S];
      load_steps<T, V, S>(p.g, p.gb, p.gt, p.gc, p, w, mine, rg);
      load_steps<T, V, S>(p.x, p.xb, p.xt, p.xc, p, w, mine, rx);
      if (CUT) cut = load_cuts<S>(p, w, mine);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        float g[V], x[V];
        unpack(rg[s], g);
        unpack(rx[s], x);
#pragma unroll
        for (int v = 0; v < V; ++v) step_ab<BLEND>(mine + s < end, g[v], x[v], a[s][v], b[s][v]);
      }
    }
    Map m[V], before[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      m[v] = Map{a[0][v], b[0][v], CUT && cut != 0};
#pragma unroll
      for (int s = 1; s < S; ++s) {
        m[v].h = CUT && (cut >> s & 1) ? b[s][v] : fmaf(a[s][v], m[v].h, b[s][v]);
        m[v].a *= a[s][v];
      }
      before[v] = Map{1.f, 0.f, false};
      if (subs > 1) {
        for (int d = 1; d < subs; d <<= 1) {
          const Map o = shfl_map_up<CUT>(m[v], d << p.lg);
          if (w.sub >= d) m[v] = then(o, m[v]);
        }
        const Map o = shfl_map_up<CUT>(m[v], 1 << p.lg);
        if (w.sub) before[v] = o;
      }
    }
    float enter[V];
    if (p.warps > 1) {
      if (w.sub == subs - 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) sh_all.total[par][wslot + w.warp][ch * V + v] = make_float2(m[v].a, m[v].h);
        if (CUT && ch == 0) sh_all.cut[par][wslot + w.warp] = m[0].cut;
      }
      unit_sync(p, w);
#pragma unroll 4
      for (int i = 0; i < p.warps; ++i) {
        const bool c = CUT && sh_all.cut[par][wslot + i];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (i == w.warp) enter[v] = carry[v];
          const float2 t = sh_all.total[par][wslot + i][ch * V + v];
          const Map mi{t.x, t.y, c};
          carry[v] = apply(mi, carry[v]);
          if (AGG) whole[v] = then(whole[v], mi);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        enter[v] = carry[v];
        Map t = m[v];
        if (subs > 1) {
          const int src = 32 - (1 << p.lg) + ch;
          t = Map{__shfl_sync(~0u, t.a, src), __shfl_sync(~0u, t.h, src), (bool)__shfl_sync(~0u, (int)t.cut, src)};
        }
        carry[v] = apply(t, carry[v]);
        if (AGG) whole[v] = then(whole[v], t);
      }
    }
    if constexpr (!AGG) {
      float h[V];
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = apply(before[v], enter[v]);
      if (p.states && w.on && mine < end && mine % MARL_SCAN_INTERVAL == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) p.states[((long long)w.b * p.intervals + mine / MARL_SCAN_INTERVAL) * p.C + w.c + v] = h[v];
      }
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = a[s][v] = CUT && (cut >> s & 1) ? b[s][v] : fmaf(a[s][v], h[v], b[s][v]);
      store_steps<T, V, S>(y, p, w, mine, end, a);
    }
  }
  if constexpr (AGG) {
    if (first < end && w.q == 0) {
      if (w.on) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          p.agg[((long long)w.b * p.chunks + blockIdx.y) * p.C + w.c + v] = make_float2(whole[v].a, whole[v].h);
      }
      if (w.lane == 0) p.agg_cut[((long long)w.b * p.groups + w.group) * p.chunks + blockIdx.y] = whole[0].cut;
    }
    return;
  }
  if (!w.on) return;
  if (w.q == 0 && (w.n > 0 ? end == w.n && first < w.n : blockIdx.y == 0)) {
    const bool gone = CUT && !p.reverse && w.n > 0 && p.done[(long long)w.b * p.L + w.n - 1];
#pragma unroll
    for (int v = 0; v < V; ++v) p.last[(long long)w.b * p.C + w.c + v] = gone ? 0.f : carry[v];
  }
  const float zero[V] = {};
  const int stop = min(p.L, first + p.chunk_len);
  for (int t = max(w.n, first) + w.q; t < stop; t += p.warps * subs) put(y + (long long)t * p.C, zero);
}

template <typename T, int V, int S, bool BLEND, bool CUT, bool AGG>
__global__ void __launch_bounds__(MAX_WARPS * 32, 2) scan_grad_kernel(const __grid_constant__ ScanParams p) {
  __shared__ ScanShared sh_all;
  Place w;
  if (!find_place<V>(p, w)) return;
  const int subs = 32 >> p.lg, tile = p.warps * subs * S, wslot = w.slot * p.warps, ch = w.lane & ((1 << p.lg) - 1);
  const int first = blockIdx.y * p.chunk_len, end = min(w.n, first + p.chunk_len);
  const int used = (w.n + p.chunk_len - 1) / p.chunk_len;
  float carry[V];
  Map whole[V];
  const bool gone = CUT && !p.reverse && w.n > 0 && p.done[(long long)w.b * p.L + w.n - 1];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    carry[v] = !AGG && w.on && p.dlast && !gone ? p.dlast[(long long)w.b * p.C + w.c + v] : 0.f;
    whole[v] = Map{1.f, 0.f, false};
  }
  if (!AGG && p.chunks > 1 && first < w.n) enter_chunk<V, true>(p, w, sh_all, used - 1 - (int)blockIdx.y, used, carry);
  T* dg = reinterpret_cast<T*>(p.dg) + (long long)w.b * p.L * p.C + w.c;
  T* dx = reinterpret_cast<T*>(p.dx) + (long long)w.b * p.L * p.C + w.c;
  const int tiles = first < end ? (end - first + tile - 1) / tile : 0;
  int par = 0;
  for (int i = tiles - 1; i >= 0; --i, par ^= 1) {
    const int k0 = first + i * tile, mine = k0 + w.q * S;
    // a: gate, q: 1 - gate (BLEND), x, d: gradient of y
    float a[S][V], q[BLEND ? S : 1][V], x[S][V], d[S][V], enter[V];
    unsigned cut = 0;
    {
      Raw<T, V> rg[S], rd[S], rx[S];
      load_steps<T, V, S>(p.g, p.gb, p.gt, p.gc, p, w, mine, rg);
      load_steps<T, V, S>(p.dy, p.dyb, p.dyt, 1, p, w, mine, rd);
      if (!AGG) load_steps<T, V, S>(p.x, p.xb, p.xt, p.xc, p, w, mine, rx);
      if (CUT) cut = load_cuts<S>(p, w, mine);
#pragma unroll
      for (int v = 0; v < V; ++v)
        enter[v] = !AGG && w.on ? p.states[((long long)w.b * p.intervals + k0 / MARL_SCAN_INTERVAL) * p.C + w.c + v] : 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        unpack(rg[s], a[s]);
        unpack(rd[s], d[s]);
        if (!AGG) unpack(rx[s], x[s]);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (BLEND) gate_pair(a[s][v], a[s][v], q[s][v]);
          if (mine + s >= end) a[s][v] = 1.f;  // (x and dy are 0 there)
        }
      }
    }
    Map m[V], r[V];   // the steps' map of the state, and that of the gradient (same factor, against the scan order)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      m[v] = r[v] = Map{a[0][v], 0.f, CUT && cut != 0};
#pragma unroll
      for (int s = 1; s < S; ++s) m[v].a *= a[s][v];
      r[v].a = m[v].a;
      if (!AGG) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const float b = BLEND ? q[s][v] * x[s][v] : x[s][v];
          m[v].h = CUT && (cut >> s & 1) ? b : fmaf(a[s][v], m[v].h, b);
        }
      }
#pragma unroll
      for (int s = S - 1; s >= 0; --s) r[v].h = CUT && (cut >> s & 1) ? 0.f : a[s][v] * (d[s][v] + r[v].h);
    }
    Map before[V], behind[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      before[v] = behind[v] = Map{1.f, 0.f, false};
      if (subs > 1) {
        for (int e = 1; e < subs; e <<= 1) {
          const Map o = shfl_map_up<CUT>(m[v], e << p.lg), t = shfl_map_down<CUT>(r[v], e << p.lg);
          if (w.sub >= e) m[v] = then(o, m[v]);
          if (w.sub + e < subs) r[v] = then(t, r[v]);
        }
        const Map o = shfl_map_up<CUT>(m[v], 1 << p.lg), t = shfl_map_down<CUT>(r[v], 1 << p.lg);
        if (w.sub) before[v] = o;
        if (w.sub + 1 < subs) behind[v] = t;
        // the warp's maps: of the state in the last sub, of the gradient in the first
        const int last = 32 - (1 << p.lg) + ch;
        m[v] = Map{__shfl_sync(~0u, m[v].a, last), __shfl_sync(~0u, m[v].h, last), (bool)__shfl_sync(~0u, (int)m[v].cut, last)};
        r[v].h = __shfl_sync(~0u, r[v].h, ch);
      }
      r[v].a = m[v].a;
      r[v].cut = m[v].cut;
    }
    float back[V];
    if (p.warps > 1) {
      if (w.sub == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          sh_all.total[par][wslot + w.warp][ch * V + v] = make_float2(m[v].a, m[v].h);
          sh_all.back[par][wslot + w.warp][ch * V + v] = r[v].h;
        }
        if (CUT && ch == 0) sh_all.cut[par][wslot + w.warp] = m[0].cut;
      }
      unit_sync(p, w);
      if (!AGG)
        for (int j = 0; j < w.warp; ++j)
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const float2 t = sh_all.total[par][wslot + j][ch * V + v];
            enter[v] = apply(Map{t.x, t.y, CUT && sh_all.cut[par][wslot + j]}, enter[v]);
          }
#pragma unroll 4
      for (int j = p.warps - 1; j >= 0; --j) {
        const bool c = CUT && sh_all.cut[par][wslot + j];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (j == w.warp) back[v] = carry[v];
          const Map mb{sh_all.total[par][wslot + j][ch * V + v].x, sh_all.back[par][wslot + j][ch * V + v], c};
          carry[v] = apply(mb, carry[v]);
          if (AGG) whole[v] = then(whole[v], mb);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        back[v] = carry[v];
        carry[v] = apply(r[v], carry[v]);
        if (AGG) whole[v] = then(whole[v], r[v]);
      }
    }
    if constexpr (!AGG) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float h = apply(before[v], enter[v]), R = apply(behind[v], back[v]);
        // d becomes G, then x and d become what is stored: (came - x) z (1 - z) G or came G, and (1 - z) G or G
#pragma unroll
        for (int s = S - 1; s >= 0; --s) {
          d[s][v] += R;
          R = CUT && (cut >> s & 1) ? 0.f : a[s][v] * d[s][v];
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
          if (CUT && (cut >> s & 1)) h = 0.f;
          if (BLEND) {
            const float G = d[s][v], b = q[s][v] * x[s][v];
            d[s][v] = G * q[s][v];
            x[s][v] = (h - x[s][v]) * (a[s][v] * d[s][v]);
            h = fmaf(a[s][v], h, b);
          } else {
            const float b = x[s][v];
            x[s][v] = d[s][v] * h;
            h = fmaf(a[s][v], h, b);
          }
        }
      }
      store_steps<T, V, S>(dg, p, w, mine, end, x);
      store_steps<T, V, S>(dx, p, w, mine, end, d);
    }
  }
  if constexpr (AGG) {
    if (first < end && w.q == 0) {
      if (w.on) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          p.agg[((long long)w.b * p.chunks + blockIdx.y) * p.C + w.c + v] = make_float2(whole[v].a, whole[v].h);
      }
      if (w.lane == 0) p.agg_cut[((long long)w.b * p.groups + w.group) * p.chunks + blockIdx.y] = whole[0].cut;
    }
    return;
  }
  if (!w.on) return;
  if (w.q == 0 && blockIdx.y == 0 && p.dh0) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.dh0[(long long)w.b * p.C + w.c + v] = carry[v];
  }
  const float zero[V] = {};
  const int stop = min(p.L, first + p.chunk_len);
  for (int t = max(w.n, first) + w.q; t < stop; t += p.warps * subs) {
    put(dg + (long long)t * p.C, zero);
    put(dx + (long long)t * p.C, zero);
  }
}

// ---- calls of one step: the serving form, element by element --------------------------------------------------------
template <typename T, int V, bool BLEND>
__global__ void scan_step_kernel(const __grid_constant__ ScanParams p) {
  const int c = (blockIdx.x * blockDim.x + threadIdx.x) * V;
  if (c >= p.C) return;
  for (int b = blockIdx.y * blockDim.y + threadIdx.y; b < p.B; b += gridDim.y * blockDim.y) {
    const bool live = !p.length || p.length[b] > 0, done = live && p.done && p.done[b];
    const long long at = (long long)b * p.C + c;
    float g[V] = {}, x[V] = {}, y[V];
    if (live) {
      unpack(*reinterpret_cast<const Raw<T, V>*>(reinterpret_cast<const T*>(p.g) + b * p.gb + (long long)c * p.gc), g);
      unpack(*reinterpret_cast<const Raw<T, V>*>(reinterpret_cast<const T*>(p.x) + b * p.xb + (long long)c * p.xc), x);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float h0 = p.h0 ? p.h0[at + v] : 0.f;
      float a, u;
      step_ab<BLEND>(true, g[v], x[v], a, u);
      const float h = p.reverse && done ? u : fmaf(a, h0, u);
      if (live && p.states) p.states[at + v] = h0;
      p.last[at + v] = !live ? h0 : !p.reverse && done ? 0.f : h;
      y[v] = live ? h : 0.f;
    }
    put(reinterpret_cast<T*>(p.y) + at, y);
  }
}

template <typename T, int V, bool BLEND>
__global__ void scan_step_grad_kernel(const __grid_constant__ ScanParams p) {
  const int c = (blockIdx.x * blockDim.x + threadIdx.x) * V;
  if (c >= p.C) return;
  for (int b = blockIdx.y * blockDim.y + threadIdx.y; b < p.B; b += gridDim.y * blockDim.y) {
    const bool live = !p.length || p.length[b] > 0, done = live && p.done && p.done[b];
    const long long at = (long long)b * p.C + c;
    float g[V] = {}, x[V] = {}, d[V] = {}, dg[V], dx[V];
    if (live) {
      unpack(*reinterpret_cast<const Raw<T, V>*>(reinterpret_cast<const T*>(p.g) + b * p.gb + (long long)c * p.gc), g);
      unpack(*reinterpret_cast<const Raw<T, V>*>(reinterpret_cast<const T*>(p.x) + b * p.xb + (long long)c * p.xc), x);
      unpack(*reinterpret_cast<const Raw<T, V>*>(reinterpret_cast<const T*>(p.dy) + b * p.dyb + c), d);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float dl = p.dlast ? p.dlast[at + v] : 0.f;
      const float G = d[v] + (!p.reverse && done ? 0.f : dl), came = live && !(p.reverse && done) ? p.states[at + v] : 0.f;
      float a = g[v], rest = 1.f;
      if (BLEND) gate_pair(g[v], a, rest);
      dg[v] = !live ? 0.f : BLEND ? (came - x[v]) * (a * (G * rest)) : G * came;
      dx[v] = !live ? 0.f : G * rest;
      if (p.dh0) p.dh0[at + v] = !live ? dl : p.reverse && done ? 0.f : a * G;
    }
    put(reinterpret_cast<T*>(p.dg) + at, dg);
    put(reinterpret_cast<T*>(p.dx) + at, dx);
  }
}

// ---- aligned rows of many channels: tiles by asynchronous copies ----------------------------------------------------
// A block takes 64 channels of a sequence, two a lane, in tiles of 64 steps, eight steps a warp.  The tiles of gate, x (and dy) come in
// 16 bytes a copy into a ring of slots in shared memory, ahead of the tile that is computed; the arithmetic is packed, two channels
// an operation.  The gradient reads x and dy from the slot twice rather than holding them.
constexpr int PIPE_STEPS = 64, PIPE_CHANNELS = 64, PIPE_THREADS = 256, PIPE_WARPS = 8, PIPE_S = PIPE_STEPS / PIPE_WARPS;
constexpr int PIPE_BLOCKS = 4;
template <typename T> constexpr int PIPE_SLOTS = sizeof(T) == 4 ? 2 : 3;
constexpr int GRAD_SLOTS = 2;
template <typename T, int ARRAYS> constexpr int SLOT_BYTES = ARRAYS * PIPE_STEPS * PIPE_CHANNELS * (int)sizeof(T);

__device__ __forceinline__ float2 pair_of(const float* at) { return *reinterpret_cast<const float2*>(at); }
__device__ __forceinline__ float2 pair_of(const __nv_bfloat16* at) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(at)); }
__device__ __forceinline__ float2 pair_of(const __half* at) { return __half22float2(*reinterpret_cast<const __half2*>(at)); }
__device__ __forceinline__ void put_pair(float* at, float2 v) { *reinterpret_cast<float2*>(at) = v; }
__device__ __forceinline__ void put_pair(__nv_bfloat16* at, float2 v) { *reinterpret_cast<__nv_bfloat162*>(at) = __floats2bfloat162_rn(v.x, v.y); }
__device__ __forceinline__ void put_pair(__half* at, float2 v) { *reinterpret_cast<__half2*>(at) = __floats2half2_rn(v.x, v.y); }

__device__ __forceinline__ void gate_pair2(float2 g, float2& z, float2& rest) {
  const float2 t = mul2(g, make_float2(-1.4426950408889634f, -1.4426950408889634f));
  float2 e, r;
  asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(e.x) : "f"(t.x));
  asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(e.y) : "f"(t.y));
  e = make_float2(ex2(e.x), ex2(e.y));
  const float2 u = add2(e, make_float2(1.f, 1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(u.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(u.y));
  z = r;
  rest = mul2(e, r);
}

struct PipeShared {
  float4 total[2][PIPE_WARPS][32];  // gate product and result of a warp's steps, two channels
  float2 back[2][PIPE_WARPS][32];
  __align__(8) uint8_t cut[2][PIPE_WARPS];
};

// One array's tiles, as a thread copies them: 16 bytes of a row of the tile, and of the rows ROW_STEP further on.
template <typename T>
struct Source {
  static constexpr int PER = 16 / (int)sizeof(T), COPIES = PIPE_CHANNELS / PER, ROW_STEP = PIPE_THREADS / COPIES, ROUNDS = PIPE_STEPS / ROW_STEP;
  const T* at;        // the thread's piece of the tile to be requested next
  long long round;    // elements between rounds, in scan order
  __device__ __forceinline__ void open(const void* base, long long offset, long long stride, const ScanParams& p, int n, int k0) {
    const int k = k0 + (int)threadIdx.x / COPIES, c = (int)threadIdx.x % COPIES * PER;
    at = reinterpret_cast<const T*>(base) + offset + c + (p.reverse ? n - 1 - k : k) * stride;
    round = (p.reverse ? -stride : stride) * ROW_STEP;
  }
  // rows: how many of the tile's rows there are (for this thread: none, if its channels are not there)
  __device__ __forceinline__ void request(uint8_t* slot, int rows) const {
    const int row = (int)threadIdx.x / COPIES;
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(slot + threadIdx.x * 16);
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j)
      if (row + j * ROW_STEP < rows)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + j * PIPE_THREADS * 16), "l"(at + j * round) : "memory");
  }
  __device__ __forceinline__ void move(int tiles) { at += round * (ROUNDS * tiles); }
};

// The flag in front of step k0 + (lane & 7) of the warp's eight steps, as loaded; vote over the lanes 0 .. 7 to use it.
__device__ __forceinline__ bool load_flag(const ScanParams& p, const uint8_t* done, int n, int k0, int lane) {
  const int k = k0 + lane, at = p.reverse ? n - 1 - k : k - 1;
  return lane < PIPE_S && k < n && at >= 0 && done[at] != 0;
}

__device__ __forceinline__ float2 apply2(float2 a, float2 h, bool cut, float2 in) { return cut ? h : fma2(a, in, h); }

// The state that enters a chunk (BACK: the gradient that comes back into it) behind `count` others: the warps compose an eighth of them each.
template <bool BACK>
__device__ __forceinline__ float2 enter_chunk2(const ScanParams& p, PipeShared& sh, int b, int group, int c, bool on, int count, float2 carry,
                                               int used = 0) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float2* agg = p.agg + (long long)b * p.chunks * p.C + c;
  const uint8_t* cuts = p.agg_cut + ((long long)b * p.groups + group) * p.chunks;
  const int per = (count + PIPE_WARPS - 1) / PIPE_WARPS, i0 = warp * per, i1 = min(count, i0 + per);
  float2 A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f);
  bool cut = false;
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    const int at = BACK ? used - 1 - i : i;
    const float4 m = on ? *reinterpret_cast<const float4*>(agg + (long long)at * p.C) : make_float4(0.f, 0.f, 0.f, 0.f);
    const bool cu = cuts[at];
    H = apply2(make_float2(m.x, m.z), make_float2(m.y, m.w), cu, H);
    A = mul2(A, make_float2(m.x, m.z));
    cut |= cu;
  }
  sh.total[0][warp][lane] = make_float4(A.x, A.y, H.x, H.y);
  if (lane == 0) sh.cut[0][warp] = cut;
  __syncthreads();
  for (int i = 0; i < PIPE_WARPS; ++i) {
    const float4 t = sh.total[0][i][lane];
    carry = apply2(make_float2(t.x, t.y), make_float2(t.z, t.w), sh.cut[0][i], carry);
  }
  __syncthreads();
  return carry;
}

// Eight steps of two channels; `cuts`: some step of the warp's has a cut in front of it.
__device__ __forceinline__ bool cut_at(unsigned cut, int s) { return cut >> s & 1; }

template <typename T, bool BLEND, bool CUT, bool AGG>
__global__ void __launch_bounds__(PIPE_THREADS, PIPE_BLOCKS) scan_pipe_kernel(const __grid_constant__ ScanParams p) {
  constexpr int SLOTS = PIPE_SLOTS<T>, S = PIPE_S;
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ PipeShared sh;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, threadIdx.x >> 5, 0);
  const int b = blockIdx.x / p.groups, group = blockIdx.x % p.groups, chan0 = group * PIPE_CHANNELS, c = chan0 + 2 * lane;
  const bool on = c < p.C;
  int n = p.length ? p.length[b] : p.L;
  n = n < 0 ? 0 : n > p.L ? p.L : n;
  const int first = blockIdx.y * p.chunk_len, end = min(n, first + p.chunk_len);
  Source<T> sg, sx;
  sg.open(p.g, b * p.gb + chan0, p.gt, p, n, first);
  sx.open(p.x, b * p.xb + chan0, p.xt, p, n, first);
  const int there = chan0 + (int)threadIdx.x % Source<T>::COPIES * Source<T>::PER < p.C ? end : first;  // (rows this thread copies end here)
  const uint8_t* done = CUT ? p.done + (long long)b * p.L : nullptr;
  auto request = [&](int k0, int slot) {
    uint8_t* at = slots + slot * SLOT_BYTES<T, 2>;
    sg.request(at, there - k0);
    sx.request(at + SLOT_BYTES<T, 1>, there - k0);
    sg.move(1);
    sx.move(1);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < SLOTS - 1; ++s) request(first + s * PIPE_STEPS, s);
  float2 carry = make_float2(0.f, 0.f), product = make_float2(1.f, 1.f);
  bool any_cut = false;
  if (!AGG && on && p.h0) carry = pair_of(p.h0 + (long long)b * p.C + c);
  if (!AGG && p.chunks > 1 && first < n) carry = enter_chunk2<false>(p, sh, b, group, c, on, blockIdx.y, carry);
  bool flag = CUT && load_flag(p, done, n, first + warp * S, lane);
  T* y = reinterpret_cast<T*>(p.y) + (long long)b * p.L * p.C + c;
  const long long row = p.reverse ? -(long long)p.C : p.C;
  T* out = y + (long long)(p.reverse ? n - 1 - first - warp * S : first + warp * S) * p.C;
  float* kept = !AGG && p.states && on && warp == 0 ? p.states + ((long long)b * p.intervals + first / MARL_SCAN_INTERVAL) * p.C + c : nullptr;
  int slot = 0, par = 0;
  for (int k0 = first; k0 < end; k0 += PIPE_STEPS, par ^= 1) {
    asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 2) : "memory");
    __syncthreads();
    request(k0 + (SLOTS - 1) * PIPE_STEPS, slot == 0 ? SLOTS - 1 : slot - 1);
    const int mine = k0 + warp * S;
    unsigned cut = 0;
    if (CUT) {
      cut = __ballot_sync(~0u, flag);
      flag = load_flag(p, done, n, mine + PIPE_STEPS, lane);
    }
    const T* tg = reinterpret_cast<const T*>(slots + slot * SLOT_BYTES<T, 2>) + warp * S * PIPE_CHANNELS + 2 * lane;
    const T* tx = tg + PIPE_STEPS * PIPE_CHANNELS;
    float2 a[S], u[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      a[s] = pair_of(tg + s * PIPE_CHANNELS);
      u[s] = pair_of(tx + s * PIPE_CHANNELS);
      if (BLEND) {
        float2 rest;
        gate_pair2(a[s], a[s], rest);
        u[s] = mul2(rest, u[s]);
      }
    }
    const bool whole = mine + S <= end;
    if (!whole) {
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (mine + s >= end) {
          a[s] = make_float2(1.f, 1.f);
          u[s] = make_float2(0.f, 0.f);
        }
    }
    float2 A = a[0], H = u[0];
#pragma unroll
    for (int s = 1; s < S; ++s) A = mul2(A, a[s]);
    if (CUT && cut) {
#pragma unroll
      for (int s = 1; s < S; ++s) H = apply2(a[s], u[s], cut_at(cut, s), H);
    } else {
#pragma unroll
      for (int s = 1; s < S; ++s) H = fma2(a[s], H, u[s]);
    }
    sh.total[par][warp][lane] = make_float4(A.x, A.y, H.x, H.y);
    if (CUT && lane == 0) sh.cut[par][warp] = cut != 0;
    __syncthreads();
    const unsigned long long cuts = CUT ? *reinterpret_cast<const unsigned long long*>(sh.cut[par]) : 0ull;
    float2 enter = carry;
    if (!CUT || cuts == 0) {
#pragma unroll
      for (int i = 0; i < PIPE_WARPS; ++i) {
        const float4 t = sh.total[par][i][lane];
        carry = fma2(make_float2(t.x, t.y), carry, make_float2(t.z, t.w));
        if (i + 1 == warp) enter = carry;
        if (AGG) product = mul2(product, make_float2(t.x, t.y));
      }
    } else {
      for (int i = 0; i < PIPE_WARPS; ++i) {
        if (i == warp) enter = carry;
        const float4 t = sh.total[par][i][lane];
        carry = apply2(make_float2(t.x, t.y), make_float2(t.z, t.w), cuts >> (8 * i) & 1, carry);
        if (AGG) product = mul2(product, make_float2(t.x, t.y));
      }
      any_cut = true;
    }
    if constexpr (!AGG) {
      if (kept) {
        put_pair(kept, enter);
        kept += p.C;
      }
      if (on) {
        float2 h = enter;
        if (whole && !(CUT && cut)) {
#pragma unroll
          for (int s = 0; s < S; ++s) {
            h = fma2(a[s], h, u[s]);
            put_pair(out + s * row, h);
          }
        } else {
#pragma unroll
          for (int s = 0; s < S; ++s) {
            h = apply2(a[s], u[s], CUT && cut_at(cut, s), h);
            if (mine + s < end) put_pair(out + s * row, h);
          }
        }
      }
      out += row * PIPE_STEPS;
    }
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if constexpr (AGG) {
    if (first < end && warp == 0) {
      if (on) *reinterpret_cast<float4*>(p.agg + ((long long)b * p.chunks + blockIdx.y) * p.C + c) = make_float4(product.x, carry.x, product.y, carry.y);
      if (lane == 0) p.agg_cut[((long long)b * p.groups + group) * p.chunks + blockIdx.y] = any_cut;
    }
    return;
  }
  if (!on) return;
  if (warp == 0 && (n > 0 ? end == n && first < n : blockIdx.y == 0)) {
    const bool gone = CUT && !p.reverse && n > 0 && done[n - 1];
    put_pair(p.last + (long long)b * p.C + c, gone ? make_float2(0.f, 0.f) : carry);
  }
  const int stop = min(p.L, first + p.chunk_len);
  for (int t = max(n, first) + warp; t < stop; t += PIPE_WARPS) put_pair(y + (long long)t * p.C, make_float2(0.f, 0.f));
}

// BLOCKS: blocks a multiprocessor, 2 (128 registers) or 3 (80).
template <typename T, bool BLEND, bool CUT, bool AGG, int BLOCKS>
__global__ void __launch_bounds__(PIPE_THREADS, BLOCKS) scan_pipe_grad_kernel(const __grid_constant__ ScanParams p) {
  constexpr int SLOTS = GRAD_SLOTS, ARRAYS = AGG ? 2 : 3, S = PIPE_S;
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ PipeShared sh;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, threadIdx.x >> 5, 0);
  const int b = blockIdx.x / p.groups, group = blockIdx.x % p.groups, chan0 = group * PIPE_CHANNELS, c = chan0 + 2 * lane;
  const bool on = c < p.C;
  int n = p.length ? p.length[b] : p.L;
  n = n < 0 ? 0 : n > p.L ? p.L : n;
  const int first = blockIdx.y * p.chunk_len, end = min(n, first + p.chunk_len), used = (n + p.chunk_len - 1) / p.chunk_len;
  const int tiles = first < end ? (end - first + PIPE_STEPS - 1) / PIPE_STEPS : 0;
  const int last0 = first + (tiles - 1) * PIPE_STEPS;  // the tiles are taken from the last to the first
  Source<T> sg, sd, sx;
  sg.open(p.g, b * p.gb + chan0, p.gt, p, n, last0);
  sd.open(p.dy, b * p.dyb + chan0, p.dyt, p, n, last0);
  if (!AGG) sx.open(p.x, b * p.xb + chan0, p.xt, p, n, last0);
  const int there = chan0 + (int)threadIdx.x % Source<T>::COPIES * Source<T>::PER < p.C ? end : first;
  const uint8_t* done = CUT ? p.done + (long long)b * p.L : nullptr;
  auto request = [&](int k0, int slot) {
    if (k0 >= first) {
      uint8_t* at = slots + slot * SLOT_BYTES<T, ARRAYS>;
      sg.request(at, there - k0);
      sd.request(at + SLOT_BYTES<T, 1>, there - k0);
      sg.move(-1);
      sd.move(-1);
      if (!AGG) {
        sx.request(at + SLOT_BYTES<T, 2>, there - k0);
        sx.move(-1);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < SLOTS - 1; ++s) request(last0 - s * PIPE_STEPS, s);
  const bool gone = CUT && !p.reverse && n > 0 && done[n - 1];
  float2 carry = make_float2(0.f, 0.f), product = make_float2(1.f, 1.f);
  bool any_cut = false;
  if (!AGG && on && p.dlast && !gone) carry = pair_of(p.dlast + (long long)b * p.C + c);
  if (!AGG && p.chunks > 1 && first < n) carry = enter_chunk2<true>(p, sh, b, group, c, on, used - 1 - (int)blockIdx.y, carry, used);
  const float* kept = p.states + ((long long)b * p.intervals + last0 / MARL_SCAN_INTERVAL) * p.C + c;
  bool flag = CUT && tiles && load_flag(p, done, n, last0 + warp * S, lane);
  float2 state = !AGG && tiles && on ? pair_of(kept) : make_float2(0.f, 0.f);
  T* dg = reinterpret_cast<T*>(p.dg) + (long long)b * p.L * p.C + c;
  T* dx = reinterpret_cast<T*>(p.dx) + (long long)b * p.L * p.C + c;
  const long long row = p.reverse ? -(long long)p.C : p.C;
  long long out = (long long)(p.reverse ? n - 1 - last0 - warp * S : last0 + warp * S) * p.C;
  int slot = 0, par = 0;
  for (int k0 = last0; k0 >= first; k0 -= PIPE_STEPS, par ^= 1) {
    const int mine = k0 + warp * S;
    asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 2) : "memory");
    __syncthreads();
    request(k0 - (SLOTS - 1) * PIPE_STEPS, slot == 0 ? SLOTS - 1 : slot - 1);
    unsigned cut = 0;
    float2 enter = state;
    if (CUT) cut = __ballot_sync(~0u, flag);
    if (k0 > first) {
      if (CUT) flag = load_flag(p, done, n, mine - PIPE_STEPS, lane);
      kept -= p.C;
      if (!AGG && on) state = pair_of(kept);
    }
    const T* tg = reinterpret_cast<const T*>(slots + slot * SLOT_BYTES<T, ARRAYS>) + warp * S * PIPE_CHANNELS + 2 * lane;
    const T *td = tg + PIPE_STEPS * PIPE_CHANNELS, *tx = td + PIPE_STEPS * PIPE_CHANNELS;
    const bool plain = mine + S <= end && !(CUT && cut);
    // PLAIN: all eight steps are there and nothing is cut.  (What a slot holds of steps behind the end is something older.)
    float2 a[S], q[BLEND ? S : 1], A, H = make_float2(0.f, 0.f), R = make_float2(0.f, 0.f);
    auto value = [&](auto tag, const T* t, int s) {
      return decltype(tag)::value || mine + s < end ? pair_of(t + s * PIPE_CHANNELS) : make_float2(0.f, 0.f);
    };
    auto reduce = [&](auto tag) {
      constexpr bool PLAIN = decltype(tag)::value;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        a[s] = value(tag, tg, s);
        if (BLEND) gate_pair2(a[s], a[s], q[s]);
        if (!PLAIN && mine + s >= end) a[s] = make_float2(1.f, 1.f);
      }
      A = a[0];
#pragma unroll
      for (int s = 1; s < S; ++s) A = mul2(A, a[s]);
      if constexpr (!AGG) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const float2 x = value(tag, tx, s), u = BLEND ? mul2(q[s], x) : x;
          H = apply2(a[s], u, !PLAIN && cut_at(cut, s), H);
        }
      }
#pragma unroll
      for (int s = S - 1; s >= 0; --s) {
        R = mul2(a[s], add2(value(tag, td, s), R));
        if (!PLAIN && cut_at(cut, s)) R = make_float2(0.f, 0.f);
      }
    };
    if (plain) reduce(std::true_type());
    else reduce(std::false_type());
    sh.total[par][warp][lane] = make_float4(A.x, A.y, H.x, H.y);
    sh.back[par][warp][lane] = R;
    if (CUT && lane == 0) sh.cut[par][warp] = cut != 0;
    __syncthreads();
    const unsigned long long cuts = CUT ? *reinterpret_cast<const unsigned long long*>(sh.cut[par]) : 0ull;
    float2 back = carry;
    if (!CUT || cuts == 0) {
#pragma unroll
      for (int j = 0; j < PIPE_WARPS - 1; ++j)
        if (!AGG && j < warp) {
          const float4 t = sh.total[par][j][lane];
          enter = fma2(make_float2(t.x, t.y), enter, make_float2(t.z, t.w));
        }
#pragma unroll
      for (int j = PIPE_WARPS - 1; j >= 0; --j) {
        const float2 f = *reinterpret_cast<const float2*>(&sh.total[par][j][lane]);
        carry = fma2(f, carry, sh.back[par][j][lane]);
        if (j - 1 == warp) back = carry;
        if (AGG) product = mul2(product, f);
      }
    } else {
      if (!AGG)
        for (int j = 0; j < warp; ++j) {
          const float4 t = sh.total[par][j][lane];
          enter = apply2(make_float2(t.x, t.y), make_float2(t.z, t.w), cuts >> (8 * j) & 1, enter);
        }
      for (int j = PIPE_WARPS - 1; j >= 0; --j) {
        if (j == warp) back = carry;
        const float2 f = *reinterpret_cast<const float2*>(&sh.total[par][j][lane]);
        carry = apply2(f, sh.back[par][j][lane], cuts >> (8 * j) & 1, carry);
        if (AGG) product = mul2(product, f);
      }
      any_cut = true;
    }
    if constexpr (!AGG) {
      auto emit = [&](auto tag) {
        constexpr bool PLAIN = decltype(tag)::value;
        float2 G[S];
#pragma unroll
        for (int s = S - 1; s >= 0; --s) {
          G[s] = add2(value(tag, td, s), back);
          back = mul2(a[s], G[s]);
          if (!PLAIN && cut_at(cut, s)) back = make_float2(0.f, 0.f);
        }
        float2 h = enter;
        T *og = dg + out, *ox = dx + out;
#pragma unroll
        for (int s = 0; s < S; ++s) {
          if (!PLAIN && cut_at(cut, s)) h = make_float2(0.f, 0.f);
          const float2 x = value(tag, tx, s);
          float2 vg, vx = G[s];
          if (BLEND) {
            vx = mul2(G[s], q[s]);
            vg = mul2(add2(h, make_float2(-x.x, -x.y)), mul2(a[s], vx));
            h = fma2(a[s], h, mul2(q[s], x));
          } else {
            vg = mul2(G[s], h);
            h = fma2(a[s], h, x);
          }
          if (on && (PLAIN || mine + s < end)) {
            put_pair(og + s * row, vg);
            put_pair(ox + s * row, vx);
          }
        }
      };
      if (plain) emit(std::true_type());
      else emit(std::false_type());
      out -= row * PIPE_STEPS;
    }
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if constexpr (AGG) {
    if (first < end && warp == 0) {
      if (on) *reinterpret_cast<float4*>(p.agg + ((long long)b * p.chunks + blockIdx.y) * p.C + c) = make_float4(product.x, carry.x, product.y, carry.y);
      if (lane == 0) p.agg_cut[((long long)b * p.groups + group) * p.chunks + blockIdx.y] = any_cut;
    }
    return;
  }
  if (!on) return;
  if (warp == 0 && blockIdx.y == 0 && p.dh0) put_pair(p.dh0 + (long long)b * p.C + c, carry);
  const int stop = min(p.L, first + p.chunk_len);
  for (int t = max(n, first) + warp; t < stop; t += PIPE_WARPS) {
    put_pair(dg + (long long)t * p.C, make_float2(0.f, 0.f));
    put_pair(dx + (long long)t * p.C, make_float2(0.f, 0.f));
  }
}

// How a call is laid out.  V: channels a lane.
static void plan(ScanParams& p, int V, bool pipe) {
  const int lanes = (p.C + V - 1) / V;
  p.pipe = pipe;
  // Lanes along the channels: 32, or fewer where that leaves at least a quarter fewer lanes idle.
  p.lg = 0;
  while ((1 << p.lg) < lanes && p.lg < 5) ++p.lg;
  for (int lg = p.lg - 1; lg >= 3; --lg) {
    const long long now = (long long)((lanes + (1 << p.lg) - 1) >> p.lg) << p.lg, then = (long long)((lanes + (1 << lg) - 1) >> lg) << lg;
    if (4 * then <= 3 * now) p.lg = lg;
  }
  p.groups = (lanes + (1 << p.lg) - 1) >> p.lg;
  const int warp_steps = (32 >> p.lg) * STEPS;
  p.warps = 1;
  while (p.warps < MAX_WARPS && p.warps * warp_steps < p.L) p.warps *= 2;
  p.units = MAX_WARPS / p.warps;
  if (pipe) {
    p.lg = 5;
    p.groups = (p.C + PIPE_CHANNELS - 1) / PIPE_CHANNELS;
    p.warps = PIPE_WARPS;
    p.units = 1;
  }
  p.intervals = (p.L + MARL_SCAN_INTERVAL - 1) / MARL_SCAN_INTERVAL;
  // Few sequences and channels: the time axis is divided over blocks, which takes a launch for the chunks' maps and reads
  // gate and x twice.
  const int tile = pipe ? PIPE_STEPS : p.warps * warp_steps;   // a multiple of MARL_SCAN_INTERVAL wherever there are two
  const long long blocks = ((long long)p.B * p.groups + p.units - 1) / p.units;
  p.chunks = 1;
  p.chunk_len = p.L > 0 ? p.L : 1;
  if (blocks > 0 && blocks < 2 * LEARNER_SMS && p.L >= 4 * tile) {
    const int tiles = (p.L + tile - 1) / tile;
    int want = (int)((pipe ? 3 : 4) * LEARNER_SMS / blocks);
    want = std::max(1, std::min(want, tiles / 2));
    const int per = (tiles + want - 1) / want;
    p.chunk_len = per * tile;
    p.chunks = (p.L + p.chunk_len - 1) / p.chunk_len;
  }
}

static size_t work_need(const ScanParams& p) {
  if (p.chunks <= 1) return 0;
  const size_t maps = (size_t)p.B * p.chunks * p.C * sizeof(float2);
  return maps + (((size_t)p.B * p.groups * p.chunks + 7) & ~(size_t)7);
}

static int check_scan(const marl_scan_t* in) {
  if (!in) return fail(MARL_EINVAL, "scan descriptor is NULL");
  if (in->B < 0 || in->L < 0 || in->C < 0) return fail(MARL_EINVAL, "B, L and C must be >= 0");
  if (in->L > (1 << 30) || in->C > (1 << 30)) return fail(MARL_EINVAL, "L and C must be at most 2^30");
  if (!dtype_known(in->dtype)) return fail(MARL_EINVAL, "unknown dtype %d", in->dtype);
  if (in->form != MARL_SCAN_RAW && in->form != MARL_SCAN_BLEND) return fail(MARL_EINVAL, "unknown form %d", in->form);
  if (in->gate_b < 0 || in->gate_t < 0 || in->x_b < 0 || in->x_t < 0) return fail(MARL_EINVAL, "a stride is negative");
  if ((in->gate_c != 0 && in->gate_c != 1) || (in->x_c != 0 && in->x_c != 1))
    return fail(MARL_EINVAL, "gate_c and x_c must be 0 or 1");
  return MARL_OK;
}

// Two channels a lane: 16-bit types whose pairs lie on 4-byte boundaries everywhere.  (One channel a lane would move 64 bytes a warp
// and step.)
static int channels_a_lane(const marl_scan_t* in) {
  const bool pairs = in->dtype != MARL_DTYPE_FP32 && in->C % 2 == 0 && in->gate_c == 1 && in->x_c == 1 && in->gate_b % 2 == 0 &&
                     in->gate_t % 2 == 0 && in->x_b % 2 == 0 && in->x_t % 2 == 0 && !misaligned(in->gate, 4) && !misaligned(in->x, 4);
  return pairs ? 2 : 1;
}

// Tiles by asynchronous copies: 16-byte pieces of rows everywhere, and enough channels and steps to fill tiles of 64 x 64.
static bool can_pipe(const marl_scan_t* in) {
  const long long es = (long long)dtype_bytes(in->dtype);
  auto whole = [&](long long elements) { return elements * es % 16 == 0; };
  return in->C >= 48 && in->L >= 32 && in->gate_c == 1 && in->x_c == 1 && whole(in->C) && whole(in->gate_b) && whole(in->gate_t) && whole(in->x_b) &&
         whole(in->x_t) && !misaligned(in->gate, 16) && !misaligned(in->x, 16) && !misaligned(in->h0, 8);
}

static ScanParams scan_params(const marl_scan_t* in, int V, bool pipe) {
  ScanParams p = {};
  p.g = in->gate; p.x = in->x;
  p.gb = in->gate_b; p.gt = in->gate_t; p.xb = in->x_b; p.xt = in->x_t;
  p.gc = in->gate_c; p.xc = in->x_c;
  p.h0 = in->h0; p.done = in->done; p.length = in->length;
  p.B = in->B; p.L = in->L; p.C = in->C; p.reverse = in->reverse != 0;
  plan(p, V, pipe);
  return p;
}

static int check_pointers(const marl_scan_t* in) {
  if (in->L > 0 && (!in->gate || !in->x)) return fail(MARL_EINVAL, "gate or x is NULL");
  const size_t es = dtype_bytes(in->dtype);
  if (misaligned(in->gate, es) || misaligned(in->x, es) || misaligned(in->h0, 4) || misaligned(in->length, 4))
    return fail(MARL_EALIGN, "an input is not aligned to its elements");
  return MARL_OK;
}

// What a caller has to bring, whatever the arrays' alignment turns out to be.
static size_t work_wanted(const marl_scan_t* in) {
  size_t need = work_need(scan_params(in, 1, false));
  if (in->dtype != MARL_DTYPE_FP32) need = std::max(need, work_need(scan_params(in, 2, false)));
  if (in->C >= 48 && in->L >= 32) need = std::max(need, work_need(scan_params(in, 2, true)));
  return need;
}

static int set_work(ScanParams& p, const marl_scan_t* in, void* work, size_t bytes) {
  if (in->L <= MARL_SCAN_INTERVAL) return MARL_OK;
  const size_t need = work_wanted(in);
  if (!need) return MARL_OK;
  if (!work || bytes < need) return fail(MARL_ENOMEM, "work: %zu bytes given, %zu needed", work ? bytes : (size_t)0, need);
  if (misaligned(work, 16)) return fail(MARL_EALIGN, "work must be 16-byte aligned");
  p.agg = reinterpret_cast<float2*>(work);
  p.agg_cut = reinterpret_cast<uint8_t*>(p.agg + (size_t)p.B * p.chunks * p.C);
  return MARL_OK;
}

static int launch_ok(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? MARL_OK : fail(MARL_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

template <typename T, int V, int S, bool BLEND, bool CUT>
static int launch_scan(const ScanParams& p, bool grad, cudaStream_t stream) {
  const long long blocks = ((long long)p.B * p.groups + p.units - 1) / p.units;
  if (blocks > INT32_MAX || p.chunks > 65535) return fail(MARL_EINVAL, "too many sequences or channels");
  const dim3 grid((unsigned)blocks, (unsigned)p.chunks);
  const int threads = p.units * p.warps * 32;
  if (!grad) {
    if (p.chunks > 1) scan_kernel<T, V, S, BLEND, CUT, true><<<grid, threads, 0, stream>>>(p);
    scan_kernel<T, V, S, BLEND, CUT, false><<<grid, threads, 0, stream>>>(p);
    return launch_ok("marl_linear_scan");
  }
  if (p.chunks > 1) scan_grad_kernel<T, V, S, BLEND, CUT, true><<<grid, threads, 0, stream>>>(p);
  scan_grad_kernel<T, V, S, BLEND, CUT, false><<<grid, threads, 0, stream>>>(p);
  return launch_ok("marl_linear_scan_backward");
}

static uint32_t g_pipe_smem[3][20][SMEM_OPTIN_DEVICES];

template <typename T, bool BLEND, bool CUT>
static int launch_pipe(const ScanParams& p, bool grad, int which, cudaStream_t stream) {
  const long long blocks = (long long)p.B * p.groups;
  if (blocks > INT32_MAX || p.chunks > 65535) return fail(MARL_EINVAL, "too many sequences or channels");
  const dim3 grid((unsigned)blocks, (unsigned)p.chunks);
  const int w = (BLEND ? 2 : 0) + (CUT ? 1 : 0);
  auto go = [&](auto kernel, int bytes, int index) {
    // (one table entry per kernel: the maps' launch of the gradient needs less than the gradient)
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (uint32_t)bytes, g_pipe_smem[which][index]);
    if (e != cudaSuccess) return e;
    kernel<<<grid, PIPE_THREADS, bytes, stream>>>(p);
    return cudaGetLastError();
  };
  cudaError_t e = cudaSuccess;
  const int slots = std::min(grad ? GRAD_SLOTS : PIPE_SLOTS<T>, (std::min(p.L, p.chunk_len) + PIPE_STEPS - 1) / PIPE_STEPS);  // no more than there are tiles
  const int two = slots * SLOT_BYTES<T, 2>, three = slots * SLOT_BYTES<T, 3>;
  if (!grad) {
    if (p.chunks > 1) e = go(scan_pipe_kernel<T, BLEND, CUT, true>, two, w);
    if (e == cudaSuccess) e = go(scan_pipe_kernel<T, BLEND, CUT, false>, two, w + 4);
  } else {
    // Three blocks a multiprocessor where their shared memory allows it and they save a wave, else two, which are faster each: 64 x 256 x 512 bf16
    // (two waves either way) 28 us with two and 33 with three, 8 x 4096 x 1024 bf16 (two waves and one) 187 and 159, 2048 x 64 x 256 fp32 (28
    // and 19) 148 and 121.
    const long long all = blocks * p.chunks;
    auto waves = [&](long long per) { return (all + per * LEARNER_SMS - 1) / (per * LEARNER_SMS); };
    const bool dense = 3 * three <= 200 * 1024 && waves(3) < waves(2);
    if (p.chunks > 1) e = go(scan_pipe_grad_kernel<T, BLEND, CUT, true, 2>, two, w + 8);
    if (e == cudaSuccess) e = dense ? go(scan_pipe_grad_kernel<T, BLEND, CUT, false, 3>, three, w + 16) : go(scan_pipe_grad_kernel<T, BLEND, CUT, false, 2>, three, w + 12);
  }
  return e == cudaSuccess ? MARL_OK : fail(MARL_ECUDA, "marl_linear_scan%s: %s", grad ? "_backward" : "", cudaGetErrorString(e));
}

template <typename T, int V, bool BLEND>
static int run_scan(const ScanParams& p, bool grad, cudaStream_t stream) {
  if (p.pipe) {
    constexpr int which = sizeof(T) == 4 ? 0 : std::is_same<T, __half>::value ? 1 : 2;
    return p.done ? launch_pipe<T, BLEND, true>(p, grad, which, stream) : launch_pipe<T, BLEND, false>(p, grad, which, stream);
  }
  if (p.L == 1) {
    const int pairs = (p.C + V - 1) / V;
    int tx = 32;
    while (tx < 256 && tx < pairs) tx *= 2;
    const dim3 threads((unsigned)tx, (unsigned)(256 / tx));
    const unsigned gy = (unsigned)std::min<long long>(((long long)p.B + threads.y - 1) / threads.y, 65535);
    const dim3 grid((unsigned)((pairs + tx - 1) / tx), gy);
    if (grad) scan_step_grad_kernel<T, V, BLEND><<<grid, threads, 0, stream>>>(p);
    else scan_step_kernel<T, V, BLEND><<<grid, threads, 0, stream>>>(p);
    return launch_ok("marl_linear_scan of one step");
  }
  return p.done ? launch_scan<T, V, STEPS, BLEND, true>(p, grad, stream) : launch_scan<T, V, STEPS, BLEND, false>(p, grad, stream);
}

static int dispatch(const ScanParams& p, int dtype, int V, bool blend, bool grad, cudaStream_t stream) {
  if (dtype == MARL_DTYPE_FP32) return blend ? run_scan<float, 1, true>(p, grad, stream) : run_scan<float, 1, false>(p, grad, stream);
  if (dtype == MARL_DTYPE_BF16) {
    if (V == 2) return blend ? run_scan<__nv_bfloat16, 2, true>(p, grad, stream) : run_scan<__nv_bfloat16, 2, false>(p, grad, stream);
    return blend ? run_scan<__nv_bfloat16, 1, true>(p, grad, stream) : run_scan<__nv_bfloat16, 1, false>(p, grad, stream);
  }
  if (V == 2) return blend ? run_scan<__half, 2, true>(p, grad, stream) : run_scan<__half, 2, false>(p, grad, stream);
  return blend ? run_scan<__half, 1, true>(p, grad, stream) : run_scan<__half, 1, false>(p, grad, stream);
}

}  // namespace marl

using namespace marl;

extern "C" int marl_linear_scan_query(const marl_scan_t* in, size_t* states_bytes, size_t* work_bytes) {
  const int rc = check_scan(in);
  if (rc != MARL_OK) return rc;
  if (states_bytes) *states_bytes = (size_t)in->B * (((size_t)in->L + MARL_SCAN_INTERVAL - 1) / MARL_SCAN_INTERVAL) * in->C * 4;
  if (work_bytes) *work_bytes = in->L <= MARL_SCAN_INTERVAL ? 0 : work_wanted(in);
  return MARL_OK;
}

extern "C" int marl_linear_scan(void* stream, const marl_scan_t* in, void* y, float* last, float* states, void* work, size_t work_bytes) {
  int rc = check_scan(in);
  if (rc != MARL_OK) return rc;
  if (in->B == 0 || in->C == 0) return MARL_OK;
  if ((rc = check_pointers(in)) != MARL_OK) return rc;
  if (!last || (in->L > 0 && !y)) return fail(MARL_EINVAL, "y or last is NULL");
  if (misaligned(y, dtype_bytes(in->dtype)) || misaligned(last, 4) || misaligned(states, 4))
    return fail(MARL_EALIGN, "an output is not aligned to its elements");
  const int V = channels_a_lane(in) == 2 && !misaligned(y, 4) ? 2 : 1;
  ScanParams p = scan_params(in, V, can_pipe(in) && !misaligned(y, 8) && !misaligned(last, 8) && !misaligned(states, 8));
  p.y = y;
  p.last = last;
  p.states = states;
  if ((rc = set_work(p, in, work, work_bytes)) != MARL_OK) return rc;
  return dispatch(p, in->dtype, V, in->form == MARL_SCAN_BLEND, false, (cudaStream_t)stream);
}

extern "C" int marl_linear_scan_backward(void* stream, const marl_scan_t* in, const float* states, const void* dy, int64_t dy_b, int64_t dy_t,
                                         const float* dlast, void* dgate, void* dx, float* dh0, void* work, size_t work_bytes) {
  int rc = check_scan(in);
  if (rc != MARL_OK) return rc;
  if (in->B == 0 || in->C == 0) return MARL_OK;
  if ((rc = check_pointers(in)) != MARL_OK) return rc;
  if (in->L > 0 && (!states || !dy || !dgate || !dx)) return fail(MARL_EINVAL, "states, dy, dgate or dx is NULL");
  if (dy_b < 0 || dy_t < 0) return fail(MARL_EINVAL, "a stride is negative");
  const size_t es = dtype_bytes(in->dtype);
  if (misaligned(states, 4) || misaligned(dlast, 4) || misaligned(dh0, 4) || misaligned(dy, es) || misaligned(dgate, es) || misaligned(dx, es))
    return fail(MARL_EALIGN, "an array is not aligned to its elements");
  const bool pairs = channels_a_lane(in) == 2 && dy_b % 2 == 0 && dy_t % 2 == 0 && !misaligned(dy, 4) && !misaligned(dgate, 4) && !misaligned(dx, 4);
  const int V = pairs ? 2 : 1;
  const bool pipe = can_pipe(in) && dy_b * (long long)es % 16 == 0 && dy_t * (long long)es % 16 == 0 && !misaligned(dy, 16) && !misaligned(dgate, 8) &&
                    !misaligned(dx, 8) && !misaligned(states, 8) && !misaligned(dlast, 8) && !misaligned(dh0, 8);
  ScanParams p = scan_params(in, V, pipe);
  p.states = const_cast<float*>(states);
  p.dy = dy;
  p.dyb = dy_b;
  p.dyt = dy_t;
  p.dlast = dlast;
  p.dg = dgate;
  p.dx = dx;
  p.dh0 = dh0;
  if ((rc = set_work(p, in, work, work_bytes)) != MARL_OK) return rc;
  return dispatch(p, in->dtype, V, in->form == MARL_SCAN_BLEND, true, (cudaStream_t)stream);
}
