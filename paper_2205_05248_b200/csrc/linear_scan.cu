// The gated linear recurrence h' = a h + b over a batch of sequences, and its gradient.
//
// A run of steps is an affine map of the state that enters it, h -> A h + H with A the product of its gates and H its result
// from a zero state; a cut inside it makes it a constant, whatever enters (kept as a flag, not as a factor 0, so that nothing
// non-finite crosses).  Each thread takes STEPS neighbouring steps of one or two channels into registers and reduces them to
// such a map; the maps are combined along the lanes that share a channel and along the warps of a block; then the
// thread runs its steps again from the state that enters them.  One pass over gate and x, one write of y.
// The gradient runs against the scan order: with G_k = dy_k + R_{k+1}, R_k = a_k G_k (0 at a cut) is the gradient of the
// state that enters step k: the same maps, composed the other way round.
#include "learner_util.cuh"
#include "launch_util.cuh"

#include <algorithm>

namespace marl {

constexpr int STEPS = 8;       // steps a thread holds
constexpr int MAX_WARPS = 8;   // warps along time
constexpr int SCAN_SMS = 148;

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

// z = 1 / (1 + e^-g) and 1 - z, each accurate where it is small.
__device__ __forceinline__ void gate_pair(float g, float& z, float& rest) {
  const float e = ex2(-fabsf(g) * 1.4426950408889634f), big = __fdividef(1.f, 1.f + e), small = e * big;
  z = g >= 0.f ? big : small;
  rest = g >= 0.f ? small : big;
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

// The cuts in front of the thread's steps k0 .. k0 + STEPS - 1 (scan order), as bits.
__device__ __forceinline__ unsigned load_cuts(const ScanParams& p, const Place& w, int k0) {
  unsigned bits = 0;
  if (!p.done) return 0;
  const uint8_t* d = p.done + (long long)w.b * p.L;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int k = k0 + s, at = p.reverse ? w.n - 1 - k : k - 1;  // done of the step before, or in reverse of this one
    if (k < w.n && at >= 0 && d[at]) bits |= 1u << s;
  }
  return bits;
}

template <typename T, int V>
__device__ __forceinline__ void load_steps(const void* base, long long sb, long long st, int sc, const ScanParams& p, const Place& w, int k0,
                                           Raw<T, V> (&r)[STEPS]) {
  const T* at = reinterpret_cast<const T*>(base) + w.b * sb + w.c * sc;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int k = k0 + s, t = p.reverse ? w.n - 1 - k : k;
    if (w.on && k < w.n) r[s] = *reinterpret_cast<const Raw<T, V>*>(at + t * st);
    else r[s] = Raw<T, V>{};
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

__device__ __forceinline__ Map shfl_map_up(const Map& m, int d) {
  return Map{__shfl_up_sync(~0u, m.a, d), __shfl_up_sync(~0u, m.h, d), (bool)__shfl_up_sync(~0u, (int)m.cut, d)};
}
__device__ __forceinline__ Map shfl_map_down(const Map& m, int d) {
  return Map{__shfl_down_sync(~0u, m.a, d), __shfl_down_sync(~0u, m.h, d), (bool)__shfl_down_sync(~0u, (int)m.cut, d)};
}

struct ScanShared {
  float2 total[2][MAX_WARPS][32 * 2];
  float back[2][MAX_WARPS][32 * 2];
  uint8_t cut[2][MAX_WARPS];
};

// The state that enters chunk `chunk` of the time axis from the maps of the chunks before it (backward: behind it).
template <int V, bool BACK>
__device__ __forceinline__ void enter_chunk(const ScanParams& p, const Place& w, int chunk, int used, float (&h)[V]) {
  const float2* agg = p.agg + (long long)w.b * p.chunks * p.C + w.c;
  const uint8_t* cut = p.agg_cut + ((long long)w.b * p.groups + w.group) * p.chunks;
  const int n = BACK ? used - 1 - chunk : chunk;
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    const int at = BACK ? used - 1 - i : i;
    const bool c = cut[at];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 m = w.on ? agg[(long long)at * p.C + v] : make_float2(0.f, 0.f);
      h[v] = apply(Map{m.x, m.y, c}, h[v]);
    }
  }
}

// AGG: only the chunk's map is computed, for the launch behind this one.
template <typename T, int V, bool BLEND, bool AGG>
__global__ void __launch_bounds__(MAX_WARPS * 32) scan_kernel(const __grid_constant__ ScanParams p) {
  __shared__ ScanShared sh_all;
  Place w;
  if (!find_place<V>(p, w)) return;
  const int subs = 32 >> p.lg, tile = p.warps * subs * STEPS, wslot = w.slot * p.warps;
  const int first = blockIdx.y * p.chunk_len, end = min(w.n, first + p.chunk_len);  // steps of this block, in scan order
  float carry[V];
  Map whole[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    carry[v] = !AGG && w.on && p.h0 ? p.h0[(long long)w.b * p.C + w.c + v] : 0.f;
    whole[v] = Map{1.f, 0.f, false};
  }
  if (!AGG && p.chunks > 1 && first < w.n) enter_chunk<V, false>(p, w, blockIdx.y, 0, carry);

  Raw<T, V> rg[STEPS], rx[STEPS];
  unsigned cuts = 0;
  if (first < end) {
    load_steps<T, V>(p.g, p.gb, p.gt, p.gc, p, w, first + w.q * STEPS, rg);
    load_steps<T, V>(p.x, p.xb, p.xt, p.xc, p, w, first + w.q * STEPS, rx);
    cuts = load_cuts(p, w, first + w.q * STEPS);
  }
  int par = 0;
  for (int k0 = first; k0 < end; k0 += tile, par ^= 1) {
    const int mine = k0 + w.q * STEPS;
    float a[STEPS][V], b[STEPS][V];
    const unsigned cut = cuts;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      float g[V], x[V];
      unpack(rg[s], g);
      unpack(rx[s], x);
#pragma unroll
      for (int v = 0; v < V; ++v) step_ab<BLEND>(mine + s < end, g[v], x[v], a[s][v], b[s][v]);
    }
    if (k0 + tile < end) {  // the next tile is on its way while this one is computed
      load_steps<T, V>(p.g, p.gb, p.gt, p.gc, p, w, mine + tile, rg);
      load_steps<T, V>(p.x, p.xb, p.xt, p.xc, p, w, mine + tile, rx);
      cuts = load_cuts(p, w, mine + tile);
    }
    Map m[V], before[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      m[v] = Map{1.f, 0.f, cut != 0};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        m[v].h = cut >> s & 1 ? b[s][v] : fmaf(a[s][v], m[v].h, b[s][v]);
        m[v].a *= a[s][v];
      }
      for (int d = 1; d < subs; d <<= 1) {
        const Map o = shfl_map_up(m[v], d << p.lg);
        if (w.sub >= d) m[v] = then(o, m[v]);
      }
      before[v] = Map{1.f, 0.f, false};
      if (subs > 1) {
        const Map o = shfl_map_up(m[v], 1 << p.lg);
        if (w.sub) before[v] = o;
      }
    }
    float enter[V];
    if (p.warps > 1) {
      if (w.sub == subs - 1) {
        const int ch = w.lane & ((1 << p.lg) - 1);
#pragma unroll
        for (int v = 0; v < V; ++v) sh_all.total[par][wslot + w.warp][ch * V + v] = make_float2(m[v].a, m[v].h);
        if (ch == 0) sh_all.cut[par][wslot + w.warp] = m[0].cut;
      }
      unit_sync(p, w);
      const int ch = w.lane & ((1 << p.lg) - 1);
#pragma unroll 4
      for (int i = 0; i < p.warps; ++i) {
        const bool c = sh_all.cut[par][wslot + i];
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
          const int src = 32 - (1 << p.lg) + (w.lane & ((1 << p.lg) - 1));
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
      T* y = reinterpret_cast<T*>(p.y) + (long long)w.b * p.L * p.C + w.c;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int k = mine + s, t = p.reverse ? w.n - 1 - k : k;
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = cut >> s & 1 ? b[s][v] : fmaf(a[s][v], h[v], b[s][v]);
        if (w.on && k < end) put(y + (long long)t * p.C, h);
      }
    }
  }
  if (AGG) {
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
    const bool gone = !p.reverse && w.n > 0 && p.done && p.done[(long long)w.b * p.L + w.n - 1];
#pragma unroll
    for (int v = 0; v < V; ++v) p.last[(long long)w.b * p.C + w.c + v] = gone ? 0.f : carry[v];
  }
  T* y = reinterpret_cast<T*>(p.y) + (long long)w.b * p.L * p.C + w.c;
  const float zero[V] = {};
  const int stop = min(p.L, first + p.chunk_len);
  for (int t = max(w.n, first) + w.q; t < stop; t += p.warps * subs) put(y + (long long)t * p.C, zero);
}

template <typename T, int V, bool BLEND, bool AGG>
__global__ void __launch_bounds__(MAX_WARPS * 32) scan_grad_kernel(const __grid_constant__ ScanParams p) {
  __shared__ ScanShared sh_all;
  Place w;
  if (!find_place<V>(p, w)) return;
  const int subs = 32 >> p.lg, tile = p.warps * subs * STEPS, wslot = w.slot * p.warps, ch = w.lane & ((1 << p.lg) - 1);
  const int first = blockIdx.y * p.chunk_len, end = min(w.n, first + p.chunk_len);
  const int used = (w.n + p.chunk_len - 1) / p.chunk_len;
  float carry[V];
  Map whole[V];
  const bool gone = !p.reverse && w.n > 0 && p.done && p.done[(long long)w.b * p.L + w.n - 1];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    carry[v] = !AGG && w.on && p.dlast && !gone ? p.dlast[(long long)w.b * p.C + w.c + v] : 0.f;
    whole[v] = Map{1.f, 0.f, false};
  }
  if (!AGG && p.chunks > 1 && first < w.n) enter_chunk<V, true>(p, w, blockIdx.y, used, carry);
  T* dg = reinterpret_cast<T*>(p.dg) + (long long)w.b * p.L * p.C + w.c;
  T* dx = reinterpret_cast<T*>(p.dx) + (long long)w.b * p.L * p.C + w.c;
  const int tiles = first < end ? (end - first + tile - 1) / tile : 0;
  int par = 0;
  for (int i = tiles - 1; i >= 0; --i, par ^= 1) {
    const int k0 = first + i * tile, mine = k0 + w.q * STEPS;
    Raw<T, V> rg[STEPS], rx[STEPS], rd[STEPS];
    load_steps<T, V>(p.g, p.gb, p.gt, p.gc, p, w, mine, rg);
    load_steps<T, V>(p.dy, p.dyb, p.dyt, 1, p, w, mine, rd);
    if (!AGG) load_steps<T, V>(p.x, p.xb, p.xt, p.xc, p, w, mine, rx);
    const unsigned cut = load_cuts(p, w, mine);
    float enter[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
      enter[v] = !AGG && w.on ? p.states[((long long)w.b * p.intervals + k0 / MARL_SCAN_INTERVAL) * p.C + w.c + v] : 0.f;
    float a[STEPS][V], x[STEPS][V], d[STEPS][V];
    Map m[V], r[V];   // the steps' map of the state, and that of the gradient (same factor, against the scan order)
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      float g[V];
      unpack(rg[s], g);
      unpack(rd[s], d[s]);
      if (!AGG) unpack(rx[s], x[s]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (BLEND) {
          float rest;
          gate_pair(g[v], a[s][v], rest);
        } else a[s][v] = g[v];
        if (mine + s >= end) a[s][v] = 1.f;  // (x and dy are 0 there)
      }
    }
    // BLEND: the input of a step is (1 - z) x; 1 - z is computed again from the gate where it is needed
    auto input = [&](int s, int v) {
      if (!BLEND) return x[s][v];
      float g[V], z, rest;
      unpack(rg[s], g);
      gate_pair(g[v], z, rest);
      return mine + s < end ? rest * x[s][v] : 0.f;
    };
#pragma unroll
    for (int v = 0; v < V; ++v) {
      m[v] = r[v] = Map{1.f, 0.f, cut != 0};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) m[v].a *= a[s][v];
      r[v].a = m[v].a;
      if (!AGG) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const float b = input(s, v);
          m[v].h = cut >> s & 1 ? b : fmaf(a[s][v], m[v].h, b);
        }
      }
#pragma unroll
      for (int s = STEPS - 1; s >= 0; --s) r[v].h = cut >> s & 1 ? 0.f : a[s][v] * (d[s][v] + r[v].h);
    }
    Map before[V], behind[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      before[v] = behind[v] = Map{1.f, 0.f, false};
      if (subs > 1) {
        for (int e = 1; e < subs; e <<= 1) {
          const Map o = shfl_map_up(m[v], e << p.lg), q = shfl_map_down(r[v], e << p.lg);
          if (w.sub >= e) m[v] = then(o, m[v]);
          if (w.sub + e < subs) r[v] = then(q, r[v]);
        }
        const Map o = shfl_map_up(m[v], 1 << p.lg), q = shfl_map_down(r[v], 1 << p.lg);
        if (w.sub) before[v] = o;
        if (w.sub + 1 < subs) behind[v] = q;
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
        if (ch == 0) sh_all.cut[par][wslot + w.warp] = m[0].cut;
      }
      unit_sync(p, w);
#pragma unroll 4
      for (int j = 0; j < p.warps; ++j) {
        const int jb = p.warps - 1 - j;
        const bool c = sh_all.cut[par][wslot + j], cb = sh_all.cut[par][wslot + jb];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (!AGG && j < w.warp) {
            const float2 t = sh_all.total[par][wslot + j][ch * V + v];
            enter[v] = apply(Map{t.x, t.y, c}, enter[v]);
          }
          if (jb == w.warp) back[v] = carry[v];
          const Map mb{sh_all.total[par][wslot + jb][ch * V + v].x, sh_all.back[par][wslot + jb][ch * V + v], cb};
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
        enter[v] = apply(before[v], enter[v]);
        back[v] = apply(behind[v], back[v]);
      }
      float came[STEPS][V];  // the state that a step's gate multiplies
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float h = enter[v];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          if (cut >> s & 1) h = 0.f;
          came[s][v] = h;
          h = fmaf(a[s][v], h, input(s, v));
        }
      }
#pragma unroll
      for (int s = STEPS - 1; s >= 0; --s) {
        const int k = mine + s, t = p.reverse ? w.n - 1 - k : k;
        float og[V], ox[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float G = d[s][v] + back[v];
          if (BLEND) {
            float g[V], z, rest;
            unpack(rg[s], g);
            gate_pair(g[v], z, rest);
            og[v] = G * (came[s][v] - x[s][v]) * (z * rest);
            ox[v] = G * rest;
          } else {
            og[v] = G * came[s][v];
            ox[v] = G;
          }
          back[v] = cut >> s & 1 ? 0.f : a[s][v] * G;
        }
        if (w.on && k < end) {
          put(dg + (long long)t * p.C, og);
          put(dx + (long long)t * p.C, ox);
        }
      }
    }
  }
  if (AGG) {
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

// How a call is laid out.  V: channels a lane.
static void plan(ScanParams& p, int V) {
  const int lanes = (p.C + V - 1) / V;
  p.lg = 0;
  while ((1 << p.lg) < lanes && p.lg < 5) ++p.lg;
  p.groups = (lanes + (1 << p.lg) - 1) >> p.lg;
  const int warp_steps = (32 >> p.lg) * STEPS;
  p.warps = 1;
  while (p.warps < MAX_WARPS && p.warps * warp_steps < p.L) p.warps *= 2;
  p.units = MAX_WARPS / p.warps;
  p.intervals = (p.L + MARL_SCAN_INTERVAL - 1) / MARL_SCAN_INTERVAL;
  // Few sequences and channels: the time axis is divided over blocks, which takes a launch for the chunks' maps and reads
  // gate and x twice.
  const int tile = p.warps * warp_steps;   // a multiple of MARL_SCAN_INTERVAL wherever there are two
  const long long blocks = ((long long)p.B * p.groups + p.units - 1) / p.units;
  p.chunks = 1;
  p.chunk_len = p.L > 0 ? p.L : 1;
  if (blocks < 2 * SCAN_SMS && p.L >= 4 * tile) {
    const int tiles = (p.L + tile - 1) / tile;
    int want = (int)((4 * SCAN_SMS + blocks - 1) / blocks);
    want = std::min(want, tiles / 2);
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

static ScanParams scan_params(const marl_scan_t* in, int V) {
  ScanParams p = {};
  p.g = in->gate; p.x = in->x;
  p.gb = in->gate_b; p.gt = in->gate_t; p.xb = in->x_b; p.xt = in->x_t;
  p.gc = in->gate_c; p.xc = in->x_c;
  p.h0 = in->h0; p.done = in->done; p.length = in->length;
  p.B = in->B; p.L = in->L; p.C = in->C; p.reverse = in->reverse != 0;
  plan(p, V);
  return p;
}

static int check_pointers(const marl_scan_t* in) {
  if (in->L > 0 && (!in->gate || !in->x)) return fail(MARL_EINVAL, "gate or x is NULL");
  const size_t es = dtype_bytes(in->dtype);
  if (misaligned(in->gate, es) || misaligned(in->x, es) || misaligned(in->h0, 4) || misaligned(in->length, 4))
    return fail(MARL_EALIGN, "an input is not aligned to its elements");
  return MARL_OK;
}

static int set_work(ScanParams& p, void* work, size_t bytes) {
  const size_t need = work_need(p);
  if (!need) return MARL_OK;
  if (!work || bytes < need) return fail(MARL_ENOMEM, "work: %zu bytes given, %zu needed", work ? bytes : (size_t)0, need);
  if (misaligned(work, 8)) return fail(MARL_EALIGN, "work must be 8-byte aligned");
  p.agg = reinterpret_cast<float2*>(work);
  p.agg_cut = reinterpret_cast<uint8_t*>(p.agg + (size_t)p.B * p.chunks * p.C);
  return MARL_OK;
}

static int launch_ok(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? MARL_OK : fail(MARL_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

template <typename T, int V, bool BLEND>
static int run_scan(const ScanParams& p, bool grad, cudaStream_t stream) {
  const long long blocks = ((long long)p.B * p.groups + p.units - 1) / p.units;
  if (blocks > INT32_MAX || p.chunks > 65535) return fail(MARL_EINVAL, "too many sequences or channels");
  const dim3 grid((unsigned)blocks, (unsigned)p.chunks);
  const int threads = p.units * p.warps * 32;
  if (!grad) {
    if (p.chunks > 1) scan_kernel<T, V, BLEND, true><<<grid, threads, 0, stream>>>(p);
    scan_kernel<T, V, BLEND, false><<<grid, threads, 0, stream>>>(p);
    return launch_ok("marl_linear_scan");
  }
  if (p.chunks > 1) scan_grad_kernel<T, V, BLEND, true><<<grid, threads, 0, stream>>>(p);
  scan_grad_kernel<T, V, BLEND, false><<<grid, threads, 0, stream>>>(p);
  return launch_ok("marl_linear_scan_backward");
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
  if (work_bytes) {  // whatever the arrays' alignment turns out to be
    const size_t one = work_need(scan_params(in, 1)), two = in->dtype == MARL_DTYPE_FP32 ? 0 : work_need(scan_params(in, 2));
    *work_bytes = std::max(one, two);
  }
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
  ScanParams p = scan_params(in, V);
  p.y = y;
  p.last = last;
  p.states = states;
  if ((rc = set_work(p, work, work_bytes)) != MARL_OK) return rc;
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
  ScanParams p = scan_params(in, V);
  p.states = const_cast<float*>(states);
  p.dy = dy;
  p.dyb = dy_b;
  p.dyt = dy_t;
  p.dlast = dlast;
  p.dg = dgate;
  p.dx = dx;
  p.dh0 = dh0;
  if ((rc = set_work(p, work, work_bytes)) != MARL_OK) return rc;
  return dispatch(p, in->dtype, V, in->form == MARL_SCAN_BLEND, true, (cudaStream_t)stream);
}
