// Log probabilities of the actions taken, entropy and best alternatives of rows of action values, and their gradient.
//
// With u_j = (x_j - m) / T for the row's largest available value m: S = sum e^u_j, log p_j = u_j - log S,
// entropy = log S - (sum e^u_j u_j) / S.  One pass over the row keeps (m, S, V = sum e^u u) and rescales S and V when m grows:
// e^(u + d) = e^u e^d, so S' = S e^d and V' = e^d (V + d S) for d = (m_old - m_new) / T.  Exponents are taken to base 2.
#include "learner_util.cuh"
#include "launch_util.cuh"

#include <algorithm>
#include <cmath>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace marl {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int LOGPROB_SMS = 148;
constexpr int KEY_NONE = INT32_MIN;          // no entry
constexpr int KEY_NEG_INF = (int)0x807FFFFF;  // the key of -infinity: entries rank above it

struct RowsParams {
  const void* x;
  const uint8_t* avail;
  const int32_t* action;
  long long rows, xs, as;
  int A, top;
  float it;    // 1 / temperature
  float c;     // log2(e) / temperature
  float *logp, *entropy;
  float2* stats;
  int32_t* top_index;
  float* top_logp;
  int parts;   // blocks a row
  int fours;   // the alternatives are written four at a time
};

struct RowsGradParams {
  RowsParams r;
  const float *g_logp, *g_entropy;
  void* dx;
  long long ds;
  int segments, seg_len;
};

// The larger value, NaN if either is one: a NaN among the available entries makes the row's maximum, and so its results, NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// An integer that orders like the value: equal for -0 and +0, NaN above +infinity.
__device__ __forceinline__ int order_key(float v) {
  const int b = __float_as_int(v + 0.0f);
  return v != v ? INT32_MAX : b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float key_value(int k) {
  if (k == -1) k = -2;  // (between the keys of zero and of the negative numbers lies that of -0, which no value has)
  return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF));
}

// Running sums of a part of a row.  Values are relative to m (to 0 while m is -infinity: every term is then 0).  Exponents below
// 2^-200 are clamped there: such a term is 0 in fp32, and stays 0 when it is multiplied by its exponent.
struct Sums {
  float m, s, v;
};
__device__ __forceinline__ float exponent(float x, float m, float c) { return max_nan((x - m) * c, -200.f); }
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void rescale(Sums& a, float m, float c) {  // m >= a.m
  const float d = a.m == m ? 0.f : exponent(a.m, base_of(m), c), f = ex2(d);
  a.v = f * (a.v + d * a.s);
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  const float m = max_nan(a.m, b.m);
  rescale(a, m, c);
  rescale(b, m, c);
  a.s += b.s;
  a.v += b.v;
  return a;
}
// The sums of all lanes, in every lane.
__device__ __forceinline__ void join_lanes(Sums& a, float c) {
  float m = a.m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(~0u, m, d));
  rescale(a, m, c);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, d);
    a.v += __shfl_xor_sync(~0u, a.v, d);
  }
}

// The row's results from its sums; x_a = the taken action's value if available, -infinity if it is not.
__device__ __forceinline__ void write_row(const RowsParams& p, long long row, const Sums& a, bool has_action, float x_a) {
  const bool empty = a.m == -INFINITY;
  const float ls = empty ? -INFINITY : logf(a.s);
  p.stats[row] = make_float2(a.m, ls);
  p.entropy[row] = empty ? 0.f : ls - a.v / a.s * LN2;
  p.logp[row] = empty || !has_action ? 0.f : (x_a - a.m) * p.it - ls;
}

// ---- the list of the best entries: one per lane of a warp, best first -----------------------------------------------
struct Entry {
  int key, idx;
};
__device__ __forceinline__ bool better(const Entry& a, const Entry& b) { return a.key > b.key || (a.key == b.key && a.idx < b.idx); }
__device__ __forceinline__ Entry entry_none() { return Entry{KEY_NONE, INT32_MAX}; }
__device__ __forceinline__ Entry shfl_entry(const Entry& e, int src) {
  return Entry{__shfl_sync(~0u, e.key, src), __shfl_sync(~0u, e.idx, src)};
}
__device__ __forceinline__ void exchange(Entry& e, int lane, int j, bool descending) {
  const Entry o{__shfl_xor_sync(~0u, e.key, j), __shfl_xor_sync(~0u, e.idx, j)};
  const bool keep_better = ((lane & j) == 0) == descending;
  if (better(o, e) == keep_better && (o.key != e.key || o.idx != e.idx)) e = o;
}
__device__ __forceinline__ void sort_list(Entry& e, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) exchange(e, lane, j, (lane & k) == 0);
}
// Both lists best first; a becomes the best 32 of both.
__device__ __forceinline__ void merge_list(Entry& a, const Entry& b, int lane) {
  const Entry o = shfl_entry(b, 31 - lane);
  if (better(o, a)) a = o;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) exchange(a, lane, j, true);
}

// Puts the values of the warp (lane l: v[0..N) at indexes i0 .. i0 + N - 1) that are at least `floor_key` into its list of the best 32;
// the top-th entry of the list decides what still enters.  Called by the whole warp.
template <int N>
__device__ __forceinline__ void take(Entry& mine, const float (&v)[N], int i0, int lane, int top, int floor_key) {
  unsigned used = 0;
  while (true) {
    const Entry worst = shfl_entry(mine, top - 1);
    Entry c = entry_none();
    int cj = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int k = order_key(v[j]);
      if (!(used >> j & 1) && k > c.key) {
        c = Entry{k, i0 + j};
        cj = j;
      }
    }
    const bool in = c.key > KEY_NEG_INF && c.key >= floor_key && better(c, worst);
    unsigned who = __ballot_sync(~0u, in);
    if (!who) return;
    if (in) used |= 1u << cj;
    if (__popc(who) <= 4) {  // one by one
      for (; who; who &= who - 1) {
        const Entry n = shfl_entry(c, __ffs(who) - 1);
        const int pos = __popc(__ballot_sync(~0u, better(mine, n)));
        const Entry up{__shfl_up_sync(~0u, mine.key, 1), __shfl_up_sync(~0u, mine.idx, 1)};
        if (lane == pos) mine = n;
        else if (lane > pos) mine = up;
      }
    } else {                 // the lanes' candidates sorted, then merged into the list
      Entry s = in ? c : entry_none();
      sort_list(s, lane);
      merge_list(mine, s, lane);
    }
  }
}

// The lanes' keys in descending order.
__device__ __forceinline__ int sort_keys(int key, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const int o = __shfl_xor_sync(~0u, key, j);
      key = ((lane & j) == 0) == ((lane & k) == 0) ? max(key, o) : min(key, o);
    }
  return key;
}
// The 32 largest of two descending lists, descending; `other` is read backwards.
__device__ __forceinline__ int merge_keys(int key, int other_reversed, int lane) {
  key = max(key, other_reversed);
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const int o = __shfl_xor_sync(~0u, key, j);
    key = (lane & j) == 0 ? max(key, o) : min(key, o);
  }
  return key;
}

// ---- 16 bytes of a row and their availability -----------------------------------------------------------------------
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <> struct Vec<__half> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
};

// N availability bytes that start anywhere, from the one or two aligned words they lie in (each holds at least one of them).
template <int N>
__device__ __forceinline__ void load_avail(const uint8_t* a, uint32_t (&w)[N / 4]) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a);
  const uint32_t* q = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3);
  const int sh = (int)(at & 3) * 8;
  uint32_t r[N / 4 + 1];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) r[i] = __ldg(q + i);
  r[N / 4] = sh ? __ldg(q + N / 4) : 0u;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) w[i] = __funnelshift_r(r[i], r[i + 1], sh);
}

// Two sums side by side (even and odd elements), in the packed fp32 arithmetic of the device.
struct Sums2 {
  float m;
  float2 s, v;
};
__device__ __forceinline__ void add_values(Sums2& a, float x0, float x1, float m, float c) {
  float2 u = mul2(add2(make_float2(x0, x1), make_float2(-m, -m)), make_float2(c, c));
  u.x = max_nan(u.x, -200.f);
  u.y = max_nan(u.y, -200.f);
  const float2 e = make_float2(ex2(u.x), ex2(u.y));
  a.s = add2(a.s, e);
  a.v = fma2(e, u, a.v);
}
template <int N>
__device__ __forceinline__ void add_values(Sums2& a, const float (&v)[N], float c) {
  float top = max_nan(v[0], v[1]);
#pragma unroll
  for (int j = 2; j < N; j += 2) top = max3_nan(top, v[j], v[j + 1]);
  if (!(top <= a.m)) {  // (also when top is NaN)
    Sums x{a.m, a.s.x, a.v.x}, y{a.m, a.s.y, a.v.y};
    top = max_nan(top, a.m);
    rescale(x, top, c);
    rescale(y, top, c);
    a = Sums2{top, make_float2(x.s, y.s), make_float2(x.v, y.v)};
  }
  const float m = base_of(a.m);
#pragma unroll
  for (int j = 0; j < N; j += 2) add_values(a, v[j], v[j + 1], m, c);
}

// ---- rows of more than SMALL_A actions ------------------------------------------------------------------------------
// WARPS warps of a block walk a row together, 16 bytes a lane, each warp every WARPS-th group of 512 bytes; with WARPS = 1 a block holds
// eight rows.  Few rows are divided over the blocks of a cluster in the same way.  A row that starts off a 16-byte boundary has up to 15
// bytes in front and behind that the first and the last warp take element by element.
// The alternatives cost the pass nothing: each lane knows the largest value that it has met, and the top-th largest of a block's such
// values is met or exceeded by at least `top` entries of the row.  Behind the pass only the lanes whose largest value reaches
// that bar are walked again, by their whole warp, from the cache.
constexpr int WIDE_THREADS = 256;

template <typename T, int WARPS, bool TOP, bool MASK>
__global__ void __launch_bounds__(WIDE_THREADS) logprob_wide_kernel(const __grid_constant__ RowsParams p) {
  constexpr int N = Vec<T>::N, ROWS = WIDE_THREADS / 32 / WARPS;
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) % WARPS, sub = (threadIdx.x >> 5) / WARPS;
  const int parts = WARPS > 1 ? p.parts : 1, rank = WARPS > 1 ? (int)(blockIdx.x % parts) : 0;
  const long long row = WARPS > 1 ? (long long)blockIdx.x / parts : (long long)blockIdx.x * ROWS + sub;
  if (row >= p.rows) return;  // (WARPS = 1 only: no barrier follows)
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs;
  const uint8_t* av = MASK ? p.avail + row * p.as : nullptr;
  const int off = (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T);
  const int head = off < p.A ? off : p.A, body = (p.A - head) / N, tail = p.A - head - body * N;
  const int stride = 32 * WARPS * parts, first = (rank * WARPS + warp) * 32;
  const bool does_head = head && first == 0, does_tail = tail && rank == parts - 1 && warp == WARPS - 1;

  Sums2 a2{-INFINITY, make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  auto load_one = [&](int i0, int n, float (&v)[N]) {  // n < N elements from i0 on, one a lane
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = -INFINITY;
    if (lane < n && (!MASK || av[i0 + lane])) v[0] = to_f32(x[i0 + lane]);
  };
  auto hide = [&](int i, float (&v)[N]) {
    uint32_t w[N / 4];
    load_avail<N>(av + head + (long long)i * N, w);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (!(w[j / 4] >> (8 * (j & 3)) & 0xFF)) v[j] = -INFINITY;
  };
  if (does_head) {
    float v[N];
    load_one(0, head, v);
    add_values<N>(a2, v, p.c);
  }
  int i = first + lane;
  for (; i + 3 * stride < body; i += 4 * stride) {  // four loads on their way at a time
    uint4 r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __ldg(xv + i + k * stride);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float v[N];
      Vec<T>::unpack(r[k], v);
      if (MASK) hide(i + k * stride, v);
      add_values<N>(a2, v, p.c);
    }
  }
  for (; i < body; i += stride) {
    float v[N];
    Vec<T>::unpack(__ldg(xv + i), v);
    if (MASK) hide(i, v);
    add_values<N>(a2, v, p.c);
  }
  __syncwarp();
  if (does_tail) {
    float v[N];
    load_one(head + body * N, tail, v);
    add_values<N>(a2, v, p.c);
  }

  const float lane_max = a2.m;
  Sums a{a2.m, a2.s.x + a2.s.y, a2.v.x + a2.v.y};
  join_lanes(a, p.c);
  __shared__ Sums part[WARPS];
  __shared__ int keys[TOP && WARPS > 1 ? WARPS : 1][32];
  __shared__ Entry lists[TOP && WARPS > 1 ? WARPS : 1][32];
  const int mine_key = TOP ? order_key(lane_max) : 0;
  int bar = TOP ? sort_keys(mine_key, lane) : 0;
  if (WARPS > 1) {
    if (lane == 0) part[warp] = a;
    if (TOP) {
#pragma unroll
      for (int w = 1; w < WARPS; w *= 2) {  // pairs of warps, pairs of pairs ...
        if (warp % (2 * w) == w) keys[warp][lane] = bar;
        __syncthreads();
        if (warp % (2 * w) == 0) bar = merge_keys(bar, keys[warp + w][31 - lane], lane);
      }
      if (warp == 0 && lane == p.top - 1) keys[0][0] = bar;
    }
    __syncthreads();
    if (TOP) bar = keys[0][0];
  } else if (TOP) bar = __shfl_sync(~0u, bar, p.top - 1);
  Entry best = entry_none();
  if (TOP) {
    float v[N];
    if (does_head) {
      load_one(0, head, v);
      take(best, v, lane, lane, p.top, bar);
    }
    // the walk of a lane is `steps` vectors, `stride` apart: as many lanes' as fit are read again at a time
    unsigned who = __ballot_sync(~0u, mine_key >= bar && mine_key > KEY_NEG_INF);
    const int steps = first < body ? (body - first + stride - 1) / stride : 0;
    int lg = 0;
    while ((1 << lg) < steps && lg < 5) ++lg;
    while (who) {
      unsigned m = who;
      for (int k = lane >> lg; k && m; --k) m &= m - 1;
      const int l = m ? __ffs(m) - 1 : 0;
      for (int s0 = 0; s0 < steps; s0 += 1 << lg) {
        const long long k = first + l + (long long)(s0 + (lane & ((1 << lg) - 1))) * stride;
        if (m && k < body) {
          Vec<T>::unpack(__ldg(xv + k), v);
          if (MASK) hide((int)k, v);
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] = -INFINITY;
        }
        take(best, v, head + (int)k * N, lane, p.top, bar);
      }
      for (int k = 32 >> lg; k && who; --k) who &= who - 1;
    }
    if (does_tail) {
      load_one(head + body * N, tail, v);
      take(best, v, head + body * N + lane, lane, p.top, bar);
    }
  }
  if (WARPS > 1) {
    if (TOP) lists[warp][lane] = best;
    __syncthreads();
    if (warp == 0) {
#pragma unroll 1
      for (int w = 1; w < WARPS; ++w) {
        a = join(a, part[w], p.c);
        if (TOP) merge_list(best, lists[w][lane], lane);
      }
    }
    if (parts > 1) {  // the blocks' sums and lists, in the order of their ranks
      cg::cluster_group cluster = cg::this_cluster();
      if (warp == 0) {
        if (lane == 0) part[0] = a;
        if (TOP) lists[0][lane] = best;
      }
      cluster.sync();
      if (rank == 0 && warp == 0) {
        for (int r = 1; r < parts; ++r) {
          a = join(a, *cluster.map_shared_rank(&part[0], r), p.c);
          if (TOP) merge_list(best, *cluster.map_shared_rank(&lists[0][lane], r), lane);
        }
      }
      cluster.sync();
      if (rank) return;
    }
    if (warp) return;
  }
  if (lane == 0) {
    const int act = p.action[row];
    const bool has = act >= 0 && act < p.A;
    write_row(p, row, a, has, has && (!MASK || av[act]) ? to_f32(x[act]) : -INFINITY);
  }
  if (TOP && lane < p.top) {
    const bool some = best.key > KEY_NEG_INF;
    p.top_index[row * p.top + lane] = some ? best.idx : -1;
    p.top_logp[row * p.top + lane] = some ? (to_f32(x[best.idx]) - a.m) * p.it - logf(a.s) : -INFINITY;
  }
}

// ---- rows of up to SMALL_A actions ----------------------------------------------------------------------------------
// A thread per row: 128 rows come in with neighbouring threads on neighbouring elements and are laid out in shared memory an odd number of
// words apart, so that the threads' walks over their rows meet no bank twice.  DENSE: rows without gaps on 16-byte boundaries (the q of a
// sampled batch) come in four elements a load.
constexpr int SMALL_A = 32, SMALL_ROWS = 128;

// i / A for i < 4096, A <= 32: inv = ceil(2^20 / A).
__device__ __forceinline__ int div_small(int i, uint32_t inv) { return (int)((uint32_t)i * inv >> 20); }

template <typename T> struct Four;
template <> struct Four<float> {
  static __device__ __forceinline__ void load(const float* at, float (&v)[4]) { *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(at); }
  static __device__ __forceinline__ void store(float* at, const float (&v)[4]) { *reinterpret_cast<float4*>(at) = *reinterpret_cast<const float4*>(v); }
};
template <typename T> struct Four16 {
  static __device__ __forceinline__ void load(const T* at, float (&v)[4]) {
    const uint2 r = *reinterpret_cast<const uint2*>(at);
    const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = to_f32(e[k]);
  }
  static __device__ __forceinline__ void store(T* at, const float (&v)[4]) {
    uint2 r;
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = from_f32<T>(v[k]);
    *reinterpret_cast<uint2*>(at) = r;
  }
};
template <> struct Four<__nv_bfloat16> : Four16<__nv_bfloat16> {};
template <> struct Four<__half> : Four16<__half> {};

template <typename T, int MA, bool DENSE>
__global__ void __launch_bounds__(SMALL_ROWS) logprob_small_kernel(const __grid_constant__ RowsParams p, uint32_t inv_a) {
  __shared__ float xs[SMALL_ROWS * (MA + 1)];
  const long long row0 = (long long)blockIdx.x * SMALL_ROWS;
  const int rows = (int)(p.rows - row0 < SMALL_ROWS ? p.rows - row0 : SMALL_ROWS), A = p.A, pitch = A | 1, pad = pitch - A;
  const T* x = reinterpret_cast<const T*>(p.x) + row0 * p.xs;
  const uint8_t* av = p.avail ? p.avail + row0 * p.as : nullptr;
  const int total = rows * A, fours = DENSE ? total >> 2 : 0;
#pragma unroll 4
  for (int q = threadIdx.x; q < fours; q += SMALL_ROWS) {
    float v[4];
    Four<T>::load(x + 4 * q, v);
    const uint32_t w = av ? __ldg(reinterpret_cast<const uint32_t*>(av) + q) : 0x01010101u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * q + e;
      xs[i + pad * div_small(i, inv_a)] = w >> (8 * e) & 0xFF ? v[e] : -INFINITY;
    }
  }
#pragma unroll 4
  for (int i = 4 * fours + threadIdx.x; i < total; i += SMALL_ROWS) {
    const int r = div_small(i, inv_a), j = i - r * A;
    float v = to_f32(x[r * p.xs + j]);
    if (av && !av[r * p.as + j]) v = -INFINITY;
    xs[r * pitch + j] = v;
  }
  __syncthreads();
  const int r = threadIdx.x;
  if (r >= rows) return;
  const float* mine = xs + r * pitch;
  float v[MA];
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < MA; ++j) {
    v[j] = j < A ? mine[j] : -INFINITY;
    m = max_nan(m, v[j]);
  }
  Sums2 a2{m, make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
  const float b = base_of(m);
#pragma unroll
  for (int j = 0; j < MA; j += 2) add_values(a2, v[j], v[j + 1], b, p.c);
  const Sums a{m, a2.s.x + a2.s.y, a2.v.x + a2.v.y};
  const long long row = row0 + r;
  const int act = p.action[row];
  const bool has = act >= 0 && act < A;
  write_row(p, row, a, has, has ? mine[act] : -INFINITY);
  if (!p.top) return;
  const float ls = logf(a.s);
  if (m != m) {  // a NaN ranks above all numbers: +infinity in its place, and that below it
#pragma unroll
    for (int j = 0; j < MA; ++j) v[j] = v[j] != v[j] ? INFINITY : v[j] == INFINITY ? 3.402823466e38f : v[j];
  }
  int out_j[4];
  float out_l[4];
  for (int k0 = 0; k0 < p.top; k0 += 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float top = -INFINITY;
      int bj = -1;
#pragma unroll
      for (int j = 0; j < MA; ++j)
        if (v[j] > top) {
          top = v[j];
          bj = j;
        }
#pragma unroll
      for (int j = 0; j < MA; ++j)
        if (j == bj) v[j] = -INFINITY;
      out_j[k] = bj;
      out_l[k] = bj >= 0 ? (mine[bj] - a.m) * p.it - ls : -INFINITY;
      if (k0 + k + 1 >= p.top) break;
    }
    int* ti = p.top_index + row * p.top + k0;
    float* tl = p.top_logp + row * p.top + k0;
    if (p.fours) {
      *reinterpret_cast<int4*>(ti) = *reinterpret_cast<int4*>(out_j);
      *reinterpret_cast<float4*>(tl) = *reinterpret_cast<float4*>(out_l);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k0 + k < p.top) {
          ti[k] = out_j[k];
          tl[k] = out_l[k];
        }
    }
  }
}

// ---- gradient -------------------------------------------------------------------------------------------------------
// With l = log2 p_j: dx_j = -p_j (k + h l), and g more at the action taken; k = g + h entropy, h in natural units of l.
struct RowGrad {
  float m, ls2, k, h, g;  // largest value, log2 S
  int action;             // -1: none
};
__device__ __forceinline__ RowGrad row_grad(const RowsGradParams& q, long long row) {
  const float2 st = q.r.stats[row];
  RowGrad r{0.f, 0.f, 0.f, 0.f, 0.f, -1};
  if (st.y == -INFINITY) return r;  // an empty row: nothing in it is available
  const int act = q.r.action[row];
  if (act >= 0 && act < q.r.A) {
    r.action = act;
    r.g = q.g_logp ? q.g_logp[row] * q.r.it : 0.f;
  }
  const float h = q.g_entropy ? q.g_entropy[row] * q.r.it : 0.f;
  r.m = st.x;
  r.ls2 = st.y * LOG2E;
  r.h = h * LN2;
  r.k = r.g + h * q.r.entropy[row];
  return r;
}
// x of an available entry, or -infinity: 0 then.
__device__ __forceinline__ float entry_grad(float m, float ls2, float k, float h, float x, float c) {
  const float l = max_nan((x - m) * c - ls2, -200.f);
  return -ex2(l) * fmaf(h, l, k);
}

// A warp per segment of a row of more than SMALL_A actions, 16 bytes of the gradient a lane.  Where the logits' rows lie otherwise than the
// gradient's from a 16-byte boundary, each lane takes its logits from the two aligned vectors that hold them, the second from the
// lane behind it.
template <typename T, bool MASK>
__global__ void __launch_bounds__(256) logprob_wide_grad_kernel(const __grid_constant__ RowsGradParams q) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long row = unit / q.segments;
  if (row >= q.r.rows) return;
  const int segment = (int)(unit - row * q.segments), A = q.r.A;
  const RowGrad g = row_grad(q, row);
  const T* x = reinterpret_cast<const T*>(q.r.x) + row * q.r.xs;
  const uint8_t* av = MASK ? q.r.avail + row * q.r.as : nullptr;
  T* d = reinterpret_cast<T*>(q.dx) + row * q.ds;
  const float c = q.r.c;
  const int off = (int)((16 - (reinterpret_cast<uintptr_t>(d) & 15)) & 15) / (int)sizeof(T);
  const int head = off < A ? off : A, body = (A - head) / N, tail = A - head - body * N;
  auto single = [&](int j) {
    float v = to_f32(x[j]);
    if (MASK && !av[j]) v = -INFINITY;
    float o = entry_grad(g.m, g.ls2, g.k, g.h, v, c);
    if (j == g.action && v != -INFINITY) o += g.g;
    d[j] = from_f32<T>(o);
  };
  if (segment == 0 && lane < head) single(lane);
  if (segment == q.segments - 1 && lane < tail) single(head + body * N + lane);
  const int i0 = segment * q.seg_len, i1 = min(body, i0 + q.seg_len);  // vectors
  const uintptr_t xa = reinterpret_cast<uintptr_t>(x + head);
  const uint4* xv = reinterpret_cast<const uint4*>(xa & ~(uintptr_t)15);
  const int shift = (int)(xa & 15);                                    // bytes
  constexpr int BATCH = 4;  // vectors on their way at a time (the gradient may be written over the logits: no load moves up past a store)
  for (int b = i0; b < i1; b += 32 * BATCH) {
    uint4 raw[BATCH], next[BATCH];
    uint32_t w[BATCH][N / 4];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b + 32 * k + lane;
      raw[k] = next[k] = make_uint4(0u, 0u, 0u, 0u);
      if (i >= i1) continue;
      raw[k] = *(xv + i);
      if (shift && (lane == 31 || i + 1 == i1)) next[k] = *(xv + i + 1);
      if (MASK) load_avail<N>(av + head + i * N, w[k]);
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b + 32 * k + lane;
      uint4 r = raw[k];
      if (shift) {
        uint4 n{__shfl_down_sync(~0u, r.x, 1), __shfl_down_sync(~0u, r.y, 1), __shfl_down_sync(~0u, r.z, 1), __shfl_down_sync(~0u, r.w, 1)};
        if (lane == 31 || i + 1 == i1) n = next[k];
        uint32_t t[8] = {r.x, r.y, r.z, r.w, n.x, n.y, n.z, n.w};
        if (shift & 8) {
#pragma unroll
          for (int e = 0; e < 6; ++e) t[e] = t[e + 2];
        }
        if (shift & 4) {
#pragma unroll
          for (int e = 0; e < 5; ++e) t[e] = t[e + 1];
        }
        const int sh = (shift & 3) * 8;
        r = make_uint4(__funnelshift_r(t[0], t[1], sh), __funnelshift_r(t[1], t[2], sh), __funnelshift_r(t[2], t[3], sh), __funnelshift_r(t[3], t[4], sh));
      }
      if (i >= i1) continue;
      float v[N], o[N];
      Vec<T>::unpack(r, v);
      const int j0 = head + i * N;
      if (MASK) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (!(w[k][j / 4] >> (8 * (j & 3)) & 0xFF)) v[j] = -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) o[j] = entry_grad(g.m, g.ls2, g.k, g.h, v[j], c);
      if ((unsigned)(g.action - j0) < (unsigned)N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j0 + j == g.action && v[j] != -INFINITY) o[j] += g.g;
      }
      uint4 s;
      T* e = reinterpret_cast<T*>(&s);
#pragma unroll
      for (int j = 0; j < N; ++j) e[j] = from_f32<T>(o[j]);
      reinterpret_cast<uint4*>(d + head)[i] = s;
    }
  }
}

// 128 rows a block, neighbouring threads on neighbouring elements, four at a time where all rows are dense.
template <typename T, bool DENSE>
__global__ void __launch_bounds__(SMALL_ROWS) logprob_small_grad_kernel(const __grid_constant__ RowsGradParams q, uint32_t inv_a) {
  __shared__ float4 gs[SMALL_ROWS];
  __shared__ float2 chosen[SMALL_ROWS];  // gradient, and place (as bits) of the action taken in the block's rows laid end to end
  const long long row0 = (long long)blockIdx.x * SMALL_ROWS;
  const int rows = (int)(q.r.rows - row0 < SMALL_ROWS ? q.r.rows - row0 : SMALL_ROWS), A = q.r.A;
  if ((int)threadIdx.x < rows) {
    const RowGrad g = row_grad(q, row0 + threadIdx.x);
    gs[threadIdx.x] = make_float4(g.m, g.ls2, g.k, g.h);
    chosen[threadIdx.x] = make_float2(g.g, __int_as_float(g.action >= 0 ? (int)threadIdx.x * A + g.action : -1));
  }
  __syncthreads();
  const T* x = reinterpret_cast<const T*>(q.r.x) + row0 * q.r.xs;
  const uint8_t* av = q.r.avail ? q.r.avail + row0 * q.r.as : nullptr;
  T* d = reinterpret_cast<T*>(q.dx) + row0 * q.ds;
  auto gradient = [&](float v, int r, int i) {
    const float4 g = gs[r];
    const float2 t = chosen[r];
    float o = entry_grad(g.x, g.y, g.z, g.w, v, q.r.c);
    if (__float_as_int(t.y) == i && v != -INFINITY) o += t.x;
    return o;
  };
  const int total = rows * A, fours = DENSE ? total >> 2 : 0;
  constexpr int BATCH = 4;
  for (int b = threadIdx.x; b < fours; b += BATCH * SMALL_ROWS) {
    float v[BATCH][4];
    uint32_t w[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b + k * SMALL_ROWS;
      if (i >= fours) break;
      Four<T>::load(x + 4 * i, v[k]);
      w[k] = av ? reinterpret_cast<const uint32_t*>(av)[i] : 0x01010101u;
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b + k * SMALL_ROWS;
      if (i >= fours) break;
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[e] = gradient(w[k] >> (8 * e) & 0xFF ? v[k][e] : -INFINITY, div_small(4 * i + e, inv_a), 4 * i + e);
      Four<T>::store(d + 4 * i, o);
    }
  }
#pragma unroll 4
  for (int i = 4 * fours + threadIdx.x; i < total; i += SMALL_ROWS) {
    const int r = div_small(i, inv_a), j = i - r * A;
    float v = to_f32(x[r * q.r.xs + j]);
    if (av && !av[r * q.r.as + j]) v = -INFINITY;
    d[r * q.ds + j] = from_f32<T>(gradient(v, r, i));
  }
}

static int check_rows(const marl_policy_rows_t* in) {
  if (!in) return fail(MARL_EINVAL, "rows descriptor is NULL");
  if (in->rows < 0 || in->rows > (1ll << 40)) return fail(MARL_EINVAL, "rows must be in [0, 2^40]");
  if (in->n_actions < 1 || in->n_actions > (1 << 30)) return fail(MARL_EINVAL, "n_actions must be in [1, 2^30]");
  if (!dtype_known(in->dtype)) return fail(MARL_EINVAL, "unknown dtype %d", in->dtype);
  if (!(in->temperature > 0.f) || !(1.f / in->temperature > 0.f) || !std::isfinite(1.f / in->temperature * LOG2E))
    return fail(MARL_EINVAL, "temperature must be positive and finite, and so its reciprocal");
  if (in->rows == 0) return MARL_OK;
  if (!in->logits || !in->action) return fail(MARL_EINVAL, "logits or action is NULL");
  if (in->row_stride < 0 || in->avail_stride < 0) return fail(MARL_EINVAL, "a row stride is negative");
  if (misaligned(in->logits, dtype_bytes(in->dtype)) || misaligned(in->action, 4))
    return fail(MARL_EALIGN, "logits or action is not aligned to its elements");
  return MARL_OK;
}

static RowsParams rows_params(const marl_policy_rows_t* in) {
  RowsParams p = {};
  p.x = in->logits;
  p.avail = in->avail;
  p.action = in->action;
  p.rows = in->rows;
  p.xs = in->row_stride;
  p.as = in->avail_stride;
  p.A = in->n_actions;
  p.it = 1.f / in->temperature;
  p.c = (float)(1.4426950408889634 / (double)in->temperature);
  return p;
}

static int launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? MARL_OK : fail(MARL_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Rows without gaps, on boundaries that four elements and four bytes of availability need.
template <typename T>
static bool rows_dense(const RowsParams& p) {
  return p.xs == p.A && !misaligned(p.x, 4 * sizeof(T)) && (!p.avail || (p.as == p.A && !misaligned(p.avail, 4)));
}

template <typename T>
static int launch_logprob(const RowsParams& p, cudaStream_t stream) {
  if (p.A <= SMALL_A) {
    const long long blocks = (p.rows + SMALL_ROWS - 1) / SMALL_ROWS;
    if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
    const uint32_t inv = ((1u << 20) + p.A - 1) / p.A;
    RowsParams q = p;
    q.fours = p.top % 4 == 0 && !misaligned(p.top_index, 16) && !misaligned(p.top_logp, 16);
    const bool dense = rows_dense<T>(p);
    auto go = [&](auto kernel) { kernel<<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(q, inv); };
    if (p.A <= 8) dense ? go(logprob_small_kernel<T, 8, true>) : go(logprob_small_kernel<T, 8, false>);
    else if (p.A <= 16) dense ? go(logprob_small_kernel<T, 16, true>) : go(logprob_small_kernel<T, 16, false>);
    else dense ? go(logprob_small_kernel<T, 32, true>) : go(logprob_small_kernel<T, 32, false>);
    return launched("marl_policy_logprob");
  }
  const bool warp_rows = p.A <= 2048;
  RowsParams q = p;
  q.parts = 1;
  if (!warp_rows)
    while (q.parts < 8 && p.rows * q.parts * 2 <= 2 * LOGPROB_SMS && p.A / (q.parts * 2) >= 4096) q.parts *= 2;
  const long long blocks = warp_rows ? (p.rows + 7) / 8 : p.rows * q.parts;
  if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)blocks);
  lc.blockDim = dim3(WIDE_THREADS);
  lc.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)q.parts;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = q.parts > 1 ? 1 : 0;
  cudaError_t err = cudaSuccess;
  auto go = [&](auto kernel) { err = cudaLaunchKernelEx(&lc, kernel, q); };
  if (warp_rows) {
    if (p.top) p.avail ? go(logprob_wide_kernel<T, 1, true, true>) : go(logprob_wide_kernel<T, 1, true, false>);
    else p.avail ? go(logprob_wide_kernel<T, 1, false, true>) : go(logprob_wide_kernel<T, 1, false, false>);
  } else {
    if (p.top) p.avail ? go(logprob_wide_kernel<T, 8, true, true>) : go(logprob_wide_kernel<T, 8, true, false>);
    else p.avail ? go(logprob_wide_kernel<T, 8, false, true>) : go(logprob_wide_kernel<T, 8, false, false>);
  }
  if (err != cudaSuccess) return fail(MARL_ECUDA, "marl_policy_logprob: %s", cudaGetErrorString(err));
  return launched("marl_policy_logprob");
}

template <typename T>
static int launch_logprob_grad(RowsGradParams q, cudaStream_t stream) {
  if (q.r.A <= SMALL_A) {
    const long long blocks = (q.r.rows + SMALL_ROWS - 1) / SMALL_ROWS;
    if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
    const uint32_t inv = ((1u << 20) + q.r.A - 1) / q.r.A;
    if (rows_dense<T>(q.r) && q.ds == q.r.A && !misaligned(q.dx, 4 * sizeof(T)))
      logprob_small_grad_kernel<T, true><<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(q, inv);
    else logprob_small_grad_kernel<T, false><<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(q, inv);
    return launched("marl_policy_logprob_backward");
  }
  q.seg_len = q.r.A > 32768 ? 1024 : 256;
  q.segments = std::max(1, (q.r.A / Vec<T>::N + q.seg_len - 1) / q.seg_len);
  const long long units = q.r.rows * q.segments, blocks = (units + 7) / 8;
  if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
  if (q.r.avail) logprob_wide_grad_kernel<T, true><<<(unsigned)blocks, 256, 0, stream>>>(q);
  else logprob_wide_grad_kernel<T, false><<<(unsigned)blocks, 256, 0, stream>>>(q);
  return launched("marl_policy_logprob_backward");
}

}  // namespace marl

using namespace marl;

extern "C" int marl_policy_logprob(void* stream, const marl_policy_rows_t* in, int32_t top, float* logp, float* entropy,
                                   float* stats, int32_t* top_index, float* top_logp) {
  const int rc = check_rows(in);
  if (rc != MARL_OK) return rc;
  if (top < 0 || top > MARL_MAX_TOP) return fail(MARL_EINVAL, "top must be in [0, %d]", MARL_MAX_TOP);
  if (in->rows == 0) return MARL_OK;
  if (!logp || !entropy || !stats || (top && (!top_index || !top_logp))) return fail(MARL_EINVAL, "an output pointer is NULL");
  if (misaligned(logp, 4) || misaligned(entropy, 4) || misaligned(stats, 8) || (top && (misaligned(top_index, 4) || misaligned(top_logp, 4))))
    return fail(MARL_EALIGN, "an output is not aligned to its elements (stats: 8 bytes)");
  RowsParams p = rows_params(in);
  p.top = top;
  p.logp = logp;
  p.entropy = entropy;
  p.stats = reinterpret_cast<float2*>(stats);
  p.top_index = top_index;
  p.top_logp = top_logp;
  return by_dtype(in->dtype, [&](auto t) { return launch_logprob<decltype(t)>(p, (cudaStream_t)stream); });
}

extern "C" int marl_policy_logprob_backward(void* stream, const marl_policy_rows_t* in, const float* stats, const float* entropy,
                                            const float* g_logp, const float* g_entropy, void* dlogits, int64_t dlogits_stride) {
  const int rc = check_rows(in);
  if (rc != MARL_OK) return rc;
  if (in->rows == 0) return MARL_OK;
  if (!stats || !entropy || !dlogits) return fail(MARL_EINVAL, "stats, entropy or dlogits is NULL");
  if (dlogits_stride < in->n_actions) return fail(MARL_EINVAL, "dlogits_stride is smaller than n_actions");
  if (misaligned(stats, 8) || misaligned(entropy, 4) || misaligned(g_logp, 4) || misaligned(g_entropy, 4) ||
      misaligned(dlogits, dtype_bytes(in->dtype)))
    return fail(MARL_EALIGN, "an array is not aligned to its elements (stats: 8 bytes)");
  RowsGradParams q = {};
  q.r = rows_params(in);
  q.r.stats = reinterpret_cast<float2*>(const_cast<float*>(stats));
  q.r.entropy = const_cast<float*>(entropy);
  q.g_logp = g_logp;
  q.g_entropy = g_entropy;
  q.dx = dlogits;
  q.ds = dlogits_stride;
  return by_dtype(in->dtype, [&](auto t) { return launch_logprob_grad<decltype(t)>(q, (cudaStream_t)stream); });
}
