// Log probabilities of the actions taken, entropy and best alternatives of rows of action values, and their gradient.
//
// With u_j = (x_j - m) / T for the row's largest available value m: S = sum e^u_j, log p_j = u_j - log S,
// entropy = log S - (sum e^u_j u_j) / S.  One pass over the row keeps (m, S, V = sum e^u u) and rescales S and V when m grows:
// e^(u + d) = e^u e^d, so S' = S e^d and V' = e^d (V + d S) for d = (m_old - m_new) / T.  Exponents are taken to base 2.
//
// Three forms of the pass: a thread per row up to 32 actions, a warp per row up to 4096, a block per row beyond, or the blocks of a cluster
// where there are few rows.  Bytes bound all of them on paper; what bounds them measured:
//   1024 x 96 x 8 rows of 14, fp32, availability: 16.6 us without alternatives (4.3 TB/s), 27.5 us with four - the ranking's integer
//     minima and maxima run at half rate - and 20.0 us for the gradient (5.9 TB/s); 52 us with four where most rows' values lie within 32 steps
//     of fp32 of each other (20 + N(0, 1e-4)) and are ranked one by one
//   2048 rows of 65537, bf16: 50 us without alternatives (5.4 TB/s), 71 us with eight - the rows' ends are chains of shuffles, barriers and
//     reads, which the other blocks of the multiprocessor cover only in part - and 94 us for the gradient (5.7 TB/s)
//   one row of 131072: 12 us on a cluster of eight blocks (49 us on one block)
#include "learner_util.cuh"
#include "launch_util.cuh"

#include <algorithm>
#include <cmath>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace marl {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
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

// An integer that orders like the value: equal for -0 and +0, NaN above +infinity.
__device__ __forceinline__ int order_key(float v) {
  const int b = __float_as_int(v + 0.0f);
  return v != v ? INT32_MAX : b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float key_value(int k) {
  if (k == -1) k = -2;  // (between the keys of zero and of the negative numbers lies that of -0, which no value has)
  return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF));
}

// Running sums of a part of a row, relative to the largest value m: the largest term is 1 exactly.
// Values below a floor are raised to it, unavailable ones among them, so that no exponent is infinite (a term of 0 times an infinite exponent
// would be NaN); m starts there.  A row whose floor is not far below its largest value - empty rows, rows of the type's lowest
// numbers, NaN, infinities, extreme temperatures (fp16: from some 630 on, its lowest number being the floor) - is walked once more, carefully, by one
// warp.  That is what such rows cost: 2048 x 65537 774 us against 54, 100000 x 200 59 us against 36.
struct Sums {
  float m, s, v;
};
// log2 of the factor between sums relative to m and to the larger m_new; 2^-200 is 0 in fp32
__device__ __forceinline__ float step_down(float m, float m_new, float c) { return max_nan((m - m_new) * c, -200.f); }
__device__ __forceinline__ void rescale(Sums& a, float m, float c) {
  const float d = step_down(a.m, m, c), f = ex2(d);
  a.v = f * (a.v + d * a.s);
  a.s *= f;
  a.m = m;
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
__device__ __forceinline__ bool trusted(const Sums& a, float floor_value, float c) {
  const float u = (floor_value - a.m) * c;
  return u <= -150.f && u >= -1.0e38f;
}
// The exponent of x relative to m, by a difference that cannot overflow to the wrong side; m = -infinity: no entry has been met.
__device__ __forceinline__ float exponent(float x, float m, float c) { return max_nan((x - (m == -INFINITY ? 0.f : m)) * c, -200.f); }

// The row's results from its sums; x_a = the taken action's value if available, -infinity if it is not.  Returns log S.
__device__ __forceinline__ float write_row(const RowsParams& p, long long row, const Sums& a, bool has_action, float x_a) {
  const bool empty = a.m == -INFINITY;
  const float ls = empty ? -INFINITY : logf(a.s);
  p.stats[row] = make_float2(a.m, ls);
  p.entropy[row] = empty ? 0.f : ls - a.v / a.s * LN2;
  p.logp[row] = empty || !has_action ? 0.f : (x_a - a.m) * p.it - ls;
  return ls;
}

// The sums of n elements, by one warp, whatever their values.
template <typename T>
__device__ __noinline__ Sums careful_sums(const T* x, const uint8_t* av, int n, float c, int lane) {
  Sums a{-INFINITY, 0.f, 0.f};
  for (int i = lane; i < n; i += 32)
    if (!av || av[i]) a.m = max_nan(a.m, to_f32(x[i]));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) a.m = max_nan(a.m, __shfl_xor_sync(~0u, a.m, d));
  for (int i = lane; i < n; i += 32) {
    const float v = to_f32(x[i]);
    if ((av && !av[i]) || v == -INFINITY) continue;
    const float u = exponent(v, a.m, c), e = ex2(u);
    a.s += e;
    a.v += e * u;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, d);
    a.v += __shfl_xor_sync(~0u, a.v, d);
  }
  return a;
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

// The n-th best of the lanes' entries, in every lane.
__device__ __forceinline__ Entry nth_best(Entry e, int n, int lane) {
  if (n > 8) {
    sort_list(e, lane);
    return shfl_entry(e, n - 1);
  }
  Entry b = entry_none();
  for (int r = 0; r < n; ++r) {
    b.key = __reduce_max_sync(~0u, e.key);
    b.idx = __reduce_min_sync(~0u, e.key == b.key ? e.idx : INT32_MAX);
    if (e.key == b.key && e.idx == b.idx) e = entry_none();
  }
  return b;
}

// The alternatives of a row, after the pass over it.  Each lane knows the largest value that it met and the vector of N entries in which
// it met it first: lane l has an entry of key k_l at an index below at_l + N.  Let (k, at) be one of these pairs with at least `top`
// pairs as good as it (higher key, or equal key and at most its index).  Then at least `top` entries are as good as (k, at + N - 1), so
// the best `top` are among those that are, and only the lanes whose pair is as good can hold one.  (A lane that met a NaN notes
// the last vector, not the first: all such lanes count.)  Those lanes' vectors are walked again, from the cache, and the entries that pass
// are collected: about `top` of them on values in no particular order, and no more for rows of equal values.
struct Bar {
  Entry e;
  float value;
};
__device__ __forceinline__ Bar make_bar(const Entry& e) { return Bar{e, e.key <= KEY_NEG_INF ? -INFINITY : e.key == INT32_MAX ? NAN : key_value(e.key)}; }
// (a lane with nothing above the floor has no pair)
__device__ __forceinline__ Entry lane_entry(float largest, int at, float floor_value) {
  return largest <= floor_value ? entry_none() : Entry{order_key(largest), at};
}
__device__ __forceinline__ bool reaches(const Entry& e, const Entry& bar) {
  return bar.key <= KEY_NEG_INF || e.key > bar.key || (e.key == bar.key && (e.idx <= bar.idx || e.key == INT32_MAX));
}
template <int N, int CAP>
__device__ __forceinline__ void collect(const float (&v)[N], int i0, const Bar& bar, Entry* found, int* count) {
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (!(v[j] < bar.value) && v[j] != -INFINITY) {
      const Entry e{order_key(v[j]), i0 + j};
      if (e.key > bar.e.key || (e.key == bar.e.key && e.idx - N < bar.e.idx)) {
        const int at = atomicAdd(count, 1);  // (their order does not matter: they are sorted by value and index)
        if (at < CAP) found[at] = e;
      }
    }
}
// The best `top` of n entries, one a lane, best first.
__device__ __forceinline__ Entry best_of(const Entry* found, int n, int top, int lane) {
  Entry best = lane < n ? found[lane] : entry_none();
  if (n <= 32 && top <= 8) {  // one by one
    Entry out = entry_none();
    for (int r = 0; r < top; ++r) {
      const int key = __reduce_max_sync(~0u, best.key), idx = __reduce_min_sync(~0u, best.key == key ? best.idx : INT32_MAX);
      if (best.idx == idx) best = entry_none();
      if (lane == r) out = Entry{key, idx};
    }
    return out;
  }
  sort_list(best, lane);
  for (int b = 32; b < n; b += 32) {
    Entry e = b + lane < n ? found[b + lane] : entry_none();
    sort_list(e, lane);
    merge_list(best, e, lane);
  }
  return best;
}
// More entries than there is room for (many large values in few lanes): the warp walks the elements [i0, i1) one by one (2048 x 65537 bf16, the large
// values eight in a row every 1024, eight alternatives: 1060 us against 75).
template <typename T>
__device__ __noinline__ void walk(Entry& best, const T* x, const uint8_t* av, int i0, int i1, int top, int lane) {
  for (int b = i0; b < i1; b += 32) {
    const int i = b + lane;
    Entry e = entry_none();
    if (i < i1 && (!av || av[i])) e = Entry{order_key(to_f32(x[i])), i};
    const Entry worst = shfl_entry(best, top - 1);
    const bool in = e.key > KEY_NEG_INF && better(e, worst);
    unsigned who = __ballot_sync(~0u, in);
    if (__popc(who) > 4) {
      if (!in) e = entry_none();
      sort_list(e, lane);
      merge_list(best, e, lane);
      continue;
    }
    for (; who; who &= who - 1) {
      const Entry n = shfl_entry(e, __ffs(who) - 1);
      const int pos = __popc(__ballot_sync(~0u, better(best, n)));
      const Entry up{__shfl_up_sync(~0u, best.key, 1), __shfl_up_sync(~0u, best.idx, 1)};
      if (lane == pos) best = n;
      else if (lane > pos) best = up;
    }
  }
}

// ---- 16 bytes of a row and their availability -----------------------------------------------------------------------
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t sel) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(r) : "r"(a), "r"(sel));
  return r;
}
// The highest bit of each byte, set where the byte is not 0.
__device__ __forceinline__ uint32_t nonzero_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w; }

// FLOOR: what values are raised to (-2^100; for fp16 its lowest number).  hide<BITS>: unavailable entries become BITS.
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t FLOOR_BITS = 0xF1800000u, NEG_INF_BITS = 0xFF800000u;
  static __device__ __forceinline__ float floor_value() { return __uint_as_float(FLOOR_BITS); }
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  }
  template <uint32_t F>
  static __device__ __forceinline__ void hide(uint4& r, const uint32_t (&w)[1]) {
    const uint32_t t = nonzero_bytes(w[0]);
    const uint32_t a = prmt(t, 0x8888), b = prmt(t, 0x9999), c = prmt(t, 0xAAAA), d = prmt(t, 0xBBBB);
    r.x = (r.x & a) | (F & ~a);
    r.y = (r.y & b) | (F & ~b);
    r.z = (r.z & c) | (F & ~c);
    r.w = (r.w & d) | (F & ~d);
  }
  static __device__ __forceinline__ uint32_t raise(uint32_t w) { return __float_as_uint(max_nan(__uint_as_float(w), floor_value())); }
  static __device__ __forceinline__ float largest(const uint4& r) {
    return max_nan(max_nan(__uint_as_float(r.x), __uint_as_float(r.y)), max_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
  }
};
template <typename T> struct Vec16 {
  static constexpr int N = 8;
  template <uint32_t F>
  static __device__ __forceinline__ void hide(uint4& r, const uint32_t (&w)[2]) {
    const uint32_t t = nonzero_bytes(w[0]), u = nonzero_bytes(w[1]);
    const uint32_t a = prmt(t, 0x9988), b = prmt(t, 0xBBAA), c = prmt(u, 0x9988), d = prmt(u, 0xBBAA);
    r.x = (r.x & a) | (F & ~a);
    r.y = (r.y & b) | (F & ~b);
    r.z = (r.z & c) | (F & ~c);
    r.w = (r.w & d) | (F & ~d);
  }
  static __device__ __forceinline__ uint32_t raise(uint32_t w) { return Vec<T>::max2(w, Vec<T>::FLOOR_BITS); }
  static __device__ __forceinline__ float largest(const uint4& r) {
    float a, b;
    Vec<T>::pair(Vec<T>::max2(Vec<T>::max2(r.x, r.y), Vec<T>::max2(r.z, r.w)), a, b);
    return max_nan(a, b);
  }
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[8]) {
    Vec<T>::pair(r.x, v[0], v[1]);
    Vec<T>::pair(r.y, v[2], v[3]);
    Vec<T>::pair(r.z, v[4], v[5]);
    Vec<T>::pair(r.w, v[6], v[7]);
  }
};
template <> struct Vec<__nv_bfloat16> : Vec16<__nv_bfloat16> {
  static constexpr uint32_t FLOOR_BITS = 0xF180F180u, NEG_INF_BITS = 0xFF80FF80u;
  static __device__ __forceinline__ float floor_value() { return __uint_as_float(0xF1800000u); }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ void pair(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
  }
};
template <> struct Vec<__half> : Vec16<__half> {
  static constexpr uint32_t FLOOR_BITS = 0xFBFFFBFFu, NEG_INF_BITS = 0xFC00FC00u;
  static __device__ __forceinline__ float floor_value() { return -65504.f; }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ void pair(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
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

// The running sums of a lane: even and odd elements side by side, in the packed fp32 arithmetic of the device, and two of these in turn.
// at: first element of the vector that brought the largest value so far.
template <typename T>
struct Run {
  static constexpr int N = Vec<T>::N;
  float m;
  float2 s[2], v[2];
  int at;
  __device__ __forceinline__ Run() {
    m = Vec<T>::floor_value();
    s[0] = s[1] = v[0] = v[1] = make_float2(0.f, 0.f);
    at = 0;
  }
  __device__ __forceinline__ Sums sums() const {
    return Sums{m, (s[0].x + s[0].y) + (s[1].x + s[1].y), (v[0].x + v[0].y) + (v[1].x + v[1].y)};
  }
  // K vectors (unavailable entries already at the floor); vector k starts at element i0 + k * step.
  template <int K>
  __device__ __forceinline__ void add(uint4 (&r)[K], int i0, int step, float c) {
    float t[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      r[k].x = Vec<T>::raise(r[k].x);
      r[k].y = Vec<T>::raise(r[k].y);
      r[k].z = Vec<T>::raise(r[k].z);
      r[k].w = Vec<T>::raise(r[k].w);
      t[k] = Vec<T>::largest(r[k]);
    }
    float top = t[0];
#pragma unroll
    for (int k = 1; k < K; ++k) top = max_nan(top, t[k]);
    if (!(top <= m)) {  // (also when top or m is NaN)
#pragma unroll
      for (int k = K - 1; k >= 0; --k)
        if (!(t[k] < top)) at = i0 + k * step;
      top = max_nan(m, top);
      const float d = step_down(m, top, c), f = ex2(d);
      const float2 f2 = make_float2(f, f), d2 = make_float2(d, d);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v[h] = mul2(f2, fma2(d2, s[h], v[h]));
        s[h] = mul2(f2, s[h]);
      }
      m = top;
    }
    const float2 c2 = make_float2(c, c), m2 = make_float2(-m, -m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float x[N];
      Vec<T>::unpack(r[k], x);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float2 u = mul2(add2(make_float2(x[j], x[j + 1]), m2), c2), e = make_float2(ex2(u.x), ex2(u.y));
        s[j / 2 & 1] = add2(s[j / 2 & 1], e);
        v[j / 2 & 1] = fma2(e, u, v[j / 2 & 1]);
      }
    }
  }
  __device__ __forceinline__ void add_one(float x, bool on, int i, float c) {  // one element a lane
    x = on ? max_nan(x, Vec<T>::floor_value()) : Vec<T>::floor_value();
    if (!(x <= m)) {
      Sums a = sums();
      rescale(a, max_nan(m, x), c);
      m = a.m;
      s[0] = make_float2(a.s, 0.f);
      v[0] = make_float2(a.v, 0.f);
      s[1] = v[1] = make_float2(0.f, 0.f);
      at = i;
    }
    const float u = (x - m) * c, e = on ? ex2(u) : 0.f;
    s[0].x += e;
    v[0].x += e * u;
  }
};

// ---- rows of more than SMALL_A actions ------------------------------------------------------------------------------
// A row that starts off a 16-byte boundary has up to 15 bytes in front of its vectors of 16 bytes and behind them, which are taken element by
// element.
template <typename T, bool MASK>
struct Row {
  static constexpr int N = Vec<T>::N;
  const T* x;
  const uint8_t* av;
  int head, body, tail;  // elements, vectors, elements
  __device__ __forceinline__ Row(const RowsParams& p, long long row) {
    x = reinterpret_cast<const T*>(p.x) + row * p.xs;
    av = MASK ? p.avail + row * p.as : nullptr;
    const int off = (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T);
    head = off < p.A ? off : p.A;
    body = (p.A - head) / N;
    tail = p.A - head - body * N;
  }
  __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(x + head); }
  // element i: its value, -infinity where it is not available
  __device__ __forceinline__ float value(int i) const { return !MASK || av[i] ? to_f32(x[i]) : -INFINITY; }
  // vector i with its unavailable entries at the floor
  __device__ __forceinline__ uint4 vector(int i) const {
    uint4 r = __ldg(vectors() + i);
    if (MASK) {
      uint32_t w[N / 4];
      load_avail<N>(av + head + i * N, w);
      Vec<T>::template hide<Vec<T>::FLOOR_BITS>(r, w);
    }
    return r;
  }
  // vector i with its unavailable entries at -infinity
  __device__ __forceinline__ void values(int i, float (&v)[N]) const {
    uint4 r = __ldg(vectors() + i);
    if (MASK) {
      uint32_t w[N / 4];
      load_avail<N>(av + head + i * N, w);
      Vec<T>::template hide<Vec<T>::NEG_INF_BITS>(r, w);
    }
    Vec<T>::unpack(r, v);
  }
};

// This lane's share of a row: vectors first, first + stride, ..., K on their way at a time.
template <int K, typename T, bool MASK>
__device__ __forceinline__ void walk_vectors(Run<T>& run, const Row<T, MASK>& r, int first, int stride, float c) {
  constexpr int N = Vec<T>::N;
  int i = first;
  if (i + (K - 1) * stride < r.body) {
    uint4 next[K];
#pragma unroll
    for (int k = 0; k < K; ++k) next[k] = r.vector(i + k * stride);
    for (;;) {
      uint4 now[K];
#pragma unroll
      for (int k = 0; k < K; ++k) now[k] = next[k];
      const int at = r.head + i * N;
      i += K * stride;
      const bool more = i + (K - 1) * stride < r.body;
      if (more) {
#pragma unroll
        for (int k = 0; k < K; ++k) next[k] = r.vector(i + k * stride);
      }
      run.template add<K>(now, at, stride * N, c);
      if (!more) break;
    }
  }
  for (; i < r.body; i += stride) {
    uint4 now[1] = {r.vector(i)};
    run.template add<1>(now, r.head + i * N, 0, c);
  }
}

// Walks a warp's qualifying lanes again: lane l's vectors are first + l, first + l + stride, ...; as many lanes' as fit are read at a time.
template <int CAP, typename T, bool MASK>
__device__ __forceinline__ void rewalk(const Row<T, MASK>& r, int first, int stride, int lane, const Entry& mine, const Bar& bar, Entry* found,
                                       int* count, uint8_t (&order)[32]) {
  constexpr int N = Vec<T>::N;
  const unsigned who = __ballot_sync(~0u, reaches(mine, bar.e));
  if (who >> lane & 1) order[__popc(who & ((1u << lane) - 1))] = (uint8_t)lane;
  const int steps = first < r.body ? (r.body - first + stride - 1) / stride : 0, lanes = __popc(who);
  int lg = 0;
  while ((1 << lg) < steps && lg < 5) ++lg;
  __syncwarp();
  for (int k = lane >> lg; k < lanes; k += 32 >> lg) {
    const int l = first + order[k];
    for (int s = lane & ((1 << lg) - 1); s < steps; s += 2 << lg) {  // two vectors on their way
      const long long i = l + (long long)s * stride, i2 = i + ((long long)stride << lg);
      float v[N], v2[N];
      if (i < r.body) r.values((int)i, v);
      if (i2 < r.body) r.values((int)i2, v2);
      if (i < r.body) collect<N, CAP>(v, r.head + (int)i * N, bar, found, count);
      if (i2 < r.body) collect<N, CAP>(v2, r.head + (int)i2 * N, bar, found, count);
    }
  }
}

// Elements in front of the vectors or behind them, one a lane, among the candidates.
template <int N, int CAP>
__device__ __forceinline__ void collect_one(float x, int i, const Bar& bar, Entry* found, int* count) {
  if (x < bar.value || x == -INFINITY) return;
  const Entry e{order_key(x), i};
  if (e.key > bar.e.key || (e.key == bar.e.key && e.idx - N < bar.e.idx)) {
    const int at = atomicAdd(count, 1);
    if (at < CAP) found[at] = e;
  }
}

// The results of a row, by one warp, from its joined sums and its list (lane k: the k-th alternative).
template <bool TOP, bool MASK, typename T>
__device__ __forceinline__ void write_results(const RowsParams& p, long long row, const Row<T, MASK>& r, Sums a, const Entry& best, int lane) {
  if (!trusted(a, Vec<T>::floor_value(), p.c)) a = careful_sums<T>(r.x, r.av, p.A, p.c, lane);
  float ls = 0.f;
  if (lane == 0) {
    const int act = p.action[row];
    const bool has = act >= 0 && act < p.A;
    ls = write_row(p, row, a, has, has ? r.value(act) : -INFINITY);
  }
  if (TOP) {
    ls = __shfl_sync(~0u, ls, 0);
    if (lane < p.top) {
      const bool some = best.key > KEY_NEG_INF;
      p.top_index[row * p.top + lane] = some ? best.idx : -1;
      p.top_logp[row * p.top + lane] = some ? ((best.key == INT32_MAX ? NAN : key_value(best.key)) - a.m) * p.it - ls : -INFINITY;
    }
  }
}

// -- a warp per row: eight rows a block.
constexpr int WARP_ROWS = 8, WARP_CAP = 96;

template <typename T, int K, bool TOP, bool MASK>
__global__ void __launch_bounds__(WARP_ROWS * 32) logprob_warp_kernel(const __grid_constant__ RowsParams p) {
  constexpr int N = Vec<T>::N;
  __shared__ Entry found_all[TOP ? WARP_ROWS : 1][WARP_CAP];
  __shared__ int count_all[WARP_ROWS];
  __shared__ uint8_t order[WARP_ROWS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * WARP_ROWS + warp;
  if (row >= p.rows) return;
  const Row<T, MASK> r(p, row);
  const int back = r.head + r.body * N;
  if (TOP && lane == 0) count_all[warp] = 0;
  Run<T> run;
  if (r.head) run.add_one(lane < r.head ? r.value(lane) : -INFINITY, lane < r.head, lane, p.c);
  walk_vectors<K>(run, r, lane, 32, p.c);
  if (r.tail) run.add_one(lane < r.tail ? r.value(back + lane) : -INFINITY, lane < r.tail, back + lane, p.c);
  __syncwarp();
  Sums a = run.sums();
  join_lanes(a, p.c);
  Entry best = entry_none();
  if constexpr (TOP) {
    Entry* found = found_all[warp];
    int* count = &count_all[warp];
    const Entry mine = lane_entry(run.m, run.at, Vec<T>::floor_value());
    const Bar bar = make_bar(nth_best(mine, p.top, lane));
    if (lane < r.head) collect_one<N, WARP_CAP>(r.value(lane), lane, bar, found, count);
    rewalk<WARP_CAP>(r, 0, 32, lane, mine, bar, found, count, order[warp]);
    if (lane < r.tail) collect_one<N, WARP_CAP>(r.value(back + lane), back + lane, bar, found, count);
    __syncwarp();
    const int n = *count;
    if (n <= WARP_CAP) best = best_of(found, n, p.top, lane);
    else walk<T>(best, r.x, r.av, 0, p.A, p.top, lane);
  }
  write_results<TOP>(p, row, r, a, best, lane);
}

// -- a block per row, or per part of a row (the parts are the blocks of a cluster).
// Eight blocks an SM (64 registers a thread) and four vectors on their way while four are computed: 2048 rows of 65537 in bf16, none / one / eight
// alternatives 50 / 57 / 72 us; with two vectors 58 / 65 / 79, with ten blocks and two vectors 60 / 67 / 83, twelve and one 82 / 88 / 106; with no
// limit on the registers (five blocks) and four vectors 68 / 72 / 90.
constexpr int EXACT_STEPS = 24;
constexpr int BLOCK_WARPS = 4, BLOCK_THREADS = BLOCK_WARPS * 32, BLOCK_CAP = 512;

template <typename T, bool TOP, bool MASK>
__global__ void __launch_bounds__(BLOCK_THREADS, 8) logprob_block_kernel(const __grid_constant__ RowsParams p) {
  constexpr int N = Vec<T>::N;
  __shared__ Sums part[BLOCK_WARPS];
  __shared__ Entry marks[BLOCK_WARPS][32];
  __shared__ uint8_t order[BLOCK_WARPS][32];
  __shared__ Entry found[TOP ? BLOCK_CAP : 1];
  __shared__ int count;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int parts = p.parts, rank = (int)(blockIdx.x % parts);
  const long long row = blockIdx.x / parts;
  const Row<T, MASK> r(p, row);
  const int back = r.head + r.body * N, stride = BLOCK_THREADS * parts, first = rank * BLOCK_THREADS + warp * 32;
  const int heads = rank == 0 && warp == 0 ? r.head : 0, tails = rank == parts - 1 && warp == BLOCK_WARPS - 1 ? r.tail : 0;
  Run<T> run;
  if (heads) run.add_one(lane < heads ? r.value(lane) : -INFINITY, lane < heads, lane, p.c);
  walk_vectors<4>(run, r, first + lane, stride, p.c);
  if (tails) run.add_one(lane < tails ? r.value(back + lane) : -INFINITY, lane < tails, back + lane, p.c);
  __syncwarp();
  Sums a = run.sums();
  join_lanes(a, p.c);
  const Entry mine = TOP ? lane_entry(run.m, run.at, Vec<T>::floor_value()) : entry_none();
  // The bar: where a lane's walk is long, the top-th best of the block's lanes; where it is short, the worst of the warps' best
  // quarters of `top`, which some half as many lanes more reach but which is sooner found.
  const bool exact = p.top > 1 && (long long)stride * EXACT_STEPS < r.body;
  Entry mark = mine;
  if (TOP) {
    if (exact) sort_list(mark, lane);
    else mark = nth_best(mark, (p.top + BLOCK_WARPS - 1) / BLOCK_WARPS, lane);
    marks[warp][lane] = mark;
  }
  if (lane == 0) {
    part[warp] = a;
    if (warp == 0) count = 0;
  }
  __syncthreads();
  if constexpr (TOP) {
    if (!exact) {
#pragma unroll
      for (int w = 0; w < BLOCK_WARPS; ++w)
        if (better(marks[w][0], mark) == (p.top == 1)) mark = marks[w][0];
    } else {
      for (int w = 0; w < BLOCK_WARPS; ++w)
        if (w != warp) merge_list(mark, marks[w][lane], lane);
      mark = shfl_entry(mark, p.top - 1);
    }
    const Bar bar = make_bar(mark);
    if (lane < heads) collect_one<N, BLOCK_CAP>(r.value(lane), lane, bar, found, &count);
    rewalk<BLOCK_CAP>(r, first, stride, lane, mine, bar, found, &count, order[warp]);
    if (lane < tails) collect_one<N, BLOCK_CAP>(r.value(back + lane), back + lane, bar, found, &count);
    __syncthreads();
  }
  Entry best = entry_none();
  if (warp == 0) {
    a = lane < BLOCK_WARPS ? part[lane] : Sums{Vec<T>::floor_value(), 0.f, 0.f};
    join_lanes(a, p.c);
    if constexpr (TOP) {
      if (count <= BLOCK_CAP) best = best_of(found, count, p.top, lane);
      else {
        if (rank == 0) walk<T>(best, r.x, r.av, 0, r.head, p.top, lane);
        for (int b = rank * BLOCK_THREADS; b < r.body; b += stride)
          walk<T>(best, r.x, r.av, r.head + b * N, r.head + min(b + BLOCK_THREADS, r.body) * N, p.top, lane);
        if (rank == parts - 1) walk<T>(best, r.x, r.av, back, p.A, p.top, lane);
      }
    }
  }
  if (parts > 1) {  // the blocks' sums and lists, in the order of their ranks
    cg::cluster_group cluster = cg::this_cluster();
    if (warp == 0) {
      __syncwarp();
      if (lane == 0) part[0] = a;
      if (TOP) found[lane] = best;
    }
    cluster.sync();
    if (rank == 0 && warp == 0) {
      a = lane < parts ? *cluster.map_shared_rank(&part[0], lane < parts ? lane : 0) : Sums{Vec<T>::floor_value(), 0.f, 0.f};
      join_lanes(a, p.c);
      if (TOP)
        for (int k = 1; k < parts; ++k) merge_list(best, *cluster.map_shared_rank(&found[lane], k), lane);
    }
    cluster.sync();
    if (rank) return;
  }
  if (warp == 0) write_results<TOP>(p, row, r, a, best, lane);
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

// Batcher's odd-even merge sort of a thread's numbers, descending; all indexes are constants, so that they stay in registers.
template <int LO, int LEN, int STEP, int N>
__device__ __forceinline__ void merge_halves(int (&a)[N]) {
  if constexpr (2 * STEP < LEN) {
    merge_halves<LO, LEN, 2 * STEP>(a);
    merge_halves<LO + STEP, LEN, 2 * STEP>(a);
#pragma unroll
    for (int i = LO + STEP; i + STEP < LO + LEN; i += 2 * STEP) {
      const int hi = max(a[i], a[i + STEP]), lo = min(a[i], a[i + STEP]);
      a[i] = hi;
      a[i + STEP] = lo;
    }
  } else {
    const int hi = max(a[LO], a[LO + STEP]), lo = min(a[LO], a[LO + STEP]);
    a[LO] = hi;
    a[LO + STEP] = lo;
  }
}
template <int LO, int LEN, int N>
__device__ __forceinline__ void sort_descending(int (&a)[N]) {
  if constexpr (LEN > 1) {
    sort_descending<LO, LEN / 2>(a);
    sort_descending<LO + LEN / 2, LEN / 2>(a);
    merge_halves<LO, LEN, 1>(a);
  }
}

// Blocks an SM: 36, 40 and 56 registers a thread, which the ranking needs.  Without the bound the look at close values makes it 48 and 76 in fp32:
// 786432 x 14, none / four alternatives 18.4 / 28.0 us against 16.6 / 27.5, in spite of the bound's spills (4 bytes; 56 for up to 32 actions).
template <typename T, int MA, bool DENSE>
__global__ void __launch_bounds__(SMALL_ROWS, MA == 8 ? 14 : MA == 16 ? 12 : 9) logprob_small_kernel(const __grid_constant__ RowsParams p, uint32_t inv_a) {
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
  Sums a{m, 0.f, 0.f};
  if (fabsf(m) < 1.0e30f) {
    float2 s2 = make_float2(0.f, 0.f), v2 = s2;
    const float2 c2 = make_float2(p.c, p.c), m2 = make_float2(-m, -m);
#pragma unroll
    for (int j = 0; j < MA; j += 2) {
      float2 u = mul2(add2(make_float2(v[j], v[j + 1]), m2), c2);
      u = make_float2(max_nan(u.x, -200.f), max_nan(u.y, -200.f));
      const float2 e = make_float2(ex2(u.x), ex2(u.y));
      s2 = add2(s2, e);
      v2 = fma2(e, u, v2);
    }
    a.s = s2.x + s2.y;
    a.v = v2.x + v2.y;
  } else {  // empty rows, NaN, infinities, numbers whose differences may overflow
    for (int j = 0; j < A; ++j) {
      if (mine[j] == -INFINITY) continue;
      const float u = exponent(mine[j], m, p.c), e = ex2(u);
      a.s += e;
      a.v += e * u;
    }
  }
  const long long row = row0 + r;
  const int act = p.action[row];
  const bool has = act >= 0 && act < A;
  const float ls = write_row(p, row, a, has, has ? mine[act] : -INFINITY);
  if (!p.top) return;
  // Keys that order like the values with their five lowest bits replaced by the index: one sort ranks them all, exactly where those bits
  // are 0 (16-bit types) and nearly always in fp32.  There, numbers that differ in those bits only come out in the order of their indexes: the
  // sorted places are looked through to the end of the group that the last wanted place lies in (a group of -infinities is in order), and where two
  // neighbours are the wrong way round, or with NaN, the alternatives are taken one by one.
  int key[MA];
#pragma unroll
  for (int j = 0; j < MA; ++j) {
    const int b = __float_as_int(v[j] + 0.0f);
    key[j] = ((b ^ ((b >> 31) & 0x7FFFFFFF)) & ~31) | (31 - j);
  }
  sort_descending<0, MA>(key);
  bool exact = m == m;
  if (sizeof(T) == 4) {
    float before = INFINITY;
    bool open = true;
#pragma unroll
    for (int k = 0; k < MA; ++k) {
      if (k > 0 && k >= p.top) open = open && (key[k] ^ key[k - 1]) >> 5 == 0 && before != -INFINITY;
      if (!open) break;
      const int j = 31 - (key[k] & 31);
      const float x = j < A ? mine[j] : -INFINITY;
      exact = exact && x <= before;
      before = x;
    }
  }
  int* ti = p.top_index + row * p.top;
  float* tl = p.top_logp + row * p.top;
  if (exact) {
#pragma unroll
    for (int k0 = 0; k0 < MA; k0 += 4) {
      if (k0 >= p.top) break;
      int out_j[4];
      float out_l[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = 31 - (key[k0 + k] & 31);
        const float x = j < A ? mine[j] : -INFINITY;
        out_j[k] = x == -INFINITY ? -1 : j;
        out_l[k] = x == -INFINITY ? -INFINITY : (x - a.m) * p.it - ls;
      }
      if (p.fours) {
        *reinterpret_cast<int4*>(ti + k0) = *reinterpret_cast<int4*>(out_j);
        *reinterpret_cast<float4*>(tl + k0) = *reinterpret_cast<float4*>(out_l);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k0 + k < p.top) {
            ti[k0 + k] = out_j[k];
            tl[k0 + k] = out_l[k];
          }
      }
    }
    for (int k = MA; k < p.top; ++k) {
      ti[k] = -1;
      tl[k] = -INFINITY;
    }
  } else {
    unsigned used = 0;
    for (int k = 0; k < p.top; ++k) {
      int bk = KEY_NEG_INF, bj = -1;
      for (int j = 0; j < A; ++j) {
        const int o = order_key(mine[j]);
        if (o > bk && !(used >> j & 1)) {
          bk = o;
          bj = j;
        }
      }
      used |= bj >= 0 ? 1u << bj : 0u;
      ti[k] = bj;
      tl[k] = bj >= 0 ? (mine[bj] - a.m) * p.it - ls : -INFINITY;
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
  const float2 st = q.r.stats[row];  // (all loads at once)
  const int act = q.r.action[row];
  const float gl = q.g_logp ? q.g_logp[row] : 0.f, ge = q.g_entropy ? q.g_entropy[row] : 0.f, entropy = q.r.entropy[row];
  RowGrad r{0.f, 0.f, 0.f, 0.f, 0.f, -1};
  if (st.y == -INFINITY) return r;  // an empty row: nothing in it is available
  if (act >= 0 && act < q.r.A) {
    r.action = act;
    r.g = gl * q.r.it;
  }
  const float h = ge * q.r.it;
  r.m = st.x;
  r.ls2 = st.y * LOG2E;
  r.h = h * LN2;
  r.k = r.g + h * entropy;
  return r;
}
// x of an available entry, or -infinity: 0 then.
__device__ __forceinline__ float entry_grad(float m, float ls2, float k, float h, float x, float c) {
  const float l = max_nan((x - m) * c - ls2, -200.f);
  return -ex2(l) * fmaf(h, l, k);
}

// Two of them, in packed arithmetic; c2 = (c, c), m2 = -(m, m) and so on.
__device__ __forceinline__ float2 entry_grad2(float2 m2, float2 c2, float2 ls2, float2 k2, float2 h2, float x0, float x1) {
  float2 l = fma2(add2(make_float2(x0, x1), m2), c2, ls2);
  l = make_float2(max_nan(l.x, -200.f), max_nan(l.y, -200.f));
  return mul2(make_float2(ex2(l.x), ex2(l.y)), fma2(h2, l, k2));
}

// A warp per segment of a row of more than SMALL_A actions, 16 bytes of the gradient a lane.  Where the logits' rows lie otherwise than the
// gradient's from a 16-byte boundary, each lane takes its logits from the two aligned vectors that hold them, the second from the
// lane behind it.
template <typename T, bool MASK>
__global__ void __launch_bounds__(256, MASK ? 5 : 4) logprob_wide_grad_kernel(const __grid_constant__ RowsGradParams q) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long row = unit / q.segments;
  if (row >= q.r.rows) return;
  const int segment = (int)(unit - row * q.segments), A = q.r.A;
  const T* x = reinterpret_cast<const T*>(q.r.x) + row * q.r.xs;
  const uint8_t* av = MASK ? q.r.avail + row * q.r.as : nullptr;
  T* d = reinterpret_cast<T*>(q.dx) + row * q.ds;
  const float c = q.r.c;
  const int off = (int)((16 - (reinterpret_cast<uintptr_t>(d) & 15)) & 15) / (int)sizeof(T);
  const int head = off < A ? off : A, body = (A - head) / N, tail = A - head - body * N;
  const int i0 = segment * q.seg_len, i1 = min(body, i0 + q.seg_len);  // vectors
  const uintptr_t xa = reinterpret_cast<uintptr_t>(x + head);
  const uint4* xv = reinterpret_cast<const uint4*>(xa & ~(uintptr_t)15);
  const int shift = (int)(xa & 15);                                    // bytes
  // BATCH vectors are on their way while BATCH are computed.  (The gradient may be written over the logits: every lane then reads
  // and writes its own vectors only, each before it is written.)
  // With availability one vector and five blocks an SM do better (1000 x 32001 fp16: 38 us against 45 with two and four) although 48 registers make
  // it spill 40 bytes a thread, without two and four (2048 x 65537 bf16: 93 us against 108; 64 registers, 4 bytes).
  constexpr int BATCH = MASK ? 1 : 2;
  uint4 raw[BATCH], next[BATCH];
  uint32_t w[BATCH][N / 4];
  auto fetch = [&](int b) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b + 32 * k + lane;
      raw[k] = next[k] = make_uint4(0u, 0u, 0u, 0u);
      if (i >= i1) continue;
      raw[k] = *(xv + i);
      if (shift && (lane == 31 || i + 1 == i1)) next[k] = *(xv + i + 1);
      if (MASK) load_avail<N>(av + head + i * N, w[k]);
    }
  };
  fetch(i0);
  const RowGrad g = row_grad(q, row);
  const float2 m2 = make_float2(-g.m, -g.m), c2 = make_float2(c, c), ls2 = make_float2(-g.ls2, -g.ls2), k2 = make_float2(-g.k, -g.k),
               h2 = make_float2(-g.h, -g.h);
  auto single = [&](int j) {
    float v = to_f32(x[j]);
    if (MASK && !av[j]) v = -INFINITY;
    float o = entry_grad(g.m, g.ls2, g.k, g.h, v, c);
    if (j == g.action && v != -INFINITY) o += g.g;
    d[j] = from_f32<T>(o);
  };
  if (segment == 0 && lane < head) single(lane);
  if (segment == q.segments - 1 && lane < tail) single(head + body * N + lane);
  for (int b = i0; b < i1; b += 32 * BATCH) {
    uint4 now[BATCH], behind[BATCH];
    uint32_t on[BATCH][N / 4];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      now[k] = raw[k];
      behind[k] = next[k];
#pragma unroll
      for (int e = 0; e < N / 4; ++e) on[k][e] = w[k][e];
    }
    if (b + 32 * BATCH < i1) fetch(b + 32 * BATCH);
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b + 32 * k + lane;
      uint4 r = now[k];
      if (shift) {
        uint4 n{__shfl_down_sync(~0u, r.x, 1), __shfl_down_sync(~0u, r.y, 1), __shfl_down_sync(~0u, r.z, 1), __shfl_down_sync(~0u, r.w, 1)};
        if (lane == 31 || i + 1 == i1) n = behind[k];
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
      if (MASK) Vec<T>::template hide<Vec<T>::NEG_INF_BITS>(r, on[k]);
      Vec<T>::unpack(r, v);
      const int j0 = head + i * N;
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float2 t = entry_grad2(m2, c2, ls2, k2, h2, v[j], v[j + 1]);
        o[j] = t.x;
        o[j + 1] = t.y;
      }
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

constexpr long long SEG_WARPS = 4 * 40ll * LEARNER_SMS;
constexpr int WARP_A = 4096;  // the longest row that one warp walks

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
  RowsParams q = p;
  q.parts = 1;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  lc.stream = stream;
  long long blocks;
  if (p.A <= WARP_A) {
    blocks = (p.rows + WARP_ROWS - 1) / WARP_ROWS;
    lc.blockDim = dim3(WARP_ROWS * 32);
  } else {
    while (q.parts < 8 && p.rows * q.parts * 2 <= 4 * LEARNER_SMS && p.A / (q.parts * 2) >= 4096) q.parts *= 2;
    blocks = p.rows * q.parts;
    lc.blockDim = dim3(BLOCK_THREADS);
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)q.parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = q.parts > 1 ? 1 : 0;
  }
  if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
  lc.gridDim = dim3((unsigned)blocks);
  cudaError_t err = cudaSuccess;
  auto go = [&](auto kernel) { err = cudaLaunchKernelEx(&lc, kernel, q); };
  if (p.A <= 32 * 4 * Vec<T>::N) {
    if (p.top) p.avail ? go(logprob_warp_kernel<T, 1, true, true>) : go(logprob_warp_kernel<T, 1, true, false>);
    else p.avail ? go(logprob_warp_kernel<T, 1, false, true>) : go(logprob_warp_kernel<T, 1, false, false>);
  } else if (p.A <= WARP_A) {
    if (p.top) p.avail ? go(logprob_warp_kernel<T, 4, true, true>) : go(logprob_warp_kernel<T, 4, true, false>);
    else p.avail ? go(logprob_warp_kernel<T, 4, false, true>) : go(logprob_warp_kernel<T, 4, false, false>);
  } else {
    if (p.top) p.avail ? go(logprob_block_kernel<T, true, true>) : go(logprob_block_kernel<T, true, false>);
    else p.avail ? go(logprob_block_kernel<T, false, true>) : go(logprob_block_kernel<T, false, false>);
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
  // Vectors a warp: as many as leave the device some four warps a slot, 64 at least.
  const long long vectors = q.r.A / Vec<T>::N;
  q.seg_len = 1024;
  while (q.seg_len > 64 && q.r.rows * ((vectors + q.seg_len - 1) / q.seg_len) < SEG_WARPS) q.seg_len /= 2;
  q.segments = (int)std::max<long long>(1, (vectors + q.seg_len - 1) / q.seg_len);
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
