// Log probabilities of the actions taken, entropy and best alternatives of rows of action values, and their gradient.
//
// With u_j = (x_j - m) / T for the row's largest available value m: S = sum e^u_j, log p_j = u_j - log S,
// entropy = log S - (sum e^u_j u_j) / S.  One pass over the row keeps (m, S, V = sum e^u u) and rescales S and V when m grows:
// e^(u + d) = e^u e^d, so S' = S e^d and V' = e^d (V + d S) for d = (m_old - m_new) / T.  Exponents are taken to base 2.
#include "learner_util.cuh"
#include "launch_util.cuh"

#include <cmath>

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
__device__ __forceinline__ Sums shuffle(const Sums& a, int mask) {
  return Sums{__shfl_xor_sync(~0u, a.m, mask), __shfl_xor_sync(~0u, a.s, mask), __shfl_xor_sync(~0u, a.v, mask)};
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

// A warp's list while it walks its part of a row in ascending order of indexes, 32 * N values at a time.  `worst` is the top-th entry;
// *shared holds the largest such key of the row's warps: an entry below it cannot be among the row's best.
template <int N>
struct TopWalk {
  Entry mine, worst;
  float bar;  // values not above it cannot enter
  __device__ __forceinline__ void reset() {
    mine = worst = entry_none();
    bar = -INFINITY;
  }
  __device__ __forceinline__ void raise(int shared_key) {
    int b = worst.key > KEY_NEG_INF ? worst.key : KEY_NEG_INF;
    if (shared_key - 1 > b) b = shared_key - 1;
    bar = b == INT32_MAX ? INFINITY : key_value(b);  // (as many NaN as entries: nothing enters behind them)
  }
  // Values of lane l: v[0..N) at indexes i0 .. i0 + N - 1 (i0 ascending with the lane).  Called by the whole warp.
  __device__ __noinline__ void take(const float (&v)[N], int i0, int lane, int top, int* shared) {
    unsigned used = 0;
    int sk = *(volatile int*)shared;
    while (true) {
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
      const bool in = c.key > KEY_NEG_INF && c.key >= sk && better(c, worst);
      unsigned who = __ballot_sync(~0u, in);
      if (!who) break;
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
      worst = shfl_entry(mine, top - 1);
    }
    if (lane == 0 && worst.key > sk) atomicMax(shared, worst.key);
    raise(sk);
  }
};

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

template <int N>
__device__ __forceinline__ void add_values(Sums& a, const float (&v)[N], float c, float& largest) {
  float top = v[0];
#pragma unroll
  for (int j = 1; j < N; ++j) top = max_nan(top, v[j]);
  largest = top;
  if (!(top <= a.m)) rescale(a, max_nan(top, a.m), c);  // (also when top is NaN)
  const float m = base_of(a.m);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float u = exponent(v[j], m, c), e = ex2(u);
    a.s += e;
    a.v += e * u;
  }
}

// ---- rows of more than SMALL_A actions ------------------------------------------------------------------------------
// WARPS warps of a block walk a row together, 16 bytes a lane, each warp every WARPS-th group of 512 bytes; with WARPS = 1 a block holds eight
// rows.  A row that starts off a 16-byte boundary has up to 15 bytes in front and behind that its first and last warp
// take element by element.
constexpr int WIDE_THREADS = 256;

template <typename T, int WARPS, bool TOP, bool MASK>
__global__ void __launch_bounds__(WIDE_THREADS) logprob_wide_kernel(const __grid_constant__ RowsParams p) {
  constexpr int N = Vec<T>::N, ROWS = WIDE_THREADS / 32 / WARPS;
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) % WARPS, sub = (threadIdx.x >> 5) / WARPS;
  const long long row = (long long)blockIdx.x * ROWS + sub;
  __shared__ int shared_key[ROWS];
  __shared__ Sums part[WARPS];
  __shared__ Entry lists[TOP && WARPS > 1 ? WARPS : 1][32];
  if (threadIdx.x < ROWS) shared_key[threadIdx.x] = KEY_NONE + 1;
  __syncthreads();
  if (row >= p.rows) return;  // (WARPS = 1 only: no barrier follows)
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs;
  const uint8_t* av = MASK ? p.avail + row * p.as : nullptr;
  const int off = (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T);
  const int head = off < p.A ? off : p.A, body = (p.A - head) / N, tail = p.A - head - body * N;

  Sums a{-INFINITY, 0.f, 0.f};
  TopWalk<N> walk;
  if (TOP) walk.reset();
  float v[N], largest;
  auto one_by_one = [&](int i0, int n) {  // n < N elements from i0 on, one per lane
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = -INFINITY;
    if (lane < n && (!MASK || av[i0 + lane])) v[0] = to_f32(x[i0 + lane]);
    add_values<N>(a, v, p.c, largest);
    if (TOP && __any_sync(~0u, !(largest <= walk.bar))) walk.take(v, i0 + lane, lane, p.top, &shared_key[sub]);
  };
  if (head && warp == 0) one_by_one(0, head);
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
#pragma unroll 2
  for (int g = warp * 32; g < body; g += 32 * WARPS) {
    const int i = g + lane, i0 = head + i * N;
    if (i < body) {
      Vec<T>::unpack(__ldg(xv + i), v);
      if (MASK) {
        uint32_t w[N / 4];
        load_avail<N>(av + i0, w);
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (!(w[j / 4] >> (8 * (j & 3)) & 0xFF)) v[j] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = -INFINITY;
    }
    add_values<N>(a, v, p.c, largest);
    if (TOP && __any_sync(~0u, !(largest <= walk.bar))) walk.take(v, i0, lane, p.top, &shared_key[sub]);
  }
  if (tail && warp == WARPS - 1) one_by_one(head + body * N, tail);

#pragma unroll
  for (int m = 16; m > 0; m >>= 1) a = join(a, shuffle(a, m), p.c);
  if (WARPS > 1) {
    if (lane == 0) part[warp] = a;
    if (TOP) lists[warp][lane] = walk.mine;
    __syncthreads();
    if (warp) return;
#pragma unroll 1
    for (int w = 1; w < WARPS; ++w) {
      a = join(a, part[w], p.c);
      if (TOP) merge_list(walk.mine, lists[w][lane], lane);
    }
  }
  if (lane == 0) {
    const int act = p.action[row];
    const bool has = act >= 0 && act < p.A;
    write_row(p, row, a, has, has && (!MASK || av[act]) ? to_f32(x[act]) : -INFINITY);
  }
  if (TOP && lane < p.top) {
    const Entry e = walk.mine;
    const bool some = e.key > KEY_NEG_INF;
    p.top_index[row * p.top + lane] = some ? e.idx : -1;
    p.top_logp[row * p.top + lane] = some ? (to_f32(x[e.idx]) - a.m) * p.it - logf(a.s) : -INFINITY;
  }
}

// ---- rows of up to SMALL_A actions ----------------------------------------------------------------------------------
// A thread per row: 128 rows come in element by element, neighbouring threads neighbouring elements, and are laid out in shared memory an
// odd number of words apart, so that the threads' walks over their rows meet no bank twice.
constexpr int SMALL_A = 32, SMALL_ROWS = 128;

template <typename T, int MA>
__global__ void __launch_bounds__(SMALL_ROWS) logprob_small_kernel(const __grid_constant__ RowsParams p, uint32_t inv_a) {
  __shared__ float xs[SMALL_ROWS * (MA + 1)];
  const long long row0 = (long long)blockIdx.x * SMALL_ROWS;
  const int rows = (int)(p.rows - row0 < SMALL_ROWS ? p.rows - row0 : SMALL_ROWS), A = p.A, pitch = A | 1;
  const T* x = reinterpret_cast<const T*>(p.x) + row0 * p.xs;
  const uint8_t* av = p.avail ? p.avail + row0 * p.as : nullptr;
#pragma unroll 8
  for (int i = threadIdx.x; i < rows * A; i += SMALL_ROWS) {
    const int r = (int)((uint32_t)i * inv_a >> 20), j = i - r * A;  // i / A: inv_a = ceil(2^20 / A), i < 4096, A <= 32
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
  const float b = base_of(m);
#pragma unroll
  for (int j = 0; j < MA; ++j) {
    const float u = exponent(v[j], b, p.c), e = ex2(u);
    a.s += e;
    a.v += e * u;
  }
  const long long row = row0 + r;
  const int act = p.action[row];
  const bool has = act >= 0 && act < A;
  write_row(p, row, a, has, has ? mine[act] : -INFINITY);
  if (!p.top) return;
  const float ls = logf(a.s);
  unsigned used = 0;
  for (int k = 0; k < p.top; ++k) {
    int bk = KEY_NEG_INF, bj = -1;
#pragma unroll
    for (int j = 0; j < MA; ++j) {
      const int key = order_key(v[j]);
      if (key > bk && !(used >> j & 1)) {
        bk = key;
        bj = j;
      }
    }
    used |= bj >= 0 ? 1u << bj : 0u;
    p.top_index[row * p.top + k] = bj;
    p.top_logp[row * p.top + k] = bj >= 0 ? (mine[bj] - a.m) * p.it - ls : -INFINITY;
  }
}

// ---- gradient -------------------------------------------------------------------------------------------------------
struct RowGrad {
  float m, ls2, gl, ge, ent2;  // largest value, log2 S, gradients over T, entropy in bits
  int action;
  bool empty;
};
__device__ __forceinline__ RowGrad row_grad(const RowsGradParams& q, long long row) {
  const float2 st = q.r.stats[row];
  RowGrad g;
  g.empty = st.y == -INFINITY;
  g.m = st.x;
  g.ls2 = st.y * LOG2E;
  const int act = q.r.action[row];
  const bool has = act >= 0 && act < q.r.A;
  g.action = has ? act : -1;
  g.gl = q.g_logp && has ? q.g_logp[row] * q.r.it : 0.f;
  g.ge = q.g_entropy ? q.g_entropy[row] * q.r.it * LN2 : 0.f;
  g.ent2 = q.r.entropy[row] * LOG2E;
  return g;
}
// x of an available entry.
__device__ __forceinline__ float entry_grad(const RowGrad& g, float x, int j, float c) {
  const float l = max_nan((x - g.m) * c - g.ls2, -200.f), pr = ex2(l);
  float d = -pr * (g.gl + g.ge * (l + g.ent2));
  if (j == g.action) d += g.gl;
  return d;
}

// A warp per segment of a row, neighbouring lanes neighbouring elements.
template <typename T>
__global__ void __launch_bounds__(256) logprob_wide_grad_kernel(const __grid_constant__ RowsGradParams q) {
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long row = unit / q.segments;
  if (row >= q.r.rows) return;
  const int j0 = (int)(unit - row * q.segments) * q.seg_len;
  const int j1 = q.r.A - j0 < q.seg_len ? q.r.A : j0 + q.seg_len;
  const RowGrad g = row_grad(q, row);
  const T* x = reinterpret_cast<const T*>(q.r.x) + row * q.r.xs;
  const uint8_t* av = q.r.avail ? q.r.avail + row * q.r.as : nullptr;
  T* d = reinterpret_cast<T*>(q.dx) + row * q.ds;
#pragma unroll 8
  for (int j = j0 + lane; j < j1; j += 32) {
    const float v = to_f32(x[j]);
    const bool on = !g.empty && v != -INFINITY && (!av || av[j]);
    d[j] = from_f32<T>(on ? entry_grad(g, v, j, q.r.c) : 0.f);
  }
}

// 128 rows a block, neighbouring threads neighbouring elements.
template <typename T>
__global__ void __launch_bounds__(SMALL_ROWS) logprob_small_grad_kernel(const __grid_constant__ RowsGradParams q, uint32_t inv_a) {
  __shared__ RowGrad gs[SMALL_ROWS];
  const long long row0 = (long long)blockIdx.x * SMALL_ROWS;
  const int rows = (int)(q.r.rows - row0 < SMALL_ROWS ? q.r.rows - row0 : SMALL_ROWS), A = q.r.A;
  if ((int)threadIdx.x < rows) gs[threadIdx.x] = row_grad(q, row0 + threadIdx.x);
  __syncthreads();
  const T* x = reinterpret_cast<const T*>(q.r.x) + row0 * q.r.xs;
  const uint8_t* av = q.r.avail ? q.r.avail + row0 * q.r.as : nullptr;
  T* d = reinterpret_cast<T*>(q.dx) + row0 * q.ds;
#pragma unroll 8
  for (int i = threadIdx.x; i < rows * A; i += SMALL_ROWS) {
    const int r = (int)((uint32_t)i * inv_a >> 20), j = i - r * A;
    const float v = to_f32(x[r * q.r.xs + j]);
    const bool on = !gs[r].empty && v != -INFINITY && (!av || av[r * q.r.as + j]);
    d[r * q.ds + j] = from_f32<T>(on ? entry_grad(gs[r], v, j, q.r.c) : 0.f);
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

template <typename T>
static int launch_logprob(const RowsParams& p, cudaStream_t stream) {
  if (p.A <= SMALL_A) {
    const long long blocks = (p.rows + SMALL_ROWS - 1) / SMALL_ROWS;
    if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
    const uint32_t inv = ((1u << 20) + p.A - 1) / p.A;
    if (p.A <= 8) logprob_small_kernel<T, 8><<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(p, inv);
    else if (p.A <= 16) logprob_small_kernel<T, 16><<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(p, inv);
    else logprob_small_kernel<T, 32><<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(p, inv);
    return launched("marl_policy_logprob");
  }
  const bool warp_rows = p.A <= 2048;
  const long long blocks = warp_rows ? (p.rows + 7) / 8 : p.rows;
  if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
  auto go = [&](auto kernel) { kernel<<<(unsigned)blocks, WIDE_THREADS, 0, stream>>>(p); };
  if (warp_rows) {
    if (p.top) p.avail ? go(logprob_wide_kernel<T, 1, true, true>) : go(logprob_wide_kernel<T, 1, true, false>);
    else p.avail ? go(logprob_wide_kernel<T, 1, false, true>) : go(logprob_wide_kernel<T, 1, false, false>);
  } else {
    if (p.top) p.avail ? go(logprob_wide_kernel<T, 8, true, true>) : go(logprob_wide_kernel<T, 8, true, false>);
    else p.avail ? go(logprob_wide_kernel<T, 8, false, true>) : go(logprob_wide_kernel<T, 8, false, false>);
  }
  return launched("marl_policy_logprob");
}

template <typename T>
static int launch_logprob_grad(RowsGradParams q, cudaStream_t stream) {
  if (q.r.A <= SMALL_A) {
    const long long blocks = (q.r.rows + SMALL_ROWS - 1) / SMALL_ROWS;
    if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
    logprob_small_grad_kernel<T><<<(unsigned)blocks, SMALL_ROWS, 0, stream>>>(q, ((1u << 20) + q.r.A - 1) / q.r.A);
    return launched("marl_policy_logprob_backward");
  }
  q.seg_len = 2048;
  q.segments = (q.r.A + q.seg_len - 1) / q.seg_len;
  const long long units = q.r.rows * q.segments, blocks = (units + 7) / 8;
  if (blocks > INT32_MAX) return fail(MARL_EINVAL, "too many rows");
  logprob_wide_grad_kernel<T><<<(unsigned)blocks, 256, 0, stream>>>(q);
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
