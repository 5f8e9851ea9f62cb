// Orthogonalised updates by Newton-Schulz products: X = G / |G|, then X <- (c0 I + c1 S + c2 S S) X with S = X X', a few times.
//
// A matrix of up to 128 x 1024 (short side m, long side n) belongs to a cluster of 1 to 8 blocks and stays in its shared memory from the
// load to the store: each block holds a slice of the long side, transposed (XT[j][i] = X[i][j], rows of the slice by
// columns of the short side).  A step is
//   each block's share of S from its slice, its rows sent to the blocks that own them
//   each block the sum of the shares of its rows (in rank order), sent to all blocks
//   each block its rows of Q = c0 I + c1 S + c2 S S, sent to all blocks
//   each block XT <- XT Q on its slice, in place (a row of XT depends on that row alone)
// Everything between blocks is sent, nothing fetched: stores into another block's shared memory are not waited for, loads from it are.
// The products are plain fp32 multiply-adds with register tiles: the polynomial's slope at 0 amplifies rounding errors of
// small singular directions (c0^5 = 485), so operands of fewer bits would show in the result: measured error 1.0e-6 (that of
// the formula in torch's fp32 products: 1.4e-6), 17 times fp32's half step; as many of bf16's would be 3 %.
// Measured, five steps: the four matrices of a hidden-64 network 37 us, 16 matrices of hidden 128 107 us (1.3 GFLOP: 12 TFLOP/s), 256 of hidden 64
// 130 us (22 TFLOP/s).  Clocks of a step of 384 x 128 on eight blocks: shares of S 8.6 k (6.1 k if every clock multiplied), S S 3.7 k (2 k), X Q
// 9 k (6.1 k), sending 10 k, barriers 5 k: the squares that every block needs whole cross the cluster three times at some 20 bytes a clock.
#include "learner_util.cuh"
#include "launch_util.cuh"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cooperative_groups.h>
#include <type_traits>

namespace cg = cooperative_groups;

namespace marl {

// 256 threads (with the products' lanes in a grid of 16 x 2: 16 matrices of hidden 128 in 115 us, with 512 threads 129; the 256 of 64 hidden-64
// networks in 143, with 128 threads 174).
constexpr int ORTHO_GROUPS = 32, ORTHO_THREADS = 256;
constexpr int ORTHO_MAX_BATCH = 1 << 24;  // matrices an entry, and a launch

struct OrthoGroup {
  const void* in;
  void* out;
  long long in_batch, in_row, out_batch, out_row;
  int first;       // index of its first matrix in the launch
  int rows, cols;
  float scale;
};
struct OrthoParams {
  OrthoGroup g[ORTHO_GROUPS];
  int groups, steps, squares;
  float c0, c1, c2, eps;
};

// Floats of shared memory: the slice, the shares received, S, and Q.  Without room for the third square Q takes the place of the shares, and a
// step ends with a barrier of the cluster.
__host__ __device__ constexpr int padded_short(int m) { return m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : 128; }
__host__ __device__ constexpr int pitch_of(int mp) { return mp + 4; }  // rows start 16 bytes further round the banks
__host__ __device__ inline int slice_of(int n, int cluster) { return ((n + cluster - 1) / cluster + 3) / 4 * 4; }
inline size_t ortho_smem(int m, int n, int cluster, int squares) {
  const int mp = padded_short(m);
  return 4 * ((size_t)slice_of(n, cluster) * pitch_of(mp) + squares * (size_t)mp * mp);
}
constexpr size_t ORTHO_SMEM_MAX = 226 * 1024;

// N neighbouring floats, 16, 8 or 4 bytes a load.
template <int N>
__device__ __forceinline__ void load_floats(const float* at, float (&v)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(&v[i]) = *reinterpret_cast<const float4*>(at + i);
  } else if constexpr (N == 2) *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(at);
  else v[0] = at[0];
}
template <int N>
__device__ __forceinline__ void store_floats(float* at, const float (&v)[N]) {
  if constexpr (N == 4) *reinterpret_cast<float4*>(at) = *reinterpret_cast<const float4*>(v);
  else if constexpr (N == 2) *reinterpret_cast<float2*>(at) = *reinterpret_cast<const float2*>(v);
  else at[0] = v[0];
}

// A warp's part of a product: acc[r][j] = sum over k0 <= k < k1 of rows[k][r] cols[k][j].  All lanes share the rows (one address: a broadcast) and
// have W neighbouring columns each, so that H W multiply-adds a lane cost H / 4 broadcasts and one load of the whole row; rows go in
// pairs through the packed multiply-add.  (Lanes in a grid of 16 x 2 with 8 x 8 elements each and single multiply-adds: 115 us for 16 matrices of
// hidden 128 against 107.)
template <int H, int W>
__device__ __forceinline__ void outer_products(const float* rows, const float* cols, int pitch, int k0, int k1, float (&acc)[H][W]) {
  float2 t[H / 2][W];
#pragma unroll
  for (int r = 0; r < H / 2; ++r)
#pragma unroll
    for (int j = 0; j < W; ++j) t[r][j] = make_float2(0.f, 0.f);
#pragma unroll 8
  for (int k = k0; k < k1; ++k) {
    float a[H], b[W];
    load_floats<H>(rows + k * pitch, a);
    load_floats<W>(cols + k * pitch, b);
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const float2 bb = make_float2(b[j], b[j]);
#pragma unroll
      for (int r = 0; r < H / 2; ++r) t[r][j] = fma2(make_float2(a[2 * r], a[2 * r + 1]), bb, t[r][j]);
    }
  }
#pragma unroll
  for (int r = 0; r < H / 2; ++r)
#pragma unroll
    for (int j = 0; j < W; ++j) {
      acc[2 * r][j] = t[r][j].x;
      acc[2 * r + 1][j] = t[r][j].y;
    }
}

template <typename T, int MP>
__device__ void ortho_matrix(const OrthoParams& p, const OrthoGroup& g, int index, float* smem) {
  // A warp has H rows of a square, a lane W of its columns (a square of 16: the upper lanes repeat the lower ones' work and store nothing).
  constexpr int PITCH = pitch_of(MP), WARPS = ORTHO_THREADS / 32, H = MP / WARPS, W = MP < 32 ? 1 : MP / 32;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), size = (int)cluster.num_blocks();
  const bool tall = g.rows > g.cols;
  const int m = tall ? g.cols : g.rows, n = tall ? g.rows : g.cols;
  const int ns = slice_of(n, size), j0 = rank * ns;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, col = (MP < 32 ? lane & (MP - 1) : lane) * W;
  const bool stores = MP >= 32 || lane < MP;
  float* xt = smem;                       // [ns][PITCH]
  float* shares = xt + ns * PITCH;        // [size][MP / size][MP] the blocks' shares of this block's rows of S
  float* s = shares + MP * MP;            // [MP][MP]
  float* qs = p.squares == 3 ? s + MP * MP : shares;
  __shared__ float exchange[2];           // largest modulus, sum of squares of the slice
  __shared__ float red[ORTHO_THREADS / 32];

  // load, transposed where the rows are the short side; zeros behind the matrix
  const T* in = reinterpret_cast<const T*>(g.in) + (long long)index * g.in_batch;
  for (int i = tid; i < ns * PITCH; i += ORTHO_THREADS) xt[i] = 0.f;
  __syncthreads();
  const int live = max(0, min(ns, n - j0));
  float top = 0.f;
  const int fast = tall ? m : live, slow = tall ? live : m;
  for (int b = tid / 32; b < slow; b += ORTHO_THREADS / 32)
    for (int a = tid & 31; a < fast; a += 32) {
      const int i = tall ? a : b, j = tall ? b : a;
      const float v = to_f32(tall ? in[(long long)(j0 + j) * g.in_row + i] : in[(long long)i * g.in_row + j0 + j]);
      xt[j * PITCH + i] = v;
      const float t = fabsf(v);
      top = t > top || t != t ? t : top;  // (a NaN stays, whatever comes behind it)
    }
  auto block_reduce = [&](float v, auto op) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(~0u, v, d));
    if ((tid & 31) == 0) red[tid >> 5] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < ORTHO_THREADS / 32; ++w) v = op(v, red[w]);
    __syncthreads();
    return v;
  };
  auto larger = [](float a, float b) { return a != a ? a : b != b ? b : fmaxf(a, b); };
  auto plus = [](float a, float b) { return a + b; };
  // |G| relative to its largest entry, so that squares neither overflow nor vanish
  top = block_reduce(top, larger);
  if (tid == 0) exchange[0] = top;
  cluster.sync();
  for (int r = 0; r < size; ++r) top = larger(top, *cluster.map_shared_rank(&exchange[0], r));
  const float inv_top = top > 0.f ? 1.f / top : 0.f;
  const bool tiny = top > 0.f && !(inv_top <= 3e38f);  // (1 / top overflows for the smallest subnormals: divide)
  float sum = 0.f;
  for (int i = tid; i < live * MP; i += ORTHO_THREADS) {
    const int j = i / MP, c = i - j * MP;
    const float v = tiny ? xt[j * PITCH + c] / top : xt[j * PITCH + c] * inv_top;
    sum += v * v;
  }
  sum = block_reduce(sum, plus);
  if (tid == 0) exchange[1] = sum;
  cluster.sync();
  sum = 0.f;
  for (int r = 0; r < size; ++r) sum += *cluster.map_shared_rank(&exchange[1], r);
  float norm = top * sqrtf(sum) + p.eps;
  if (top > 0.f && !(norm >= FLT_MIN && norm <= FLT_MAX)) {
    // beyond fp32's numbers, or below its normal ones, although no entry is: entries and eps relative to the largest entry
#pragma unroll 1
    for (int i = tid; i < live * MP; i += ORTHO_THREADS) xt[i / MP * PITCH + i % MP] /= top;
    norm = sqrtf(sum) + p.eps / top;
  }
  for (int i = tid; i < live * MP; i += ORTHO_THREADS) {
    const int j = i / MP, c = i - j * MP;
    float& v = xt[j * PITCH + c];
    v = top == 0.f ? 0.f : v / norm;
  }
  if (p.steps == 0) cluster.sync();  // (a block must not end while others read its sum)
  __syncthreads();

  const int rs = MP / size, row0 = rank * rs;    // this block's rows of S and Q
  for (int step = 0; step < p.steps; ++step) {
    {  // this block's share of S
      float acc[H][W];
      outer_products<H, W>(xt + warp * H, xt + col, PITCH, 0, ns, acc);
      if (stores)
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const int row = warp * H + i, owner = row / rs;
          store_floats<W>(cluster.map_shared_rank(shares, owner) + (rank * rs + row - owner * rs) * MP + col, acc[i]);
        }
    }
    cluster.sync();
    for (int i = tid; i < rs * MP / 4; i += ORTHO_THREADS) {
      float4 t = reinterpret_cast<const float4*>(shares)[i];
      for (int r = 1; r < size; ++r) {
        const float4 o = reinterpret_cast<const float4*>(shares + r * rs * MP)[i];
        t.x += o.x;
        t.y += o.y;
        t.z += o.z;
        t.w += o.w;
      }
      for (int r = 0; r < size; ++r) reinterpret_cast<float4*>(cluster.map_shared_rank(s, r) + row0 * MP)[i] = t;
    }
    cluster.sync();
    // This block's rows of S S, into `shares` (which is free now): its MP / size rows are `bands` tiles of H, and the warps that are left take parts
    // of the sum over k, which are added up in their order.  (S is symmetric: its rows are read.)
    const int bands = rs / H, parts = WARPS / bands, len = MP / parts;
    {
      const int band = warp % bands, part = warp / bands;
      float acc[H][W];
      outer_products<H, W>(s + row0 + band * H, s + col, MP, part * len, (part + 1) * len, acc);
      if (stores)
#pragma unroll
        for (int r = 0; r < H; ++r) store_floats<W>(shares + (part * rs + band * H + r) * MP + col, acc[r]);
    }
    __syncthreads();
    // this block's rows of Q, to every block
    float4 q[MP * MP / 4 / ORTHO_THREADS > 0 ? MP * MP / 4 / ORTHO_THREADS : 1];
    int held = 0;
#pragma unroll
    for (int h = 0; h < (int)(sizeof(q) / sizeof(q[0])); ++h) {
      const int i = tid + h * ORTHO_THREADS;
      if (i >= rs * MP / 4) break;
      float4 t = reinterpret_cast<const float4*>(shares)[i];
      for (int r = 1; r < parts; ++r) {
        const float4 o = reinterpret_cast<const float4*>(shares + r * rs * MP)[i];
        t.x += o.x;
        t.y += o.y;
        t.z += o.z;
        t.w += o.w;
      }
      const int row = row0 + i / (MP / 4), c = i % (MP / 4) * 4;
      const float4 a = *reinterpret_cast<const float4*>(s + row * MP + c);
      q[h] = make_float4(fmaf(p.c2, t.x, p.c1 * a.x) + (c == row ? p.c0 : 0.f), fmaf(p.c2, t.y, p.c1 * a.y) + (c + 1 == row ? p.c0 : 0.f),
                         fmaf(p.c2, t.z, p.c1 * a.z) + (c + 2 == row ? p.c0 : 0.f), fmaf(p.c2, t.w, p.c1 * a.w) + (c + 3 == row ? p.c0 : 0.f));
      held = h + 1;
    }
    if (p.squares != 3) cluster.sync();  // (Q takes the place of the parts, of every block)
#pragma unroll
    for (int h = 0; h < (int)(sizeof(q) / sizeof(q[0])); ++h) {
      if (h >= held) break;
      for (int r = 0; r < size; ++r) reinterpret_cast<float4*>(cluster.map_shared_rank(qs, r) + row0 * MP)[tid + h * ORTHO_THREADS] = q[h];
    }
    cluster.sync();
    // XT <- XT Q: a row belongs to one warp, whose lanes have all read it before any of them writes it
    auto times_q = [&](auto count) {
      constexpr int R = decltype(count)::value;
      for (int b = warp * R; b < ns; b += WARPS * R) {
        float acc[R][W];
        const float* rows[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          rows[i] = xt + min(b + i, ns - 1) * PITCH;
#pragma unroll
          for (int j = 0; j < W; ++j) acc[i][j] = 0.f;
        }
#pragma unroll 2
        for (int k = 0; k < MP; k += 4) {
          float a[R][4];
#pragma unroll
          for (int i = 0; i < R; ++i) *reinterpret_cast<float4*>(a[i]) = *reinterpret_cast<const float4*>(rows[i] + k);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            float q[W];
            load_floats<W>(qs + (k + kk) * MP + col, q);
#pragma unroll
            for (int i = 0; i < R; ++i) {
              if constexpr (W % 2 == 0) {
                const float2 aa = make_float2(a[i][kk], a[i][kk]);
#pragma unroll
                for (int j = 0; j < W; j += 2) {
                  const float2 t = fma2(aa, make_float2(q[j], q[j + 1]), make_float2(acc[i][j], acc[i][j + 1]));
                  acc[i][j] = t.x;
                  acc[i][j + 1] = t.y;
                }
              } else {
#pragma unroll
                for (int j = 0; j < W; ++j) acc[i][j] = fmaf(a[i][kk], q[j], acc[i][j]);
              }
            }
          }
        }
        __syncwarp();
        if (stores)
#pragma unroll
          for (int i = 0; i < R; ++i)
            if (b + i < ns) store_floats<W>(xt + (b + i) * PITCH + col, acc[i]);
        __syncwarp();
      }
    };
    const int rows_a_warp = (ns + WARPS - 1) / WARPS;
    if (rows_a_warp > 6) times_q(std::integral_constant<int, 8>());
    else if (rows_a_warp > 4) times_q(std::integral_constant<int, 6>());
    else if (rows_a_warp > 3) times_q(std::integral_constant<int, 4>());
    else if (rows_a_warp > 2) times_q(std::integral_constant<int, 3>());
    else times_q(std::integral_constant<int, 2>());
    if (p.squares == 3) __syncthreads();
    else cluster.sync();
  }

  T* out = reinterpret_cast<T*>(g.out) + (long long)index * g.out_batch;
  for (int b = tid / 32; b < slow; b += ORTHO_THREADS / 32)
    for (int a = tid & 31; a < fast; a += 32) {
      const int i = tall ? a : b, j = tall ? b : a;
      T* at = tall ? out + (long long)(j0 + j) * g.out_row + i : out + (long long)i * g.out_row + j0 + j;
      *at = from_f32<T>(g.scale * xt[j * PITCH + i]);
    }
}

// MOST: the largest padded short side of the list.  Up to 64 two blocks share a multiprocessor.
template <typename T, int MOST>
__global__ void __launch_bounds__(ORTHO_THREADS, MOST == 128 ? 1 : 2) orthogonalise_kernel(const __grid_constant__ OrthoParams p) {
  extern __shared__ __align__(16) float ortho_smem_buf[];
  const int matrix = (int)(blockIdx.x / cg::this_cluster().num_blocks());
  int at = 0;
  while (at + 1 < p.groups && matrix >= p.g[at + 1].first) ++at;
  const OrthoGroup& g = p.g[at];
  const int m = min(g.rows, g.cols), index = matrix - g.first;
  if (m <= 16) ortho_matrix<T, 16>(p, g, index, ortho_smem_buf);
  else if (m <= 32) ortho_matrix<T, 32>(p, g, index, ortho_smem_buf);
  else if (MOST == 64 || m <= 64) ortho_matrix<T, 64>(p, g, index, ortho_smem_buf);
  else if constexpr (MOST == 128) ortho_matrix<T, 128>(p, g, index, ortho_smem_buf);
}

static uint32_t g_ortho_smem[6][SMEM_OPTIN_DEVICES];

template <typename T, int MOST>
static int launch_ortho(const OrthoParams& p, int matrices, int cluster, size_t smem, int which, cudaStream_t stream) {
  auto* kernel = &orthogonalise_kernel<T, MOST>;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (uint32_t)smem, g_ortho_smem[which]);
  if (e != cudaSuccess) return fail(MARL_ECUDA, "marl_orthogonalise: %s", cudaGetErrorString(e));
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3((unsigned)(matrices * cluster));
  c.blockDim = dim3(ORTHO_THREADS);
  c.dynamicSmemBytes = smem;
  c.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  c.attrs = at;
  c.numAttrs = 1;
  e = cudaLaunchKernelEx(&c, kernel, p);
  return e == cudaSuccess ? MARL_OK : fail(MARL_ECUDA, "marl_orthogonalise: %s", cudaGetErrorString(e));
}

}  // namespace marl

using namespace marl;

extern "C" int marl_orthogonalise(void* stream, const marl_matrix_t* list, int32_t count, int32_t dtype, int32_t steps, const float* coeffs,
                                  float eps) {
  if (count < 0 || (count > 0 && !list)) return fail(MARL_EINVAL, "the list is NULL or its length negative");
  if (!dtype_known(dtype)) return fail(MARL_EINVAL, "unknown dtype %d", dtype);
  if (steps < 0 || steps > 64) return fail(MARL_EINVAL, "steps must be in [0, 64]");
  if (!coeffs) return fail(MARL_EINVAL, "coeffs is NULL");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MARL_EINVAL, "eps must be >= 0 and finite");
  for (int i = 0; i < count; ++i) {
    const marl_matrix_t& g = list[i];
    if (g.batch < 0) return fail(MARL_EINVAL, "matrix %d: batch is negative", i);
    if (g.rows < 1 || g.cols < 1 || std::min(g.rows, g.cols) > MARL_ORTHO_MAX_SHORT || std::max(g.rows, g.cols) > MARL_ORTHO_MAX_LONG)
      return fail(MARL_EINVAL, "matrix %d: %d x %d is outside 1 x 1 .. %d x %d (either way round)", i, g.rows, g.cols, MARL_ORTHO_MAX_SHORT,
                  MARL_ORTHO_MAX_LONG);
    if (g.batch > ORTHO_MAX_BATCH) return fail(MARL_EINVAL, "matrix %d: batch is larger than 2^24", i);
    if (g.batch == 0) continue;
    if (!g.in || !g.out) return fail(MARL_EINVAL, "matrix %d: in or out is NULL", i);
    if (g.in_batch < 0 || g.in_row < 0) return fail(MARL_EINVAL, "matrix %d: a stride is negative", i);
    if ((g.rows > 1 && g.out_row < g.cols) || (g.batch > 1 && g.out_batch < (g.rows - 1) * g.out_row + g.cols))
      return fail(MARL_EINVAL, "matrix %d: rows or matrices of the output overlap", i);
    if (misaligned(g.in, dtype_bytes(dtype)) || misaligned(g.out, dtype_bytes(dtype)))
      return fail(MARL_EALIGN, "matrix %d is not aligned to its elements", i);
    for (int j = 0; j < i; ++j)
      if (list[j].batch > 0 && list[j].out == g.out) return fail(MARL_EINVAL, "matrices %d and %d have the same output", j, i);
  }
  for (int i0 = 0; i0 < count;) {
    OrthoParams p = {};
    p.steps = steps;
    p.c0 = coeffs[0];
    p.c1 = coeffs[1];
    p.c2 = coeffs[2];
    p.eps = eps;
    long long matrices = 0;
    int i = i0;
    for (; i < count && p.groups < ORTHO_GROUPS; ++i) {
      const marl_matrix_t& g = list[i];
      if (g.batch == 0) continue;
      if (matrices + g.batch > ORTHO_MAX_BATCH) break;  // (no single entry is larger: the first of a launch always fits)
      p.g[p.groups++] = OrthoGroup{g.in, g.out, g.in_batch, g.in_row, g.out_batch, g.out_row, (int)matrices, g.rows, g.cols, g.scale};
      matrices += g.batch;
    }
    auto smem_for = [&](int cluster, int squares) {
      size_t need = 0;
      for (int k = 0; k < p.groups; ++k)
        need = std::max(need, ortho_smem(std::min(p.g[k].rows, p.g[k].cols), std::max(p.g[k].rows, p.g[k].cols), cluster, squares));
      return need;
    };
    i0 = i;
    if (p.groups == 0) continue;
    // Few matrices: as many blocks a matrix as the device has room for; more: as few as their shared memory allows.
    p.squares = 3;
    int cluster = 1;
    while (cluster < 8 && smem_for(cluster, 3) > ORTHO_SMEM_MAX) cluster *= 2;
    if (smem_for(cluster, 3) > ORTHO_SMEM_MAX) p.squares = 2;
    while (cluster < 8 && matrices * cluster * 2 <= LEARNER_SMS) cluster *= 2;
    const size_t smem = smem_for(cluster, p.squares);
    int rc;
    int most = 0;
    for (int k = 0; k < p.groups; ++k) most = std::max(most, std::min(p.g[k].rows, p.g[k].cols));
    rc = by_dtype(dtype, [&](auto t) {
      using T = decltype(t);
      return most <= 64 ? launch_ortho<T, 64>(p, (int)matrices, cluster, smem, dtype, (cudaStream_t)stream)
                        : launch_ortho<T, 128>(p, (int)matrices, cluster, smem, dtype + 3, (cudaStream_t)stream);
    });
    if (rc != MARL_OK) return rc;
  }
  return MARL_OK;
}
