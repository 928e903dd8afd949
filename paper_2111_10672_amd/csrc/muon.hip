// One optimiser step over the partial gradients of several workers: matrices take an update orthogonalised by Newton-Schulz
// products, everything else AdamW.
//
//   g = mean of the contributors' gradients (added in the order given)
//   matrices   m = mu m + g;  u = g + mu m or m;  X = u / (|u|_F + eps), the shorter side first;  `steps` times
//                  A = X X^T,  B = b A + c A A,  X = a X + B X      (a, b, c = 3.4445, -4.7750, 2.0315)
//              which moves every singular value of u towards 1;  w = w (1 - rate wd) - rate rms sqrt(longer side) X
//   others     m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w = w (1 - rate wd) - rate (m / c1) / (sqrt(v / c2) + eps)
//
// The elementwise half is memory-bound and one launch over a table of tensors (update_kernel); for matrices it leaves u
// (float32) and the partial sums of |u|^2 (float64, so that neither tiny nor huge gradients leave the range) in the workspace.  24 matrices of
// 4096 x 1024 with one worker: 279 us, 5.8 TB/s; AdamW of 23.4 million bfloat16 with four: 146 us, 5.8 TB/s.
// The products are bound by the matrix cores where there are many tiles (24 of 1024 x 4096 x 1024: 207 us, 1.0 PFLOP/s; the symmetric ones
// of 48 of 768 x 768, 0.53 PFLOP/s of useful work in 41 us, are two rounds of tiles of 128, each with a start and stores that nothing covers), by launches and latency where there
// are few; kernels for each are below.  All matrices of one padding go through a product in one launch, whichever
// tensors and blocks they come from, and the two symmetric products form the tiles on and below the diagonal only and
// write each twice: a step of an r x c matrix costs r^2 c + r^3 + 2 r^2 c operations instead of 2 r^2 c + 2 r^3 + 2 r^2 c.
//
// Number formats.  X, A and B are stored as float16 between the products, which accumulate in float32: at the same matrix
// rate as bfloat16 it carries three bits more, and the step is a polynomial of a matrix of norm near 1, whose entries a fixed power of two
// (sigma, tau) keeps in range: |X| <= 1.3 in the spectral norm throughout, so sigma |x| <= 1.3 * 2^14 and tau |b| <= 2^14.
// For a bfloat16 parameter that leaves the orthogonalised matrix 0.9e-3 to 1.2e-3 off in the Frobenius norm (48 of 768 x 768, 24 of 4096 x 1024; up to 4e-3 where a few
// directions stand far above the rest), where float32 in its place leaves 2e-6 to 3e-6 and rounding it to bfloat16 would leave 1.7e-3.  Added to the parameter it is not seen: that is
// 1.66e-3 from the one in 64 bits either way, its own rounding, and 5e-4 to 7e-4 from the one with float32 in between (roundings that fall to the other side).
// A float32 parameter would show the 2^-11 of that format: its X, A and B are stored as two float16 (value and remainder, the remainder
// scaled by 2^11), and a product is three: value x remainder, remainder x value, their sum scaled by 2^-11, value x value.
#include <algorithm>
#include <cmath>

#include "gemm_dma_impl.h"

namespace spb {
namespace {

using gemm_detail::f32x16;
using gemm_detail::f32x4;
using gemm_detail::u32x4;
using gemm_detail::xcd_tile;
using gemm_dma_detail::krow_rot;
using gemm_dma_detail::wait_loads_and_barrier;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
// the same as they lie at any element's address: one access all the same (gfx950 takes global addresses of any alignment)
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_t;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kThreads = 256;
constexpr int kTileK = 64;
constexpr float kTau = 1024.f;            // A and B are stored times this
constexpr float kLoScale = 2048.f;        // remainders are stored times this

// One matrix of the step, written by update_kernel for the kernels behind it.
struct Matrix {
  void* w;                 // first element of the matrix in its parameter
  const float* u;          // [rows, cols] dense
  const double* partial;   // [parts] sums of u^2
  int parts, rows, cols, bf16;
  float keep, step;        // w = keep * w - step * X
  double eps;
};

// ---- elementwise half ---------------------------------------------------------------------------------------------

constexpr int kMaxTensors = 16;
constexpr int kPiece = 1024;              // elements a workgroup takes at a time
constexpr int kMaxParts = 256;            // workgroups of one matrix

struct Tensor {
  void* w; float* m; float* v;
  const float* g[kMaxAggWorkers];
  float* u;                // matrices: the workspace's [rows, cols]; null: AdamW
  double* partial;
  Matrix* out;
  long long numel;         // of one block
  long long chunk;         // elements of one workgroup
  int blocks, parts;       // matrices, workgroups of each
  int first_block, count, bf16, rows, cols;
  float rate, keep, step;   // keep = 1 - rate * weight decay
};
struct Table {
  Tensor t[kMaxTensors];
  int n, nesterov;
  float momentum, beta1, beta2, new1, new2, inv_c1, inv_c2, adam_eps;   // new1 = 1 - beta1
  double ns_eps;
};

__device__ __forceinline__ float bf(uint16_t v) { return __uint_as_float(((uint32_t)v) << 16); }

template <bool MATRIX>
__device__ __forceinline__ void step_element(const Table& tab, const Tensor& t, float g, float& m, float& v, float& w, float& u) {
  if constexpr (MATRIX) {
    m = tab.momentum * m + g;
    u = tab.nesterov ? g + tab.momentum * m : m;
  } else {
    m = tab.beta1 * m + tab.new1 * g;
    v = tab.beta2 * v + tab.new2 * (g * g);
    w = w * t.keep - t.rate * ((m * tab.inv_c1) / (sqrtf(v * tab.inv_c2) + tab.adam_eps));
  }
}

// Four elements of a thread, all of their loads requested before the first is used.  C gradients, MATRIX: momentum and u, otherwise AdamW.
template <int C, bool MATRIX>
__device__ __forceinline__ void step_vector(const Table& tab, const Tensor& t, long long e0, float inv, double& sq) {
  f32x4 x[C], v = {}, w = {};
#pragma unroll
  for (int j = 0; j < C; ++j) x[j] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(t.g[j] + e0));   // read once
  f32x4 m = *reinterpret_cast<const f32x4_any*>(t.m + e0);
  u32x2_any wb = {};
  if constexpr (!MATRIX) {
    v = *reinterpret_cast<const f32x4_any*>(t.v + e0);
    if (t.bf16) wb = *reinterpret_cast<const u32x2_any*>(static_cast<const uint16_t*>(t.w) + e0);
    else w = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(t.w) + e0);
  }
  f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = {};
#pragma unroll
  for (int j = 0; j < C; ++j) g += x[j];   // workers added in the order given
  if (!MATRIX && t.bf16) w = f32x4{__uint_as_float(wb.x << 16), __uint_as_float(wb.x & 0xFFFF0000u), __uint_as_float(wb.y << 16), __uint_as_float(wb.y & 0xFFFF0000u)};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float me = m[e], ve = v[e], we = w[e], ue = 0.f;
    step_element<MATRIX>(tab, t, g[e] * inv, me, ve, we, ue);
    m[e] = me; v[e] = ve; w[e] = we; u[e] = ue;
  }
  *reinterpret_cast<f32x4_any*>(t.m + e0) = m;
  if constexpr (MATRIX) {
    *reinterpret_cast<f32x4_any*>(t.u + e0) = u;
#pragma unroll
    for (int e = 0; e < 4; ++e) sq += (double)u[e] * (double)u[e];
  } else {
    *reinterpret_cast<f32x4_any*>(t.v + e0) = v;
    if (t.bf16) *reinterpret_cast<u32x2_any*>(static_cast<uint16_t*>(t.w) + e0) = u32x2_any{bf16_pack2(w[0], w[1]), bf16_pack2(w[2], w[3])};
    else *reinterpret_cast<f32x4_any*>(static_cast<float*>(t.w) + e0) = w;
  }
}
// The same element by element: the last three at most.  (Element by element throughout, 11.9 million float32 of six workers took 352 us, where four at a time take
// 94.)
template <bool MATRIX>
__device__ __forceinline__ void step_scalar(const Table& tab, const Tensor& t, long long e0, long long end, float inv, double& sq) {
  for (long long at = e0; at < end; ++at) {
    float g = 0.f, m = t.m[at], v = 0.f, w = 0.f, u = 0.f;
    for (int j = 0; j < t.count; ++j) g += t.g[j][at];
    if (!MATRIX) {
      v = t.v[at];
      w = t.bf16 ? bf(static_cast<const uint16_t*>(t.w)[at]) : static_cast<const float*>(t.w)[at];
    }
    step_element<MATRIX>(tab, t, g * inv, m, v, w, u);
    t.m[at] = m;
    if (MATRIX) {
      t.u[at] = u;
      sq += (double)u * (double)u;
    } else {
      t.v[at] = v;
      if (t.bf16) static_cast<uint16_t*>(t.w)[at] = bf16_round(w);
      else static_cast<float*>(t.w)[at] = w;
    }
  }
}
template <int C, bool MATRIX>
__device__ __forceinline__ void step_range(const Table& tab, const Tensor& t, long long begin, long long end, double& sq) {
  const float inv = 1.f / (float)t.count;
  for (long long e0 = begin + threadIdx.x * 4; e0 < end; e0 += kThreads * 4) {
    if (e0 + 4 <= end) step_vector<C, MATRIX>(tab, t, e0, inv, sq);
    else step_scalar<MATRIX>(tab, t, e0, end, inv, sq);
  }
}
template <bool MATRIX>
__device__ __forceinline__ void step_tensor(const Table& tab, const Tensor& t, long long begin, long long end, double& sq) {
  switch (t.count) {   // uniform over the workgroup
    case 1: step_range<1, MATRIX>(tab, t, begin, end, sq); return;
    case 2: step_range<2, MATRIX>(tab, t, begin, end, sq); return;
    case 3: step_range<3, MATRIX>(tab, t, begin, end, sq); return;
    case 4: step_range<4, MATRIX>(tab, t, begin, end, sq); return;
    case 5: step_range<5, MATRIX>(tab, t, begin, end, sq); return;
    case 6: step_range<6, MATRIX>(tab, t, begin, end, sq); return;
    case 7: step_range<7, MATRIX>(tab, t, begin, end, sq); return;
    default: step_range<kMaxAggWorkers, MATRIX>(tab, t, begin, end, sq);
  }
}

__global__ __launch_bounds__(kThreads) void update_kernel(Table tab) {
  int ti = 0;
  for (int i = 1; i < tab.n; ++i)
    if ((int)blockIdx.x >= tab.t[i].first_block) ti = i;
  const Tensor& t = tab.t[ti];
  const int local = (int)blockIdx.x - t.first_block;
  const int mat = local / t.parts, part = local - mat * t.parts;
  const long long base = mat * t.numel;
  const long long begin = base + part * t.chunk, end = base + min(t.numel, (part + 1) * t.chunk);
  double sq = 0.0;
  if (t.u) step_tensor<true>(tab, t, begin, end, sq);
  else step_tensor<false>(tab, t, begin, end, sq);
  if (!t.u) return;   // uniform over the workgroup
  __shared__ double sums[kThreads / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sq += __shfl_xor(sq, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sq;
  __syncthreads();
  if (threadIdx.x == 0) {
    t.partial[(long long)mat * t.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    if (part == 0)
      t.out[mat] = Matrix{t.bf16 ? (void*)(static_cast<uint16_t*>(t.w) + base) : (void*)(static_cast<float*>(t.w) + base), t.u + base,
                          t.partial + (long long)mat * t.parts, t.parts, t.rows, t.cols, t.bf16, t.keep, t.step, tab.ns_eps};
  }
}

// A factor on its way to float32 as two: the second is 1 unless the first would leave float32's range, where it takes a power of two.
struct Factor { float main, lift; };
__device__ __forceinline__ Factor factor_of(double f) {
  const double lift = f > 0x1p100 ? 0x1p100 : f < 0x1p-100 ? 0x1p-100 : 1.0;
  return Factor{(float)(f / lift), (float)lift};
}
// by / (|u| + eps) from the sum of u's squares; a u of zeros stays one whatever eps is.
__device__ __forceinline__ double over_norm(double by, double squares, double eps) { return squares == 0.0 ? 0.0 : by / (sqrt(squares) + eps); }

// ---- matrices of one padded shape -----------------------------------------------------------------------------------

constexpr int kMaxGroups = 24;
struct Group {
  _Float16* x[2];          // [count][planes][mp][np], this step's and the next one's
  _Float16* a;             // [count][planes][mp][mp]
  _Float16* b;
  const Matrix* matrices;
  int mp, np, count;       // padded sides, the shorter first
  int first_block, per_matrix;
  float sigma;             // X is stored times this
};
struct Groups {
  Group g[kMaxGroups];
  int n;
};

// EARLY: by value, the first group at once, which saves small launches a second round trip to the kernel's arguments (66 -> 58 us for a step of one
// 100 x 300 matrix); the large kernels lose 5 % to holding it.
template <bool EARLY>
__device__ __forceinline__ std::conditional_t<EARLY, Group, const Group&> group_of(const Groups& t, int block, int& mat, int& tile) {
  if constexpr (EARLY) {
    Group g = t.g[0];
    for (int j = 1; j < t.n; ++j)
      if (block >= t.g[j].first_block) g = t.g[j];
    const int local = block - g.first_block;
    mat = local / g.per_matrix;
    tile = local - mat * g.per_matrix;
    return g;
  } else {
    int i = 0;
    for (int j = 1; j < t.n; ++j)
      if (block >= t.g[j].first_block) i = j;
    const Group& g = t.g[i];
    const int local = block - g.first_block;
    mat = local / g.per_matrix;
    tile = local - mat * g.per_matrix;
    return g;
  }
}

// A value that is about to be split is rounded to float32 here, once.  Left to itself the compiler contracts the product it comes from with one of the
// two conversions to float16 and not with the other; next to a tie the stored value and the one the remainder is taken from are then a float16 step apart.
__device__ __forceinline__ void settle(float& v) { asm volatile("" : "+v"(v)); }

// value and remainder of v at p and, with two planes, p + plane
template <int PLANES>
__device__ __forceinline__ void split8(float (&v)[8], _Float16* p, size_t plane) {
  if constexpr (PLANES == 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) settle(v[e]);
  }
  f16x8 hi;
#pragma unroll
  for (int e = 0; e < 8; ++e) hi[e] = (_Float16)v[e];
  *reinterpret_cast<f16x8*>(p) = hi;
  if constexpr (PLANES == 2) {
    f16x8 lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[e] = (_Float16)((v[e] - (float)hi[e]) * kLoScale);
    *reinterpret_cast<f16x8*>(p + plane) = lo;
  }
}
template <int PLANES>
__device__ __forceinline__ void join8(const u32x4 (&w)[PLANES], float (&v)[8]) {
  const f16x8 hi = __builtin_bit_cast(f16x8, w[0]);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)hi[e];
  if constexpr (PLANES == 2) {
    const f16x8 lo = __builtin_bit_cast(f16x8, w[1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += (float)lo[e] * (1.f / kLoScale);
  }
}

// Where entry (row, col) of a matrix of `ld` columns lies in blocks of 16 rows and 32 columns, col a multiple of 8: the 16 bytes of each lane of a wavefront's operand
// behind one another, so that a wavefront loads an operand as 1 KB in a row, without LDS.
__device__ __forceinline__ size_t place(int ld, int row, int col) {
  return ((size_t)(row >> 4) * (ld >> 5) + (col >> 5)) * 512 + (((col >> 3) & 3) * 16 + (row & 15)) * 8;
}

// X = sigma u / (|u| + eps), shorter side first, zeros in the padding.  A workgroup per 64 x 64 entries.  BLOCKS: X lies as `place` says.
template <int PLANES, bool BLOCKS>
__global__ __launch_bounds__(kThreads) void normalise_kernel(Groups groups) {
  __shared__ float tile_s[64][65];
  __shared__ double sums[kThreads / 64];
  int mat, tile;
  const Group g = group_of<true>(groups, blockIdx.x, mat, tile);
  const Matrix d = g.matrices[mat];
  double s = (int)threadIdx.x < d.parts ? d.partial[threadIdx.x] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  const int tiles_n = g.np / 64, i0 = tile / tiles_n * 64, j0 = (tile - tile / tiles_n * tiles_n) * 64;
  const bool tall = d.rows > d.cols;
  // rows of u: those of X, or, the matrix being tall, its columns
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  f32x4 in[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = k * 16 + (threadIdx.x >> 4), c = (threadIdx.x & 15) * 4;
    const float* src = d.u + (size_t)(r0 + r) * d.cols + c0 + c;
    in[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (r0 + r >= d.rows) continue;
    if (c0 + c + 4 <= d.cols) in[k] = *reinterpret_cast<const f32x4_any*>(src);
    else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c0 + c + e < d.cols) in[k][e] = src[e];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) tile_s[k * 16 + (threadIdx.x >> 4)][(threadIdx.x & 15) * 4 + e] = in[k][e];
  __syncthreads();
  const Factor scale = factor_of(over_norm((double)g.sigma, (sums[0] + sums[1]) + (sums[2] + sums[3]), d.eps));
  const size_t plane = (size_t)g.mp * g.np;
  _Float16* x = g.x[0] + mat * PLANES * plane;
  for (int k = threadIdx.x; k < 64 * 8; k += kThreads) {
    const int i = BLOCKS ? (k >> 7) * 16 + (k & 15) : k >> 3, j = BLOCKS ? ((k >> 4) & 7) * 8 : (k & 7) * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (tall ? tile_s[j + e][i] : tile_s[i][j + e]) * scale.lift * scale.main;
    split8<PLANES>(v, x + (BLOCKS ? place(g.np, i0 + i, j0 + j) : (size_t)(i0 + i) * g.np + j0 + j), plane);
  }
}

// 8 entries of one row of the parameter (bfloat16 with one plane, float32 with two) as they are before the step, requested ahead where they are whole
// 16-byte pieces.
template <int PLANES> struct Entries { u32x4 c[PLANES]; };
__device__ __forceinline__ bool whole8(const Matrix& d, int row, int col) { return row < d.rows && col + 8 <= d.cols; }
template <int PLANES>
__device__ __forceinline__ void request8(const Matrix& d, int row, int col, Entries<PLANES>& to) {
  if (!whole8(d, row, col)) return;
  const char* w = static_cast<const char*>(d.w) + ((size_t)row * d.cols + col) * (PLANES == 2 ? 4 : 2);
#pragma unroll
  for (int h = 0; h < PLANES; ++h) to.c[h] = *reinterpret_cast<const u32x4_any*>(w + 16 * h);
}
// w = keep * w - step * X; v: sigma X.
template <int PLANES>
__device__ __forceinline__ void apply8(const Matrix& d, float inv_sigma, const float (&v)[8], int row, int col, const Entries<PLANES>& old) {
  if (row >= d.rows || col >= d.cols) return;
  const float step = d.step * inv_sigma;
  const size_t at = (size_t)row * d.cols + col;
  if constexpr (PLANES == 1) {
    uint16_t* w = static_cast<uint16_t*>(d.w) + at;
    if (whole8(d, row, col)) {
      u32x4 out;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        out[e] = bf16_pack2(d.keep * __uint_as_float(old.c[0][e] << 16) - step * v[2 * e], d.keep * __uint_as_float(old.c[0][e] & 0xFFFF0000u) - step * v[2 * e + 1]);
      *reinterpret_cast<u32x4_any*>(w) = out;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < d.cols) w[e] = bf16_round(d.keep * bf(w[e]) - step * v[e]);
    }
  } else {
    float* w = static_cast<float*>(d.w) + at;
    if (whole8(d, row, col)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = d.keep * __uint_as_float(old.c[h][e]) - step * v[4 * h + e];
        *reinterpret_cast<f32x4_any*>(w + 4 * h) = out;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < d.cols) w[e] = d.keep * w[e] - step * v[e];
    }
  }
}

// One operand panel of a tile on its way to LDS: ROWS rows with k contiguous (RowK), or k-rows of ROWS columns (KRow), fetched by NW wavefronts.
template <int ROWS, Layout L, int NW>
struct Panel {
  static constexpr int kInstr = ROWS / (8 * NW);   // direct-to-LDS instructions of a wavefront: 64 chunks of 16 bytes each
  static_assert(ROWS % (8 * NW) == 0 && kInstr >= 1, "panel rows must fill whole wave instructions");
  const char* base;
  size_t step;
  uint32_t voff[kInstr];
  __device__ __forceinline__ void init(const _Float16* p, int ld, int row0, int wave, int lane) {
    step = L == Layout::RowK ? (size_t)kTileK * 2 : (size_t)kTileK * ld * 2;
    base = reinterpret_cast<const char*>(L == Layout::RowK ? p + (size_t)row0 * ld : p + row0);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int slot = (i * NW + wave) * 64 + lane;
      if constexpr (L == Layout::RowK) {
        const int row = slot >> 3, pc = slot & 7;
        voff[i] = (uint32_t)row * ld * 2u + (uint32_t)((((pc ^ row ^ ((row >> 3) & 3)) & 7) << 3) * 2);   // the inverse of lds_offset
      } else {
        constexpr int kRowChunks = ROWS / 8;
        const int k = slot / kRowChunks, pc = slot % kRowChunks;
        voff[i] = (uint32_t)k * ld * 2u + (uint32_t)((((pc - krow_rot<ROWS>(k) + kRowChunks) % kRowChunks) << 3) * 2);
      }
    }
  }
  __device__ __forceinline__ void load(int i, const char* at, char* tile, int wave) const {
    const uint32_t dst = (uint32_t)(uintptr_t)(gemm_dma_detail::lds_ptr_t)(tile + (i * NW + wave) * 1024);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(voff[i]), "s"(at), "s"(dst) : "m0", "memory");
  }
};

enum Mode { kGram = 0, kPoly = 1, kUpdate = 2, kFinal = 3 };

// Row and column of a matrix's tile number `tile`: those on and below the diagonal of a symmetric result, or all, down the columns.
template <int MODE>
__device__ __forceinline__ void place_tile(int tile, int tiles_m, int& ti, int& tj) {
  if constexpr (MODE == kGram || MODE == kPoly) {
    ti = (int)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    tj = tile - ti * (ti + 1) / 2;
  } else {
    tj = tile / tiles_m;
    ti = tile - tj * tiles_m;
  }
}

// From the sums of a product to what is stored, for 8 entries; s: kPoly's entries of A; diagonal: which of the 8 lies on the diagonal, if any.
template <int MODE, int PLANES>
__device__ __forceinline__ void finish8(float (&v)[8], float inv_sigma, const u32x4 (&s)[PLANES], int diagonal) {
  const float by = MODE == kGram ? kTau * inv_sigma * inv_sigma : MODE == kPoly ? kC / kTau : 1.f / kTau;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= by;
  if constexpr (MODE == kPoly) {
    float f[8];
    join8<PLANES>(s, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += kB * f[e] + (e == diagonal ? kA * kTau : 0.f);
  }
}

// kGram: A = X X^T.  kPoly: B = a I + b A + c A A.  kUpdate: X' = B X.  kFinal: the same, applied to the parameter.
// (a I inside B, so that the update reads nothing but the product's operands: X behind the tile loop once more was 200 MB of 24 matrices of 1024 x 4096, and
// its latency stood between the loop and the stores.)
// The matrices are padded to whole tiles with zeros, so nothing in the loop has an edge.
//
// Tile loop: a ring of STAGES tiles of 64 k, filled by direct-to-LDS loads.  A block is the MFMAs of one k-group (16 of k) on the
// fragments fetched during the block before; between them the wave issues the LDS reads of the next k-group and its share of a
// later tile's loads.  One barrier a tile, in front of its last k-group: by then the wave holds all of the tile in registers, so the
// buffer may be overwritten, and its own loads of the next tile have landed, so everybody may read that.
template <int MODE, int PLANES, int BT, int STAGES, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void product_kernel(Groups groups) {
  constexpr int NW = WAVES_M * WAVES_N;
  constexpr int WM = BT / WAVES_M, WN = BT / WAVES_N, TM = WM / 32, TN = WN / 32;
  static_assert(WM % 32 == 0 && WN % 32 == 0, "wave tile is a multiple of 32 x 32");
  constexpr int kPanelBytes = BT * 128, kStageBytes = 2 * PLANES * kPanelBytes;
  constexpr Layout LQ = MODE == kGram || MODE == kPoly ? Layout::RowK : Layout::KRow;
  constexpr int PARTS = STAGES >= 3 ? 4 : 2;           // a tile's loads: in every block, or in the two after the barrier
  constexpr int kSets = PLANES == 2 ? 3 : 1;           // products of planes
  constexpr int kMfma = kSets * TM * TN, kReads = PLANES * (TM + TN), kReadsPerSlot = (kReads + kMfma - 1) / kMfma;
  using SourceP = Panel<BT, Layout::RowK, NW>;
  using SourceQ = Panel<BT, LQ, NW>;
  constexpr int kLoads = 2 * PLANES * SourceP::kInstr;
  static_assert((STAGES - 2) * kLoads < 64, "vmcnt range");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int mat, tile;
  const Group& g = group_of<false>(groups, xcd_tile(blockIdx.x, gridDim.x), mat, tile);
  int ti, tj;
  place_tile<MODE>(tile, g.mp / BT, ti, tj);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WAVES_M, wn = wave / WAVES_M;
  const size_t plane_x = (size_t)g.mp * g.np, plane_a = (size_t)g.mp * g.mp;
  const _Float16* x = g.x[0] + mat * PLANES * plane_x;
  _Float16* a = g.a + mat * PLANES * plane_a;
  _Float16* b = g.b + mat * PLANES * plane_a;
  const size_t plane_p = (MODE == kGram ? plane_x : plane_a) * 2, plane_q = (MODE == kPoly ? plane_a : plane_x) * 2;   // bytes
  const int n = (MODE == kGram ? g.np : g.mp) / kTileK;

  SourceP sp;
  SourceQ sq;
  sp.init(MODE == kGram ? x : MODE == kPoly ? a : b, MODE == kGram ? g.np : g.mp, ti * BT, wave, lane);
  sq.init(MODE == kPoly ? a : x, MODE == kPoly ? g.mp : g.np, tj * BT, wave, lane);
  auto stage_of = [&](int t) { return lds + (t % STAGES) * kStageBytes; };
  auto issue_part = [&](int t, int part) {
    if (t >= n) return;
    char* stage = stage_of(t);
#pragma unroll
    for (int pl = 0; pl < PLANES; ++pl)
#pragma unroll
      for (int i = 0; i < SourceP::kInstr; ++i) {
        if ((2 * (pl * SourceP::kInstr + i)) % PARTS == part) sp.load(i, sp.base + t * sp.step + pl * plane_p, stage + pl * kPanelBytes, wave);
        if ((2 * (pl * SourceP::kInstr + i) + 1) % PARTS == part) sq.load(i, sq.base + t * sq.step + pl * plane_q, stage + (PLANES + pl) * kPanelBytes, wave);
      }
  };
  f32x16 acc[TM][TN], acc_lo[PLANES == 2 ? TM : 1][PLANES == 2 ? TN : 1];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        acc[i][j][r] = 0.f;
        if constexpr (PLANES == 2) acc_lo[i][j][r] = 0.f;
      }

  auto pin = [] { __builtin_amdgcn_sched_barrier(0); };   // the instruction scheduler moves nothing across this point
  auto lds_done = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
  u32x4 fp[2][PLANES * TM], fq[2][PLANES * TN];
  auto keep = [&](int set) {
#pragma unroll
    for (int i = 0; i < PLANES * TM; ++i) asm volatile("" : "+v"(fp[set][i]));
#pragma unroll
    for (int j = 0; j < PLANES * TN; ++j) asm volatile("" : "+v"(fq[set][j]));
  };
  using ReaderP = gemm_dma_detail::FragmentReader<BT, Layout::RowK, TM>;
  using ReaderQ = gemm_dma_detail::FragmentReader<BT, LQ, TN>;
  ReaderP reader_p;
  ReaderQ reader_q;
  reader_p.init(wm * WM, lane);
  reader_q.init(wn * WN, lane);
  struct At { uint32_t p[PLANES][ReaderP::kN], q[PLANES][ReaderQ::kN]; };
  At at, next;                                             // the tile being multiplied, the tile after it
  auto locate = [&](int t, At& where) {
    const uint32_t base = (uint32_t)(uintptr_t)(gemm_dma_detail::lds_ptr_t)stage_of(t);
#pragma unroll
    for (int pl = 0; pl < PLANES; ++pl) { reader_p.at(base + pl * kPanelBytes, where.p[pl]); reader_q.at(base + (PLANES + pl) * kPanelBytes, where.q[pl]); }
  };
  // read number R of k-group KG into set S
  auto fetch = [&](auto set, auto kg, auto r, const At& where) {
    constexpr int S = decltype(set)::value, KG = decltype(kg)::value, R = decltype(r)::value;
    if constexpr (R < PLANES * TM) fp[S][R] = ReaderP::template read<R % TM, KG>(where.p[R / TM]);
    else if constexpr (R < kReads) fq[S][R - PLANES * TM] = ReaderQ::template read<(R - PLANES * TM) % TN, KG>(where.q[(R - PLANES * TM) / TN]);
  };

#pragma unroll
  for (int t = 0; t < STAGES - 1; ++t)
#pragma unroll
    for (int part = 0; part < PARTS; ++part) issue_part(t, part);
  issue_part(STAGES - 1, 0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  pin();
  __builtin_amdgcn_s_barrier();
  pin();
  locate(0, next);
  gemm_detail::static_for<kReads>([&](auto r) { fetch(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, r, next); });

  for (int t = 0; t < n; ++t) {
    const bool more = t + 1 < n;
    locate(t, at);
    gemm_detail::static_for<4>([&](auto blk_c) {
      constexpr int blk = decltype(blk_c)::value, cur = blk & 1, nxt = cur ^ 1;
      constexpr bool last = blk == 3;
      lds_done();
      keep(cur);
      if constexpr (last) {
        if (STAGES >= 3 && t + STAGES - 1 < n) __builtin_amdgcn_s_waitcnt(gemm_dma_detail::waitcnt_imm((STAGES - 2) * kLoads, 15));
        else __builtin_amdgcn_s_waitcnt(gemm_dma_detail::waitcnt_imm(0, 15));
        pin();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        locate(t + 1, next);
      }
      pin();
      const bool fetching = !last || more;
      const int load_tile = last ? t + STAGES : t + STAGES - 1;
      constexpr int load_part = last ? 0 : blk + 1;
      gemm_detail::static_for<kMfma>([&](auto idx_c) {
        constexpr int idx = decltype(idx_c)::value;
        constexpr int set = idx / (TM * TN), i = (idx / TN) % TM, j = idx % TN;
        // with two planes: remainder x value, value x remainder, value x value.  (Operands exchanged: a lane then holds runs of four columns of one row.)
        constexpr int qi = (PLANES == 2 && set == 0 ? TN : 0) + j, pi = (PLANES == 2 && set == 1 ? TM : 0) + i;
        auto& into = [&]() -> f32x16& {
          if constexpr (PLANES == 2 && set < 2) return acc_lo[i][j];
          else return acc[i][j];
        }();
        into = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, fq[cur][qi]), __builtin_bit_cast(f16x8, fp[cur][pi]), into, 0, 0, 0);
        if (fetching)
          gemm_detail::static_for<kReadsPerSlot>([&](auto k) {
            constexpr int r = idx * kReadsPerSlot + decltype(k)::value;
            fetch(std::integral_constant<int, nxt>{}, std::integral_constant<int, last ? 0 : blk + 1>{}, std::integral_constant<int, r>{}, last ? next : at);
          });
        if constexpr (idx == 0 && load_part < PARTS) issue_part(load_tile, load_part);
        pin();
      });
    });
  }
  wait_loads_and_barrier<0>();   // every wave is done with the ring
  // What is stored, rounded to its planes in the registers, goes through the wave's own part of LDS, so that it moves in 16-byte pieces: as it
  // lies, and for a mirror image or a tall parameter transposed by the reads (ds_read_b64_tr_b16: of 4 rows of 16 columns each of 16 lanes gets
  // a column).  The whole tile at once: 32 rows at a time in float32 were four round trips to LDS, a third of the time of a product over k = 768.
  constexpr int kRow = WN * 2, kChunks = WN / 8, kPlane = WM * kRow;   // bytes of a row, its 16-byte chunks, bytes of a plane
  constexpr int kUnits = WM * WN / 512, kBatch = kUnits < 8 ? kUnits : 8;   // pieces of 8 entries of a lane
  static_assert(NW * PLANES * kPlane <= STAGES * kStageBytes, "the results fit in the ring");
  char* mine = lds + wave * (PLANES * kPlane);
  // a row's chunks are permuted by the row, so that the 32 rows of a fragment lie in different banks
  auto spot = [&](int row, int col) {
    constexpr int kShift = kChunks == 8 ? 1 : 2;
    return mine + row * kRow + ((((col >> 3) ^ (row >> kShift)) & (kChunks - 1)) << 4) + (col & 7) * 2;
  };
  const float inv_sigma = 1.f / g.sigma;
  const Matrix d = MODE == kFinal ? g.matrices[mat] : Matrix{};
  const bool turn = MODE == kFinal ? d.rows > d.cols : ti != tj;   // a mirror image to write, or a tall parameter
  const int row0 = ti * BT + wm * WM, col0 = tj * BT + wn * WN;
  // piece k of the lane: along the rows, and along the columns
  auto along_row = [&](int k, int& r, int& c) { r = (k * 64 + lane) / kChunks; c = (k * 64 + lane) % kChunks * 8; };
  auto along_col = [&](int k, int& r, int& c) { r = k / (WN / 16) * 32 + (lane >> 4) * 8; c = k % (WN / 16) * 16 + (lane & 15); };
  if constexpr (MODE == kPoly) {   // the entries of A, in the places of what they become part of
#pragma unroll
    for (int k0 = 0; k0 < kUnits; k0 += kBatch) {
      u32x4 in[kBatch][PLANES];
      int r, c;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        along_row(k0 + k, r, c);
#pragma unroll
        for (int pl = 0; pl < PLANES; ++pl) in[k][pl] = *reinterpret_cast<const u32x4*>(a + pl * plane_a + (size_t)(row0 + r) * g.mp + col0 + c);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        along_row(k0 + k, r, c);
#pragma unroll
        for (int pl = 0; pl < PLANES; ++pl) *reinterpret_cast<u32x4*>(spot(r, c) + pl * kPlane) = in[k][pl];
      }
    }
    gemm_dma_detail::lanes_together();
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int r = i * 32 + (lane & 31), c = j * 32 + 2 * e + 4 * (lane >> 5);
        char* place = spot(r, c);
        const float by = MODE == kGram ? kTau * inv_sigma * inv_sigma : MODE == kPoly ? kC / kTau : 1.f / kTau;
        f32x4 v = f32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        if constexpr (PLANES == 2) v += f32x4{acc_lo[i][j][e], acc_lo[i][j][e + 1], acc_lo[i][j][e + 2], acc_lo[i][j][e + 3]} * (1.f / kLoScale);
        v *= by;
        if constexpr (MODE == kPoly) {
          f32x4 s = __builtin_convertvector(*reinterpret_cast<const f16x4*>(place), f32x4);
          if constexpr (PLANES == 2) s += __builtin_convertvector(*reinterpret_cast<const f16x4*>(place + kPlane), f32x4) * (1.f / kLoScale);
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] += kB * s[q] + (row0 + r == col0 + c + q ? kA * kTau : 0.f);
        }
        if constexpr (PLANES == 2) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float one = v[q];
            settle(one);
            v[q] = one;
          }
        }
        const f16x4 hi = __builtin_convertvector(v, f16x4);
        *reinterpret_cast<f16x4*>(place) = hi;
        if constexpr (PLANES == 2) *reinterpret_cast<f16x4*>(place + kPlane) = __builtin_convertvector((v - __builtin_convertvector(hi, f32x4)) * kLoScale, f16x4);
      }
  gemm_dma_detail::lanes_together();
  // where entry (row, col) of the result lies
  auto result = [&](int row, int col) -> _Float16* {
    if constexpr (MODE == kUpdate) return g.x[1] + mat * PLANES * plane_x + (size_t)row * g.np + col;
    else return (MODE == kGram ? a : b) + (size_t)row * g.mp + col;
  };
  constexpr size_t kNone = 0;
  const size_t plane_out = MODE == kUpdate ? plane_x : MODE == kFinal ? kNone : plane_a;
  if (MODE != kFinal || !turn) {
#pragma unroll
    for (int k0 = 0; k0 < kUnits; k0 += kBatch) {
      Entries<PLANES> old[kBatch];
      int r, c;
      if constexpr (MODE == kFinal) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          along_row(k0 + k, r, c);
          request8<PLANES>(d, row0 + r, col0 + c, old[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        along_row(k0 + k, r, c);
        u32x4 w[PLANES];
#pragma unroll
        for (int pl = 0; pl < PLANES; ++pl) w[pl] = *reinterpret_cast<const u32x4*>(spot(r, c) + pl * kPlane);
        if constexpr (MODE == kFinal) {
          float v[8];
          join8<PLANES>(w, v);
          apply8<PLANES>(d, inv_sigma, v, row0 + r, col0 + c, old[k]);
        } else {
#pragma unroll
          for (int pl = 0; pl < PLANES; ++pl) *reinterpret_cast<u32x4*>(result(row0 + r, col0 + c) + pl * plane_out) = w[pl];
        }
      }
    }
  }
  if constexpr (MODE != kUpdate) {
    if (!turn) return;   // uniform over the workgroup
#pragma unroll
    for (int k0 = 0; k0 < kUnits; k0 += kBatch) {
      Entries<PLANES> old[kBatch];
      int r, c;
      if constexpr (MODE == kFinal) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          along_col(k0 + k, r, c);
          request8<PLANES>(d, col0 + c, row0 + r, old[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        along_col(k0 + k, r, c);
        u32x4 w[PLANES];
#pragma unroll
        for (int pl = 0; pl < PLANES; ++pl)
#pragma unroll
          for (int h = 0; h < 2; ++h) {   // this lane's word: 4 columns of row (lane % 16) / 4 of the 4
            const char* word = spot(r + 4 * h + ((lane & 15) >> 2), (c & ~15) + 4 * (lane & 3)) + pl * kPlane;
            const s16x4 got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(__attribute__((address_space(3))) const char*)word);
            const uint2 bits = __builtin_bit_cast(uint2, got);
            w[pl][2 * h] = bits.x; w[pl][2 * h + 1] = bits.y;
          }
        if constexpr (MODE == kFinal) {
          float v[8];
          join8<PLANES>(w, v);
          apply8<PLANES>(d, inv_sigma, v, col0 + c, row0 + r, old[k]);
        } else {
#pragma unroll
          for (int pl = 0; pl < PLANES; ++pl) *reinterpret_cast<u32x4*>(result(col0 + c, row0 + r) + pl * plane_out) = w[pl];
        }
      }
    }
  }
}

// The same products where there are few tiles and a product is a chain of latencies: tiles of 32 x 32, so that more CUs have one, whose k range
// the four wavefronts share.  Each has a ring of its own and waits on its own loads only; their partial tiles are added up through LDS, in
// wavefront order.  (One float32 matrix of 256 x 784: A = X X^T 10.1 us in tiles of 64 by four wavefronts in step.)
template <int MODE, int PLANES, int SW>
__global__ __launch_bounds__(kThreads) void small_product_kernel(Groups groups) {
  constexpr int BT = 32, NW = 4, LD = BT + 4;
  constexpr int kPanelBytes = BT * 128, kStageBytes = 2 * PLANES * kPanelBytes, kLoads = 2 * PLANES * (BT / 8);
  static_assert((SW - 1) * kLoads < 64, "vmcnt range");
  static_assert((size_t)NW * BT * LD * 4 <= (size_t)NW * SW * kStageBytes, "partial tiles fit in the rings");
  constexpr Layout LQ = MODE == kGram || MODE == kPoly ? Layout::RowK : Layout::KRow;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int mat, tile, ti, tj;
  const Group g = group_of<true>(groups, xcd_tile(blockIdx.x, gridDim.x), mat, tile);
  place_tile<MODE>(tile, g.mp / BT, ti, tj);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t plane_x = (size_t)g.mp * g.np, plane_a = (size_t)g.mp * g.mp;
  const _Float16* x = g.x[0] + mat * PLANES * plane_x;
  _Float16* a = g.a + mat * PLANES * plane_a;
  _Float16* b = g.b + mat * PLANES * plane_a;
  const size_t plane_p = (MODE == kGram ? plane_x : plane_a) * 2, plane_q = (MODE == kPoly ? plane_a : plane_x) * 2;   // bytes
  const int k_tiles = (MODE == kGram ? g.np : g.mp) / kTileK, per_wave = (k_tiles + NW - 1) / NW;
  const int first = min(wave * per_wave, k_tiles), n = min(first + per_wave, k_tiles) - first;
  char* ring = lds + wave * (SW * kStageBytes);
  Panel<BT, Layout::RowK, 1> sp;
  Panel<BT, LQ, 1> sq;
  sp.init(MODE == kGram ? x : MODE == kPoly ? a : b, MODE == kGram ? g.np : g.mp, ti * BT, 0, lane);
  sq.init(MODE == kPoly ? a : x, MODE == kPoly ? g.mp : g.np, tj * BT, 0, lane);
  auto issue = [&](int t) {
    char* stage = ring + (t % SW) * kStageBytes;
#pragma unroll
    for (int pl = 0; pl < PLANES; ++pl)
#pragma unroll
      for (int i = 0; i < BT / 8; ++i) {
        sp.load(i, sp.base + (first + t) * sp.step + pl * plane_p, stage + pl * kPanelBytes, 0);
        sq.load(i, sq.base + (first + t) * sq.step + pl * plane_q, stage + (PLANES + pl) * kPanelBytes, 0);
      }
  };
  // what this thread's 8 entries are combined with (threads of the first two wavefronts)
  const int r = (threadIdx.x & 127) >> 2, c = (threadIdx.x & 3) * 8;
  const Matrix d = MODE == kFinal ? g.matrices[mat] : Matrix{};
  const bool turn = MODE == kFinal ? d.rows > d.cols : ti != tj, finishes = threadIdx.x < 128;
  u32x4 held[PLANES];
  Entries<PLANES> old;
  if (finishes) {
    if constexpr (MODE == kPoly) {
#pragma unroll
      for (int pl = 0; pl < PLANES; ++pl) held[pl] = *reinterpret_cast<const u32x4*>(a + pl * plane_a + (size_t)(ti * BT + r) * g.mp + tj * BT + c);
    } else if constexpr (MODE == kFinal) {
      request8<PLANES>(d, (turn ? tj : ti) * BT + r, (turn ? ti : tj) * BT + c, old);
    }
  }
#pragma unroll
  for (int s = 0; s < SW; ++s)
    if (s < n) issue(s);
  f32x16 acc, acc_lo;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = acc_lo[e] = 0.f;
  using ReaderP = gemm_dma_detail::FragmentReader<BT, Layout::RowK, 1>;
  using ReaderQ = gemm_dma_detail::FragmentReader<BT, LQ, 1>;
  ReaderP reader_p;
  ReaderQ reader_q;
  reader_p.init(0, lane);
  reader_q.init(0, lane);
  for (int t = 0; t < n; ++t) {
    asm volatile("" ::: "memory");
    if (t + SW <= n) __builtin_amdgcn_s_waitcnt(gemm_dma_detail::waitcnt_imm((SW - 1) * kLoads, 15));
    else __builtin_amdgcn_s_waitcnt(gemm_dma_detail::waitcnt_imm(0, 15));
    asm volatile("" ::: "memory");
    const uint32_t base = (uint32_t)(uintptr_t)(gemm_dma_detail::lds_ptr_t)(ring + (t % SW) * kStageBytes);
    u32x4 fp[4 * PLANES], fq[4 * PLANES];
    gemm_detail::static_for<PLANES>([&](auto pl_c) {
      constexpr int pl = decltype(pl_c)::value;
      uint32_t at_p[ReaderP::kN], at_q[ReaderQ::kN];
      reader_p.at(base + pl * kPanelBytes, at_p);
      reader_q.at(base + (PLANES + pl) * kPanelBytes, at_q);
      gemm_detail::static_for<4>([&](auto kg) {
        fp[pl * 4 + decltype(kg)::value] = ReaderP::template read<0, decltype(kg)::value>(at_p);
        fq[pl * 4 + decltype(kg)::value] = ReaderQ::template read<0, decltype(kg)::value>(at_q);
      });
    });
    gemm_dma_detail::fragments_ready(fp, fq);
    if (t + SW < n) issue(t + SW);   // over the tile that is in registers now
#pragma unroll
    for (int kg = 0; kg < 4; ++kg) {
      auto mfma = [&](const u32x4& qf, const u32x4& pf, f32x16& into) {
        into = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, qf), __builtin_bit_cast(f16x8, pf), into, 0, 0, 0);
      };
      mfma(fq[kg], fp[kg], acc);
      if constexpr (PLANES == 2) {
        mfma(fq[4 + kg], fp[kg], acc_lo);
        mfma(fq[kg], fp[4 + kg], acc_lo);
      }
    }
  }
  if constexpr (PLANES == 2) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += acc_lo[e] * (1.f / kLoScale);
  }
  __syncthreads();   // every ring is dead
  float* parts = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int e = 0; e < 16; e += 4)
    *reinterpret_cast<f32x4*>(parts + wave * (BT * LD) + (lane & 31) * LD + 2 * e + 4 * (lane >> 5)) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  __syncthreads();
  const float inv_sigma = 1.f / g.sigma;
  if (finishes) {
    float* at_s = parts + r * LD + c;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = ((at_s[e] + at_s[BT * LD + e]) + at_s[2 * BT * LD + e]) + at_s[3 * BT * LD + e];
    const int row = ti * BT + r, col = tj * BT + c;
    finish8<MODE, PLANES>(v, inv_sigma, held, row - col);
    if constexpr (MODE == kGram) split8<PLANES>(v, a + (size_t)row * g.mp + col, plane_a);
    else if constexpr (MODE == kPoly) split8<PLANES>(v, b + (size_t)row * g.mp + col, plane_a);
    else if constexpr (MODE == kUpdate) split8<PLANES>(v, g.x[1] + mat * PLANES * plane_x + (size_t)row * g.np + col, plane_x);
    else if (!turn) apply8<PLANES>(d, inv_sigma, v, row, col, old);
#pragma unroll
    for (int e = 0; e < 8; ++e) at_s[e] = v[e];
  }
  if constexpr (MODE != kUpdate) {
    if (!turn) return;   // uniform over the workgroup
    __syncthreads();
    if (!finishes) return;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = parts[(c + e) * LD + r];
    const int row = tj * BT + r, col = ti * BT + c;
    if constexpr (MODE == kGram) split8<PLANES>(v, a + (size_t)row * g.mp + col, plane_a);
    else if constexpr (MODE == kPoly) split8<PLANES>(v, b + (size_t)row * g.mp + col, plane_a);
    else apply8<PLANES>(d, inv_sigma, v, row, col, old);
  }
}

// ---- steps of two launches ------------------------------------------------------------------------------------------

// Matrices of a padded shorter side of at most 256, as long as there are few of them: what a step takes is launches, 3 us and more each whatever they do, and
// latency.  X and A lie in blocks (`place`), so that operands go from memory to registers.  One step of the optimiser against three launches a step: 4 of 60 x 60 in
// bfloat16 41 us (60), one of 256 x 784 51 (66), in float32 69 (83), 24 of 128 x 512 in float32 66 (96), 4 of 128 x 4000 in float32 100 (149).
constexpr int kStrip = 16;                // columns of a workgroup of pair_kernel
constexpr int kShareThreads = 512;

// A = X X^T in tiles of T x T, those on and below the diagonal; eight wavefronts share the long side and have their next AHEAD pieces of 64 of it in flight.  Their
// partial tiles are added up in wavefront order.  256 x 784 in float32: 3.8 us, where tiles of 32 through LDS by four wavefronts take 5.9.
template <int PLANES, int T, int AHEAD>
__global__ __launch_bounds__(kShareThreads) void share_gram_kernel(Groups groups) {
  constexpr int NW = kShareThreads / 64, TB = T / 16, LD = T + 4;
  __shared__ __attribute__((aligned(16))) float parts[NW * T * LD];
  int mat, tile, ti, tj;
  const Group g = group_of<true>(groups, xcd_tile(blockIdx.x, gridDim.x), mat, tile);
  place_tile<kGram>(tile, g.mp / T, ti, tj);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t plane_x = (size_t)g.mp * g.np, plane_a = (size_t)g.mp * g.mp;
  const int pieces = g.np / 64, first = wave * pieces / NW, n = (wave + 1) * pieces / NW - first;
  const _Float16* x = g.x[0] + mat * PLANES * plane_x + (size_t)first * 1024 + lane * 8;
  const _Float16* p = x + (size_t)(ti * TB) * (g.np / 32) * 512;   // the blocks of a row of blocks lie behind one another
  const _Float16* q = x + (size_t)(tj * TB) * (g.np / 32) * 512;
  u32x4 fp[AHEAD][2][TB][PLANES], fq[AHEAD][2][TB][PLANES];
  auto load = [&](auto slot, int u) {
    constexpr int S = decltype(slot)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int pl = 0; pl < PLANES; ++pl) {
          const size_t at = pl * plane_x + (size_t)i * (g.np / 32) * 512 + (size_t)(2 * u + h) * 512;
          fp[S][h][i][pl] = *reinterpret_cast<const u32x4*>(p + at);
          fq[S][h][i][pl] = *reinterpret_cast<const u32x4*>(q + at);
        }
  };
  f32x4 acc[TB][TB] = {}, lo[TB][TB] = {};
  gemm_detail::static_for<AHEAD>([&](auto slot) {
    if (decltype(slot)::value < n) load(slot, decltype(slot)::value);
  });
  for (int u = 0; u < n; u += AHEAD)
    gemm_detail::static_for<AHEAD>([&](auto slot) {
      constexpr int S = decltype(slot)::value;
      if (u + S < n) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < TB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) {   // (operands exchanged: a lane then holds four columns of one row)
              auto mfma = [&](int pq, int pp, f32x4& into) {
                into = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, fq[S][h][j][pq]), __builtin_bit_cast(f16x8, fp[S][h][i][pp]), into, 0, 0, 0);
              };
              mfma(0, 0, acc[i][j]);
              if constexpr (PLANES == 2) {
                mfma(1, 0, lo[i][j]);
                mfma(0, 1, lo[i][j]);
              }
            }
        if (u + S + AHEAD < n) load(slot, u + S + AHEAD);
      }
    });
#pragma unroll
  for (int i = 0; i < TB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      if constexpr (PLANES == 2) acc[i][j] += lo[i][j] * (1.f / kLoScale);
      *reinterpret_cast<f32x4*>(&parts[wave * (T * LD) + (16 * i + (lane & 15)) * LD + 16 * j + 4 * (lane >> 4)]) = acc[i][j];
    }
  __syncthreads();
  constexpr int kFinish = T * T / 8;      // threads with 8 entries each
  const int r = (threadIdx.x & (kFinish - 1)) % T, c = (threadIdx.x & (kFinish - 1)) / T * 8;
  const float inv_sigma = 1.f / g.sigma;
  _Float16* a = g.a + mat * PLANES * plane_a;
  float* at_s = parts + r * LD + c;
  float v[8];
  if (threadIdx.x < kFinish) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float sum = at_s[e];
#pragma unroll
      for (int w = 1; w < NW; ++w) sum += at_s[w * (T * LD) + e];
      v[e] = sum * (kTau * inv_sigma * inv_sigma);
      at_s[e] = v[e];
    }
    split8<PLANES>(v, a + place(g.mp, ti * T + r, tj * T + c), plane_a);
  }
  if (ti == tj) return;
  __syncthreads();
  if (threadIdx.x >= kFinish) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = parts[(c + e) * LD + r];
  split8<PLANES>(v, a + place(g.mp, tj * T + r, ti * T + c), plane_a);
}

// The second and third product of a step in one launch: X' = a X + A Z with Z = b X + c A X, for a strip of 16 columns, whose products need nothing of the other
// strips.  A wavefront has 32 rows; its part of A, the left operand of both products, goes from memory to registers and stays there, and the strip's X and Z
// lie transposed in LDS, k contiguous.  Z takes the place of B as what is rounded to float16 in between: |Z| <= 2.9 in the spectral norm where X stays
// below 1.3, so sigma |z| <= 2.9 * 2^14.  256 x 784 takes 7.9 us in float32 and 4.5 in bfloat16 on 52 CUs, and 13 and 7.3 with A in rows, where a quarter of a wavefront's
// load asks for 16 lines.  No rate bounds it: of the 7.9 the least launch is 3, the load of A at 64 bytes a clock into a CU 1.7 and the multiplications 1.3 (in bfloat16
// 0.9 and 0.4 of 4.5); the rest is a chain of loads, LDS round trips and three barriers that wait for one another.
template <bool FINAL, int PLANES, int MP>
__device__ __forceinline__ void pair_strip(const Group& g, int mat, int strip, char* lds) {
  constexpr int W = kStrip, LD = MP + 8, LF = MP + 4, STEPS = MP / 32;
  if (threadIdx.x >= 2 * MP) return;   // whole wavefronts: the workgroup has as many as the largest matrix of the launch needs
  _Float16* xt = reinterpret_cast<_Float16*>(lds);
  _Float16* zt = xt + PLANES * W * LD;
  float* out = reinterpret_cast<float*>(zt + PLANES * W * LD);
  const int lane = threadIdx.x & 63, row0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 32, col0 = strip * W;
  const size_t plane_x = (size_t)MP * g.np;
  constexpr size_t plane_a = (size_t)MP * MP;
  const _Float16* x = g.x[0] + mat * PLANES * plane_x;
  const _Float16* a = g.a + mat * PLANES * plane_a;
  const Matrix d = FINAL ? g.matrices[mat] : Matrix{};
  const bool turn = FINAL && d.rows > d.cols;
  const int row = (threadIdx.x >> 5) * 16 + (threadIdx.x & 15), c = ((threadIdx.x >> 4) & 1) * 8;   // this thread's 8 entries of X and, as they lie, of X'
  const int tn = threadIdx.x / (MP / 8), tc = threadIdx.x % (MP / 8) * 8;                             // and of a tall parameter
  u32x4 in[PLANES];
#pragma unroll
  for (int pl = 0; pl < PLANES; ++pl) in[pl] = *reinterpret_cast<const u32x4*>(x + pl * plane_x + place(g.np, row, col0 + c));
  u32x4 fa[2][STEPS][PLANES];
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int pl = 0; pl < PLANES; ++pl)   // `place` of row row0 + 16 i + lane % 16, column 32 s + 8 (lane / 16)
        fa[i][s][pl] = *reinterpret_cast<const u32x4*>(a + pl * plane_a + ((size_t)((row0 >> 4) + i) * STEPS + s) * 512 + lane * 8);
  Entries<PLANES> old;
  if (FINAL) request8<PLANES>(d, turn ? col0 + tn : row, turn ? tc : col0 + c, old);
#pragma unroll
  for (int pl = 0; pl < PLANES; ++pl) {
    const f16x8 w = __builtin_bit_cast(f16x8, in[pl]);
#pragma unroll
    for (int e = 0; e < 8; ++e) xt[pl * W * LD + (c + e) * LD + row] = w[e];
  }
  __syncthreads();
  const int n = lane & 15, kg = lane >> 4;
  f32x4 acc[2];
  auto multiply = [&](const _Float16* right) {
    f32x4 lo[2] = {};
    acc[0] = acc[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      f16x8 q[PLANES];
#pragma unroll
      for (int pl = 0; pl < PLANES; ++pl) q[pl] = *reinterpret_cast<const f16x8*>(right + pl * W * LD + n * LD + s * 32 + kg * 8);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f16x8 p = __builtin_bit_cast(f16x8, fa[i][s][0]);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q[0], acc[i], 0, 0, 0);
        if constexpr (PLANES == 2) {
          lo[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, fa[i][s][1]), q[0], lo[i], 0, 0, 0);
          lo[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q[1], lo[i], 0, 0, 0);
        }
      }
    }
    if constexpr (PLANES == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i] += lo[i] * (1.f / kLoScale);
    }
  };
  multiply(xt);
  f32x4 own[2];   // of X, where this lane has sums
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = n * LD + row0 + 16 * i + 4 * kg;
    own[i] = __builtin_convertvector(*reinterpret_cast<const f16x4*>(xt + at), f32x4);
    if constexpr (PLANES == 2) own[i] += __builtin_convertvector(*reinterpret_cast<const f16x4*>(xt + W * LD + at), f32x4) * (1.f / kLoScale);
    f32x4 z;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float one = kB * own[i][q] + kC / kTau * acc[i][q];
      if constexpr (PLANES == 2) settle(one);
      z[q] = one;
    }
    const f16x4 hi = __builtin_convertvector(z, f16x4);
    *reinterpret_cast<f16x4*>(zt + at) = hi;
    if constexpr (PLANES == 2) *reinterpret_cast<f16x4*>(zt + W * LD + at) = __builtin_convertvector((z - __builtin_convertvector(hi, f32x4)) * kLoScale, f16x4);
  }
  __syncthreads();
  multiply(zt);
#pragma unroll
  for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4*>(out + n * LF + row0 + 16 * i + 4 * kg) = kA * own[i] + acc[i] * (1.f / kTau);
  __syncthreads();
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = turn ? out[tn * LF + tc + e] : out[(c + e) * LF + row];
  if constexpr (FINAL) apply8<PLANES>(d, 1.f / g.sigma, v, turn ? col0 + tn : row, turn ? tc : col0 + c, old);
  else split8<PLANES>(v, g.x[1] + mat * PLANES * plane_x + place(g.np, row, col0 + c), plane_x);
}
// MOST: the largest shorter side of the launch.
template <bool FINAL, int PLANES, int MOST>
__global__ __launch_bounds__(2 * MOST) void pair_kernel(Groups groups) {
  __shared__ __attribute__((aligned(16))) char lds[kStrip * (2 * PLANES * 2 * (MOST + 8) + 4 * (MOST + 4))];
  int mat, strip;
  const Group g = group_of<true>(groups, xcd_tile(blockIdx.x, gridDim.x), mat, strip);
  if (g.mp == 64) return pair_strip<FINAL, PLANES, 64>(g, mat, strip, lds);
  if constexpr (MOST >= 128)
    if (g.mp == 128) return pair_strip<FINAL, PLANES, 128>(g, mat, strip, lds);
  if constexpr (MOST >= 256) {
    if (g.mp == 192) return pair_strip<FINAL, PLANES, 192>(g, mat, strip, lds);
    return pair_strip<FINAL, PLANES, 256>(g, mat, strip, lds);
  }
}

// ---- matrices with a short side of at most 32 or 48 -----------------------------------------------------------------

// The steps' polynomials commute with A = X X^T, so for a matrix of a short side the whole chain can run on that one small matrix: with
// B_k = a I + b A_k + c A_k^2,  A_{k+1} = A_k B_k^2  and  X_steps = (B_{steps-1} ... B_0) X_0.  That squares singular values, and rounding in A_0 grows
// up to a^2 = 11.9 times a step where they are small: in float32 too much of it, in float64 at most 1e-16 * 11.9^7 = 3e-9 by the eighth step, which
// is where it is used.  Three launches in place of three a step: the entries of A in float64 from slices of the long side, one workgroup a matrix
// for the chain, the product with u and the update.  The chain is bound by one CU's float64 matrix rate and
// LDS.  A step of the optimiser, and in brackets as products of the whole matrix: 16 x 100 25 us (41), 32 x 300 33 (42), 16 of 32 x 2000 42 (51), in float32 40 (68); from 33
// on bfloat16 ones no longer gain (48 x 300: 48 (43)), and float32 ones, whose products are three, about as much as they lose (48 x 300: 47 (45), 16 of 48 x 2000: 59 (71)).
constexpr int narrow_side(int planes) { return planes == 2 ? 48 : 32; }
constexpr int kNarrow = narrow_side(2), kNarrowLong = 8192, kNarrowSteps = 8, kNarrowCount = 256, kMaxSlices = 16, kNarrowTiles = 6;
typedef double f64x4 __attribute__((ext_vector_type(4)));

struct NarrowGroup {
  const Matrix* matrices;
  double* partial;         // [count][slices][tiles][256]: 16 x 16 tiles of u u^T on and below the diagonal
  float* q;                // [count][shorter][shorter], and behind the matrices [count] factors 1 / (|u| + eps) in two
  int shorter, longer, count, tiles, slices, first_block;
};
struct NarrowGroups {
  NarrowGroup g[kMaxGroups];
  int n;
};
// which matrix of which group, and which of its `per` workgroups
template <class F>
__device__ __forceinline__ NarrowGroup narrow_group(const NarrowGroups& t, int block, F&& per, int& mat, int& part) {
  NarrowGroup g = t.g[0];
  for (int j = 1; j < t.n; ++j)
    if (block >= t.g[j].first_block) g = t.g[j];
  const int local = block - g.first_block, p = per(g);
  mat = local / p;
  part = local - mat * p;
  return g;
}
// Row and column of tile number t on and below the diagonal (at most six).
__device__ __forceinline__ void lower_tile(int t, int& ti, int& tj) {
  ti = t >= 3 ? 2 : t >= 1 ? 1 : 0;
  tj = t - ti * (ti + 1) / 2;
}
// u's entries of P positions of the long side from `at` on, P / 4 of them a thread; which row of the short side and which position entry k of the thread is.
template <int P>
struct NarrowChunk {
  static constexpr int kEach = P / 4;
  int shorter, longer;
  float inv;               // 1 / shorter: entries are numbered below 2^12, which float32 divides exactly
  bool tall;
  __device__ __forceinline__ bool place(int k, int& i, int& j) const {
    const int e = k * kThreads + threadIdx.x;
    if (tall) { j = (int)(((float)e + 0.5f) * inv); i = e - j * shorter; }
    else { i = e / P; j = e % P; }
    return i < shorter && j < P;
  }
  __device__ __forceinline__ void load(const float* u, int at, float (&v)[kEach]) const {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      int i, j;
      const bool has = place(k, i, j) && at + j < longer;
      v[k] = has ? u[tall ? (size_t)(at + j) * shorter + i : (size_t)i * longer + at + j] : 0.f;
    }
  }
  // to[i][j] = by * v
  template <int LD>
  __device__ __forceinline__ void park(const float (&v)[kEach], float by, float (*to)[LD]) const {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      int i, j;
      if (place(k, i, j)) to[i][j] = v[k] * by;
    }
  }
};

__global__ __launch_bounds__(kThreads) void narrow_gram_kernel(NarrowGroups groups) {
  __shared__ float xs[kNarrow][65];
  __shared__ double sums[4 * kNarrowTiles * 256];   // [4 wavefronts][tiles][256]
  int mat, slice;
  const NarrowGroup g = narrow_group(groups, blockIdx.x, [](const NarrowGroup& q) { return q.slices; }, mat, slice);
  const Matrix d = g.matrices[mat];
  const NarrowChunk<64> chunk = {g.shorter, g.longer, 1.f / (float)g.shorter, d.rows > d.cols};
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m16 = (g.shorter + 15) / 16;
  for (int e = threadIdx.x; e < kNarrow * 65; e += kThreads) (&xs[0][0])[e] = 0.f;   // rows beyond the short side stay so
  f64x4 acc[kNarrowTiles];
#pragma unroll
  for (int t = 0; t < kNarrowTiles; ++t) acc[t] = f64x4{0.0, 0.0, 0.0, 0.0};
  float next[16];
  const int step = 64 * g.slices;
  chunk.load(d.u, slice * 64, next);
  for (int at = slice * 64; at < g.longer; at += step) {
    __syncthreads();
    chunk.park(next, 1.f, xs);
    __syncthreads();
    chunk.load(d.u, at + step, next);
    // a wavefront takes a quarter of the positions, for all tiles
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int j = wave * 16 + s * 4 + (lane >> 4);
      double row[kNarrow / 16];
#pragma unroll
      for (int t = 0; t < kNarrow / 16; ++t) row[t] = t < m16 ? (double)xs[t * 16 + (lane & 15)][j] : 0.0;
#pragma unroll
      for (int t = 0; t < kNarrowTiles; ++t) {
        int ti, tj;
        lower_tile(t, ti, tj);
        if (ti < m16) acc[t] = __builtin_amdgcn_mfma_f64_16x16x4f64(row[ti], row[tj], acc[t], 0, 0, 0);   // uniform
      }
    }
  }
  double* mine = sums + wave * (kNarrowTiles * 256);
#pragma unroll
  for (int t = 0; t < kNarrowTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) mine[t * 256 + (4 * r + (lane >> 4)) * 16 + (lane & 15)] = acc[t][r];
  __syncthreads();
  double* out = g.partial + ((size_t)mat * g.slices + slice) * g.tiles * 256;
  for (int e = threadIdx.x; e < g.tiles * 256; e += kThreads)
    out[e] = (sums[e] + sums[kNarrowTiles * 256 + e]) + (sums[2 * kNarrowTiles * 256 + e] + sums[3 * kNarrowTiles * 256 + e]);
}

// doubles from row to row in LDS: 16 rows of 4 consecutive entries, as an operand is read, lie in as many places
constexpr int narrow_pitch(int m16) { return 16 * m16 + 4; }
constexpr size_t narrow_lds(int m16) { return (4 * 16 * (size_t)m16 * narrow_pitch(m16) + 2) * sizeof(double); }

// A wavefront a tile on and below the diagonal: the matrix cores of a CU take them in turn.
constexpr int kChainThreads = 64 * kNarrowTiles;
template <int M16>
__device__ __forceinline__ void narrow_chain(const NarrowGroup& g, int mat, int steps, double* a) {
  constexpr int kPitch = narrow_pitch(M16), kSize = 16 * M16 * kPitch, kTiles = M16 * (M16 + 1) / 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double* b = a + kSize;
  double* t = b + kSize;
  double* q = t + kSize;
  double* norm = q + kSize;
  auto put = [&](double* m, int i, int j, double v) { m[i * kPitch + j] = v; m[j * kPitch + i] = v; };
  for (int e = threadIdx.x; e < kTiles * 256; e += kChainThreads) {
    int ti, tj;
    lower_tile(e >> 8, ti, tj);
    const double* p = g.partial + (size_t)mat * g.slices * kTiles * 256 + e;
    double s = 0.0;
#pragma unroll 8
    for (int i = 0; i < g.slices; ++i) s += p[(size_t)i * kTiles * 256];
    const int i = ti * 16 + ((e >> 4) & 15), j = tj * 16 + (e & 15);
    if (i >= j) put(a, i, j, s);
  }
  __syncthreads();
  if (wave == 0) {   // the trace is |u|^2
    double s = lane < 16 * M16 ? a[lane * kPitch + lane] : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) *norm = over_norm(1.0, s, g.matrices[mat].eps);
  }
  __syncthreads();
  const double inv = *norm;
  for (int e = threadIdx.x; e < kSize; e += kChainThreads) a[e] = a[e] * inv * inv;
  __syncthreads();
  int ti, tj;
  lower_tile(wave, ti, tj);
  // out = finish(p r) for symmetric p and r whose product is symmetric: tiles on and below the diagonal, each written twice
  auto product = [&](const double* p, const double* r, double* out, auto finish) {
    if (wave < kTiles) {
      const double* pi = p + (ti * 16 + (lane & 15)) * kPitch + (lane >> 4);
      const double* rj = r + (tj * 16 + (lane & 15)) * kPitch + (lane >> 4);
      double x[4 * M16], y[4 * M16];
#pragma unroll
      for (int s = 0; s < 4 * M16; ++s) { x[s] = pi[4 * s]; y[s] = rj[4 * s]; }
      f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int s = 0; s < 4 * M16; ++s) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(x[s], y[s], acc, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = ti * 16 + 4 * e + (lane >> 4), j = tj * 16 + (lane & 15);
        if (i >= j) put(out, i, j, finish(acc[e], i, j));
      }
    }
    __syncthreads();
  };
  auto as_is = [](double v, int, int) { return v; };
  for (int k = 0; k < steps; ++k) {
    product(a, a, b, [&](double v, int i, int j) { return (double)kC * v + (double)kB * a[i * kPitch + j] + (i == j ? (double)kA : 0.0); });
    if (k > 0) {
      product(q, b, t, as_is);
      double* old = q;
      q = t; t = old;
    }
    if (k + 1 == steps) break;
    product(a, b, t, as_is);
    product(t, b, a, as_is);
    if (k == 0) {            // the chain's product so far is B itself
      double* spare = q;
      q = b; b = spare;
    }
  }
  const double* chain = steps == 1 ? b : q;
  float* out = g.q + (size_t)mat * g.shorter * g.shorter;
  for (int e = threadIdx.x; e < g.shorter * g.shorter; e += kChainThreads) out[e] = (float)chain[(e / g.shorter) * kPitch + e % g.shorter];
  if (threadIdx.x == 0) reinterpret_cast<Factor*>(g.q + (size_t)g.count * g.shorter * g.shorter)[mat] = factor_of(inv);
}

__global__ __launch_bounds__(kChainThreads) void narrow_chain_kernel(NarrowGroups groups, int steps) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int mat, none;
  const NarrowGroup g = narrow_group(groups, blockIdx.x, [](const NarrowGroup&) { return 1; }, mat, none);
  double* a = reinterpret_cast<double*>(lds);
  switch (g.tiles) {   // uniform over the workgroup
    case 1: narrow_chain<1>(g, mat, steps, a); break;
    case 3: narrow_chain<2>(g, mat, steps, a); break;
    default: narrow_chain<3>(g, mat, steps, a);
  }
}

// w = keep * w - step * Q u / (|u| + eps), 32 positions of the long side a workgroup, 4 x 2 entries a thread.
constexpr int kApply = 32;
__global__ __launch_bounds__(kThreads) void narrow_apply_kernel(NarrowGroups groups) {
  __shared__ __attribute__((aligned(16))) float us[kNarrow][kApply + 4], qs[kNarrow][64 + 4];   // [k][j], [k][i]
  int mat, part;
  const NarrowGroup g = narrow_group(groups, blockIdx.x, [](const NarrowGroup& q) { return (q.longer + kApply - 1) / kApply; }, mat, part);
  const Matrix d = g.matrices[mat];
  const float* q = g.q + (size_t)mat * g.shorter * g.shorter;
  const Factor inv = reinterpret_cast<const Factor*>(g.q + (size_t)g.count * g.shorter * g.shorter)[mat];
  constexpr int kRows = kNarrow / 4;
  float qv[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int row = k * 4 + (threadIdx.x >> 6), i = threadIdx.x & 63;
    qv[k] = row < g.shorter && i < g.shorter ? q[row * g.shorter + i] : 0.f;   // (symmetric)
  }
  const bool tall = d.rows > d.cols;
  const NarrowChunk<kApply> chunk = {g.shorter, g.longer, 1.f / (float)g.shorter, tall};
  float v[kApply / 4];
  chunk.load(d.u, part * kApply, v);
  // the entries of a run of lanes lie side by side in the parameter
  const int i0 = (tall ? threadIdx.x & 15 : threadIdx.x >> 4) * 4, j0 = (tall ? threadIdx.x >> 4 : threadIdx.x & 15) * 2;
  auto place = [&](int i, int j, size_t& at) {
    i += i0; j += part * kApply + j0;
    at = tall ? (size_t)j * g.shorter + i : (size_t)i * g.longer + j;
    return i < g.shorter && j < g.longer;
  };
  float old[4][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      size_t at;
      old[i][j] = 0.f;
      if (place(i, j, at)) old[i][j] = d.bf16 ? bf(static_cast<const uint16_t*>(d.w)[at]) : static_cast<const float*>(d.w)[at];
    }
#pragma unroll
  for (int k = 0; k < kRows; ++k) qs[k * 4 + (threadIdx.x >> 6)][threadIdx.x & 63] = qv[k];
#pragma unroll
  for (int k = 0; k < kApply / 4; ++k) v[k] *= inv.lift;
  chunk.park(v, inv.main, us);
  __syncthreads();
  float acc[4][2] = {};
#pragma unroll 8
  for (int k = 0; k < g.shorter; ++k) {
    const f32x4 qi = *reinterpret_cast<const f32x4*>(&qs[k][i0]);
    const float2 uj = *reinterpret_cast<const float2*>(&us[k][j0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) { acc[i][0] += qi[i] * uj.x; acc[i][1] += qi[i] * uj.y; }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      size_t at;
      if (!place(i, j, at)) continue;
      const float w = d.keep * old[i][j] - d.step * acc[i][j];
      if (d.bf16) static_cast<uint16_t*>(d.w)[at] = bf16_round(w);
      else static_cast<float*>(d.w)[at] = w;
    }
}

// ---- plan -----------------------------------------------------------------------------------------------------------

// What a product of `count` matrices in tiles of `tile` takes, in us, from these kernels' times over 1 to 64 matrices of 64 x 64 to 4096 x 4096: rounds of
// workgroups over the 256 CUs, each a start and an end (2 to 8 us) and so much for every 64 of k, less where a round is alone.  The short rounds of tiles of 32 run into one
// another: a tenth or a third of a round on top, not a whole one (one product of 1024 x 1024 x 1024 in bfloat16, 528 tiles: 7 us, with tiles of 64 9).  Tiles of 64 and of 256 have a CU to
// themselves (rings of 96 and 128 KB); those of 128 share one with another once there are more than CUs (24 products of 1024 x 4096 x 1024: 272 us so, 345 us
// alone on a ring of four), and have it to themselves before (136 tiles over k = 2048: 26 against 23).  One float32 product of 1024 x 1024 x 1024: tiles
// of 64 13 us, of 128 24; 16 of them: 175 and 112.  Symmetric ones in many rounds: 19 matrices
// of 617 x 1467, both products of a step in tiles of 64 145 us, of 128 126 (the 0.7 rests on this one shape).  One of 256 x 256 x 784: tiles of 32 6.0 us, of 64 10.5; one bfloat16 product of 512 cubed 4.2 and 6.2, of 2048
// cubed 80 and 55, and in tiles of 128 25.  48 of 768 x 768 x 768: tiles of 128 62 us, of 256 53; their symmetric halves 44 and 53.
double product_cost(int mode, long long tiles, int tile, int planes, int k) {
  const double steps = k / 64;
  auto rounds = [&](int at_once) { return (double)((tiles + at_once - 1) / at_once); };
  const bool alone = tiles <= 256;
  if (planes == 2) {
    if (tile == 32) return alone ? 3.6 + 0.16 * steps : (tiles / 256.0 + 0.35) * (3.2 + 0.26 * steps);
    if (tile == 64) return alone ? 4.7 + 0.42 * steps : rounds(256) * (2.0 + (mode == kGram || mode == kPoly ? 0.7 : 0.56) * steps);
    return rounds(256) * (5.0 + 1.44 * steps);
  }
  if (tile == 32) return alone ? 2.8 + 0.09 * steps : std::max(tiles / 512.0 + 0.1, 1.0) * (2.0 + 0.24 * steps);
  if (tile == 64) return alone ? 4.2 + 0.29 * steps : rounds(256) * (2.8 + 0.29 * steps);
  if (tile == 128) return alone ? 5.0 + 0.6 * steps : rounds(512) * (6.0 + 1.0 * steps);
  return rounds(256) * (8.0 + 1.64 * steps);
}

constexpr double kLaunch = 1.0;            // of a launch, us, beside its kernel's start
constexpr int kMostPair = 256;              // the longest shorter side that pair_kernel holds in registers

long long tiles_of(int mode, int mp, int np, int tile) {
  const long long m = mp / tile, n = np / tile;
  return mode == kGram || mode == kPoly ? m * (m + 1) / 2 : m * n;
}

constexpr int largest_tile(int planes) { return planes == 2 ? 128 : 256; }

// The cheapest tile among those that divide the padded sides, for all groups of a launch together.
template <class Sizes>
int pick_tile(int mode, int planes, int pad, const Sizes& groups, int n, double* cost = nullptr) {
  int best = 32;
  double least = 0.0;
  for (int tile = 32; tile <= std::min(pad, largest_tile(planes)); tile *= 2) {
    long long tiles = 0;
    int k = 0;
    for (int i = 0; i < n; ++i) {
      tiles += tiles_of(mode, groups[i].mp, groups[i].np, tile) * groups[i].count;
      k = std::max(k, mode == kGram ? groups[i].np : groups[i].mp);
    }
    const double c = product_cost(mode, tiles, tile, planes, k);
    if (tile == 32 || c < least) { best = tile; least = c; }
  }
  if (cost) *cost = least;
  return best;
}

struct Plan {
  struct G { int planes, shorter, longer, pad, mp, np, count = 0, first = 0; size_t x[2], a, b, partial, q; float sigma; bool narrow, pair = false; };   // matrices of one shape and type
  std::vector<G> groups;
  std::vector<int> group_of_tensor, first_of_tensor, parts;
  std::vector<size_t> u, partial;
  size_t matrices = 0, total = 0;
  int n_matrices = 0;
};

long long parts_of(long long numel, long long* chunk) {
  long long c = (numel + kMaxParts - 1) / kMaxParts;
  c = (c + kPiece - 1) / kPiece * kPiece;
  *chunk = c;
  return (numel + c - 1) / c;
}

int narrow_tiles(int shorter) {
  const int m16 = (shorter + 15) / 16;
  return m16 * (m16 + 1) / 2;
}

void pad_to(Plan::G& g, int pad) {
  g.pad = pad;
  g.mp = (g.shorter + pad - 1) / pad * pad;
  g.np = (g.longer + pad - 1) / pad * pad;
}

// What share_gram_kernel and pair_kernel take for a step of the groups, in us, from their times over 1 to 24 matrices of 64 x 300 to 256 x 4000.  The strips' part grows
// with the cube of the shorter side: its square in operands and products, and fewer workgroups at a time on a CU for the registers that hold A.  24 matrices
// of 128 x 4000 in bfloat16: strips 14 us, where the second and third product take 18; one of 256 x 784 in float32 8 against 9, 16 of them 24 against 20.
int share_tile(long long tiles_of_16) { return tiles_of_16 <= 512 ? 16 : 32; }   // tiles of 16 as long as a CU has two at most: 4 of 128 x 4000 in float32 7.4 us, of 32 13
double pair_cost(const std::vector<Plan::G>& groups, int planes) {
  long long tiles[2] = {0, 0};
  int steps = 0;
  double strips = 0.0;
  for (const auto& g : groups) {
    for (int h = 0; h < 2; ++h) tiles[h] += tiles_of(kGram, g.mp, g.np, 16 << h) * g.count;
    steps = std::max(steps, g.np / 64);
    strips += (double)(g.np / kStrip) * g.count / 256.0 * (0.3 + (planes == 2 ? 0.010 : 0.004) * std::pow(g.mp / 32.0, 3.0));
  }
  const int tile = share_tile(tiles[0]);
  const double piece = (planes == 2 ? 0.06 : 0.03) * (tile == 16 ? 1.0 : 2.7);
  return 3.0 + piece * steps * std::ceil(tiles[tile == 32] / 256.0) + 3.0 + strips + 2 * kLaunch;
}

// A step of the groups of one type, those of one padding launched together, and those of two launches a step.
double step_cost(const std::vector<Plan::G>& groups, int planes) {
  double sum = 0.0;
  std::vector<Plan::G> some;
  auto select = [&](auto&& which) {
    some.clear();
    for (const auto& g : groups)
      if (g.planes == planes && !g.narrow && which(g)) some.push_back(g);
    return !some.empty();
  };
  if (select([](const Plan::G& g) { return g.pair; })) sum += pair_cost(some, planes);
  for (int pad = 64; pad <= largest_tile(planes); pad *= 2) {
    if (!select([&](const Plan::G& g) { return !g.pair && g.pad == pad; })) continue;
    for (int mode : {kGram, kPoly, kUpdate}) {
      double cost;
      pick_tile(mode, planes, pad, some, (int)some.size(), &cost);
      sum += cost + kLaunch;
    }
  }
  return sum;
}

// Sides padded to multiples of 64, 128 or 256, which is what lets a product use tiles of that size, and steps of two or three launches: each group as is
// cheapest for it alone, or the paddings all alike, or no group in two launches, whichever makes the step cheapest.
void choose_padding(std::vector<Plan::G>& groups, int planes) {
  std::vector<Plan::G> best, own = groups;
  double least = 0.0;
  auto consider = [&](const std::vector<Plan::G>& now) {
    const double cost = step_cost(now, planes);
    if (best.empty() || cost < least) { best = now; least = cost; }
  };
  std::vector<char> pair(groups.size(), 0);
  for (size_t i = 0; i < own.size(); ++i) {
    Plan::G& g = own[i];
    if (g.planes != planes) continue;
    double cheapest = 0.0;
    Plan::G pick = g;
    auto alone = [&](Plan::G q, int pad) {
      pad_to(q, pad);
      q.narrow = false;   // (a narrow one of many steps)
      const double cost = step_cost({q}, planes);
      if (cheapest == 0.0 || cost < cheapest) { pick.pair = q.pair; if (!q.pair) pad_to(pick, pad); cheapest = cost; }
    };
    for (int pad = 64; pad <= largest_tile(planes); pad *= 2) alone(g, pad);
    Plan::G two = g;
    pad_to(two, 64);
    two.pair = two.mp <= kMostPair;
    if (two.pair) alone(two, 64);
    pair[i] = pick.pair;
    pick.pair = false;
    g = pick;
  }
  for (int two = 0; two < 2; ++two) {
    auto with_pairs = [&](std::vector<Plan::G> now) {
      for (size_t i = 0; i < now.size(); ++i)
        if (two && now[i].planes == planes && pair[i]) { now[i].pair = true; pad_to(now[i], 64); }
      consider(now);
    };
    with_pairs(own);
    for (int pad = 64; pad <= largest_tile(planes); pad *= 2) {
      std::vector<Plan::G> alike = groups;
      for (auto& g : alike)
        if (g.planes == planes) pad_to(g, pad);
      with_pairs(alike);
    }
  }
  groups = std::move(best);
}

Plan make_plan(const MuonTensor* t, int n) {
  Plan p;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += (bytes + 255) / 256 * 256; return o; };
  p.group_of_tensor.assign(n, -1); p.first_of_tensor.assign(n, 0); p.parts.assign(n, 0);
  p.u.assign(n, 0); p.partial.assign(n, 0);
  for (int i = 0; i < n; ++i) {
    if (t[i].blocks == 0) continue;
    const long long r = t[i].rows / t[i].blocks, c = t[i].cols;
    Plan::G g;
    g.planes = t[i].dtype == DType::F32 ? 2 : 1;
    g.shorter = (int)std::min(r, c);
    g.longer = (int)std::max(r, c);
    size_t k = 0;
    while (k < p.groups.size() && !(p.groups[k].planes == g.planes && p.groups[k].shorter == g.shorter && p.groups[k].longer == g.longer)) ++k;
    if (k == p.groups.size()) p.groups.push_back(g);
    p.group_of_tensor[i] = (int)k;
    p.first_of_tensor[i] = p.groups[k].count;
    p.groups[k].count += t[i].blocks;
    p.n_matrices += t[i].blocks;
  }
  int first = 0;
  for (auto& g : p.groups) { g.first = first; first += g.count; }
  for (auto& g : p.groups) g.narrow = g.shorter <= narrow_side(g.planes) && g.longer <= kNarrowLong && g.count <= kNarrowCount;
  for (int planes = 1; planes <= 2; ++planes) choose_padding(p.groups, planes);
  p.matrices = take(sizeof(Matrix) * (size_t)p.n_matrices);
  for (int i = 0; i < n; ++i) {
    if (t[i].blocks == 0) continue;
    long long chunk;
    const long long numel = t[i].rows / t[i].blocks * t[i].cols;
    p.parts[i] = (int)parts_of(numel, &chunk);
    p.first_of_tensor[i] += p.groups[p.group_of_tensor[i]].first;
    p.partial[i] = take(sizeof(double) * (size_t)p.parts[i] * t[i].blocks);
    p.u[i] = take(sizeof(float) * (size_t)(t[i].rows * t[i].cols));
  }
  for (auto& g : p.groups) {
    const size_t x = (size_t)g.count * g.planes * g.mp * g.np * 2, a = (size_t)g.count * g.planes * g.mp * g.mp * 2;
    g.x[0] = take(x); g.x[1] = take(x); g.a = take(a); g.b = take(g.pair ? 0 : a);
    if (g.narrow) {   // (many steps take the other way)
      g.partial = take((size_t)g.count * kMaxSlices * narrow_tiles(g.shorter) * 256 * sizeof(double));
      g.q = take((size_t)g.count * ((size_t)g.shorter * g.shorter * sizeof(float) + sizeof(Factor)));
    }
    // a power of two that brings entries of the size a flat matrix of norm 1 has to about 1
    g.sigma = std::exp2((float)std::min(14, (int)std::lround(0.5 * std::log2((double)g.mp * g.np))));
  }
  p.total = off;
  return p;
}

template <int MODE, int PLANES, int BT, int STAGES, int WAVES_M, int WAVES_N>
hipError_t launch_product(const Groups& t, int blocks, hipStream_t s) {
  auto* kernel = product_kernel<MODE, PLANES, BT, STAGES, WAVES_M, WAVES_N>;
  constexpr size_t lds = (size_t)STAGES * 2 * PLANES * BT * 128;
  if (lds > 64 * 1024)
    if (hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * WAVES_M * WAVES_N), lds, s, t);
  return hipGetLastError();
}

constexpr long long kMostBlocks = 1 << 23;   // of a launch: a grid has fewer than 2^32 threads

// Lays the workgroups of a launch out over the groups; the number of them, or -1 if it is too large for one.
template <class F>
int lay_out(Groups& t, F&& per_matrix) {
  long long blocks = 0;
  for (int i = 0; i < t.n; ++i) {
    const long long per = per_matrix(t.g[i]);
    if (blocks + per * t.g[i].count > kMostBlocks) return -1;   // (a caller with so many has been refused before)
    t.g[i].first_block = (int)blocks;
    t.g[i].per_matrix = (int)per;
    blocks += per * t.g[i].count;
  }
  return (int)blocks;
}

template <int MODE, int PLANES>
hipError_t launch_small_product(const Groups& t, int blocks, hipStream_t s) {
  constexpr int SW = 2;
  auto* kernel = small_product_kernel<MODE, PLANES, SW>;
  constexpr size_t lds = (size_t)4 * SW * 2 * PLANES * 32 * 128;
  if (lds > 64 * 1024)
    if (hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), lds, s, t);
  return hipGetLastError();
}

template <int MODE, int PLANES>
hipError_t product(Groups& t, int pad, hipStream_t s) {
  const int tile = pick_tile(MODE, PLANES, pad, t.g, t.n);
  const int blocks = lay_out(t, [&](const Group& g) { return tiles_of(MODE, g.mp, g.np, tile); });
  if (blocks < 0) return hipErrorInvalidValue;
  if (tile == 32) return launch_small_product<MODE, PLANES>(t, blocks, s);
  if constexpr (PLANES == 1) {
    if (tile == 256) return launch_product<MODE, 1, 256, 2, 2, 4>(t, blocks, s);
    if (tile == 128) return blocks <= 256 ? launch_product<MODE, 1, 128, 4, 2, 2>(t, blocks, s) : launch_product<MODE, 1, 128, 2, 2, 2>(t, blocks, s);
    return launch_product<MODE, 1, 64, 6, 2, 2>(t, blocks, s);
  } else {
    if (tile == 128) return launch_product<MODE, 2, 128, 2, 2, 2>(t, blocks, s);
    return launch_product<MODE, 2, 64, 4, 2, 2>(t, blocks, s);
  }
}

template <bool FINAL, int PLANES>
hipError_t launch_pair(Groups& t, hipStream_t s) {
  int most = 0;
  for (int i = 0; i < t.n; ++i) most = std::max(most, t.g[i].mp);
  const int blocks = lay_out(t, [](const Group& g) { return g.np / kStrip; });
  if (blocks < 0) return hipErrorInvalidValue;
  auto go = [&](auto size) {
    constexpr int MOST = decltype(size)::value;
    hipLaunchKernelGGL((pair_kernel<FINAL, PLANES, MOST>), dim3((unsigned)blocks), dim3(2 * MOST), 0, s, t);
    return hipGetLastError();
  };
  if (most <= 64) return go(std::integral_constant<int, 64>{});
  if (most <= 128) return go(std::integral_constant<int, 128>{});
  return go(std::integral_constant<int, 256>{});
}
template <int PLANES>
hipError_t launch_share_gram(Groups& t, hipStream_t s) {
  auto tiles = [&](int tile) { return lay_out(t, [&](const Group& g) { return tiles_of(kGram, g.mp, g.np, tile); }); };
  int blocks = tiles(16);
  if (blocks >= 0 && share_tile(blocks) == 16) {
    hipLaunchKernelGGL((share_gram_kernel<PLANES, 16, PLANES == 2 ? 3 : 4>), dim3((unsigned)blocks), dim3(kShareThreads), 0, s, t);
    return hipGetLastError();
  }
  blocks = tiles(32);
  if (blocks < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((share_gram_kernel<PLANES, 32, PLANES == 2 ? 2 : 3>), dim3((unsigned)blocks), dim3(kShareThreads), 0, s, t);
  return hipGetLastError();
}

hipError_t narrow_steps(NarrowGroups t, int steps, hipStream_t s) {
  size_t chain_lds = 0;
  auto lay_out = [&](auto per_matrix) {
    long long blocks = 0;
    for (int i = 0; i < t.n; ++i) {
      t.g[i].first_block = (int)blocks;
      blocks += (long long)per_matrix(t.g[i]) * t.g[i].count;
      chain_lds = std::max(chain_lds, narrow_lds((t.g[i].shorter + 15) / 16));
    }
    return dim3((unsigned)blocks);   // at most kMaxGroups * kNarrowCount * kNarrowLong / kApply
  };
  dim3 blocks = lay_out([](const NarrowGroup& g) { return g.slices; });
  hipLaunchKernelGGL(narrow_gram_kernel, blocks, dim3(kThreads), 0, s, t);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  blocks = lay_out([](const NarrowGroup&) { return 1; });
  if (chain_lds > 64 * 1024)
    if (hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(narrow_chain_kernel), narrow_lds(kNarrow / 16)); e != hipSuccess) return e;
  hipLaunchKernelGGL(narrow_chain_kernel, blocks, dim3(kChainThreads), chain_lds, s, t, steps);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  blocks = lay_out([](const NarrowGroup& g) { return (g.longer + kApply - 1) / kApply; });
  hipLaunchKernelGGL(narrow_apply_kernel, blocks, dim3(kThreads), 0, s, t);
  return hipGetLastError();
}

template <int PLANES, bool PAIR>
hipError_t orthogonalise(Groups t, int pad, int steps, hipStream_t s) {
  int blocks = lay_out(t, [](const Group& g) { return (long long)(g.mp / 64) * (g.np / 64); });
  if (blocks < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((normalise_kernel<PLANES, PAIR>), dim3((unsigned)blocks), dim3(kThreads), 0, s, t);
  hipError_t e = hipGetLastError();
  for (int k = 0; k < steps && e == hipSuccess; ++k) {
    const bool last = k + 1 == steps;
    if constexpr (PAIR) {
      e = launch_share_gram<PLANES>(t, s);
      if (e == hipSuccess) e = last ? launch_pair<true, PLANES>(t, s) : launch_pair<false, PLANES>(t, s);
    } else {
      e = product<kGram, PLANES>(t, pad, s);
      if (e == hipSuccess) e = product<kPoly, PLANES>(t, pad, s);
      if (e == hipSuccess) e = last ? product<kFinal, PLANES>(t, pad, s) : product<kUpdate, PLANES>(t, pad, s);
    }
    for (int i = 0; i < t.n; ++i) std::swap(t.g[i].x[0], t.g[i].x[1]);
  }
  return e;
}

}  // namespace

size_t muon_workspace_size(const MuonTensor* tensors, int n) { return make_plan(tensors, n).total; }

hipError_t launch_muon_step(const MuonTensor* tensors, int n, const spb_muon_config& c, void* workspace, hipStream_t stream) {
  const Plan p = make_plan(tensors, n);
  char* ws = static_cast<char*>(workspace);
  Matrix* matrices = reinterpret_cast<Matrix*>(ws + p.matrices);
  int i = 0;
  while (i < n) {
    Table tab = {};
    tab.nesterov = c.nesterov; tab.momentum = (float)c.momentum; tab.adam_eps = (float)c.adam_eps; tab.ns_eps = c.ns_eps;
    tab.beta1 = (float)c.beta1; tab.beta2 = (float)c.beta2; tab.new1 = (float)(1.0 - c.beta1); tab.new2 = (float)(1.0 - c.beta2);
    tab.inv_c1 = (float)(1.0 / (1.0 - std::pow(c.beta1, (double)c.step)));
    tab.inv_c2 = (float)(1.0 / (1.0 - std::pow(c.beta2, (double)c.step)));
    long long blocks = 0;
    for (; i < n && tab.n < kMaxTensors; ++i) {
      const MuonTensor& s = tensors[i];
      const bool matrix = s.blocks > 0;
      long long chunk = kPiece;
      const long long numel = s.rows * s.cols / (matrix ? s.blocks : 1);
      const long long parts = matrix ? parts_of(numel, &chunk) : (numel + kPiece - 1) / kPiece;
      if (blocks && blocks + parts * (matrix ? s.blocks : 1) > kMostBlocks) break;
      Tensor& d = tab.t[tab.n++];
      d.w = s.w; d.m = s.m; d.v = s.v; d.count = s.count; d.bf16 = s.dtype == DType::BF16; d.rate = (float)s.rate; d.keep = (float)(1.0 - s.rate * c.weight_decay);
      d.blocks = matrix ? s.blocks : 1;
      d.numel = numel; d.parts = (int)parts; d.chunk = chunk;
      d.rows = (int)(matrix ? s.rows / s.blocks : 0); d.cols = (int)(matrix ? s.cols : 0);
      d.first_block = (int)blocks;
      for (int j = 0; j < s.count; ++j) d.g[j] = s.g[j];
      if (matrix) {
        d.u = reinterpret_cast<float*>(ws + p.u[i]);
        d.partial = reinterpret_cast<double*>(ws + p.partial[i]);
        d.out = matrices + p.first_of_tensor[i];
        d.step = (float)(s.rate * c.rms * std::sqrt((double)std::max(d.rows, d.cols)));
      }
      blocks += parts * d.blocks;
    }
    hipLaunchKernelGGL(update_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, tab);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const bool few_steps = c.ns_steps <= kNarrowSteps;
  for (size_t k = 0; few_steps && k < p.groups.size();) {
    NarrowGroups t = {};
    for (; k < p.groups.size() && t.n < kMaxGroups; ++k) {
      const Plan::G& s = p.groups[k];
      if (!s.narrow) continue;
      NarrowGroup& d = t.g[t.n++];
      d.matrices = matrices + s.first;
      d.partial = reinterpret_cast<double*>(ws + s.partial); d.q = reinterpret_cast<float*>(ws + s.q);
      d.shorter = s.shorter; d.longer = s.longer; d.count = s.count; d.tiles = narrow_tiles(s.shorter);
      d.slices = std::min((s.longer + 127) / 128, kMaxSlices);
    }
    if (t.n == 0) break;
    if (hipError_t e = narrow_steps(t, c.ns_steps, stream); e != hipSuccess) return e;
  }
  // pad 0: the groups of two launches a step
  auto steps_of = [&](int planes, int pad) {
    for (size_t k = 0; k < p.groups.size();) {
      Groups t = {};
      for (; k < p.groups.size() && t.n < kMaxGroups; ++k) {
        const Plan::G& s = p.groups[k];
        if (s.planes != planes || (s.pair ? 0 : s.pad) != pad || (s.narrow && few_steps)) continue;
        Group& d = t.g[t.n++];
        d.x[0] = reinterpret_cast<_Float16*>(ws + s.x[0]); d.x[1] = reinterpret_cast<_Float16*>(ws + s.x[1]);
        d.a = reinterpret_cast<_Float16*>(ws + s.a); d.b = reinterpret_cast<_Float16*>(ws + s.b);
        d.matrices = matrices + s.first;
        d.mp = s.mp; d.np = s.np; d.count = s.count; d.sigma = s.sigma;
      }
      if (t.n == 0) break;
      const hipError_t e = pad == 0 ? planes == 1 ? orthogonalise<1, true>(t, pad, c.ns_steps, stream) : orthogonalise<2, true>(t, pad, c.ns_steps, stream)
                                    : planes == 1 ? orthogonalise<1, false>(t, pad, c.ns_steps, stream) : orthogonalise<2, false>(t, pad, c.ns_steps, stream);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  for (int planes = 1; planes <= 2; ++planes) {
    if (hipError_t e = steps_of(planes, 0); e != hipSuccess) return e;
    for (int pad = 64; pad <= largest_tile(planes); pad *= 2)
      if (hipError_t e = steps_of(planes, pad); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace spb
