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
// (float32) and the partial sums of |u|^2 (float64, so that neither tiny nor huge gradients leave the range) in the workspace.
// The products are bound by the matrix cores.  All matrices of one padded shape go through a product in one launch, whichever
// tensors and blocks they come from, and the two symmetric products form the tiles on and below the diagonal only and
// write each twice: a step of an r x c matrix costs r^2 c + r^3 + 2 r^2 c operations instead of 2 r^2 c + 2 r^3 + 2 r^2 c.
//
// Number formats.  X, A and B are stored as float16 between the products, which accumulate in float32: at the same matrix
// rate as bfloat16 it carries three bits more, and the step is a polynomial of a matrix of norm near 1, whose entries a fixed power of two
// (sigma, tau) keeps in range: |X| <= 1.3 in the spectral norm throughout, so sigma |x| <= 1.3 * 2^14 and tau |b| <= 2^14.
// A float32 parameter would show the 2^-11 of that format: its X, A and B are stored as two float16 (value and remainder, the remainder
// scaled by 2^11), and a product is three: value x remainder, remainder x value, their sum scaled by 2^-11, value x value.
#include <algorithm>
#include <cmath>

#include "gemm_dma_impl.h"

namespace spb {
namespace {

using gemm_detail::f32x16;
using gemm_detail::f32x4;
using gemm_detail::lds_offset;
using gemm_detail::u32x4;
using gemm_detail::xcd_tile;
using gemm_dma_detail::fragments_ready;
using gemm_dma_detail::krow_rot;
using gemm_dma_detail::read_fragment;
using gemm_dma_detail::wait_loads_and_barrier;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

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
  float keep, step, eps;   // w = keep * w - step * X
};

// ---- elementwise half ---------------------------------------------------------------------------------------------

constexpr int kMaxTensors = 16;
constexpr int kPiece = 2048;              // elements a workgroup takes at a time
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
  int first_block, count, bf16, rows, cols, vector;
  float rate, keep, step;   // keep = 1 - rate * weight decay
};
struct Table {
  Tensor t[kMaxTensors];
  int n, nesterov;
  float momentum, beta1, beta2, new1, new2, inv_c1, inv_c2, adam_eps, ns_eps;   // new1 = 1 - beta1
};

__device__ __forceinline__ float bf(uint16_t v) { return __uint_as_float(((uint32_t)v) << 16); }

__device__ __forceinline__ void step_element(const Table& tab, const Tensor& t, float g, float& m, float& v, float& w, float& u) {
  if (t.u) {
    m = tab.momentum * m + g;
    u = tab.nesterov ? g + tab.momentum * m : m;
  } else {
    m = tab.beta1 * m + tab.new1 * g;
    v = tab.beta2 * v + tab.new2 * (g * g);
    w = w * t.keep - t.rate * ((m * tab.inv_c1) / (sqrtf(v * tab.inv_c2) + tab.adam_eps));
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
  const float inv = 1.f / (float)t.count;
  double sq = 0.0;
  for (long long e0 = begin + threadIdx.x * 4; e0 < end; e0 += kThreads * 4) {
    float g[4] = {0.f, 0.f, 0.f, 0.f}, m[4] = {}, v[4] = {}, w[4] = {}, u[4] = {};
    const int live = (int)min(end - e0, 4ll);
    if (t.vector) {
      for (int j = 0; j < t.count; ++j) {
        const f32x4 x = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(t.g[j] + e0));
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] += x[e];
      }
      const f32x4 mm = *reinterpret_cast<const f32x4*>(t.m + e0);
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = mm[e];
      if (!t.u) {
        const f32x4 vv = *reinterpret_cast<const f32x4*>(t.v + e0);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = vv[e];
        if (t.bf16) {
          const uint2 b = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(t.w) + e0);
          w[0] = __uint_as_float(b.x << 16); w[1] = __uint_as_float(b.x & 0xFFFF0000u);
          w[2] = __uint_as_float(b.y << 16); w[3] = __uint_as_float(b.y & 0xFFFF0000u);
        } else {
          const f32x4 ww = *reinterpret_cast<const f32x4*>(static_cast<const float*>(t.w) + e0);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = ww[e];
        }
      }
    } else {
      for (int j = 0; j < t.count; ++j)
        for (int e = 0; e < live; ++e) g[e] += t.g[j][e0 + e];
      for (int e = 0; e < live; ++e) m[e] = t.m[e0 + e];
      if (!t.u)
        for (int e = 0; e < live; ++e) {
          v[e] = t.v[e0 + e];
          w[e] = t.bf16 ? bf(static_cast<const uint16_t*>(t.w)[e0 + e]) : static_cast<const float*>(t.w)[e0 + e];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      step_element(tab, t, g[e] * inv, m[e], v[e], w[e], u[e]);
      if (e < live) sq += (double)u[e] * (double)u[e];
    }
    if (t.vector) {
      *reinterpret_cast<f32x4*>(t.m + e0) = f32x4{m[0], m[1], m[2], m[3]};
      if (t.u) *reinterpret_cast<f32x4*>(t.u + e0) = f32x4{u[0], u[1], u[2], u[3]};
      else {
        *reinterpret_cast<f32x4*>(t.v + e0) = f32x4{v[0], v[1], v[2], v[3]};
        if (t.bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(t.w) + e0) = uint2{bf16_pack2(w[0], w[1]), bf16_pack2(w[2], w[3])};
        else *reinterpret_cast<f32x4*>(static_cast<float*>(t.w) + e0) = f32x4{w[0], w[1], w[2], w[3]};
      }
    } else {
      for (int e = 0; e < live; ++e) {
        t.m[e0 + e] = m[e];
        if (t.u) { t.u[e0 + e] = u[e]; continue; }
        t.v[e0 + e] = v[e];
        if (t.bf16) static_cast<uint16_t*>(t.w)[e0 + e] = bf16_round(w[e]);
        else static_cast<float*>(t.w)[e0 + e] = w[e];
      }
    }
  }
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

__device__ __forceinline__ const Group& group_of(const Groups& t, int block, int& mat, int& tile) {
  int i = 0;
  for (int j = 1; j < t.n; ++j)
    if (block >= t.g[j].first_block) i = j;
  const Group& g = t.g[i];
  const int local = block - g.first_block;
  mat = local / g.per_matrix;
  tile = local - mat * g.per_matrix;
  return g;
}

// value and remainder of v at p and, with two planes, p + plane
template <int PLANES>
__device__ __forceinline__ void split8(const float (&v)[8], _Float16* p, size_t plane) {
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
__device__ __forceinline__ void join8(const _Float16* p, size_t plane, float (&v)[8]) {
  const f16x8 hi = *reinterpret_cast<const f16x8*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)hi[e];
  if constexpr (PLANES == 2) {
    const f16x8 lo = *reinterpret_cast<const f16x8*>(p + plane);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += (float)lo[e] * (1.f / kLoScale);
  }
}

// X = sigma u / (|u| + eps), shorter side first, zeros in the padding.  A workgroup per 64 x 64 entries.
template <int PLANES>
__global__ __launch_bounds__(kThreads) void normalise_kernel(Groups groups) {
  __shared__ float tile_s[64][65];
  __shared__ double sums[kThreads / 64];
  int mat, tile;
  const Group& g = group_of(groups, blockIdx.x, mat, tile);
  const Matrix d = g.matrices[mat];
  double s = (int)threadIdx.x < d.parts ? d.partial[threadIdx.x] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  const int tiles_n = g.np / 64, i0 = tile / tiles_n * 64, j0 = (tile - tile / tiles_n * tiles_n) * 64;
  const bool tall = d.rows > d.cols;
  // rows of u: those of X, or, the matrix being tall, its columns
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  for (int k = threadIdx.x; k < 64 * 64; k += kThreads) {
    const int r = k >> 6, c = k & 63;
    tile_s[r][c] = r0 + r < d.rows && c0 + c < d.cols ? d.u[(size_t)(r0 + r) * d.cols + c0 + c] : 0.f;
  }
  __syncthreads();
  const float scale = (float)((double)g.sigma / (sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)d.eps));
  const size_t plane = (size_t)g.mp * g.np;
  _Float16* x = g.x[0] + mat * PLANES * plane;
  for (int k = threadIdx.x; k < 64 * 8; k += kThreads) {
    const int i = k >> 3, j = (k & 7) * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (tall ? tile_s[j + e][i] : tile_s[i][j + e]) * scale;
    split8<PLANES>(v, x + (size_t)(i0 + i) * g.np + j0 + j, plane);
  }
}

// One operand panel of a tile on its way to LDS: ROWS rows with k contiguous (RowK), or k-rows of ROWS columns (KRow).
template <int ROWS, Layout L>
struct Panel {
  static constexpr int kInstr = ROWS / 32;   // four wavefronts of 64 chunks of 16 bytes
  const char* base;
  size_t step;
  uint32_t voff[kInstr];
  __device__ __forceinline__ void init(const _Float16* p, int ld, int row0, int wave, int lane) {
    step = L == Layout::RowK ? (size_t)kTileK * 2 : (size_t)kTileK * ld * 2;
    base = reinterpret_cast<const char*>(L == Layout::RowK ? p + (size_t)row0 * ld : p + row0);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int slot = (i * 4 + wave) * 64 + lane;
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
  __device__ __forceinline__ void load(const char* at, char* tile, int wave) const {
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const uint32_t dst = (uint32_t)(uintptr_t)(gemm_dma_detail::lds_ptr_t)(tile + (i * 4 + wave) * 1024);
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(voff[i]), "s"(at), "s"(dst) : "m0", "memory");
    }
  }
};

enum Mode { kGram = 0, kPoly = 1, kUpdate = 2, kFinal = 3 };

template <int BT, int STAGES>
constexpr size_t product_lds = std::max((size_t)STAGES * 2 * BT * 128, (size_t)BT * (BT + 4) * 4);

// kGram: A = X X^T.  kPoly: B = b A + c A A.  kUpdate: X' = a X + B X.  kFinal: the same, applied to the parameter.
// Tiles of BT x BT by four wavefronts of BT/2 x BT/2; k in steps of 64 through a ring of STAGES tiles filled by direct-to-LDS loads.  The
// matrices are padded to whole tiles with zeros, so nothing in the loop has an edge.
template <int MODE, int PLANES, int BT, int STAGES>
__global__ __launch_bounds__(kThreads) void product_kernel(Groups groups) {
  constexpr int T = BT / 64;                  // 32 x 32 fragments of a wavefront, each way
  constexpr int kStageBytes = 2 * BT * 128;
  constexpr int kLoads = 2 * (BT / 32);
  constexpr Layout LQ = MODE == kGram || MODE == kPoly ? Layout::RowK : Layout::KRow;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int mat, tile;
  const Group& g = group_of(groups, xcd_tile(blockIdx.x, gridDim.x), mat, tile);
  int ti, tj;
  if constexpr (MODE == kGram || MODE == kPoly) {   // on and below the diagonal
    ti = (int)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    tj = tile - ti * (ti + 1) / 2;
  } else {
    const int tiles_m = g.mp / BT;
    tj = tile / tiles_m;
    ti = tile - tj * tiles_m;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  const size_t plane_x = (size_t)g.mp * g.np, plane_a = (size_t)g.mp * g.mp;
  const _Float16* x = g.x[0] + mat * PLANES * plane_x;
  _Float16* a = g.a + mat * PLANES * plane_a;
  _Float16* b = g.b + mat * PLANES * plane_a;
  const _Float16* p = MODE == kGram ? x : MODE == kPoly ? a : b;
  const _Float16* q = MODE == kPoly ? a : x;
  const int ldp = MODE == kGram ? g.np : g.mp, ldq = MODE == kPoly ? g.mp : g.np;
  const size_t plane_p = (MODE == kGram ? plane_x : plane_a) * 2, plane_q = (MODE == kPoly ? plane_a : plane_x) * 2;   // bytes
  const int k_tiles = (MODE == kGram ? g.np : g.mp) / kTileK;
  const int n_steps = (PLANES == 2 ? 3 : 1) * k_tiles;

  Panel<BT, Layout::RowK> sp;
  Panel<BT, LQ> sq;
  sp.init(p, ldp, ti * BT, wave, lane);
  sq.init(q, ldq, tj * BT, wave, lane);
  // the next tile to be requested: its step and, with two planes, which planes of the operands it multiplies
  int next = 0, next_k = 0, pass = 0;
  auto issue = [&]() {
    char* stage = lds + (next % STAGES) * kStageBytes;
    const char* at_p = sp.base + next_k * sp.step;
    const char* at_q = sq.base + next_k * sq.step;
    if constexpr (PLANES == 2) {
      if (pass == 0) at_q += plane_q;
      if (pass == 1) at_p += plane_p;
    }
    sp.load(at_p, stage, wave);
    sq.load(at_q, stage + BT * 128, wave);
    ++next;
    if (++next_k == k_tiles) { next_k = 0; ++pass; }
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < n_steps) issue();
  f32x16 acc[T][T];
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  for (int t = 0; t < n_steps; ++t) {
    if (t + STAGES - 2 < n_steps) wait_loads_and_barrier<(STAGES - 2) * kLoads>();
    else wait_loads_and_barrier<0>();
    if (t + STAGES - 1 < n_steps) issue();
    if (PLANES == 2 && t == 2 * k_tiles) {   // the products with remainders are complete
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] *= 1.f / kLoScale;
    }
    const char* ps = lds + (t % STAGES) * kStageBytes;
    const char* qs = ps + BT * 128;
    constexpr int kBatch = T == 1 ? 4 : 2;
#pragma unroll
    for (int kb = 0; kb < 4; kb += kBatch) {
      u32x4 pf[kBatch * T], qf[kBatch * T];
#pragma unroll
      for (int h = 0; h < kBatch; ++h) {
#pragma unroll
        for (int i = 0; i < T; ++i) pf[h * T + i] = read_fragment<BT, Layout::RowK>(ps, (wm * T + i) * 32, kb + h, lane);
#pragma unroll
        for (int j = 0; j < T; ++j) qf[h * T + j] = read_fragment<BT, LQ>(qs, (wn * T + j) * 32, kb + h, lane);
      }
      if constexpr (LQ == Layout::KRow) fragments_ready(pf, qf);
#pragma unroll
      for (int h = 0; h < kBatch; ++h)
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
          for (int j = 0; j < T; ++j)   // operands exchanged: a lane then holds runs of four columns of one row
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, qf[h * T + j]), __builtin_bit_cast(f16x8, pf[h * T + i]),
                                                               acc[i][j], 0, 0, 0);
    }
  }
  wait_loads_and_barrier<0>();   // every wave is done with the ring

  // The tile in float32 through LDS, so that what it is combined with and what it becomes move in 16-byte pieces.
  constexpr int LD = BT + 4;
  float* tile_s = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<f32x4*>(tile_s + ((wm * T + i) * 32 + (lane & 31)) * LD + (wn * T + j) * 32 + 2 * r + 4 * (lane >> 5)) =
            f32x4{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
  __syncthreads();
  const float inv_sigma = 1.f / g.sigma;
  constexpr int kUnits = BT * BT / 8;
  if constexpr (MODE == kGram || MODE == kPoly) {
    _Float16* out = MODE == kGram ? a : b;
    auto finish = [&](float (&v)[8], size_t at) {
      if constexpr (MODE == kGram) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= kTau * inv_sigma * inv_sigma;
      } else {
        float s[8];
        join8<PLANES>(a + at, plane_a, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = kB * s[e] + (kC / kTau) * v[e];
      }
      split8<PLANES>(v, out + at, plane_a);
    };
    for (int k = threadIdx.x; k < kUnits; k += kThreads) {
      const int i = k / (BT / 8), j = (k % (BT / 8)) * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile_s[i * LD + j + e];
      finish(v, (size_t)(ti * BT + i) * g.mp + tj * BT + j);
    }
    if (ti != tj)
      for (int k = threadIdx.x; k < kUnits; k += kThreads) {   // its mirror image: 16 columns of the tile by 4 pieces of 8 rows at a time
        const int c = k & 15, quad = (k >> 4) & 3, rest = k >> 6;
        const int i = (rest % (BT / 16)) * 16 + c, j = ((rest / (BT / 16)) * 4 + quad) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile_s[(j + e) * LD + i];
        finish(v, (size_t)(tj * BT + i) * g.mp + ti * BT + j);
      }
  } else {
    _Float16* next_x = g.x[1] + mat * PLANES * plane_x;
    const Matrix d = MODE == kFinal ? g.matrices[mat] : Matrix{};
    const bool tall = d.rows > d.cols;
    for (int k = threadIdx.x; k < kUnits; k += kThreads) {
      const int i = k / (BT / 8), j = (k % (BT / 8)) * 8;
      const size_t at = (size_t)(ti * BT + i) * g.np + tj * BT + j;
      float v[8], s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile_s[i * LD + j + e];
      join8<PLANES>(x + at, plane_x, s);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = kA * s[e] + (1.f / kTau) * v[e];
      if constexpr (MODE == kUpdate) split8<PLANES>(v, next_x + at, plane_x);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e) tile_s[i * LD + j + e] = v[e];   // (each entry by the thread that read it)
      }
    }
    if constexpr (MODE == kFinal) {
      __syncthreads();
      const float step = d.step * inv_sigma;
      for (int k = threadIdx.x; k < BT * BT; k += kThreads) {
        const int hi = k / BT, lo = k % BT;                 // row of the parameter's tile, column
        const int i = tall ? lo : hi, j = tall ? hi : lo;
        const int row = (tall ? tj : ti) * BT + hi, col = (tall ? ti : tj) * BT + lo;
        if (row >= d.rows || col >= d.cols) continue;
        const size_t at = (size_t)row * d.cols + col;
        const float v = tile_s[i * LD + j];
        if (d.bf16) {
          uint16_t* w = static_cast<uint16_t*>(d.w) + at;
          *w = bf16_round(d.keep * bf(*w) - step * v);
        } else {
          float* w = static_cast<float*>(d.w) + at;
          *w = d.keep * *w - step * v;
        }
      }
    }
  }
}

// ---- plan -----------------------------------------------------------------------------------------------------------

struct Plan {
  struct Mat { int tensor, first; };                  // of a matrix tensor: its first entry of the matrix table
  struct G { int planes, tile, mp, np, count = 0, first = 0; size_t x[2], a, b; float sigma; };
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

Plan make_plan(const MuonTensor* t, int n) {
  Plan p;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += (bytes + 255) / 256 * 256; return o; };
  p.group_of_tensor.assign(n, -1); p.first_of_tensor.assign(n, 0); p.parts.assign(n, 0);
  p.u.assign(n, 0); p.partial.assign(n, 0);
  for (int i = 0; i < n; ++i) {
    if (t[i].blocks == 0) continue;
    const long long r = t[i].rows / t[i].blocks, c = t[i].cols;
    const int shorter = (int)std::min(r, c), longer = (int)std::max(r, c);
    const int tile = shorter > 64 ? 128 : 64;
    Plan::G g;
    g.planes = t[i].dtype == DType::F32 ? 2 : 1;
    g.tile = tile;
    g.mp = (shorter + tile - 1) / tile * tile;
    g.np = (longer + tile - 1) / tile * tile;
    size_t k = 0;
    while (k < p.groups.size() && !(p.groups[k].planes == g.planes && p.groups[k].mp == g.mp && p.groups[k].np == g.np)) ++k;
    if (k == p.groups.size()) p.groups.push_back(g);
    p.group_of_tensor[i] = (int)k;
    p.first_of_tensor[i] = p.groups[k].count;
    p.groups[k].count += t[i].blocks;
    p.n_matrices += t[i].blocks;
  }
  int first = 0;
  for (auto& g : p.groups) { g.first = first; first += g.count; }
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
    g.x[0] = take(x); g.x[1] = take(x); g.a = take(a); g.b = take(a);
    // a power of two that brings entries of the size a flat matrix of norm 1 has to about 1
    g.sigma = std::exp2((float)std::min(14, (int)std::lround(0.5 * std::log2((double)g.mp * g.np))));
  }
  p.total = off;
  return p;
}

template <int MODE, int PLANES, int BT, int STAGES>
hipError_t launch_product(Groups t, int blocks, hipStream_t s) {
  auto* kernel = product_kernel<MODE, PLANES, BT, STAGES>;
  constexpr size_t lds = product_lds<BT, STAGES>;
  if (lds > 64 * 1024)
    if (hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), lds, s, t);
  return hipGetLastError();
}

template <int PLANES, int BT, int STAGES>
hipError_t orthogonalise(Groups t, int steps, hipStream_t s) {
  auto blocks_for = [&](auto per_matrix) {
    int blocks = 0;
    for (int i = 0; i < t.n; ++i) {
      t.g[i].first_block = blocks;
      t.g[i].per_matrix = per_matrix(t.g[i]);
      blocks += t.g[i].per_matrix * t.g[i].count;
    }
    return blocks;
  };
  auto lower = [](const Group& g) { const int n = g.mp / BT; return n * (n + 1) / 2; };
  auto all = [](const Group& g) { return (g.mp / BT) * (g.np / BT); };
  int blocks = blocks_for([](const Group& g) { return (g.mp / 64) * (g.np / 64); });
  hipLaunchKernelGGL(normalise_kernel<PLANES>, dim3((unsigned)blocks), dim3(kThreads), 0, s, t);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  for (int k = 0; k < steps; ++k) {
    blocks = blocks_for(lower);
    if (hipError_t e = launch_product<kGram, PLANES, BT, STAGES>(t, blocks, s); e != hipSuccess) return e;
    if (hipError_t e = launch_product<kPoly, PLANES, BT, STAGES>(t, blocks, s); e != hipSuccess) return e;
    blocks = blocks_for(all);
    const hipError_t e = k + 1 < steps ? launch_product<kUpdate, PLANES, BT, STAGES>(t, blocks, s) : launch_product<kFinal, PLANES, BT, STAGES>(t, blocks, s);
    if (e != hipSuccess) return e;
    for (int i = 0; i < t.n; ++i) std::swap(t.g[i].x[0], t.g[i].x[1]);
  }
  return hipSuccess;
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
    tab.nesterov = c.nesterov; tab.momentum = (float)c.momentum; tab.adam_eps = (float)c.adam_eps; tab.ns_eps = (float)c.ns_eps;
    tab.beta1 = (float)c.beta1; tab.beta2 = (float)c.beta2; tab.new1 = (float)(1.0 - c.beta1); tab.new2 = (float)(1.0 - c.beta2);
    tab.inv_c1 = (float)(1.0 / (1.0 - std::pow(c.beta1, (double)c.step)));
    tab.inv_c2 = (float)(1.0 / (1.0 - std::pow(c.beta2, (double)c.step)));
    int blocks = 0;
    for (; i < n && tab.n < kMaxTensors; ++i) {
      const MuonTensor& s = tensors[i];
      Tensor& d = tab.t[tab.n++];
      const bool matrix = s.blocks > 0;
      d.w = s.w; d.m = s.m; d.v = s.v; d.count = s.count; d.bf16 = s.dtype == DType::BF16; d.rate = (float)s.rate; d.keep = (float)(1.0 - s.rate * c.weight_decay);
      d.blocks = matrix ? s.blocks : 1;
      d.numel = s.rows * s.cols / d.blocks;
      d.rows = (int)(matrix ? s.rows / s.blocks : 0); d.cols = (int)(matrix ? s.cols : 0);
      d.first_block = blocks;
      uintptr_t bits = (uintptr_t)s.w | (uintptr_t)s.m | (uintptr_t)s.v;
      for (int j = 0; j < s.count; ++j) { d.g[j] = s.g[j]; bits |= (uintptr_t)s.g[j]; }
      d.vector = (bits & 15) == 0 && d.numel % 4 == 0;
      if (matrix) {
        d.parts = (int)parts_of(d.numel, &d.chunk);
        d.u = reinterpret_cast<float*>(ws + p.u[i]);
        d.partial = reinterpret_cast<double*>(ws + p.partial[i]);
        d.out = matrices + p.first_of_tensor[i];
        d.step = (float)(s.rate * c.rms * std::sqrt((double)std::max(d.rows, d.cols)));
      } else {
        d.chunk = kPiece;
        d.parts = (int)((d.numel + kPiece - 1) / kPiece);
      }
      blocks += d.parts * d.blocks;
    }
    hipLaunchKernelGGL(update_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, tab);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  for (int planes = 1; planes <= 2; ++planes)
    for (int tile = 64; tile <= 128; tile += 64) {
      size_t k = 0;
      while (k < p.groups.size()) {
        Groups t = {};
        for (; k < p.groups.size() && t.n < kMaxGroups; ++k) {
          const Plan::G& s = p.groups[k];
          if (s.planes != planes || s.tile != tile) continue;
          Group& d = t.g[t.n++];
          d.x[0] = reinterpret_cast<_Float16*>(ws + s.x[0]); d.x[1] = reinterpret_cast<_Float16*>(ws + s.x[1]);
          d.a = reinterpret_cast<_Float16*>(ws + s.a); d.b = reinterpret_cast<_Float16*>(ws + s.b);
          d.matrices = matrices + s.first;
          d.mp = s.mp; d.np = s.np; d.count = s.count; d.sigma = s.sigma;
        }
        if (t.n == 0) break;
        const hipError_t e = tile == 128 ? (planes == 1 ? orthogonalise<1, 128, 2>(t, c.ns_steps, stream) : orthogonalise<2, 128, 2>(t, c.ns_steps, stream))
                                         : (planes == 1 ? orthogonalise<1, 64, 3>(t, c.ns_steps, stream) : orthogonalise<2, 64, 3>(t, c.ns_steps, stream));
        if (e != hipSuccess) return e;
      }
    }
  return hipSuccess;
}

}  // namespace spb
