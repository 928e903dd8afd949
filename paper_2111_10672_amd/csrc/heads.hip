// The rows of query and key heads between projection and attention: a layer norm of each head's row, a rotation of
// its pairs by the token's positions, or both in one pass, and the gradient of that.
//
//   norm      xh = (x - mean) / sqrt(var + eps) over the head's elements;  n = gamma xh + beta
//   rotation  pair j turns by t_j = freq_j * pos[axis_j]:  (u, v) -> (u cos t - v sin t, u sin t + v cos t)
//   backward  g = the gradient turned by -t;  dbeta = sum g;  dgamma = sum g xh;  h = g gamma;
//             dx = (h - mean(h) - xh mean(h xh)) / sqrt(var + eps)
//
// Memory-bound: every element is read once and written once, statistics are formed from the row in registers (the
// backward pass forms them again rather than read them).  32792 tokens of 32 heads of 128 in bfloat16, normed and half of each head turned: 107 us, 5.0 TB/s;
// backward, 16384 tokens of 24 + 8 heads of 128 normed and turned: 91 us and 4 us for the sums, 4.2 TB/s.  What threatens to bound it instead is the angles: cosine and
// sine of a far position in enough bits take some hundred instruction slots a pair.  So a workgroup takes all heads of a
// few tokens and works the angles out once per token and pair, into LDS, where every head of the token reads them.
//
// An angle is formed as a fraction of a turn in float64: positions are whole numbers, so position times turns per unit, less
// the nearest whole number, keeps 2^-53 * |position| turns (2^-22 at the far end of int32), and only the fraction in
// [-1/2, 1/2] is rounded to float32.  Everything else is float32, rounded once where the result is stored.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace spb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kMaxTokensPerBlock = 64, kMaxTurnedTokens = 16;
constexpr int kMaxAnglesPerBlock = 2048;    // 16 KB of LDS

struct bf16_t { uint16_t bits; };
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16_t v) { return __uint_as_float(((uint32_t)v.bits) << 16); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(bf16_t* p, float v) { p->bits = bf16_round(v); }

// A chunk of V elements, 4 to 16 bytes, as it lies in memory.
template <typename T, int V>
struct Chunk {
  static constexpr int kWords = V * (int)sizeof(T) / 4;
  typedef uint32_t Raw __attribute__((ext_vector_type(kWords < 2 ? 2 : kWords)));   // (of one word: the first of two)
  static __device__ __forceinline__ Raw load(const T* p) {
    if constexpr (kWords == 1) return Raw{*reinterpret_cast<const uint32_t*>(p), 0u};
    else return *reinterpret_cast<const Raw*>(p);
  }
  static __device__ __forceinline__ void store(T* p, const Raw& w) {
    if constexpr (kWords == 1) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<Raw*>(p) = w;
  }
  static __device__ __forceinline__ void unpack(const Raw& w, float (&f)[V]) {
#pragma unroll
    for (int d = 0; d < kWords; ++d) {
      if constexpr (sizeof(T) == 2) { f[2 * d] = __uint_as_float(w[d] << 16); f[2 * d + 1] = __uint_as_float(w[d] & 0xFFFF0000u); }
      else f[d] = __uint_as_float(w[d]);
    }
  }
  static __device__ __forceinline__ Raw pack(const float (&f)[V]) {
    Raw o = {};
#pragma unroll
    for (int d = 0; d < kWords; ++d) {
      if constexpr (sizeof(T) == 2) o[d] = bf16_pack2(f[2 * d], f[2 * d + 1]);
      else o[d] = __float_as_uint(f[d]);
    }
    return o;
  }
};

struct Args {
  const void* x;          // forward: the input; backward: the forward pass's input (null without norm)
  const void* dy;         // backward only
  void* out;              // forward: y; backward: dx
  void* keep;             // forward, optional: x once more, [token][heads][dim] dense
  const int32_t* pos;
  const void* gamma; const void* beta;
  float* partial;         // backward with norm: [blocks][2][groups * dim]
  long long pos_axis, pos_batch;
  long long xs[3], gs[3], os[3];   // strides in elements (batch, token, head) of x, dy and out
  int tokens, seq, heads_q, heads, dim, pairs, interleaved, norm, inverse, tokens_per_block, tokens_per_block_k;
  float eps;
  uint8_t axis[SPB_MAX_PAIRS];
  double turns[SPB_MAX_PAIRS];     // turns per unit of position
};

struct Token { long long x, g, o, pos; };

// Which token of a block and which of `heads` heads (or pairs) row r is: r < 2^20, so float32 divides it exactly.
__device__ __forceinline__ void place_of(int r, int heads, float inv_heads, int& token, int& head) {
  token = (int)(((float)r + 0.5f) * inv_heads);
  head = r - token * heads;
}

// Cosine and sine of `turn` turns, |turn| <= 1/2: the nearest quarter aside, the series at most an eighth of a turn from zero, up to the ninth and the
// tenth power, whose remainders are below 2^-29.
__device__ __forceinline__ float2 cos_sin(float turn) {
  constexpr double T = 2.0 * M_PI, T2 = T * T;
  const float quarter = rintf(4.f * turn), y = fmaf(quarter, -0.25f, turn), z = y * y;   // (y is exact)
  float s = (float)(T * T2 * T2 * T2 * T2 / 362880.0);
  s = fmaf(s, z, (float)(-T * T2 * T2 * T2 / 5040.0));
  s = fmaf(s, z, (float)(T * T2 * T2 / 120.0));
  s = fmaf(s, z, (float)(-T * T2 / 6.0));
  s = fmaf(s, z, (float)T) * y;
  float c = (float)(-T2 * T2 * T2 * T2 * T2 / 3628800.0);
  c = fmaf(c, z, (float)(T2 * T2 * T2 * T2 / 40320.0));
  c = fmaf(c, z, (float)(-T2 * T2 * T2 / 720.0));
  c = fmaf(c, z, (float)(T2 * T2 / 24.0));
  c = fmaf(c, z, (float)(-T2 / 2.0));
  c = fmaf(c, z, 1.f);
  const int q = (int)quarter;
  const float cn = q & 1 ? s : c, sn = q & 1 ? c : s;
  return make_float2((q + 1) & 2 ? -cn : cn, q & 2 ? -sn : sn);
}

// Offsets of the tokens of a block and the cosines and sines of their pairs, into LDS.
__device__ __forceinline__ void load_tokens(const Args& a, unsigned first, int n, Token* tok, float2* cs) {
  if ((int)threadIdx.x < n) {
    const unsigned t = first + threadIdx.x, b = t / (unsigned)a.seq, s = t - b * a.seq;
    tok[threadIdx.x] = Token{(long long)b * a.xs[0] + (long long)s * a.xs[1], (long long)b * a.gs[0] + (long long)s * a.gs[1],
                             (long long)b * a.os[0] + (long long)s * a.os[1], (long long)b * a.pos_batch + s};
  }
  __syncthreads();
  const float inv_pairs = 1.f / (float)a.pairs;
  for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
    int k, j;
    place_of(i, a.pairs, inv_pairs, k, j);
    double turn = (double)a.pos[a.axis[j] * a.pos_axis + tok[k].pos] * a.turns[j];
    turn -= rint(turn);
    const float2 t = cos_sin((float)turn);
    cs[i] = make_float2(t.x, a.inverse ? -t.y : t.y);
  }
}

// Which two chunks of its row lane l holds.  Pairs as halves: chunk l and the chunk its partners are in, as far as pairs reach, then the
// rest two by two; interleaved pairs lie inside a chunk.
__device__ __forceinline__ void chunks_of(int l, int rotated_half, int interleaved, int& c0, int& c1) {
  if (interleaved) { c0 = 2 * l; c1 = 2 * l + 1; }
  else if (l < rotated_half) { c0 = l; c1 = l + rotated_half; }
  else { c0 = 2 * rotated_half + 2 * (l - rotated_half); c1 = c0 + 1; }
}

// Rotates the two chunks a lane holds; cs: the token's pairs.
template <int V>
__device__ __forceinline__ void turn(float (&u)[V], float (&v)[V], const float2* cs, int c0, int c1, int rotated, int interleaved) {
  if (interleaved) {
    if (c0 < rotated) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 t = cs[(c0 * V + e) >> 1];
        const float p = u[e], q = u[e + 1];
        u[e] = p * t.x - q * t.y; u[e + 1] = p * t.y + q * t.x;
      }
    }
    if (c1 < rotated) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 t = cs[(c1 * V + e) >> 1];
        const float p = v[e], q = v[e + 1];
        v[e] = p * t.x - q * t.y; v[e + 1] = p * t.y + q * t.x;
      }
    }
  } else if (c0 < rotated / 2) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float2 t = cs[c0 * V + e];
      const float p = u[e], q = v[e];
      u[e] = p * t.x - q * t.y; v[e] = p * t.y + q * t.x;
    }
  }
}

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <int V>
__device__ __forceinline__ float sum_of(const float (&u)[V], const float (&v)[V]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) s += u[e] + v[e];
  return s;
}

// mean and 1 / sqrt(var + eps) of a row spread over G lanes; u, v become x - mean (zero where the lane holds nothing).
template <int G, int V>
__device__ __forceinline__ float centre(float (&u)[V], float (&v)[V], bool has0, bool has1, float inv_dim, float eps) {
  const float mean = group_sum<G>(sum_of(u, v)) * inv_dim;
  float sq = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    u[e] = has0 ? u[e] - mean : 0.f;
    v[e] = has1 ? v[e] - mean : 0.f;
    sq += u[e] * u[e] + v[e] * v[e];
  }
  return 1.f / sqrtf(group_sum<G>(sq) * inv_dim + eps);
}

// The two chunks of a row that a lane holds.
template <typename T, int V> struct Pair { typename Chunk<T, V>::Raw c[2]; };
template <typename T, int V>
__device__ __forceinline__ Pair<T, V> load_pair(const T* row, int c0, int c1, bool has0, bool has1) {
  Pair<T, V> p = {};
  if (has0) p.c[0] = Chunk<T, V>::load(row + c0 * V);
  if (has1) p.c[1] = Chunk<T, V>::load(row + c1 * V);
  return p;
}
template <typename T, int V>
__device__ __forceinline__ void store_pair(T* row, const Pair<T, V>& p, int c0, int c1, bool has0, bool has1) {
  if (has0) Chunk<T, V>::store(row + c0 * V, p.c[0]);
  if (has1) Chunk<T, V>::store(row + c1 * V, p.c[1]);
}

// Rows of whole chunks of V elements: G lanes a row, two chunks a lane.  Also the backward pass without norm (a rotation by -t).  With norm, queries and
// keys one after the other, so that a lane holds the weights of its elements; the next row is requested before this one is worked on.
template <typename T, int V, int G>
__global__ __launch_bounds__(kThreads) void heads_forward_kernel(Args a) {
  constexpr int S = kThreads / G;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Token* tok = reinterpret_cast<Token*>(lds);
  float2* cs = reinterpret_cast<float2*>(lds + sizeof(Token) * kMaxTokensPerBlock);
  const int l = threadIdx.x % G, chunks = a.dim / V;
  const int rotated = 2 * a.pairs / V, half = a.pairs ? rotated / 2 : chunks / 2;
  int c0, c1;
  chunks_of(l, half, a.interleaved, c0, c1);
  const bool has0 = c0 < chunks, has1 = c1 < chunks;
  const float inv_dim = 1.f / (float)a.dim;
  for (unsigned first = blockIdx.x * (unsigned)a.tokens_per_block; first < (unsigned)a.tokens; first += gridDim.x * (unsigned)a.tokens_per_block) {
    const int n = min(a.tokens_per_block, a.tokens - (int)first);
    if (first != blockIdx.x * (unsigned)a.tokens_per_block) __syncthreads();   // the last block's angles are done with
    load_tokens(a, first, n, tok, cs);
    __syncthreads();
    for (int g = 0; g < (a.norm ? 2 : 1); ++g) {
      const int heads = !a.norm ? a.heads : g ? a.heads - a.heads_q : a.heads_q, h0 = g ? a.heads_q : 0, rows = n * heads;
      if (rows == 0) break;
      const float inv_heads = 1.f / (float)heads;
      auto request = [&](int r) {
        int k, h;
        place_of(min(r, rows - 1), heads, inv_heads, k, h);
        return load_pair<T, V>(static_cast<const T*>(a.x) + tok[k].x + (h0 + h) * a.xs[2], c0, c1, has0, has1);
      };
      Pair<T, V> next = request(threadIdx.x / G), gam = {}, bet = {};
      if (a.norm) {
        gam = load_pair<T, V>(static_cast<const T*>(a.gamma) + g * a.dim, c0, c1, has0, has1);
        if (a.beta) bet = load_pair<T, V>(static_cast<const T*>(a.beta) + g * a.dim, c0, c1, has0, has1);
      }
      for (int r = threadIdx.x / G; r < rows; r += S) {
        int k, h;
        place_of(r, heads, inv_heads, k, h);
        h += h0;
        const Pair<T, V> now = next;
        next = request(r + S);
        if (a.keep) store_pair<T, V>(static_cast<T*>(a.keep) + ((size_t)(first + k) * a.heads + h) * a.dim, now, c0, c1, has0, has1);
        float u[V], v[V];
        Chunk<T, V>::unpack(now.c[0], u);
        Chunk<T, V>::unpack(now.c[1], v);
        if (a.norm) {
          const float rstd = centre<G>(u, v, has0, has1, inv_dim, a.eps);
          float w[V], z[V];
          Chunk<T, V>::unpack(gam.c[0], w);
          Chunk<T, V>::unpack(bet.c[0], z);
#pragma unroll
          for (int e = 0; e < V; ++e) u[e] = w[e] * (u[e] * rstd) + z[e];
          Chunk<T, V>::unpack(gam.c[1], w);
          Chunk<T, V>::unpack(bet.c[1], z);
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = w[e] * (v[e] * rstd) + z[e];
        }
        if (a.pairs) turn(u, v, cs + k * a.pairs, c0, c1, rotated, a.interleaved);
        Pair<T, V> out;
        out.c[0] = Chunk<T, V>::pack(u);
        out.c[1] = Chunk<T, V>::pack(v);
        store_pair<T, V>(static_cast<T*>(a.out) + tok[k].o + h * a.os[2], out, c0, c1, has0, has1);
      }
    }
  }
}

// Backward pass with norm, queries (blockIdx.y = 0) and keys apart.  Workgroups walk over blocks of tokens and keep the sums for dgamma and dbeta of the
// elements their lanes hold in registers (one kernel for both kinds of head held twice the sums: two wavefronts a SIMD instead of four, 4096 tokens of
// 12 + 12 heads of 64 16.4 us); at the end each adds its lanes up through LDS in a fixed order and writes its part of a partial row.
template <typename T, int V, int G>
__global__ __launch_bounds__(kThreads) void heads_norm_backward_kernel(Args a) {
  constexpr int S = kThreads / G;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Token* tok = reinterpret_cast<Token*>(lds);
  float2* cs = reinterpret_cast<float2*>(lds + sizeof(Token) * kMaxTokensPerBlock);
  const int l = threadIdx.x % G, chunks = a.dim / V;
  const int rotated = 2 * a.pairs / V, half = a.pairs ? rotated / 2 : chunks / 2;
  int c0, c1;
  chunks_of(l, half, a.interleaved, c0, c1);
  const bool has0 = c0 < chunks, has1 = c1 < chunks;
  const float inv_dim = 1.f / (float)a.dim;
  const int g = blockIdx.y, heads = g ? a.heads - a.heads_q : a.heads_q, h0 = g ? a.heads_q : 0, per_block = g ? a.tokens_per_block_k : a.tokens_per_block;
  const float inv_heads = 1.f / (float)heads;
  const Pair<T, V> gam = load_pair<T, V>(static_cast<const T*>(a.gamma) + g * a.dim, c0, c1, has0, has1);
  float dgam[2][V], dbet[2][V];
#pragma unroll
  for (int e = 0; e < V; ++e) dgam[0][e] = dgam[1][e] = dbet[0][e] = dbet[1][e] = 0.f;
  for (unsigned first = blockIdx.x * (unsigned)per_block; first < (unsigned)a.tokens; first += gridDim.x * (unsigned)per_block) {
    const int n = min(per_block, a.tokens - (int)first), rows = n * heads;
    __syncthreads();
    load_tokens(a, first, n, tok, cs);
    __syncthreads();
    struct Both { Pair<T, V> x, dy; };
    auto request = [&](int r) {
      int k, h;
      place_of(min(r, rows - 1), heads, inv_heads, k, h);
      return Both{load_pair<T, V>(static_cast<const T*>(a.x) + tok[k].x + (h0 + h) * a.xs[2], c0, c1, has0, has1),
                  load_pair<T, V>(static_cast<const T*>(a.dy) + tok[k].g + (h0 + h) * a.gs[2], c0, c1, has0, has1)};
    };
    Both next = request(threadIdx.x / G);
    for (int r = threadIdx.x / G; r < rows; r += S) {
      int k, h;
      place_of(r, heads, inv_heads, k, h);
      h += h0;
      const Both now = next;
      next = request(r + S);
      float u[V], v[V], p[V], q[V], w[V];
      Chunk<T, V>::unpack(now.x.c[0], u);
      Chunk<T, V>::unpack(now.x.c[1], v);
      Chunk<T, V>::unpack(now.dy.c[0], p);
      Chunk<T, V>::unpack(now.dy.c[1], q);
      const float rstd = centre<G>(u, v, has0, has1, inv_dim, a.eps);
      if (a.pairs) turn(p, q, cs + k * a.pairs, c0, c1, rotated, a.interleaved);
      float s1 = 0.f, s2 = 0.f;
      Chunk<T, V>::unpack(gam.c[0], w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        u[e] *= rstd;
        dgam[0][e] += p[e] * u[e];
        dbet[0][e] += p[e];
        p[e] *= w[e];
        s1 += p[e];
        s2 += p[e] * u[e];
      }
      Chunk<T, V>::unpack(gam.c[1], w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[e] *= rstd;
        dgam[1][e] += q[e] * v[e];
        dbet[1][e] += q[e];
        q[e] *= w[e];
        s1 += q[e];
        s2 += q[e] * v[e];
      }
      const float m1 = group_sum<G>(s1) * inv_dim, m2 = group_sum<G>(s2) * inv_dim;
#pragma unroll
      for (int e = 0; e < V; ++e) { u[e] = (p[e] - m1 - u[e] * m2) * rstd; v[e] = (q[e] - m1 - v[e] * m2) * rstd; }
      Pair<T, V> out;
      out.c[0] = Chunk<T, V>::pack(u);
      out.c[1] = Chunk<T, V>::pack(v);
      store_pair<T, V>(static_cast<T*>(a.out) + tok[k].o + h * a.os[2], out, c0, c1, has0, has1);
    }
  }
  // [lane groups][2][dim] floats, rows 16 bytes further apart than that, so that the lane groups of a wavefront write to different banks.  A column's lane groups are added up by as many threads as there are columns for, each a stretch of
  // them in order, and the stretches in order.
  float* sums = reinterpret_cast<float*>(lds);
  __shared__ float part[kThreads];
  const int columns = 2 * a.dim, pitch = columns + 4, width = (int)gridDim.y * a.dim, slot = threadIdx.x / G;
  int stretches = 1;
  while (stretches < S && 2 * stretches * columns <= kThreads) stretches *= 2;
  const int per = S / stretches;
  __syncthreads();
  float* mine = sums + slot * pitch;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if (has0) { mine[c0 * V + e] = dgam[0][e]; mine[a.dim + c0 * V + e] = dbet[0][e]; }
    if (has1) { mine[c1 * V + e] = dgam[1][e]; mine[a.dim + c1 * V + e] = dbet[1][e]; }
  }
  __syncthreads();
  auto file = [&](int c, float s) {
    const int which = c >= a.dim;
    a.partial[((size_t)blockIdx.x * 2 + which) * width + g * a.dim + c - which * a.dim] = s;
  };
  if (stretches == 1) {
    for (int c = threadIdx.x; c < columns; c += kThreads) {
      float s = 0.f;
#pragma unroll 8
      for (int i = 0; i < S; ++i) s += sums[i * pitch + c];
      file(c, s);
    }
  } else {
    const int c = threadIdx.x % columns, stretch = threadIdx.x / columns;
    float s = 0.f;
    if (stretch < stretches) {
#pragma unroll 8
      for (int i = 0; i < per; ++i) s += sums[(stretch * per + i) * pitch + c];
    }
    part[threadIdx.x] = s;
    __syncthreads();
    if ((int)threadIdx.x < columns) {
      for (int i = 1; i < stretches; ++i) s += part[i * columns + threadIdx.x];
      file(threadIdx.x, s);
    }
  }
}

// Any head size, stride and alignment: a wavefront takes a row; lane l holds pairs l and l + 64 and elements l, l + 64, ... behind
// the last pair.  The same arithmetic with loads and stores of single elements.
struct Row {
  float u[2], v[2], w[4];
};
struct Places {
  int pu[2], pv[2], pw[4];   // element of the head, or -1
  __device__ __forceinline__ void init(int lane, int dim, int pairs, int interleaved) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = lane + 64 * i;
      pu[i] = j < pairs ? (interleaved ? 2 * j : j) : -1;
      pv[i] = j < pairs ? (interleaved ? 2 * j + 1 : j + pairs) : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 2 * pairs + lane + 64 * i;
      pw[i] = e < dim ? e : -1;
    }
  }
};
template <typename T>
__device__ __forceinline__ void load_row(const T* p, const Places& at, Row& r) {
#pragma unroll
  for (int i = 0; i < 2; ++i) { r.u[i] = at.pu[i] >= 0 ? to_float(p[at.pu[i]]) : 0.f; r.v[i] = at.pv[i] >= 0 ? to_float(p[at.pv[i]]) : 0.f; }
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = at.pw[i] >= 0 ? to_float(p[at.pw[i]]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_row(T* p, const Places& at, const Row& r) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (at.pu[i] >= 0) { store(p + at.pu[i], r.u[i]); store(p + at.pv[i], r.v[i]); }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (at.pw[i] >= 0) store(p + at.pw[i], r.w[i]);
}
// f(element of r, element of s, whether the lane holds it)
template <class F>
__device__ __forceinline__ void each(const Places& at, Row& r, const Row& s, F&& f) {
#pragma unroll
  for (int i = 0; i < 2; ++i) { f(r.u[i], s.u[i], at.pu[i] >= 0); f(r.v[i], s.v[i], at.pv[i] >= 0); }
#pragma unroll
  for (int i = 0; i < 4; ++i) f(r.w[i], s.w[i], at.pw[i] >= 0);
}
__device__ __forceinline__ float centre_row(const Places& at, Row& r, float inv_dim, float eps) {
  float s = 0.f;
  each(at, r, r, [&](float& a, float, bool) { s += a; });
  const float mean = group_sum<64>(s) * inv_dim;
  float sq = 0.f;
  each(at, r, r, [&](float& a, float, bool has) { a = has ? a - mean : 0.f; sq += a * a; });
  return 1.f / sqrtf(group_sum<64>(sq) * inv_dim + eps);
}
__device__ __forceinline__ void turn_row(Row& r, const Places& at, const float2* cs, int lane) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (at.pu[i] < 0) continue;
    const float2 t = cs[lane + 64 * i];
    const float p = r.u[i], q = r.v[i];
    r.u[i] = p * t.x - q * t.y; r.v[i] = p * t.y + q * t.x;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void heads_forward_any_kernel(Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Token* tok = reinterpret_cast<Token*>(lds);
  float2* cs = reinterpret_cast<float2*>(lds + sizeof(Token) * kMaxTokensPerBlock);
  const int lane = threadIdx.x & 63;
  Places at;
  at.init(lane, a.dim, a.pairs, a.interleaved);
  const float inv_dim = 1.f / (float)a.dim;
  for (unsigned first = blockIdx.x * (unsigned)a.tokens_per_block; first < (unsigned)a.tokens; first += gridDim.x * (unsigned)a.tokens_per_block) {
    const int n = min(a.tokens_per_block, a.tokens - (int)first);
    if (first != blockIdx.x * (unsigned)a.tokens_per_block) __syncthreads();
    load_tokens(a, first, n, tok, cs);
    __syncthreads();
    for (int r = threadIdx.x >> 6; r < n * a.heads; r += kThreads / 64) {
      const int k = r / a.heads, h = r - k * a.heads;
      Row x;
      load_row(static_cast<const T*>(a.x) + tok[k].x + h * a.xs[2], at, x);
      if (a.keep) store_row(static_cast<T*>(a.keep) + ((size_t)(first + k) * a.heads + h) * a.dim, at, x);
      if (a.norm) {
        const float rstd = centre_row(at, x, inv_dim, a.eps);
        const int row = (h >= a.heads_q) * a.dim;
        Row w;
        load_row(static_cast<const T*>(a.gamma) + row, at, w);
        each(at, x, w, [&](float& v, float g, bool) { v = g * (v * rstd); });
        if (a.beta) {
          load_row(static_cast<const T*>(a.beta) + row, at, w);
          each(at, x, w, [&](float& v, float b, bool) { v += b; });
        }
      }
      if (a.pairs) turn_row(x, at, cs + k * a.pairs, lane);
      store_row(static_cast<T*>(a.out) + tok[k].o + h * a.os[2], at, x);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void heads_norm_backward_any_kernel(Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Token* tok = reinterpret_cast<Token*>(lds);
  float2* cs = reinterpret_cast<float2*>(lds + sizeof(Token) * kMaxTokensPerBlock);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Places at;
  at.init(lane, a.dim, a.pairs, a.interleaved);
  const float inv_dim = 1.f / (float)a.dim;
  const int g = blockIdx.y, heads = g ? a.heads - a.heads_q : a.heads_q, h0 = g ? a.heads_q : 0, per_block = g ? a.tokens_per_block_k : a.tokens_per_block;
  Row dgam, dbet, gam;
  each(at, dgam, dgam, [](float& v, float, bool) { v = 0.f; });
  each(at, dbet, dbet, [](float& v, float, bool) { v = 0.f; });
  load_row(static_cast<const T*>(a.gamma) + g * a.dim, at, gam);
  for (unsigned first = blockIdx.x * (unsigned)per_block; first < (unsigned)a.tokens; first += gridDim.x * (unsigned)per_block) {
    const int n = min(per_block, a.tokens - (int)first);
    __syncthreads();
    load_tokens(a, first, n, tok, cs);
    __syncthreads();
    for (int r = wave; r < n * heads; r += kThreads / 64) {
      const int k = r / heads, h = h0 + r - k * heads;
      Row x, d;
      load_row(static_cast<const T*>(a.x) + tok[k].x + h * a.xs[2], at, x);
      load_row(static_cast<const T*>(a.dy) + tok[k].g + h * a.gs[2], at, d);
      const float rstd = centre_row(at, x, inv_dim, a.eps);
      if (a.pairs) turn_row(d, at, cs + k * a.pairs, lane);
      each(at, x, x, [&](float& v, float, bool) { v *= rstd; });
      each(at, dbet, d, [](float& s, float v, bool) { s += v; });
      Row dh = d;
      each(at, dh, x, [](float& v, float xh, bool) { v *= xh; });
      each(at, dgam, dh, [](float& s, float v, bool) { s += v; });
      each(at, d, gam, [](float& v, float w, bool) { v *= w; });
      float s1 = 0.f, s2 = 0.f;
      each(at, d, x, [&](float& v, float xh, bool) { s1 += v; s2 += v * xh; });
      const float m1 = group_sum<64>(s1) * inv_dim, m2 = group_sum<64>(s2) * inv_dim;
      each(at, d, x, [&](float& v, float xh, bool) { v = (v - m1 - xh * m2) * rstd; });
      store_row(static_cast<T*>(a.out) + tok[k].o + h * a.os[2], at, d);
    }
  }
  float* sums = reinterpret_cast<float*>(lds);   // [4 wavefronts][2][dim]
  const int width = (int)gridDim.y * a.dim;
  __syncthreads();
  store_row(sums + wave * 2 * a.dim, at, dgam);
  store_row(sums + wave * 2 * a.dim + a.dim, at, dbet);
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * a.dim; c += kThreads) {
    const int which = c >= a.dim;
    a.partial[((size_t)blockIdx.x * 2 + which) * width + g * a.dim + c - which * a.dim] =
        ((sums[c] + sums[2 * a.dim + c]) + sums[4 * a.dim + c]) + sums[6 * a.dim + c];
  }
}

struct Route {
  int lanes = 0, elements = 0;   // lanes a row and elements a chunk of the kernels of whole chunks, 0: the general kernels
  int tokens_per_block = 1, tokens_per_block_k = 1;
  long long blocks = 0;
  int kinds = 1;             // blockIdx.y: queries, keys (backward with norm)
  size_t lds = 0;
};

// Tokens of a workgroup: so many that its rows make four rounds of its lanes (three in the backward pass with norm), which is when waiting for
// the angles and the first rows stops to count, as long as 1024 workgroups (256 with norm backward) are left.  16389 tokens of 32 heads of 128: 53 us with
// 4 tokens, 60 with 8; 8192 of 24 heads of 64: 10.5 with 8, 12.0 with 4 (one round and a half).
// A backward pass with norm takes at most 512 workgroups a kind of head, which walk over the blocks and keep their sums: 16384 tokens of 32 heads of
// 128: 91 us, with 256 122, with 1024 98; and the 512 partial rows take 4 us to add up.
constexpr long long kBackwardBlocks = 512;
constexpr long long kMostBlocks = 1 << 20;   // a grid has fewer than 2^32 threads

Route route_of(const HeadsProblem& q, bool sums) {
  Route r;
  const long long tokens = (long long)q.batch * q.seq;
  // the widest chunks of 16, 8 or 4 bytes that divide the head, the pairs and every stride, from aligned addresses
  const int size = q.dtype == DType::BF16 ? 2 : 4;
  const uintptr_t bits = (uintptr_t)q.x | (uintptr_t)q.dy | (uintptr_t)q.out | (uintptr_t)q.gamma | (uintptr_t)q.beta | (uintptr_t)q.keep;
  for (int v = 16 / size; v >= 2 && !r.lanes; v /= 2) {
    auto whole = [&](const long long (&s)[3]) { return s[0] % v == 0 && s[1] % v == 0 && s[2] % v == 0; };
    const bool strides = whole(q.x_stride) && whole(q.out_stride) && (!q.dy || whole(q.dy_stride));
    const bool pairs = q.interleaved ? 2 * q.pairs % v == 0 : q.pairs % v == 0;
    if (q.head_dim % v || !strides || bits % (v * size) || !pairs) continue;
    r.elements = v;
    r.lanes = v == 16 / size ? 1 : v == 2 ? 8 : 4;   // (few lanes only where all of a head is little: with wide chunks)
    while (r.lanes * 2 * v < q.head_dim) r.lanes *= 2;
  }
  const int at_once = r.lanes ? kThreads / r.lanes : kThreads / 64;   // rows a workgroup works on at a time
  const int most = sums || !q.pairs ? std::min(kMaxTokensPerBlock, kMaxAnglesPerBlock / std::max(q.pairs, 1)) : kMaxTurnedTokens;
  auto tokens_for = [&](int heads) {
    const long long want = ((long long)(sums ? 3 : 4) * at_once + heads - 1) / heads;
    return (int)std::max<long long>(1, std::min<long long>({want, most, tokens / (sums ? 256 : 1024)}));
  };
  r.tokens_per_block = tokens_for(sums ? q.heads_q : q.heads_q + q.heads_k);
  if (sums && q.heads_k) r.tokens_per_block_k = tokens_for(q.heads_k);
  r.blocks = (tokens + r.tokens_per_block - 1) / r.tokens_per_block;
  r.blocks = std::min(r.blocks, kMostBlocks);   // workgroups walk over the rest
  if (sums) {
    r.blocks = std::min(r.blocks, kBackwardBlocks);
    r.kinds = q.heads_k ? 2 : 1;
  }
  r.lds = sizeof(Token) * kMaxTokensPerBlock + sizeof(float2) * (size_t)std::max(r.tokens_per_block, r.tokens_per_block_k) * q.pairs;
  if (sums) r.lds = std::max(r.lds, (size_t)at_once * (2 * q.head_dim + 4) * sizeof(float));
  return r;
}

Args args_of(const HeadsProblem& q, const Route& r, bool inverse) {
  Args a = {};
  a.x = q.x; a.dy = q.dy; a.out = q.out; a.keep = q.keep; a.pos = q.pos; a.gamma = q.gamma; a.beta = q.beta; a.partial = q.partial;
  a.pos_axis = q.pos_axis_stride; a.pos_batch = q.pos_batch_stride;
  for (int i = 0; i < 3; ++i) { a.xs[i] = q.x_stride[i]; a.gs[i] = q.dy_stride[i]; a.os[i] = q.out_stride[i]; }
  a.tokens = q.batch * q.seq;
  a.seq = q.seq; a.heads_q = q.heads_q; a.heads = q.heads_q + q.heads_k; a.dim = q.head_dim;
  a.pairs = q.pairs; a.interleaved = q.pairs ? q.interleaved : 0; a.norm = q.norm; a.inverse = inverse; a.tokens_per_block = r.tokens_per_block; a.tokens_per_block_k = r.tokens_per_block_k;
  a.eps = q.eps;
  for (int j = 0; j < q.pairs; ++j) { a.axis[j] = (uint8_t)q.axis[j]; a.turns[j] = q.freq[j] / (2.0 * M_PI); }
  return a;
}

template <typename F>
hipError_t launch(F* kernel, const Route& r, const Args& a, hipStream_t s) {
  if (r.lds > 64 * 1024)
    if (hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), r.lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)r.blocks, (unsigned)r.kinds), dim3(kThreads), r.lds, s, a);
  return hipGetLastError();
}

template <typename T, int V, int G>
hipError_t launch_lanes(bool backward, const Route& r, const Args& a, hipStream_t s) {
  if (r.lanes == G) return backward ? launch(heads_norm_backward_kernel<T, V, G>, r, a, s) : launch(heads_forward_kernel<T, V, G>, r, a, s);
  if constexpr (2 * G * V < SPB_MAX_HEAD_DIM) return launch_lanes<T, V, 2 * G>(backward, r, a, s);   // a longer head
  else return hipErrorInvalidValue;
}
// backward: with norm
template <typename T>
hipError_t launch_heads(bool backward, const Route& r, const Args& a, hipStream_t s) {
  constexpr int kWide = 16 / (int)sizeof(T);
  if (r.lanes == 0) return backward ? launch(heads_norm_backward_any_kernel<T>, r, a, s) : launch(heads_forward_any_kernel<T>, r, a, s);
  if (r.elements == kWide) return launch_lanes<T, kWide, 1>(backward, r, a, s);
  if (r.elements == 2) return launch_lanes<T, 2, 8>(backward, r, a, s);
  if constexpr (kWide == 8) return launch_lanes<T, 4, 4>(backward, r, a, s);
  return hipErrorInvalidValue;
}

bool valid(const HeadsProblem& q) {
  return q.batch > 0 && q.seq > 0 && q.heads_q > 0 && q.heads_k >= 0 && q.head_dim > 0 && q.head_dim <= SPB_MAX_HEAD_DIM && q.pairs >= 0 &&
         2 * q.pairs <= q.head_dim && (long long)q.batch * q.seq <= 0x7FFFFFFFll && q.out;
}

}  // namespace

hipError_t launch_heads_forward(const HeadsProblem& q, hipStream_t s) {
  if (!valid(q) || !q.x) return hipErrorInvalidValue;
  const Route r = route_of(q, false);
  const Args a = args_of(q, r, false);
  return q.dtype == DType::BF16 ? launch_heads<bf16_t>(false, r, a, s) : launch_heads<float>(false, r, a, s);
}

size_t heads_partial_floats(int batch, int seq, int heads_k, int head_dim) {
  const long long tokens = (long long)batch * seq;
  return (size_t)std::min(std::max<long long>(tokens, 1), kBackwardBlocks) * 2 * (heads_k ? 2 : 1) * head_dim;
}

hipError_t launch_heads_backward(const HeadsProblem& q, hipStream_t s, ReduceTask* deferred) {
  if (!valid(q) || !q.dy) return hipErrorInvalidValue;
  if (!q.norm) {   // a rotation back
    HeadsProblem b = q;
    b.x = q.dy; b.dy = nullptr; b.keep = nullptr; b.gamma = b.beta = nullptr;
    for (int i = 0; i < 3; ++i) b.x_stride[i] = q.dy_stride[i];
    const Route r = route_of(b, false);
    const Args a = args_of(b, r, true);
    return q.dtype == DType::BF16 ? launch_heads<bf16_t>(false, r, a, s) : launch_heads<float>(false, r, a, s);
  }
  if (!q.x || !q.partial || !q.dgamma || !q.dbeta) return hipErrorInvalidValue;
  const Route r = route_of(q, true);
  const Args a = args_of(q, r, true);
  const hipError_t e = q.dtype == DType::BF16 ? launch_heads<bf16_t>(true, r, a, s) : launch_heads<float>(true, r, a, s);
  if (e != hipSuccess) return e;
  ReduceTask task;
  task.kind = ReduceTask::kPairs;
  task.partial = q.partial; task.count = (int)r.blocks; task.width = (q.heads_k ? 2 : 1) * q.head_dim;
  task.out = q.dgamma; task.out_b = q.dbeta;
  task.blocks = reduce_pairs_blocks(task.width);
  if (deferred) { *deferred = task; return hipSuccess; }
  return launch_unit_reduce(&task, 1, s);
}

}  // namespace spb
