// Tenant split and tenant-private action heads (fp32):
//   pool       mean of each sample's valid rows of the shared feature, written
//              in tenant order (the split of the shared features by slices)
//   head_gemm  one launch per head layer and direction for all tenants, fp32
//              matrix-core tiles: forward (bias, GELU or the squared-error loss
//              and its gradient fused), weight gradient (bias gradient fused)
//              and data gradient (GELU derivative fused); tenant row ranges are
//              read from the device maps, so the host needs no per-tenant counts
// Every reduction runs in a fixed order: results are bitwise reproducible.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "jn_device.h"
#include "jn_internal.h"
#include "jn_kv.h"

namespace jnx {

// ------------------------------------------------------------------ pool ---

// Block = (sample, 512-column chunk); 256 threads = 4 wavefronts, lane l
// owning columns 8 l .. 8 l + 7 (one 16-byte load covers 1 KB of a row per
// wave).  Wave w sums rows w, w+4, w+8, ... of the sample in that order, eight
// loads in flight per lane; the four wave sums are combined as
// (s0 + s1) + (s2 + s3).  The order depends only on the sample's own length,
// so a sample pools to the same bits in any batch.  Bound by HBM, one read of
// every valid row, non-temporal: 256 samples of ~296 rows of 4 KB 69 -> 50 us
// (6.2 TB/s).
typedef uint32_t u32x4h __attribute__((ext_vector_type(4)));
constexpr int kPoolCols = 512;
constexpr int kPoolWaves = 4;

__global__ __launch_bounds__(256) void pool_kernel(const uint16_t* __restrict__ hidden,
                                                   const int32_t* __restrict__ seqlens,
                                                   const int32_t* __restrict__ cu_seqlens,
                                                   const int32_t* __restrict__ rank, int32_t d,
                                                   float* __restrict__ pooled) {
  __shared__ float red[kPoolWaves][kPoolCols];
  const int32_t chunks = (d + kPoolCols - 1) / kPoolCols;
  const int32_t i = blockIdx.x / chunks;
  const int32_t c0 = (blockIdx.x % chunks) * kPoolCols;
  const int32_t L = seqlens[i];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int32_t col = c0 + lane * 8;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  if (col < d) {
    const uint16_t* base = hidden + (int64_t)cu_seqlens[i] * d + col;
    auto add = [&](const u32x4h& q) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[2 * e] += __uint_as_float(q[e] << 16);
        acc[2 * e + 1] += __uint_as_float(q[e] & 0xffff0000u);
      }
    };
    auto load = [&](int32_t j) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4h*>(base + (int64_t)j * d)); };
    int32_t j = w;
    for (; j + 7 * kPoolWaves < L; j += 8 * kPoolWaves) {
      u32x4h q[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) q[k] = load(j + k * kPoolWaves);
#pragma unroll
      for (int k = 0; k < 8; ++k) add(q[k]);
    }
    for (; j + 3 * kPoolWaves < L; j += 4 * kPoolWaves) {
      u32x4h q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = load(j + k * kPoolWaves);
#pragma unroll
      for (int k = 0; k < 4; ++k) add(q[k]);
    }
    for (; j < L; j += kPoolWaves) add(load(j));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) red[w][lane * 8 + e] = acc[e];
  __syncthreads();
  const float inv = 1.0f / (float)L;
  for (int t = threadIdx.x; t < kPoolCols; t += 256) {
    if (c0 + t < d)
      pooled[(int64_t)rank[i] * d + c0 + t] = ((red[0][t] + red[1][t]) + (red[2][t] + red[3][t])) * inv;
  }
}

hipError_t launch_pool(hipStream_t s, const void* hidden, const int32_t* seqlens, const int32_t* cu_seqlens,
                       const int32_t* rank, int32_t N, int32_t d, float* pooled) {
  const int64_t blocks = (int64_t)((d + kPoolCols - 1) / kPoolCols) * N;
  if (d % 8 != 0 || N < 1 || blocks > 0x7fffffff) return hipErrorInvalidValue;
  dim3 grid((unsigned)blocks);
  pool_kernel<<<grid, 256, 0, s>>>(reinterpret_cast<const uint16_t*>(hidden), seqlens, cu_seqlens, rank, d, pooled);
  return hipGetLastError();
}

// ------------------------------------------------------------- head gemm ---

// fp32 matrix cores (v_mfma_f32_16x16x4_f32, the heads' precision), operands
// loaded from global memory straight into the MFMA layout: lane l supplies
// A(m = l & 15, k = l >> 4), and which k a step and lane quad stand for, or
// which column a block and lane stand for, is free as long as both operands
// agree, so every operand loads whole vectors along its contiguous dimension.
//   FWD    C[m][n] = X[m][k] W[n][k]: 16-byte loads along k (step s of a
//          16-wide k block is k = 4 quad + s)
//   DGRAD  C[m][n] = dZ[m][k] W[k][n]: 16-byte loads of dZ along k, 8-byte
//          loads of W along n (block b holds columns 2 j + b)
//   WGRAD  C[m][n] = sum_k dZ[k][m] X[k][n]: 4-byte loads along m, 16-byte
//          along n (step = 4 rows, one per quad)
// A workgroup has 8 wavefronts.  FWD and DGRAD: a 32 x 32 tile, the waves each
// take a K range (ceil(K / 8) rounded up to 32) and the eight partial tiles
// are added through LDS in wave order, so a long contraction needs neither
// partial sums in memory nor a second launch.  WGRAD (K is a tenant's row
// count): 64 x 256 tile, 32 x 64 per wave over all rows; long contractions
// (head_long_rows) by eight workgroups, 32 x 64 each, the waves again sharing K: in
// one wave they are a serial chain that a few workgroups walk on an empty chip.
// The order of every sum depends on the layer's sizes and the tenant's rows alone,
// so a tenant's bits do not depend on the batch.
// Bound by the weights' and gradients' HBM traffic (one read, one write) and by
// launches: with LDS staging, K ranges as workgroups and a reduction launch
// after each, the heads of 8 tenants x 32 rows on 2,048-wide features took
// thirteen launches and 276 us after the pool; now six launches and 141 us
// (forward 26 + 15 + 15, backward 24 + 33 + 28 us).  Per launch about 4.7 us go
// to the launch and the first descriptor, 2.5 us to the last tile's store.
typedef float f32x4h __attribute__((ext_vector_type(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows need not be 16-byte aligned
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));

__device__ __forceinline__ f32x4h head_mfma(float a, float b, f32x4h c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

constexpr int kHeadWaves = 8;
constexpr int kHeadDepth = 4;  // slabs in flight per wave
constexpr int kHeadRed = kHeadTile + 4;  // LDS row stride of a partial tile

// A tenant's first row of the loss sums.
__device__ __forceinline__ float* head_lpart(const HeadGemm& D, int32_t off, int32_t tenant) {
  return D.lpart + (int64_t)(off / kHeadTile + tenant) * D.ldp;
}

// Epilogue of the 32 x 32 tile: sum of the waves' partials, then per element
// bias, GELU' (DGRAD), GELU copy, or -- a training forward's last layer -- the
// loss: actions, dL/dy and the tile's sum of squared errors.
__device__ __forceinline__ void head_finish(const HeadGemm& D, const float* red, float* scratch, int32_t off, int32_t ng,
                                            int32_t m0, int32_t n0, int32_t M, float* lpart) {
  const int tid = threadIdx.x;
  const int32_t r = tid >> 4, c = (tid & 15) * 2;
  const int32_t m = m0 + r;
  float ss = 0.f;
  if (m < M) {
    float v[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      v[e] = red[r * kHeadRed + c + e];
#pragma unroll
      for (int w = 1; w < kHeadWaves; ++w) v[e] += red[(w * kHeadTile + r) * kHeadRed + c + e];
    }
    const int64_t row = (int64_t)(off + m) * D.ldc;
    const float scale = 2.0f / ((float)ng * (float)D.N);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int32_t n = n0 + c + e;
      if (n >= D.N) break;
      float y = v[e];
      if (D.bias) y += D.bias[n];
      if (D.Zg) y *= gelu_grad_f(D.Zg[row + n]);
      if (D.target) {
        const int64_t i = (int64_t)m * D.N + n;
        const float diff = y - D.target[i];
        D.actions[i] = y;
        D.C[row + n] = scale * diff;
        ss = fmaf(diff, diff, ss);
      } else {
        D.C[row + n] = y;
        if (D.Cact) D.Cact[row + n] = gelu_f(y);
      }
    }
  }
  if (D.target) {
    ss = wave_sum(ss);
    if ((tid & 63) == 0) scratch[tid >> 6] = ss;
    __syncthreads();
    if (tid == 0) {
      float s = 0.f;
      for (int w = 0; w < kHeadWaves; ++w) s += scratch[w];
      *lpart = s;
    }
  }
}

// Weight gradients over more rows than this are shared by a workgroup's waves.  One
// tenant's short contractions want the wide tiles' less traffic and its long ones
// more workgroups, small gradients sooner: 768 x 256 over 256, 512 and 4,096 rows
// in the whole call 80, 125 and 794 us unshared, 41, 48 and 179 shared; 2048 x 1024 x
// 1024 over 512 and 4,096 264 and 1,796, 174 and 1,068 -- but eight tenants of it over
// 64, 275 and 1,000 rows (16 tenants) 205, 711 and 4,644 unshared, 252, 736 and 4,617
// shared.  The line is the layer's own, so a tenant's bits do not depend on its batch.
__device__ __forceinline__ int32_t head_long_rows(int32_t M, int32_t N) {
  const int32_t tiles = (M + kHeadWgradM - 1) / kHeadWgradM * ((N + kHeadWgradN - 1) / kHeadWgradN);
  return tiles > 32 ? 2 * kHeadLongRows : kHeadLongRows;
}

// The K range of a wave; its whole slabs of S end at `kw` (kb where the tile
// cannot take vector loads), the rest goes four k at a time with element loads.
struct HeadRange {
  int32_t kb, kw, ke;
};
template <int S>
__device__ __forceinline__ HeadRange head_range(int32_t K, int wave, bool vectors) {
  const int32_t kc = ((K + kHeadWaves - 1) / kHeadWaves + 31) / 32 * 32;
  HeadRange r;
  r.kb = min(K, wave * kc);
  r.ke = min(K, r.kb + kc);
  r.kw = vectors ? r.kb + (r.ke - r.kb) / S * S : r.kb;
  return r;
}

__device__ __forceinline__ void head_fwd_tile(const HeadGemm& D, float* red, int32_t off, int32_t m0, int32_t n0, int32_t M) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15, quad = lane >> 4;
  const HeadRange R = head_range<32>(D.K, wave, true);
  const float *A[2], *B[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    A[i] = D.A + (int64_t)(off + min(m0 + 16 * i + j, M - 1)) * D.lda;
    B[i] = D.B + (int64_t)min(n0 + 16 * i + j, D.N - 1) * D.ldb;
  }
  f32x4h acc[2][2] = {};
  f32x4h a[kHeadDepth][2][2], b[kHeadDepth][2][2];  // [slab in flight][16-wide k block][operand block]
  auto load = [&](int u, int32_t k0) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[u][h][i] = *reinterpret_cast<const f32x4u*>(A[i] + k0 + 16 * h + 4 * quad);
        b[u][h][i] = *reinterpret_cast<const f32x4u*>(B[i] + k0 + 16 * h + 4 * quad);
      }
  };
#pragma unroll
  for (int u = 0; u < kHeadDepth; ++u)
    if (R.kb + 32 * u < R.kw) load(u, R.kb + 32 * u);
  for (int32_t k0 = R.kb; k0 < R.kw; k0 += 32 * kHeadDepth) {
#pragma unroll
    for (int u = 0; u < kHeadDepth; ++u) {
      if (k0 + 32 * u >= R.kw) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int x = 0; x < 2; ++x) acc[y][x] = head_mfma(b[u][h][y][s], a[u][h][x][s], acc[y][x]);
      if (k0 + 32 * (u + kHeadDepth) < R.kw) load(u, k0 + 32 * (u + kHeadDepth));
    }
  }
  for (int32_t k0 = R.kw; k0 < R.ke; k0 += 4) {
    const int32_t k = min(k0 + quad, R.ke - 1);
    const bool live = k0 + quad < R.ke;
    float av[2], bv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float x = A[i][k], w = B[i][k];
      av[i] = live ? x : 0.f;
      bv[i] = live ? w : 0.f;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int x = 0; x < 2; ++x) acc[y][x] = head_mfma(bv[y], av[x], acc[y][x]);
  }
  // lane: columns n = 16 y + 4 quad .. +3 of row m = 16 x + j
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int x = 0; x < 2; ++x)
      *reinterpret_cast<f32x4h*>(red + (wave * kHeadTile + 16 * x + j) * kHeadRed + 16 * y + 4 * quad) = acc[y][x];
}

__device__ __forceinline__ void head_dgrad_tile(const HeadGemm& D, float* red, int32_t off, int32_t m0, int32_t n0,
                                                int32_t M) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15, quad = lane >> 4;
  const HeadRange R = head_range<16>(D.K, wave, n0 + kHeadTile <= D.N);
  const float* A[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) A[i] = D.A + (int64_t)(off + min(m0 + 16 * i + j, M - 1)) * D.lda;
  const int64_t ldb = D.ldb;
  const uint32_t bo = 4 * quad * (uint32_t)ldb + n0 + 2 * j;
  f32x4h acc[2][2] = {};
  f32x4h a[kHeadDepth][2];
  f32x2u b[kHeadDepth][4];
  auto load = [&](int u, int32_t k0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) a[u][i] = *reinterpret_cast<const f32x4u*>(A[i] + k0 + 4 * quad);
    const float* p = D.B + (int64_t)k0 * ldb;  // uniform; 32-bit lane offsets
#pragma unroll
    for (int s = 0; s < 4; ++s) b[u][s] = *reinterpret_cast<const f32x2u*>(p + s * ldb + bo);
  };
#pragma unroll
  for (int u = 0; u < kHeadDepth; ++u)
    if (R.kb + 16 * u < R.kw) load(u, R.kb + 16 * u);
  for (int32_t k0 = R.kb; k0 < R.kw; k0 += 16 * kHeadDepth) {
#pragma unroll
    for (int u = 0; u < kHeadDepth; ++u) {
      if (k0 + 16 * u >= R.kw) break;
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int x = 0; x < 2; ++x) acc[y][x] = head_mfma(b[u][s][y], a[u][x][s], acc[y][x]);
      if (k0 + 16 * (u + kHeadDepth) < R.kw) load(u, k0 + 16 * (u + kHeadDepth));
    }
  }
#pragma unroll 4
  for (int32_t k0 = R.kw; k0 < R.ke; k0 += 4) {
    const int32_t k = min(k0 + quad, R.ke - 1);
    const bool live = k0 + quad < R.ke;
    float av[2], bv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float x = A[i][k], w = D.B[(int64_t)k * ldb + min(n0 + 2 * j + i, D.N - 1)];
      av[i] = live ? x : 0.f;
      bv[i] = live ? w : 0.f;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int x = 0; x < 2; ++x) acc[y][x] = head_mfma(bv[y], av[x], acc[y][x]);
  }
  // lane: columns n = 8 quad + 2 e + y of row m = 16 x + j
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    float* p = red + (wave * kHeadTile + 16 * x + j) * kHeadRed + 8 * quad;
    *reinterpret_cast<f32x4h*>(p) = f32x4h{acc[0][x][0], acc[1][x][0], acc[0][x][1], acc[1][x][1]};
    *reinterpret_cast<f32x4h*>(p + 4) = f32x4h{acc[0][x][2], acc[1][x][2], acc[0][x][3], acc[1][x][3]};
  }
}

// piece: which 32 x 64 of the tile; where `shared`, the whole workgroup's, each wave
// a K range, else the wave's own over all rows.
__device__ __forceinline__ void head_wgrad_tile(const HeadGemm& D, float* red, int32_t off, int32_t tm, int32_t tn,
                                                int32_t rows, int piece, bool shared) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15, quad = lane >> 4;
  const int32_t M = D.M, N = D.N;
  const int32_t m0 = tm * kHeadWgradM + 32 * (piece >> 2), n0 = tn * kHeadWgradN + 64 * (piece & 3);
  if (m0 >= M || n0 >= N) return;
  int32_t K = rows, kb = 0;  // the wave's rows, from off + kb
  if (shared) {
    const int32_t kc = ((rows + kHeadWaves - 1) / kHeadWaves + 15) / 16 * 16;
    kb = min(rows, wave * kc);
    K = min(kc, rows - kb);
  }
  const int64_t lda = D.lda, ldb = D.ldb;
  const float *const A = D.A + (int64_t)(off + kb) * lda, *const B = D.B + (int64_t)(off + kb) * ldb;
  const uint32_t a0 = quad * (uint32_t)lda + min(m0 + j, M - 1), a1 = quad * (uint32_t)lda + min(m0 + 16 + j, M - 1);
  const int cj = n0 + 4 * ((j >> 2) + 4 * (j & 3));  // this lane's four columns
  const uint32_t bo = quad * (uint32_t)ldb + cj;
  const bool whole = n0 + 64 <= N;  // uniform: vector loads along n
  f32x4h acc[4][2] = {};            // [column block b][row block a]
  float cs[2] = {0.f, 0.f};         // bias gradient: this quad's rows of columns m0 + j, m0 + 16 + j
  float a[2][4][2];                 // [16 rows in flight][step][row block]
  f32x4h b[2][4];
  auto load = [&](int u, int32_t k0) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float *pa = A + (int64_t)(k0 + 4 * s) * lda, *pb = B + (int64_t)(k0 + 4 * s) * ldb;  // uniform
      a[u][s][0] = pa[a0];
      a[u][s][1] = pa[a1];
      b[u][s] = *reinterpret_cast<const f32x4u*>(pb + bo);
    }
  };
  const int32_t kw = whole ? K / 16 * 16 : 0;
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (16 * u < kw) load(u, 16 * u);
  for (int32_t k0 = 0; k0 < kw; k0 += 32) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (k0 + 16 * u >= kw) break;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
#pragma unroll
        for (int x = 0; x < 2; ++x) cs[x] += a[u][s][x];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int x = 0; x < 2; ++x) acc[y][x] = head_mfma(b[u][s][y], a[u][s][x], acc[y][x]);
      }
      if (k0 + 16 * (u + 2) < kw) load(u, k0 + 16 * (u + 2));
    }
  }
#pragma unroll 2
  for (int32_t k0 = kw; k0 < K; k0 += 4) {
    const int64_t k = min(k0 + quad, K - 1);
    const bool live = k0 + quad < K;
    float av[2] = {A[k * lda + min(m0 + j, M - 1)], A[k * lda + min(m0 + 16 + j, M - 1)]};
    float bv[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) bv[y] = B[k * ldb + min(cj + y, N - 1)];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      av[x] = live ? av[x] : 0.f;
      cs[x] += av[x];
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      bv[y] = live ? bv[y] : 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x) acc[y][x] = head_mfma(bv[y], av[x], acc[y][x]);
    }
  }
  // lane: columns n0 + 16 e + 4 quad + y of rows m0 + 16 x + j (the loads' column
  // order makes a store instruction cover 64 contiguous bytes of 16 rows)
  float bias[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) bias[x] = sum_xor32(sum_xor16(cs[x]));
  if (shared) {
    // the waves' partials, added in wave order: 16 rows at a time, then the bias
    constexpr int kLd = 68;  // LDS row stride
    static_assert(kHeadWaves * 16 * kLd <= kHeadWaves * kHeadTile * kHeadRed, "partials fit");
    const int t = threadIdx.x, c = 2 * (t & 31), r = t >> 5;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4h*>(red + (wave * 16 + j) * kLd + 16 * e + 4 * quad) =
            f32x4h{acc[0][x][e], acc[1][x][e], acc[2][x][e], acc[3][x][e]};
      __syncthreads();
      const int32_t m = m0 + 16 * x + r;
      if (m < M) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float v = red[r * kLd + c + i];
#pragma unroll
          for (int w = 1; w < kHeadWaves; ++w) v += red[(w * 16 + r) * kLd + c + i];
          if (n0 + c + i < N) D.C[(int64_t)m * D.ldc + n0 + c + i] = v;
        }
      }
    }
    if (n0 == 0) {
      __syncthreads();
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (quad == 0) red[wave * 32 + 16 * x + j] = bias[x];
      __syncthreads();
      if (t < 32 && m0 + t < M) {
        float v = red[t];
#pragma unroll
        for (int w = 1; w < kHeadWaves; ++w) v += red[w * 32 + t];
        D.db[m0 + t] = v;
      }
    }
    return;
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int32_t m = m0 + 16 * x + j;
    if (m >= M) break;
    float* p = D.C + (int64_t)m * D.ldc + n0 + 4 * quad;
    if (whole) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4u*>(p + 16 * e) = f32x4h{acc[0][x][e], acc[1][x][e], acc[2][x][e], acc[3][x][e]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (n0 + 16 * e + 4 * quad + y < N) p[16 * e + y] = acc[y][x][e];
    }
    if (n0 == 0 && quad == 0) D.db[m] = bias[x];
  }
}

// FORWARD: FWD tiles only (one workgroup per CU on the 2048-wide heads,
// its slabs in flight are what hides the weights' latency); otherwise the
// backward modes, in at most 128 registers so that two workgroups share a CU.
// Workgroup b < nrow * tms: row tile tm0 + b / nrow of entry b % nrow.  The list
// holds a column of tiles once, not once per row tile of the largest tenant: 32
// tenants of up to 4,096 samples would list 110,000 tiles.
template <bool FORWARD>
__global__ __launch_bounds__(64 * kHeadWaves, FORWARD ? 2 : 4) void head_gemm_kernel(const HeadGemm* __restrict__ descs,
                                                                                     const HeadTile* __restrict__ tiles,
                                                                                     const int32_t* __restrict__ tso,
                                                                                     int32_t nrow, int32_t tms,
                                                                                     int32_t tm0, int32_t nown,
                                                                                     int32_t parts) {
  __shared__ __attribute__((aligned(16))) float red[kHeadWaves * kHeadTile * kHeadRed];
  __shared__ float scratch[kHeadWaves];
  const int32_t b = blockIdx.x;
  const bool own = !FORWARD && b >= nrow * tms;
  const int32_t row = own ? 0 : b / nrow;
  // own tiles: `parts` workgroups of each, tile fastest (workgroups are dealt to the
  // XCDs in turn: where only the first of a tile's eight has work, piece fastest
  // would leave seven XCDs idle)
  const int32_t at = b - nrow * tms, piece = own ? at / nown : 0;
  const HeadTile tile = tiles[own ? nrow + at - piece * nown : b - row * nrow];
  const int32_t off = tso[tile.tenant], ng = tso[tile.tenant + 1] - off;
  const HeadGemm D = descs[tile.desc];
  if (!FORWARD && own) {
    const bool shared = parts > 1 && ng > head_long_rows(D.M, D.N);
    if (piece > 0 && (!shared || tile.tm == kHeadLossTile)) return;
    if (tile.tm != kHeadLossTile) {
      head_wgrad_tile(D, red, off, tile.tm, tile.tn, ng,
                      shared ? piece : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), shared);
      return;
    }
    // the tenant's loss from its tiles' sums, in tile order per thread, then a fixed tree
    const int32_t tn = (D.M + kHeadTile - 1) / kHeadTile, n = (ng + kHeadTile - 1) / kHeadTile * tn;
    const float* const part = head_lpart(D, off, tile.tenant);
    float s = 0.f;
    for (int32_t i = threadIdx.x; i < n; i += 64 * kHeadWaves) s += part[(int64_t)(i / tn) * D.ldp + i % tn];
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      float t = 0.f;
      for (int w = 0; w < kHeadWaves; ++w) t += scratch[w];
      D.loss[0] = t / ((float)ng * (float)D.M);
    }
    return;
  }
  const int32_t tm = tm0 + row, m0 = tm * kHeadTile, n0 = tile.tn * kHeadTile;
  if (m0 >= ng) return;  // tiles past a tenant's row count (upper-bound grid)
  if (FORWARD)
    head_fwd_tile(D, red, off, m0, n0, ng);
  else
    head_dgrad_tile(D, red, off, m0, n0, ng);
  __syncthreads();
  head_finish(D, red, scratch, D.own_rows ? 0 : off, ng, m0, n0, ng,
              head_lpart(D, off, tile.tenant) + (int64_t)tm * D.ldp + tile.tn);
}

hipError_t launch_head_gemm(hipStream_t s, const HeadGemm* descs, const HeadTile* tiles, const HeadLaunch& n,
                            int32_t tms, const int32_t* tso, bool forward) {
  tiles += n.first;
  // a dispatch holds at most 2^32 - 1 threads: row tiles beyond it in further launches
  constexpr int64_t kMost = 0xffffffffll / (64 * kHeadWaves);
  if (n.nrow + (int64_t)n.nown > kMost) return hipErrorInvalidValue;
  const bool longer = tms * (int64_t)kHeadTile > kHeadLongRows && n.nrow + (int64_t)n.nown * kHeadWaves <= kMost;
  const int32_t parts = longer ? kHeadWaves : 1, all = n.nown * parts;
  const int32_t step = n.nrow ? (int32_t)std::min<int64_t>(tms, (kMost - all) / n.nrow) : 0;
  for (int32_t tm0 = 0, own = all;; own = 0) {
    const int32_t rows = std::min(step, tms - tm0);
    const dim3 grid((unsigned)(n.nrow * (int64_t)rows + own));
    if (forward)
      head_gemm_kernel<true><<<grid, 64 * kHeadWaves, 0, s>>>(descs, tiles, tso, n.nrow, rows, tm0, n.nown, parts);
    else
      head_gemm_kernel<false><<<grid, 64 * kHeadWaves, 0, s>>>(descs, tiles, tso, n.nrow, rows, tm0, n.nown, parts);
    const hipError_t e = hipGetLastError();
    tm0 += rows;
    if (e != hipSuccess || n.nrow == 0 || tm0 >= tms) return e;
  }
}

// ------------------------------------------------------------ token heads ---
// The small kernels around a token head's products (k_gemm.hip): targets in, the
// softmax parts of a row's columns joined, results out.

// Last tenant whose targets start at or before i; tenants without any share a
// start with the next one.
__device__ __forceinline__ int32_t tok_tenant(const TokDesc* __restrict__ d, int32_t G, int32_t i) {
  int32_t lo = 0, hi = G - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (d[mid].first <= i) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One wavefront per target: rows without a target become zeros here, whatever the
// feature holds there, so that nothing behind this reads them.  The G workgroups
// behind them count the targets of a tenant each, the last one lays the table
// down.  BYVAL: the descriptors are at the start of the table's bytes, else
// (larger tables, laid down before, another launch) in device memory.
constexpr size_t kTableBytes = 4000;  // a launch's arguments hold 4 KB
struct alignas(16) TokTable {
  uint32_t w[kTableBytes / 4];
};
__global__ __launch_bounds__(256) void tok_table_kernel(uint32_t* __restrict__ dst, TokTable t, int32_t n) {
  for (int32_t i = threadIdx.x; i < n; i += 256) dst[i] = t.w[i];
}

typedef uint32_t u32x4t __attribute__((ext_vector_type(4)));
template <bool BYVAL>
__global__ __launch_bounds__(256) void tok_gather_kernel(uint32_t* __restrict__ dst, TokTable t, int32_t words, int32_t G,
                                                         int32_t N, const u32x4t* __restrict__ hidden, int32_t T,
                                                         int32_t chunks, u32x4t* __restrict__ h,
                                                         int32_t* __restrict__ labels, float* __restrict__ inv) {
  const TokDesc* const desc = reinterpret_cast<const TokDesc*>(BYVAL ? t.w : dst);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int32_t rows = (N + 3) / 4;
  if ((int32_t)blockIdx.x >= rows + (inv ? G : 0)) {
    for (int32_t i = threadIdx.x; i < words; i += 256) dst[i] = t.w[i];
    return;
  }
  if ((int32_t)blockIdx.x >= rows) {
    const TokDesc& d = desc[blockIdx.x - rows];
    __shared__ int32_t part[4];
    int32_t n = 0;
    for (int32_t i = threadIdx.x; i < d.n; i += 256) {
      const int32_t r = d.rows[i], at = d.targets[i];
      n += r >= 0 && r < T && at >= 0 && at < d.vocab;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, kWave);
    if (lane == 0) part[w] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      n = part[0] + part[1] + part[2] + part[3];
      inv[blockIdx.x - rows] = n > 0 ? 1.f / (float)n : 0.f;
    }
    return;
  }
  const int32_t i = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + w);
  if (i >= N) return;
  const TokDesc& d = desc[tok_tenant(desc, G, i)];
  const int32_t r = d.rows[i - d.first], at = d.targets ? d.targets[i - d.first] : 0;
  const bool live = r >= 0 && r < T && at >= 0 && at < d.vocab;
  if (lane == 0) labels[i] = live ? at : -1;
  for (int32_t c = lane; c < chunks; c += 64)
    h[(int64_t)i * chunks + c] = live ? hidden[(int64_t)r * chunks + c] : u32x4t{0, 0, 0, 0};
}

hipError_t launch_tok_table(hipStream_t s, void* dst, const void* table, size_t bytes) {
  TokTable t{};
  for (size_t at = 0; at < bytes; at += kTableBytes) {
    const size_t n = std::min(bytes - at, kTableBytes);
    std::memcpy(t.w, static_cast<const char*>(table) + at, n);
    tok_table_kernel<<<1, 256, 0, s>>>(static_cast<uint32_t*>(dst) + at / 4, t, (int32_t)(n / 4));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_tok_gather(hipStream_t s, void* dst, const void* table, size_t bytes, int32_t G, int32_t N,
                             const void* hidden, int32_t T, int32_t width, uint16_t* h, int32_t* labels, float* inv) {
  TokTable t{};
  uint32_t* const to = static_cast<uint32_t*>(dst);
  const unsigned blocks = (N + 3) / 4 + (inv ? G : 0);
  auto go = [&](auto byval, int32_t words) {
    tok_gather_kernel<byval()><<<blocks + (words > 0), 256, 0, s>>>(
        to, t, words, G, N, static_cast<const u32x4t*>(hidden), T, width / 8, reinterpret_cast<u32x4t*>(h), labels, inv);
    return hipGetLastError();
  };
  if (bytes <= kTableBytes) {
    std::memcpy(t.w, table, bytes);
    return go(std::true_type(), (int32_t)(bytes / 4));
  }
  const hipError_t e = launch_tok_table(s, dst, table, bytes);
  return e != hipSuccess ? e : go(std::false_type(), 0);
}

// Parts {m, rest} of two sets of columns joined (TokPart).
__device__ __forceinline__ void part_join(float& m, float& rest, float m2, float rest2) {
  const float hi = __builtin_elementwise_maximum(m, m2), lo = __builtin_elementwise_minimum(m, m2);
  const float base = hi == -INFINITY ? 0.f : hi;
  const bool first = m >= m2;
  rest = (first ? rest : rest2) + (1.f + (first ? rest2 : rest)) * __builtin_amdgcn_exp2f((lo - base) * 1.4426950408889634f);
  m = hi;
}

// The same where a side may be empty ({-inf, 0}: no value).
__device__ __forceinline__ void part_merge(float& m, float& rest, float m2, float rest2) {
  if (m == -INFINITY && rest == 0.f) {
    m = m2;
    rest = rest2;
  } else if (!(m2 == -INFINITY && rest2 == 0.f)) {
    part_join(m, rest, m2, rest2);
  }
}

// 16 rows per workgroup, read as runs of 16 parts (128 bytes) of a column block,
// 64 blocks at a time; joined in a fixed order.
constexpr int kJoinThreads = 1024, kJoinWaves = kJoinThreads / 64;
template <bool PICK>
__global__ __launch_bounds__(kJoinThreads) void tok_join_kernel(const TokDesc* __restrict__ desc, int32_t G, int32_t N,
                                                                const int32_t* __restrict__ labels,
                                                                const float* __restrict__ zlab,
                                                                TokRow* __restrict__ rows) {
  __shared__ float sm[kJoinWaves][16], sr[kJoinWaves][16];
  __shared__ int32_t sa[PICK ? kJoinWaves : 1][16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int32_t i = blockIdx.x * 16 + (lane & 15);
  const TokDesc d = desc[tok_tenant(desc, G, min(i, N - 1))];
  float m = -INFINITY, rest = 0.f;
  int32_t at = 0x7fffffff;
  auto join = [&](float m2, float rest2, int32_t at2) __attribute__((always_inline)) {
    if constexpr (PICK) at = m2 > m ? at2 : m2 == m ? min(at, at2) : at;
    part_merge(m, rest, m2, rest2);
  };
  if (i < N) {
    const int64_t col = i - d.first;
#pragma unroll 4
    for (int32_t b = w * 4 + (lane >> 4); b < d.blocks; b += 4 * kJoinWaves) {
      const TokPart p = d.part[(int64_t)b * d.n + col];
      join(p.m, p.rest, PICK ? d.index[(int64_t)b * d.n + col] : 0);
    }
  }
#pragma unroll
  for (int o = 16; o <= 32; o <<= 1) {
    const float m2 = __shfl_xor(m, o, kWave), rest2 = __shfl_xor(rest, o, kWave);
    const int32_t at2 = PICK ? __shfl_xor(at, o, kWave) : 0;
    join(m2, rest2, at2);
  }
  if (lane < 16) {
    sm[w][lane] = m;
    sr[w][lane] = rest;
    if constexpr (PICK) sa[w][lane] = at;
  }
  __syncthreads();
  if (threadIdx.x >= 16 || i >= N) return;
  for (int k = 1; k < kJoinWaves; ++k) join(sm[k][lane], sr[k][lane], PICK ? sa[k][lane] : 0);
  const int32_t label = labels[i];
  const float tail = log1pf(rest);
  if constexpr (PICK) {
    // (a row of NaN has no largest value: any token of the vocabulary)
    d.token[i - d.first] = label < 0 ? -1 : min(at, d.vocab - 1);
    d.logp[i - d.first] = label < 0 ? 0.f : -tail + 0.f * m;
  } else {
    const float logp = label < 0 ? 0.f : (zlab[i] - m) - tail;
    d.logp[i - d.first] = logp;
    rows[i] = TokRow{label < 0 ? INFINITY : (m + tail) * 1.4426950408889634f, label, expm1f(logp)};
  }
}

hipError_t launch_tok_join(hipStream_t s, const TokDesc* d, int32_t G, int32_t N, const int32_t* labels,
                           const float* zlab, TokRow* rows) {
  tok_join_kernel<false><<<(N + 15) / 16, kJoinThreads, 0, s>>>(d, G, N, labels, zlab, rows);
  return hipGetLastError();
}

hipError_t launch_tok_pick(hipStream_t s, const TokDesc* d, int32_t G, int32_t N, const int32_t* labels) {
  tok_join_kernel<true><<<(N + 15) / 16, kJoinThreads, 0, s>>>(d, G, N, labels, nullptr, nullptr);
  return hipGetLastError();
}

// The kept logits (kKeepSteps) to their gradient p - 1: p = exp(z - m) exp(m - lse),
// `own` in the target's column, rounded to bf16 here and nowhere else; 8 columns a thread.  The
// next G workgroups sum a tenant's logp each, those behind them clear dW of
// tenants without entries.
__global__ __launch_bounds__(256) void tok_grad_kernel(const TokDesc* __restrict__ desc, int32_t G, int32_t N,
                                                       const float* __restrict__ inv, const TokRow* __restrict__ rows,
                                                       int32_t blocks, int32_t zeros) {
  int32_t b = blockIdx.x;
  if (b < blocks) {
    int32_t lo = 0, hi = G - 1;  // as tok_tenant
    while (lo < hi) {
      const int32_t mid = (lo + hi + 1) >> 1;
      if (desc[mid].grad_block <= b) lo = mid; else hi = mid - 1;
    }
    const TokDesc& d = desc[lo];
    const int32_t per = (d.kept_n8() + 255) / 256, n = (b - d.grad_block) / per, i = d.first + n;
    const int32_t c = (b - d.grad_block - n * per) * 256 + threadIdx.x;
    if (c >= d.kept_n8()) return;
    const TokRow row = rows[i];
    uint4* const at = reinterpret_cast<uint4*>(d.keep) + (int64_t)n * d.kept_n8() + c;
    if (row.label < 0) {  // (whatever W made of the zeros in its place)
      *at = make_uint4(0, 0, 0, 0);
      return;
    }
    const int32_t v0 = 8 * c;
    const float m = d.part[(int64_t)(v0 / d.width) * d.n + n].m;
    // (a block without a column has m = -inf)
    const float f = v0 < d.kept ? fmaf(m, 1.4426950408889634f, -row.lse2) : -INFINITY;
    const uint4 q = *at;
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t u = k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffffu;
      v[k] = __builtin_amdgcn_exp2f(u == kKeepNone ? -INFINITY + f : fmaf((float)u, -1.f / kKeepSteps, f));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = row.label == v0 + k ? row.own : v[k];
    *at = make_uint4(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7]));
    return;
  }
  b -= blocks;
  if (b < G) {
    const TokDesc& d = desc[b];
    __shared__ float part[4];
    float v = 0.f;
    for (int32_t i = threadIdx.x; i < d.n; i += 256) v += d.logp[i];
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) d.loss[0] = -((part[0] + part[1]) + (part[2] + part[3])) * inv[b];
    return;
  }
  for (int32_t g = 0; g < G; ++g)
    if (desc[g].zero_n8 > 0)
      for (int64_t e = (int64_t)(b - G) * 256 + threadIdx.x; e < desc[g].zero_n8; e += (int64_t)zeros * 256)
        reinterpret_cast<uint4*>(desc[g].keep)[e] = make_uint4(0, 0, 0, 0);
}

hipError_t launch_tok_grad(hipStream_t s, const TokDesc* d, int32_t G, int32_t N, const float* inv, const TokRow* rows,
                           int32_t blocks, int64_t zero8) {
  const int32_t zeros = (int32_t)std::min<int64_t>((zero8 + 1023) / 1024, 2048);
  tok_grad_kernel<<<(unsigned)(blocks + G + zeros), 256, 0, s>>>(d, G, N, inv, rows, blocks, zeros);
  return hipGetLastError();
}

// Eight elements of dh per STR lanes, the sum of the planes' PARTS rows of an entry
// (two where its logits' gradient is two bf16); they share the planes (many planes
// are those of few rows) and are added in pairs, against one lane each: 60 rows, 120,000 x
// 128 74 -> 70 us a call, 20 of 100,003 x 128 147 -> 58, 5 of 60,000 x 2,048 176 -> 162;
// 701 rows of 10 planes, 32,003 x 2,048 330 -> 339.
template <int STR, int PARTS>
__global__ __launch_bounds__(256) void tok_rows_kernel(const TokDesc* __restrict__ desc, int32_t G, int32_t N,
                                                       int32_t T, const float* __restrict__ inv, const float4* __restrict__ acc,
                                                       int32_t chunks) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) / STR, plane = (int64_t)N * chunks;
  if (e >= plane) return;
  const int32_t i = (int32_t)(e / chunks), c = (int32_t)(e - (int64_t)i * chunks), t = tok_tenant(desc, G, i);
  const TokDesc& d = desc[t];
  if (!d.dh) return;
  const int32_t r = d.rows[i - d.first], to = d.targets[i - d.first];
  const bool live = r >= 0 && r < T && to >= 0 && to < d.vocab;
  float v[8] = {};
#pragma unroll 4
  for (int32_t k = threadIdx.x % STR; k < d.planes; k += STR) {
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      const float4* const at = acc + 2 * (PARTS * (k * plane + (int64_t)i * chunks) + (int64_t)part * chunks + c);
      const float4 x = at[0], y = at[1];
      const float w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += w[j];
    }
  }
#pragma unroll
  for (int o = 1; o < STR; o <<= 1)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += __shfl_xor(v[j], o, kWave);
  if (threadIdx.x % STR != 0) return;
  const float f = inv[t];
  reinterpret_cast<uint4*>(d.dh)[(int64_t)(i - d.first) * chunks + c] =
      live ? make_uint4(pack_bf2(v[0] * f, v[1] * f), pack_bf2(v[2] * f, v[3] * f), pack_bf2(v[4] * f, v[5] * f),
                        pack_bf2(v[6] * f, v[7] * f))
           : make_uint4(0, 0, 0, 0);
}

hipError_t launch_tok_rows(hipStream_t s, const TokDesc* d, int32_t G, int32_t N, int32_t T, const float* inv,
                           const float* acc, int32_t planes, int32_t width, bool pairs) {
  const int64_t all = (int64_t)N * (width / 8);
  auto go = [&](auto str, auto parts) {
    tok_rows_kernel<str(), parts()><<<(unsigned)((all * str() + 255) / 256), 256, 0, s>>>(
        d, G, N, T, inv, reinterpret_cast<const float4*>(acc), width / 8);
    return hipGetLastError();
  };
  auto rows = [&](auto str) {
    return pairs ? go(str, std::integral_constant<int, 2>()) : go(str, std::integral_constant<int, 1>());
  };
  return planes > 16 && all < (1 << 20) ? rows(std::integral_constant<int, 16>()) : rows(std::integral_constant<int, 1>());
}

// ---- tenants of few rows ----
// With up to 64 rows a call is bound by memory, W in and dW out once each, and the
// smallest ones by their launches.

typedef __bf16 bf16x8h __attribute__((ext_vector_type(8)));
typedef float f32x4h __attribute__((ext_vector_type(4)));
constexpr int kSmallThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;

template <bool ONCE, typename V>
__device__ __forceinline__ void put_once(V v, V* p) {
  if constexpr (ONCE)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}

// LDS written before is read behind it; loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int C>
__device__ __forceinline__ int32_t small_tenant(const TokSmallArgs<C>& s, int32_t wg, bool grads) {
  int32_t g = 0;
  while (g + 1 < s.G && (grads ? s.t[g + 1].gwg0 : s.t[g + 1].wg0) <= wg) ++g;
  return g;
}

// The feature's row of entry i, or -1 where it has no target.
__device__ __forceinline__ int32_t small_row(const TokSmall& d, int32_t i, int32_t T) {
  if (i >= d.n) return -1;
  const int32_t r = d.rows[i], at = d.targets ? d.targets[i] : 0;
  return r >= 0 && r < T && at >= 0 && at < d.vocab ? r : -1;
}

// z = W h for up to 16 NB rows.  8 wavefronts: WK share the contraction (at most 8
// CH steps of 32 each, whose row fragments stay in registers for the whole
// launch) and 8 / WK take 16 vocabulary rows each; W goes straight from memory to
// the matrix cores' operands, 8 loads of 1 KB a wavefront ahead of the 8 in use
// (128 KB of a CU in flight), and is read by nobody twice.  The shares are added
// in LDS, in pairs, which also rounds less than one long chain of additions.
// Every thread then owns one row and some of the vocabulary's, and keeps a running
// maximum and the sum of the others' exponentials, as TokPart.
template <int WK, int CH, int NB, int C>
__global__ __launch_bounds__(kSmallThreads, 2) void small_scores_kernel(TokSmallArgs<C> set, int32_t ldz,
                                                                        const uint16_t* __restrict__ hidden, int32_t T,
                                                                        int32_t width) {
  constexpr int WV = 8 / WK, TOK = 16 * NB, LD = TOK + 4, ROWS = 16 * WV, PER = kSmallThreads / TOK;
  __shared__ __attribute__((aligned(16))) float red[2][8][16 * LD];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wk = w % WK, wv = w / WK, quad = lane >> 4, row = lane & 15;
  const TokSmall& d = set.t[small_tenant(set, blockIdx.x, false)];
  const int32_t V = d.vocab, n = d.n, wg = blockIdx.x - d.wg0;
  const int32_t blocks = (V + ROWS - 1) / ROWS;
  const int32_t b0 = (int32_t)((int64_t)blocks * wg / d.wgs), b1 = (int32_t)((int64_t)blocks * (wg + 1) / d.wgs);
  const int32_t S = width / 32, s0 = S * wk / WK, ns = S * (wk + 1) / WK - s0;
  bf16x8h w0[8], w1[8];
  auto fetch = [&](bf16x8h(&to)[8], int32_t b, int c) __attribute__((always_inline)) {
    const int32_t v = min((b * WV + wv) * 16 + row, V - 1);
    const uint16_t* const p = d.W + (int64_t)v * width + (s0 + 8 * c) * 32 + 8 * quad;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (8 * c + s < ns)
        to[s] = *reinterpret_cast<const bf16x8h*>(p + 32 * s);
      else if constexpr (CH > 2)  // (else zeros from the start: a register takes one chunk; with 0 * inf a product too many shows)
        to[s] = bf16x8h{};
    }
  };
#pragma unroll
  for (int s = 0; s < 8; ++s) w0[s] = w1[s] = bf16x8h{};
  if (b0 < b1) fetch(w0, b0, 0);
  bf16x8h x[8 * CH][NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    // (loads without a condition: rows without a target read W instead)
    const int32_t r = small_row(d, 16 * j + row, T);
    const uint16_t* const p = (r >= 0 ? hidden + (int64_t)r * width : d.W) + s0 * 32 + 8 * quad;
#pragma unroll
    for (int s = 0; s < 8 * CH; ++s) {
      x[s][j] = bf16x8h{};
      if (s < ns) {
        const uint4 v = *reinterpret_cast<const uint4*>(p + 32 * s);
        x[s][j] = __builtin_bit_cast(bf16x8h, r >= 0 ? v : make_uint4(0, 0, 0, 0));
      }
    }
  }
  const int32_t tok = threadIdx.x % TOK;
  const int32_t label = d.targets && tok < n ? d.targets[tok] : -1;
  float m = -INFINITY, rest = 0.f;
  // the thread's first token, so that logits that are all -inf pick their lowest
  const int32_t first = threadIdx.x / TOK;
  int32_t at = first < ROWS && b0 < b1 && b0 * ROWS + first < V ? b0 * ROWS + first : 0x7fffffff;
  f32x4h acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = f32x4h{0.f, 0.f, 0.f, 0.f};
  int buf = 0;
  // chunk c of block b, from `use`; the next one into `next`
  auto chunk = [&](auto c_, bf16x8h(&use)[8], bf16x8h(&next)[8], int32_t b) __attribute__((always_inline)) {
    constexpr int c = decltype(c_)::value;
    if (c + 1 < CH)
      fetch(next, b, c + 1);
    else if (b + 1 < b1)
      fetch(next, b + 1, 0);
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(use[s], x[8 * c + s][j], acc[j], 0, 0, 0);
    if (c + 1 < CH) return;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) red[buf][w][(4 * quad + e) * LD + 16 * j + row] = acc[j][e];
      acc[j] = f32x4h{0.f, 0.f, 0.f, 0.f};
    }
    lds_barrier();
#pragma unroll
    for (int u = 0; u < (ROWS + PER - 1) / PER; ++u) {
      const int32_t r = threadIdx.x / TOK + u * PER;
      if (ROWS % PER != 0 && r >= ROWS) break;
      float p[WK];
#pragma unroll
      for (int k = 0; k < WK; ++k) p[k] = red[buf][(r >> 4) * WK + k][(r & 15) * LD + tok];
#pragma unroll
      for (int h = 1; h < WK; h <<= 1)
#pragma unroll
        for (int k = 0; k < WK; k += 2 * h) p[k] += p[k + h];
      const float z = p[0];
      const int32_t v = b * ROWS + r;
      if (v >= V) continue;
      if (d.z) d.z[(int64_t)v * ldz + tok] = z;
      if (v == label) d.zlab[tok] = z;
      const float e = __builtin_amdgcn_exp2f(-fabsf(z - m) * kLog2e);
      if (z > m) {
        rest = (rest + 1.f) * e;  // (from -inf: e = 0)
        m = z;
        at = v;
      } else {
        rest += z == -INFINITY ? 0.f : e;  // (as the first of a thread's values: e = NaN)
      }
    }
    buf ^= 1;
  };
  if constexpr (CH == 1) {
    for (int32_t b = b0; b < b1; b += 2) {
      chunk(std::integral_constant<int, 0>(), w0, w1, b);
      if (b + 1 < b1) chunk(std::integral_constant<int, 0>(), w1, w0, b + 1);
    }
  } else {
    for (int32_t b = b0; b < b1; ++b) {
      chunk(std::integral_constant<int, 0>(), w0, w1, b);
      chunk(std::integral_constant<int, 1>(), w1, w0, b);
      if constexpr (CH == 4) {
        chunk(std::integral_constant<int, 2>(), w0, w1, b);
        chunk(std::integral_constant<int, 3>(), w1, w0, b);
      }
    }
  }
  // the lanes of a row, then its wavefronts
  auto join = [&](float m2, float rest2, int32_t at2) __attribute__((always_inline)) {
    at = m2 > m ? at2 : m2 == m ? min(at, at2) : at;
    part_merge(m, rest, m2, rest2);
  };
#pragma unroll
  for (int o = TOK; o < 64; o <<= 1) {
    const float m2 = __shfl_xor(m, o, kWave), rest2 = __shfl_xor(rest, o, kWave);
    join(m2, rest2, __shfl_xor(at, o, kWave));
  }
  lds_barrier();  // the last step's shares are read
  float* const sm = red[0][0];
  float* const sr = sm + 8 * TOK;
  int32_t* const sa = reinterpret_cast<int32_t*>(sr + 8 * TOK);
  static_assert(3 * 8 * TOK <= 2 * 8 * 16 * LD, "joins in the same memory");
  if (lane < TOK) {
    sm[w * TOK + lane] = m;
    sr[w * TOK + lane] = rest;
    sa[w * TOK + lane] = at;
  }
  lds_barrier();
  if (threadIdx.x >= TOK || tok >= n) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) join(sm[k * TOK + tok], sr[k * TOK + tok], sa[k * TOK + tok]);
  d.part[(int64_t)wg * n + tok] = TokPart{m, rest};
  if (d.index) d.index[(int64_t)wg * n + tok] = at;
}

// Parts of TOK rows from row `first` on joined by a workgroup: thread t < TOK ends
// with row first + t's.
template <int TOK>
struct SmallJoin {
  float m[8][TOK], rest[8][TOK];
  int32_t at[8][TOK];
};
template <int TOK>
__device__ __forceinline__ void small_join(const TokSmall& d, int32_t first, float& m, float& rest, int32_t& at,
                                           SmallJoin<TOK>& l) {
  constexpr int PER = kSmallThreads / TOK;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, t = threadIdx.x % TOK;
  const int32_t tok = first + t;
  m = -INFINITY;
  rest = 0.f;
  at = 0x7fffffff;
  auto join = [&](float m2, float rest2, int32_t at2) __attribute__((always_inline)) {
    at = m2 > m ? at2 : m2 == m ? min(at, at2) : at;
    part_merge(m, rest, m2, rest2);
  };
  if (tok < d.n) {
#pragma unroll 8
    for (int32_t p = threadIdx.x / TOK; p < d.wgs; p += PER) {
      const TokPart q = d.part[(int64_t)p * d.n + tok];
      join(q.m, q.rest, d.index ? d.index[(int64_t)p * d.n + tok] : 0);
    }
  }
#pragma unroll
  for (int o = TOK; o < 64; o <<= 1) {
    const float m2 = __shfl_xor(m, o, kWave), rest2 = __shfl_xor(rest, o, kWave);
    join(m2, rest2, __shfl_xor(at, o, kWave));
  }
  if (lane < TOK) {
    l.m[w][t] = m;
    l.rest[w][t] = rest;
    l.at[w][t] = at;
  }
  lds_barrier();
  if (threadIdx.x < TOK) {
#pragma unroll
    for (int k = 1; k < 8; ++k) join(l.m[k][t], l.rest[k][t], l.at[k][t]);
  }
}

// 16 rows per workgroup.
template <int C>
__global__ __launch_bounds__(kSmallThreads) void small_pick_kernel(TokSmallArgs<C> set, int32_t T) {
  __shared__ SmallJoin<16> l;
  const TokSmall& d = set.t[blockIdx.x];
  const int32_t first = 16 * blockIdx.y;
  if (first >= d.n) return;
  float m, rest;
  int32_t at;
  const int32_t i = first + threadIdx.x;
  const bool live = threadIdx.x < 16 && small_row(d, i, T) >= 0;
  small_join<16>(d, first, m, rest, at, l);
  if (threadIdx.x >= 16 || i >= d.n) return;
  // (a row of NaN has no largest value: any token of the vocabulary)
  d.token[i] = live ? min(at, d.vocab - 1) : -1;
  d.logp[i] = live ? -log1pf(rest) + 0.f * m : 0.f;
}

// dW = dz^T H / count for up to 32 NS rows: the contraction is the rows, so one or
// two matrix instructions make 16 vocabulary rows x 16 columns, and the kernel is
// bound by writing dW.  A lane's fragments of H^T stay in registers: it reads 8
// columns (16 bytes) of 8 rows and turns them, so that row i = 4 q + e of
// instruction j is column 32 e + 8 q + j of a group of 128: the 8 results of a lane
// for one e are 8 adjacent columns, turned around in LDS so that a store instruction
// writes 256 adjacent bytes of 4 rows.  60 rows, 120,000 x 2,048 (491 MB): 187 us with 16
// bytes in each of four places a row and instruction, 152 with 64 adjacent ones, 120
// so, non-temporally (93 with plain stores, whose lines the next call then waits
// for: 260 us a call instead of 243).  dz of 128
// vocabulary rows at a time is formed from z and the rows' joined sums by the
// workgroup's threads together, 8 rows of the feature each, and shared through LDS as
// two bf16, the nearest one and what is left: a row of dW is made of few terms here, of
// one where a tenant has one target, and one bf16's rounding would stay in an fp32 dW
// (up to 2^-8 of it; two hold 2^-16).  A second matrix instruction takes the rest: 60
// rows, 120,000 x 2,048 236 -> 238 us a call, 5 rows, 60,000 x 2,048 with row gradients
// 158 -> 160, 60 of 120,000 x 2,048 346 -> 360.  The next rows of z are on their way
// meanwhile.
// rows: those of a chunk, 128 or, of small vocabularies, fewer (a multiple of 16), so
// that there are workgroups for the chip.  blockIdx.y: 2,048 columns each.
constexpr int kGradRows = kSmallGradRows;
template <int GP, int NS, int C, bool F32, bool ONCE>
__global__ __launch_bounds__(kSmallThreads, 2) void small_grads_kernel(TokSmallArgs<C> set, int32_t ldz,
                                                                       const uint16_t* __restrict__ hidden, int32_t T,
                                                                       int32_t width, int32_t rows) {
  constexpr int TG = 4 * NS, U = kGradRows * TG / kSmallThreads, LD = 32 * NS + 8;  // groups of 8 rows; passes; elements of a line
  __shared__ SmallJoin<32 * NS> l;
  __shared__ __attribute__((aligned(16))) uint16_t dz[2][2][kGradRows * LD];  // of two chunks: nearest, rest
  __shared__ u32x4t stage[8][256];
  __shared__ __attribute__((aligned(16))) float lse[64], own[64];
  __shared__ __attribute__((aligned(16))) int32_t lab[64];
  __shared__ float scale;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quad = lane >> 4, col = lane & 15;
  const TokSmall& d = set.t[small_tenant(set, blockIdx.x, true)];
  const int32_t V = d.vocab, wg = blockIdx.x - d.gwg0, n = d.n;
  // column groups of this slice, and how many wavefronts share them
  const int32_t g0 = 16 * blockIdx.y, groups = min((width + 127) / 128 - g0, 16);
  const int32_t WC = groups > 4 ? 8 : groups > 2 ? 4 : groups, WV = 8 / WC, wc = w % WC, wv = w / WC;
  u32x4t* const mine16 = stage[w];
  const int32_t mine = small_row(d, lane, T);  // of row `lane`
  uint4 q[GP][NS][8];
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int32_t r = __shfl(mine, 32 * s + 8 * quad + t, kWave);
#pragma unroll
      for (int p = 0; p < GP; ++p) {
        // (a load without a condition: rows without a target, and columns past the end, read W instead)
        const int32_t k = 128 * (g0 + wc + 8 * p) + 32 * (col & 3) + 8 * (col >> 2);
        const bool in = r >= 0 && k < width;
        const uint4 v = *reinterpret_cast<const uint4*>(in ? hidden + (int64_t)r * width + k : d.W);
        q[p][s][t] = in ? v : make_uint4(0, 0, 0, 0);
      }
    }
  {
    float m, rest;
    int32_t at;
    const bool live = mine >= 0;
    const float zl = w == 0 && live ? d.zlab[lane] : 0.f;
    const int32_t label = w == 0 && live ? d.targets[lane] : -1;
    small_join<32 * NS>(d, 0, m, rest, at, l);
    if (w == 0) {
      // (of 32 rows the upper lanes have none)
      const float tail = log1pf(rest), logp = live ? (zl - m) - tail : 0.f;
      lse[lane] = live ? (m + tail) * kLog2e : INFINITY;  // (no target: z = 0, and p = 0)
      own[lane] = expm1f(logp);
      lab[lane] = label;
      const int32_t count = __popcll(__builtin_amdgcn_ballot_w64(live));
      const float inv = count > 0 ? 1.f / (float)count : 0.f, sum = wave_sum(logp);
      if (wg == 0 && blockIdx.y == 0) {
        if (lane < n) d.logp[lane] = logp;
        if (lane == 0) {
          d.loss[0] = -sum * inv;
          *d.inv = inv;
        }
      }
      if (lane == 0) scale = inv;
    }
    lds_barrier();
  }
  bf16x8h h[GP][NS][8];
#pragma unroll
  for (int p = 0; p < GP; ++p)
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t f[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t lo = reinterpret_cast<const uint32_t*>(&q[p][s][2 * t])[j >> 1];
          const uint32_t hi = reinterpret_cast<const uint32_t*>(&q[p][s][2 * t + 1])[j >> 1];
          f[t] = __builtin_amdgcn_perm(hi, lo, (j & 1) ? 0x07060302u : 0x05040100u);
        }
        h[p][s][j] = __builtin_bit_cast(bf16x8h, make_uint4(f[0], f[1], f[2], f[3]));
      }
  // this thread's 8 rows of the feature, and its vocabulary rows r0 + u 512 / TG of a chunk
  const int32_t tg = threadIdx.x % TG, r0 = threadIdx.x / TG;
  float l2[8], ow[8];
  int32_t lb[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    l2[t] = lse[8 * tg + t];
    ow[t] = own[8 * tg + t];
    lb[t] = lab[8 * tg + t];
  }
  const float inv = scale;
  const bool held = n > 0 && 8 * tg < ldz;  // z has these columns
  const int32_t chunks = (V + rows - 1) / rows;
  const int32_t c0 = (int32_t)((int64_t)chunks * wg / d.gwgs), c1 = (int32_t)((int64_t)chunks * (wg + 1) / d.gwgs);
  float4 z[U][2];
  auto fetch = [&](int32_t c) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      z[u][0] = z[u][1] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (held && r0 + u * (kSmallThreads / TG) < rows) {
        const int32_t v = min(c * rows + r0 + u * (kSmallThreads / TG), V - 1);
        const float4* const p = reinterpret_cast<const float4*>(d.z + (int64_t)v * ldz + 8 * tg);
        z[u][0] = p[0];
        z[u][1] = p[1];
      }
    }
  };
  if (c0 < c1) fetch(c0);
  for (int32_t c = c0; c < c1; ++c) {
    uint16_t* const line = dz[(c - c0) & 1][0];
    uint16_t* const rest = dz[(c - c0) & 1][1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t r = r0 + u * (kSmallThreads / TG), v = c * rows + r;
      if (r >= rows) break;
      float p[8] = {z[u][0].x, z[u][0].y, z[u][0].z, z[u][0].w, z[u][1].x, z[u][1].y, z[u][1].z, z[u][1].w};
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        p[t] = __builtin_amdgcn_exp2f(fmaf(p[t], kLog2e, -l2[t]));
        p[t] = lb[t] == v ? ow[t] : lb[t] < 0 ? 0.f : p[t];  // (no target: zeros also where W is not finite)
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        hi[t] = pack_bf2_cvt(p[2 * t], p[2 * t + 1]);
        lo[t] = pack_bf2_cvt(p[2 * t] - __uint_as_float(hi[t] << 16), p[2 * t + 1] - __uint_as_float(hi[t] & 0xffff0000u));
      }
      *reinterpret_cast<uint4*>(line + r * LD + 8 * tg) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(rest + r * LD + 8 * tg) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      if (d.grad && blockIdx.y == 0 && v < V && 8 * tg < ldz) {
        uint32_t w[8];  // both of a row side by side
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          w[2 * t] = __builtin_amdgcn_perm(lo[t], hi[t], 0x05040100u);
          w[2 * t + 1] = __builtin_amdgcn_perm(lo[t], hi[t], 0x07060302u);
        }
        uint4* const to = reinterpret_cast<uint4*>(d.grad + 2 * ((int64_t)v * ldz + 8 * tg));
        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
    lds_barrier();  // (the other line's readers passed the barrier before this one)
    if (c + 1 < c1) fetch(c + 1);
    for (int32_t b = wv; b < rows / 16; b += WV) {
#pragma unroll
      for (int p = 0; p < GP; ++p) {
        f32x4h a[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = f32x4h{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            __builtin_amdgcn_sched_barrier(0);  // (one fragment of dz at a time: more spill)
            const bf16x8h g = *reinterpret_cast<const bf16x8h*>((part ? line : rest) + (16 * b + col) * LD + 32 * s + 8 * quad);
#pragma unroll
            for (int j = 0; j < 8; ++j) a[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[p][s][j], g, a[j], 0, 0, 0);
          }
        if (wc + 8 * p >= groups) continue;
        // turned around in LDS: a store instruction writes 256 adjacent bytes of 4 rows
        constexpr int HALVES = F32 ? 2 : 1, COLS = 128 / HALVES;
#pragma unroll
        for (int f = 0; f < HALVES; ++f) {
#pragma unroll
          for (int e = f * 4 / HALVES; e < (f + 1) * 4 / HALVES; ++e) {
            const int chunk = F32 ? 8 * (e & 1) + 2 * quad : 4 * e + quad;
            if constexpr (F32) {
              mine16[col * 16 + (chunk ^ col)] = __builtin_bit_cast(u32x4t, f32x4h{a[0][e] * inv, a[1][e] * inv, a[2][e] * inv, a[3][e] * inv});
              mine16[col * 16 + ((chunk + 1) ^ col)] = __builtin_bit_cast(u32x4t, f32x4h{a[4][e] * inv, a[5][e] * inv, a[6][e] * inv, a[7][e] * inv});
            } else {
              mine16[col * 16 + (chunk ^ col)] = u32x4t{pack_bf2_cvt(a[0][e] * inv, a[1][e] * inv), pack_bf2_cvt(a[2][e] * inv, a[3][e] * inv),
                                                        pack_bf2_cvt(a[4][e] * inv, a[5][e] * inv), pack_bf2_cvt(a[6][e] * inv, a[7][e] * inv)};
            }
          }
          __builtin_amdgcn_wave_barrier();  // (a wave's LDS operations stay in order)
          const int32_t k = 128 * (g0 + wc + 8 * p) + COLS * f + COLS / 16 * col;
          u32x4t o[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) o[r] = mine16[(4 * r + quad) * 16 + (col ^ (4 * r + quad))];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int32_t v = c * rows + 16 * b + 4 * r + quad;
            if (v < V && k < width)
              put_once<ONCE>(o[r], reinterpret_cast<u32x4t*>(static_cast<char*>(d.dW) + ((int64_t)v * width + k) * (F32 ? 4 : 2)));
          }
          __builtin_amdgcn_wave_barrier();
        }
      }
    }
  }
}

static int small_share(int32_t d) { return d <= 256 ? 1 : d <= 512 ? 2 : d <= 1024 ? 4 : 8; }  // WK
int32_t small_score_rows(int32_t d) { return 16 * (8 / small_share(d)); }
int32_t small_grad_rows(int32_t d, int64_t vocab) {
  const int32_t groups = (d + 127) / 128, least = groups > 4 ? 16 : groups > 2 ? 32 : 128 / groups;  // of all wavefronts
  const int64_t each = (vocab + kSmallGroups - 1) / kSmallGroups;
  return (int32_t)std::max<int64_t>(least, std::min<int64_t>(kSmallGradRows, (each + 15) / 16 * 16));
}
// Kernel arguments of two tenants take 0.3 KB, of kSmallTenants 3 KB.
template <typename F>
static hipError_t with_tenants(const TokSmallSet& set, F&& f) {
  if (set.G > 2) return f(set);
  TokSmallArgs<2> few;
  few.t[0] = set.t[0];
  few.t[1] = set.t[1];
  few.G = set.G;
  return f(few);
}

hipError_t launch_small_scores(hipStream_t s, const TokSmallSet& all, int32_t wgs, int32_t ldz, const void* hidden,
                               int32_t T, int32_t d) {
  const uint16_t* const h = static_cast<const uint16_t*>(hidden);
  if (d > 8192 || d % 64 != 0) return hipErrorInvalidValue;
  return with_tenants(all, [&](const auto& set) {
    constexpr int C = sizeof(set.t) / sizeof(set.t[0]);
    auto go = [&](auto wk, auto ch, auto nb) {
      small_scores_kernel<wk(), ch(), nb(), C><<<wgs, kSmallThreads, 0, s>>>(set, ldz, h, T, d);
      return hipGetLastError();
    };
    auto rows = [&](auto wk, auto ch) {
      if (ldz == 16) return go(wk, ch, std::integral_constant<int, 1>());
      if constexpr (decltype(ch)::value <= 2)
        if (ldz == 32) return go(wk, ch, std::integral_constant<int, 2>());
      if constexpr (decltype(ch)::value == 1)
        if (ldz == 64) return go(wk, ch, std::integral_constant<int, 4>());
      return hipErrorInvalidValue;
    };
    const auto one = std::integral_constant<int, 1>();
    switch (small_share(d)) {
      case 1: return rows(std::integral_constant<int, 1>(), one);
      case 2: return rows(std::integral_constant<int, 2>(), one);
      case 4: return rows(std::integral_constant<int, 4>(), one);
      default:
        if (d <= 2048) return rows(std::integral_constant<int, 8>(), one);
        if (d <= 4096) return rows(std::integral_constant<int, 8>(), std::integral_constant<int, 2>());
        return rows(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
    }
  });
}

hipError_t launch_small_grads(hipStream_t s, const TokSmallSet& all, int32_t wgs, int32_t ldz, const void* hidden,
                              int32_t T, int32_t d, int32_t rows, bool f32) {
  if (rows < 16 || rows > kSmallGradRows || rows % 16 != 0) return hipErrorInvalidValue;
  const uint16_t* const h = static_cast<const uint16_t*>(hidden);
  const dim3 grid(wgs, (d + 2047) / 2048);
  // dW stored non-temporally where W, read before, and dW pass the last-level cache:
  // the next call's W then need not push dW out (5 rows, 60,000 x 2,048 129 -> 115 us)
  int64_t bytes = 0;
  for (int32_t g = 0; g < all.G; ++g) bytes += (f32 ? 6ll : 4ll) * all.t[g].vocab * d;
  return with_tenants(all, [&](const auto& set) {
    constexpr int C = sizeof(set.t) / sizeof(set.t[0]);
    auto go = [&](auto gp, auto ns) {
      auto kind = [&](auto f32_, auto once) {
        small_grads_kernel<gp(), ns(), C, f32_(), once()><<<grid, kSmallThreads, 0, s>>>(set, ldz, h, T, d, rows);
        return hipGetLastError();
      };
      auto type = [&](auto once) { return f32 ? kind(std::true_type(), once) : kind(std::false_type(), once); };
      return bytes > kStreamBytes ? type(std::true_type()) : type(std::false_type());
    };
    auto steps = [&](auto gp) {
      return ldz > 32 ? go(gp, std::integral_constant<int, 2>()) : go(gp, std::integral_constant<int, 1>());
    };
    return d <= 1024 ? steps(std::integral_constant<int, 1>()) : steps(std::integral_constant<int, 2>());
  });
}

hipError_t launch_small_pick(hipStream_t s, const TokSmallSet& all, int32_t ldz, int32_t T) {
  return with_tenants(all, [&](const auto& set) {
    constexpr int C = sizeof(set.t) / sizeof(set.t[0]);
    small_pick_kernel<C><<<dim3(set.G, ldz / 16), kSmallThreads, 0, s>>>(set, T);
    return hipGetLastError();
  });
}

// ------------------------------------------------ verification of drafts ---
// Rejecting children drawn from q leaves max(p_k - q, 0) / T of the node's
// distribution p_k; with p_k = max(p - a q, 0) / T that is max(p - (a + T) q, 0) over its
// sum, so that a node's state is the two numbers a and T, and a rejected drawn child costs
// one pass over the node's rows for the next T. Drafts that were picked need no pass:
// their p is taken off T. At last the next token needs one pass over the last node's row.
// A pass over a row by one workgroup would take 25 us for 160,001 tokens of p and q, so passes
// are launches of their own: tok_sums_kernel, `chunks` workgroups to a tree, each of
// which walks the tree for itself until it needs a sum, and sums its piece of that row.
// The next launch goes on from there (VerifyState), and tok_pick_next_kernel to the end,
// with passes of its own where the launches were too few; it finds the token in the pieces.
// What a walk needs of a node is one entry of its parent's rows: all nodes' are
// fetched together, then the walk is a wavefront's, a child after the other.
// All sums are formed in 64 bits: a border between two tokens lies where the
// definition has it, whatever order the terms are added in.
// Bound by latency: a chain over 32,003 tokens 5.7 + 5.0 us, 64 trees of 25 picked drafts
// 13.3 (their scattered entries) + 7.6, 16 trees of 9 drawn ones over 160,001 five launches of
// 3.5 to 10 and 7.6. (One workgroup a tree for everything took 78, 75 and 439.)
constexpr int kSumThreads = 256, kPickThreads = 1024;
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// Elements of a row's piece: pieces are whole multiples of 4.
__device__ __forceinline__ int32_t verify_piece(int32_t vocab, int32_t chunks) {
  return ((vocab + chunks - 1) / chunks + 3) / 4 * 4;
}

// Shared by a workgroup: the window's nodes, rejected tokens, where the walk is.
struct VerifyNodes {
  int32_t parent[JN_KV_TREE_ROWS], token[JN_KV_TREE_ROWS];
  float u[JN_KV_TREE_ROWS], p[JN_KV_TREE_ROWS], q[JN_KV_TREE_ROWS];
  int32_t gone[JN_KV_TREE_ROWS];
  VerifyState walk;
};

__device__ __forceinline__ VerifyState verify_start(const TokVerify& d) {
  VerifyState w{};
  w.count = 1;
  w.T = 1.;
  w.over = d.max_path == 1;
  return w;
}

// Sum of pieces by a wavefront.
__device__ __forceinline__ double verify_sum(const double* part, int32_t chunks, int32_t lane) {
  double v = 0.;
  for (int32_t c = lane; c < chunks; c += 64) v += part[c];
  return wave_sum64(v);
}

// The walk of a tree of n nodes by the first wavefront, on from w, until it needs a sum
// (w.waits) or is over; every thread gets the end. path (or null) receives standing nodes.
template <int THREADS>
__device__ VerifyState verify_walk(VerifyNodes& s, const TokVerify& d, int32_t first, int32_t n, VerifyState w, int32_t* path) {
  const int tid = threadIdx.x, lane = tid & 63;
  for (int32_t w0 = w.at / JN_KV_TREE_ROWS * JN_KV_TREE_ROWS; w0 < n; w0 += JN_KV_TREE_ROWS) {  // (of a long chain)
    const int32_t m = min(n - w0, JN_KV_TREE_ROWS);
    __syncthreads();
    for (int32_t i = tid; i < m; i += THREADS) {
      const int32_t j = w0 + i, up = j == 0 ? -1 : d.parents ? kv_parent(d.parents + first, j) : j - 1;
      const int32_t x = d.tokens[first + j];
      const bool on = up >= 0 && x >= 0 && x < d.vocab;
      s.parent[i] = on ? up : -1;
      s.token[i] = x;
      if (d.p) {
        s.u[i] = on ? d.u[first + j] : 0.f;
        s.p[i] = on ? d.p[(first + up) * d.ldp + x] : 0.f;
        s.q[i] = on && d.q ? d.q[(first + up) * d.ldq + x] : 0.f;
      } else {
        s.p[i] = on && d.greedy[first + up] == x ? 1.f : 0.f;
      }
    }
    __syncthreads();
    if (tid >= 64) continue;
#pragma unroll 1
    for (int32_t b0 = max(0, w.at - w0) & ~63; b0 < m && !w.over && !w.waits; b0 += 64) {
      const int32_t i = b0 + lane;
      const bool in = i < m;
      const int32_t parent = in ? s.parent[i] : -1, token = in ? s.token[i] : -1;
      const float pv = in ? s.p[i] : 0.f, qv = in ? s.q[i] : 0.f, uv = in && d.p ? s.u[i] : 0.f;
      const int32_t done = w.at - w0 - b0;  // nodes of the block before the one to go on with
      uint64_t left = done <= 0 ? ~0ull : ~0ull << done;
      while (true) {
        const uint64_t kids = __ballot(parent == w.cur) & left;
        if (kids == 0) break;
        const int k = __builtin_ctzll(kids);
        left = k == 63 ? 0 : ~0ull << (k + 1);
        const int32_t j = w0 + b0 + k, x = __builtin_amdgcn_readlane(token, k);
        w.at = j + 1;
        const double p = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pv), k));
        const double q = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(qv), k));
        const double u = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(uv), k));
        bool stands;
        if (!d.p) {
          stands = p > 0.;
        } else if (d.q) {
          const double rest = p - w.a * q;
          stands = u * q * w.T < (rest > 0. ? rest : 0.);
          if (!stands && w.T > 0.) {
            w.before = w.a;
            w.a += w.T;
            w.waits = 1;
            break;
          }
        } else {
          bool was = false;
          for (int32_t g = lane; g < w.ngone; g += 64) was |= s.gone[g] == x;
          const double rest = __any(was) || !(p > 0.) ? 0. : p;
          stands = u * w.T < rest;
          if (!stands && rest > 0.) {  // (of others nothing is taken: the last one gone is the last that had a weight)
            w.T -= rest;
            if (lane == 0) s.gone[w.ngone] = x;
            ++w.ngone;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          }
        }
        if (stands) {
          if (path && lane == 0) path[w.count] = j;
          w.cur = j;
          ++w.count;
          w.ngone = 0;
          w.a = w.before = 0.;
          w.T = 1.;
          if (w.count == d.max_path) {
            w.over = 1;
            break;
          }
        }
      }
    }
  }
  if (tid < 64) {
    if (!w.waits) w.over = 1;
    if (lane == 0) s.walk = w;
  }
  __syncthreads();
  return s.walk;
}

// Weights of elements i .. i + 3 of the row of node c.
__device__ __forceinline__ void verify_weights(const TokVerify& d, const VerifyNodes& s, int64_t row, double a,
                                               int32_t ngone, int32_t i, double (&w)[4]) {
  const float* const p = d.p + row * d.ldp + i;
  f32x4u x{0.f, 0.f, 0.f, 0.f}, y{0.f, 0.f, 0.f, 0.f};
  const bool whole = i + 4 <= d.vocab;
  if (whole) {
    x = *reinterpret_cast<const f32x4u*>(p);
    if (d.q) y = *reinterpret_cast<const f32x4u*>(d.q + row * d.ldq + i);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < d.vocab) {
        x[e] = p[e];
        if (d.q) y[e] = d.q[row * d.ldq + i + e];
      }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double v = d.q ? (double)x[e] - a * (double)y[e] : (double)x[e];
    w[e] = v > 0. ? v : 0.;
  }
  for (int32_t g = 0; g < ngone; ++g) {
    const uint32_t e = s.gone[g] - i;
    if (e < 4u) w[e] = 0.;
  }
}

__device__ __forceinline__ const TokVerify& verify_tenant(const TokVerifySet& set, int32_t tree) {
  int32_t g = 0;
  while (g + 1 < set.G && set.t[g + 1].tree0 <= tree) ++g;
  return set.t[g];
}
__device__ __forceinline__ int32_t verify_nodes(const TokVerify& d, int32_t t, int32_t& first) {
  first = min(max(d.cu[t], 0), d.n);
  return min(max(min(d.cu[t + 1], d.n) - first, 0), d.parents ? JN_KV_TREE_ROWS : d.max_path);
}

// Launch `phase`: every tree's walk on to the next sum that it needs, and its pieces.
__global__ __launch_bounds__(kSumThreads) void tok_sums_kernel(TokVerifySet set, VerifySums v, int32_t phase) {
  __shared__ VerifyNodes s;
  __shared__ double red[4];
  const int tid = threadIdx.x, lane = tid & 63;
  const int32_t tree = blockIdx.x / set.chunks, c = blockIdx.x - tree * set.chunks;
  const TokVerify& d = verify_tenant(set, tree);
  const int32_t t = tree - d.tree0;
  int32_t first;
  const int32_t n = verify_nodes(d, t, first);
  if (n == 0 || !d.p) return;
  const int now = phase & 1;
  VerifyState w = phase == 0 ? verify_start(d) : v.state[(now ^ 1) * set.trees + tree];
  int32_t* const path = c == 0 ? d.path + (int64_t)t * d.max_path : nullptr;
  if (path && phase == 0)
    for (int32_t k = tid; k < d.max_path; k += kSumThreads) path[k] = k == 0 ? 0 : -1;
  bool sum = false;
  if (!w.ends) {
    if (phase > 0) {
      w.T = verify_sum(v.part + ((int64_t)(now ^ 1) * set.trees + tree) * set.chunks, set.chunks, lane);
      w.waits = 0;
      w.slot = now ^ 1;
    }
    const double a = w.a;
    w = verify_walk<kSumThreads>(s, d, first, n, w, path);
    // at its end it needs the next token's sum, unless that is the one it has just taken
    w.ends = !w.waits;
    sum = w.waits || !(d.q && w.a > 0. && w.a == a);
    if (sum) w.slot = now;
  }
  if (c == 0) {
    if (tid == 0) v.state[now * set.trees + tree] = w;
    if (phase == 0 && w.ngone > 0)
      for (int32_t k = tid; k < w.ngone; k += kSumThreads) v.gone[(int64_t)tree * JN_KV_TREE_ROWS + k] = s.gone[k];
  }
  if (!sum) return;
  const int32_t piece = verify_piece(d.vocab, set.chunks), i0 = min(c * piece, d.vocab), i1 = min(i0 + piece, d.vocab);
  double y = 0.;
#pragma unroll 4
  for (int32_t i = i0 + 4 * tid; i < i1; i += 4 * kSumThreads) {
    double x[4];
    verify_weights(d, s, first + w.cur, w.a, w.ngone, i, x);
    y += (x[0] + x[1]) + (x[2] + x[3]);
  }
  y = wave_sum64(y);
  if (lane == 0) red[tid >> 6] = y;
  __syncthreads();
  if (tid == 0) v.part[((int64_t)now * set.trees + tree) * set.chunks + c] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kPickThreads) void tok_pick_next_kernel(TokVerifySet set, VerifySums vs, int32_t phases) {
  __shared__ VerifyNodes s;
  __shared__ double sums[kVerifyChunks], red[16];
  __shared__ int32_t pick[2], lasts[16], hits16[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t tree = blockIdx.x;
  const TokVerify& d = verify_tenant(set, tree);
  const int32_t t = tree - d.tree0;
  int32_t first;
  const int32_t n = verify_nodes(d, t, first);
  int32_t* const path = d.path + (int64_t)t * d.max_path;
  const bool begun = phases > 0 && d.p && n > 0;
  if (!begun)
    for (int32_t k = tid; k < d.max_path; k += kPickThreads) path[k] = k == 0 && n > 0 ? 0 : -1;
  if (n == 0) {
    if (tid == 0) {
      d.n_path[t] = 0;
      d.next[t] = -1;
    }
    return;
  }
  const int32_t piece = verify_piece(d.vocab, set.chunks);
  // pieces' sums of what is left at (c, a)
  auto pieces = [&](const VerifyState& w, double a) {
    __syncthreads();
    for (int32_t c = wave; c < set.chunks; c += 16) {
      const int32_t i0 = min(c * piece, d.vocab), i1 = min(i0 + piece, d.vocab);
      double v = 0.;
#pragma unroll 4
      for (int32_t i = i0 + 4 * lane; i < i1; i += 256) {
        double x[4];
        verify_weights(d, s, first + w.cur, a, w.ngone, i, x);
        v += (x[0] + x[1]) + (x[2] + x[3]);
      }
      v = wave_sum64(v);
      if (lane == 0) sums[c] = v;
    }
    __syncthreads();
  };
  VerifyState w;
  if (begun) {
    w = vs.state[((phases - 1) & 1) * set.trees + tree];
    const double* const from = vs.part + ((int64_t)w.slot * set.trees + tree) * set.chunks;
    for (int32_t c = tid; c < set.chunks; c += kPickThreads) sums[c] = from[c];
    for (int32_t k = tid; k < w.ngone; k += kPickThreads) s.gone[k] = vs.gone[(int64_t)tree * JN_KV_TREE_ROWS + k];
    __syncthreads();
  } else {
    w = verify_walk<kPickThreads>(s, d, first, n, verify_start(d), path);
    if (!d.p) {
      if (tid == 0) {
        d.n_path[t] = w.count;
        d.next[t] = d.greedy[first + w.cur];
      }
      return;
    }
    pieces(w, w.a);
  }
  while (w.waits) {  // more sums than launches: `sums` are what it waits for
    const double a = w.a;
    w.T = verify_sum(sums, set.chunks, lane);
    w.waits = 0;
    w = verify_walk<kPickThreads>(s, d, first, n, w, path);
    if (w.waits || w.a != a || !(w.a > 0.)) pieces(w, w.a);
  }
  double a = w.a;
  if (d.q && a > 0. && w.T == 0.) {
    a = w.before;
    pieces(w, a);
  }
  if (tid == 0) d.n_path[t] = w.count;
  // the piece that passes r of the whole, and in it every thread's run
  if (wave == 0) {
    double up = 0.;  // before the lane's pieces
    const int32_t per = (set.chunks + 63) / 64, c0 = min(lane * per, set.chunks), c1 = min(c0 + per, set.chunks);
    double v = 0.;
    for (int32_t c = c0; c < c1; ++c) v += sums[c];
    up = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(up, o, kWave);
      if (lane >= o) up += x;
    }
    const double want = (double)d.r[t] * __shfl(up, 63, kWave);
    double at = up - v;
    int32_t hit = -1, last = -1;
    double base = 0., lbase = 0.;
    for (int32_t c = c0; c < c1; ++c) {
      if (sums[c] > 0.) {
        last = c;
        lbase = at;
      }
      at += sums[c];
      if (hit < 0 && sums[c] > 0. && at > want) {
        hit = c;
        base = at - sums[c];
      }
    }
    // the first such piece; where rounding leaves none the last one with a weight
    const uint64_t hits = __ballot(hit >= 0), some = __ballot(last >= 0);
    const int l = hits ? __builtin_ctzll(hits) : some ? 63 - __builtin_clzll(some) : 0;
    if (lane == l) {
      pick[0] = hits ? hit : last;
      pick[1] = hits != 0;
      red[0] = want - (hits ? base : lbase);
    }
  }
  __syncthreads();
  const int32_t c = pick[0];
  const bool found = pick[1] != 0;
  const double want = red[0];
  __syncthreads();
  if (c < 0) {  // (of picked drafts the token that was taken last is all that was there before)
    if (tid == 0) d.next[t] = !d.q && w.ngone > 0 ? s.gone[w.ngone - 1] : -1;
    return;
  }
  const int32_t i0 = c * piece, i1 = min(i0 + piece, d.vocab);
  const int32_t run = ((i1 - i0 + kPickThreads - 1) / kPickThreads + 3) / 4 * 4;
  const int32_t r0 = min(i0 + tid * run, i1), r1 = min(r0 + run, i1);
  double v = 0., x[4];
  for (int32_t i = r0; i < r1; i += 4) {
    verify_weights(d, s, first + w.cur, a, w.ngone, i, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) v += i + e < i1 ? x[e] : 0.;
  }
  double up = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(up, o, kWave);
    if (lane >= o) up += y;
  }
  if (lane == 63) red[wave] = up;
  __syncthreads();
  double at = 0.;
  for (int k = 0; k < wave; ++k) at += red[k];
  at += up - v;
  int32_t last = -1, hit = -1;
  for (int32_t i = r0; i < r1; i += 4) {
    verify_weights(d, s, first + w.cur, a, w.ngone, i, x);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < i1 && x[e] > 0.) {
        at += x[e];
        last = i + e;
        if (hit < 0 && at > want) hit = i + e;
      }
  }
  // runs ascend with the threads: the first with a hit has the lowest, the last with a weight the highest
  const uint64_t some = __ballot(last >= 0), ones = __ballot(hit >= 0 && found);
  if (lane == 0) lasts[wave] = hits16[wave] = -1;
  if (some != 0 && lane == 63 - __builtin_clzll(some)) lasts[wave] = last;
  if (ones != 0 && lane == __builtin_ctzll(ones)) hits16[wave] = hit;
  __syncthreads();
  if (tid == 0) {
    int32_t next = -1;
    for (int k = 0; k < 16; ++k) next = max(next, lasts[k]);
    for (int k = 15; k >= 0; --k) next = hits16[k] >= 0 ? hits16[k] : next;
    d.next[t] = next;
  }
}

hipError_t launch_tok_verify(hipStream_t s, const TokVerifySet& set, int32_t phases, const VerifySums& v) {
  for (int32_t k = 0; k < phases; ++k) tok_sums_kernel<<<set.trees * set.chunks, kSumThreads, 0, s>>>(set, v, k);
  tok_pick_next_kernel<<<set.trees, kPickThreads, 0, s>>>(set, v, phases);
  return hipGetLastError();
}

}  // namespace jnx
