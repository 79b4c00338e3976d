// RMSNorm over rows of the packed batch: one wavefront per row, the row held
// in registers between the sum-of-squares pass and the scaling pass, a
// butterfly wave reduction (deterministic order), fp32 math, bf16 output.
#include <algorithm>
#include <type_traits>

#include "jn_device.h"
#include "jn_internal.h"

namespace jnx {

constexpr int kNormRowsPerBlock = 4;  // 4 waves, one row each

// Vectors of the non-temporal loads.
template <int W>
struct NormVec {
  typedef float f __attribute__((ext_vector_type(W)));
};

// Load VEC bf16 values starting at element `e` of a bf16 row.
template <int VEC>
__device__ __forceinline__ void load_bf(const uint16_t* row, int e, float* v) {
  if constexpr (VEC == 8) {
    uint4 q = *reinterpret_cast<const uint4*>(row + e);
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  } else if constexpr (VEC == 4) {
    uint2 q = *reinterpret_cast<const uint2*>(row + e);
    v[0] = __uint_as_float(q.x << 16);
    v[1] = __uint_as_float(q.x & 0xffff0000u);
    v[2] = __uint_as_float(q.y << 16);
    v[3] = __uint_as_float(q.y & 0xffff0000u);
  } else {
    uint32_t q = *reinterpret_cast<const uint32_t*>(row + e);
    v[0] = __uint_as_float(q << 16);
    v[1] = __uint_as_float(q & 0xffff0000u);
  }
}

template <int VEC, bool STREAM = false>
__device__ __forceinline__ void load_f32(const float* row, int e, float* v) {
  constexpr int W = VEC % 4 == 0 ? 4 : 2;
  typedef typename NormVec<W>::f V;
#pragma unroll
  for (int k = 0; k < VEC; k += W) {
    const V* p = reinterpret_cast<const V*>(row + e + k);
    V q;
    if constexpr (STREAM)
      q = __builtin_nontemporal_load(p);
    else
      q = *p;
#pragma unroll
    for (int i = 0; i < W; ++i) v[k + i] = q[i];
  }
}

template <int VEC>
__device__ __forceinline__ void store_f32(float* row, int e, const float* v) {
#pragma unroll
  for (int k = 0; k < VEC; k += 2) *reinterpret_cast<float2*>(row + e + k) = make_float2(v[k], v[k + 1]);
}

template <int VEC>
__device__ __forceinline__ void store_bf(uint16_t* row, int e, const float* v) {
  if constexpr (VEC == 8) {
    *reinterpret_cast<uint4*>(row + e) =
        make_uint4(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7]));
  } else if constexpr (VEC == 4) {
    *reinterpret_cast<uint2*>(row + e) = make_uint2(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]));
  } else {
    *reinterpret_cast<uint32_t*>(row + e) = pack_bf2(v[0], v[1]);
  }
}

// IN_BF16: x is bf16 (the packed tokens); its fp32 widening is also written to
// x_out (the residual stream).  Otherwise x is the fp32 residual stream.
// Each lane owns elements (c*64 + lane)*VEC .. +VEC for c < NC.  HBM-bound; the
// fp32 rows are read non-temporal, so that h, which the next GEMM reads, is what
// the caches keep: 295,606 x 768 236 -> 212 us (6.4 TB/s), 75,776 x 2048 159 ->
// 153.  (A non-temporal store of x_out: 239 -> 255 us on the latter.)
template <int VEC, int NC, bool IN_BF16>
__global__ __launch_bounds__(256) void rmsnorm_kernel(const void* __restrict__ xin, float* __restrict__ x_out,
                                                      const uint16_t* __restrict__ g, uint16_t* __restrict__ h,
                                                      int32_t rows, int32_t d, float eps) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * kNormRowsPerBlock + (threadIdx.x >> 6);
  if (row >= rows) return;
  float v[NC][VEC];
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int e = (c * 64 + lane) * VEC;
    if constexpr (IN_BF16)
      load_bf<VEC>(reinterpret_cast<const uint16_t*>(xin) + row * d, e, v[c]);
    else
      load_f32<VEC, true>(reinterpret_cast<const float*>(xin) + row * d, e, v[c]);
#pragma unroll
    for (int k = 0; k < VEC; ++k) ss += v[c][k] * v[c][k];
  }
  ss = wave_sum(ss);
  const float r = rsqrtf(ss / (float)d + eps);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int e = (c * 64 + lane) * VEC;
    if constexpr (IN_BF16) store_f32<VEC>(x_out + row * d, e, v[c]);
    float gv[VEC], o[VEC];
    load_bf<VEC>(g, e, gv);
#pragma unroll
    for (int k = 0; k < VEC; ++k) o[k] = v[c][k] * r * gv[k];
    store_bf<VEC>(h + row * d, e, o);
  }
}

// Reduction of a split residual projection and the norm after it in one pass:
// v = x + ((part[0] + part[1]) + ...), written back to x, then the norm of v in
// rmsnorm_kernel's order (which every wave forms for itself from the row in LDS).
// One workgroup per row, its column blocks dealt to up to four wavefronts: these
// batches have few rows, and the S + 1 reads of a row are what it waits for.  As two
// launches, in one wavefront per row, and now: 1 row of 4096, S = 8, 10.3, 17.3 and
// 5.8 us; 100 rows 9.7, 17.0 and 6.5; 300 rows of 2048, S = 8, 9.8, 6.6 and 6.4;
// 2,468 rows 39 (S = 8), 19.9 and 19.8 (S = 3).
constexpr int split_waves(int nc) { return nc < 4 ? nc : 4; }
template <int VEC, int NC>
__global__ __launch_bounds__(64 * split_waves(NC)) void rmsnorm_split_kernel(
    float* __restrict__ x, const float* __restrict__ part, int32_t S, int64_t stride, const uint16_t* __restrict__ g,
    uint16_t* __restrict__ h, int32_t d, float eps) {
  constexpr int W = split_waves(NC), CW = (NC + W - 1) / W;
  __shared__ __attribute__((aligned(16))) float line[NC * 64 * VEC];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = blockIdx.x;
  auto at = [&](int i) { return ((w + W * i) * 64 + lane) * VEC; };  // the wave's column block i
  auto mine = [&](int i) { return NC % W == 0 || w + W * i < NC; };
  float v[CW][VEC], a[CW][VEC];
#pragma unroll
  for (int i = 0; i < CW; ++i)
    if (mine(i)) {
      load_f32<VEC>(x + row * d, at(i), v[i]);
      load_f32<VEC>(part + row * d, at(i), a[i]);
    }
#pragma unroll 4
  for (int32_t s = 1; s < S; ++s) {
#pragma unroll
    for (int i = 0; i < CW; ++i)
      if (mine(i)) {
        float q[VEC];
        load_f32<VEC>(part + s * stride + row * d, at(i), q);
#pragma unroll
        for (int k = 0; k < VEC; ++k) a[i][k] += q[k];
      }
  }
#pragma unroll
  for (int i = 0; i < CW; ++i)
    if (mine(i)) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[i][k] += a[i][k];
      store_f32<VEC>(x + row * d, at(i), v[i]);
      store_f32<VEC>(line, at(i), v[i]);
    }
  __syncthreads();
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float q[VEC];
    load_f32<VEC>(line, (c * 64 + lane) * VEC, q);
#pragma unroll
    for (int k = 0; k < VEC; ++k) ss += q[k] * q[k];
  }
  ss = wave_sum(ss);
  const float r = rsqrtf(ss / (float)d + eps);
#pragma unroll
  for (int i = 0; i < CW; ++i)
    if (mine(i)) {
      float gv[VEC], o[VEC];
      load_bf<VEC>(g, at(i), gv);
#pragma unroll
      for (int k = 0; k < VEC; ++k) o[k] = v[i][k] * r * gv[k];
      store_bf<VEC>(h + row * d, at(i), o);
    }
}

// Calls f<VEC, NC>() with the lane layout of row width d: a multiple of 128 up
// to 4096; widths without a layout of their own take two elements per lane.
template <typename F>
static hipError_t with_width(int32_t d, F&& f) {
#define JN_RMS(VEC, NC) \
  if (d == 64 * (VEC) * (NC)) return f(std::integral_constant<int, VEC>(), std::integral_constant<int, NC>());
  JN_RMS(2, 1)   // 128
  JN_RMS(4, 1)   // 256
  JN_RMS(4, 2)   // 512
  JN_RMS(4, 3)   // 768
  JN_RMS(8, 2)   // 1024
  JN_RMS(8, 3)   // 1536
  JN_RMS(8, 4)   // 2048
  JN_RMS(8, 5)   // 2560
  JN_RMS(8, 6)   // 3072
  JN_RMS(8, 8)   // 4096
#define JN_RMS2(NC) JN_RMS(2, NC)
  JN_RMS2(3) JN_RMS2(5) JN_RMS2(7) JN_RMS2(9) JN_RMS2(10) JN_RMS2(11) JN_RMS2(13) JN_RMS2(14) JN_RMS2(15)
  JN_RMS2(17) JN_RMS2(18) JN_RMS2(19) JN_RMS2(20) JN_RMS2(21) JN_RMS2(22) JN_RMS2(23) JN_RMS2(25)
  JN_RMS2(26) JN_RMS2(27) JN_RMS2(28) JN_RMS2(29) JN_RMS2(30) JN_RMS2(31)
#undef JN_RMS2
#undef JN_RMS
  return hipErrorInvalidValue;
}

template <bool IN_BF16>
static hipError_t launch_rms(hipStream_t s, const void* x, float* x_out, const void* g, void* h, int32_t rows,
                             int32_t d, float eps) {
  const dim3 grid((rows + kNormRowsPerBlock - 1) / kNormRowsPerBlock);
  return with_width(d, [&](auto vec, auto nc) {
    rmsnorm_kernel<vec(), nc(), IN_BF16><<<grid, 256, 0, s>>>(x, x_out, reinterpret_cast<const uint16_t*>(g),
                                                              reinterpret_cast<uint16_t*>(h), rows, d, eps);
    return hipGetLastError();
  });
}

hipError_t launch_rmsnorm_split(hipStream_t s, float* x, const float* part, int32_t S, const void* g, void* h,
                                int32_t rows, int32_t d, float eps) {
  return with_width(d, [&](auto vec, auto nc) {
    rmsnorm_split_kernel<vec(), nc()><<<dim3(rows), 64 * split_waves(nc()), 0, s>>>(
        x, part, S, (int64_t)rows * d, reinterpret_cast<const uint16_t*>(g), reinterpret_cast<uint16_t*>(h), d, eps);
    return hipGetLastError();
  });
}

hipError_t launch_rmsnorm_bf16in(hipStream_t s, const void* x_bf16, float* x_out, const void* g, void* h,
                                 int32_t rows, int32_t d, float eps) {
  return launch_rms<true>(s, x_bf16, x_out, g, h, rows, d, eps);
}

hipError_t launch_rmsnorm_f32in(hipStream_t s, const float* x, const void* g, void* h, int32_t rows, int32_t d,
                                float eps) {
  return launch_rms<false>(s, x, nullptr, g, h, rows, d, eps);
}

// ------------------------------------- head norms and rotary positions ---
// Queries and keys of a fused q | k | v row, per head x of hd elements:
//   y = R(u), u = g x r, r = 1 / sqrt(mean(x^2) + eps)        (NORM; else u = x)
// R turns the pair (u_i, u_{i + hd/2}) by pos[axis(i)] * theta^(-2i/hd).  Its
// gradients, with du = R^T dy and xh = x r:
//   dx = r (g du - xh mean(xh g du)),   dg = sum over rows and heads of du xh
//
// One wavefront per row (or per part of a row's heads, where rows are few).  P2
// lanes hold a head: lane q its elements E q .. E q + E - 1 of both halves, so that
// a pair lies in one lane, and the 64 / P2 heads of one step are reduced together
// by log2 P2 lane exchanges.  A row's sines and cosines are formed once, one pair
// per lane, and shared through LDS.  Angles: turns = pos * f in 64 bits (f =
// theta^(-2i/hd) / 2 pi), of which the whole turns are dropped before anything is
// rounded to 32 bits, so positions of any size lose nothing; then sincospi.
// Everything else is fp32; y and dx are rounded to bf16 once.
// Bound by memory; with E = 4 a step holds fewer heads, so that less of the last
// one is idle (18 heads: 5 steps of 4, not 3 of 8), and the gradients' sums, gains
// and rows fit the registers of four wavefronts a SIMD: 75,923 rows forward 129 ->
// 124 us, gradients 262 -> 223.  The rows' loads are issued before the sines.  A
// vector instruction takes four cycles, so instructions count too: with the row
// and the step's offsets in scalar registers, 1 / hd multiplied in, the keys' gains
// chosen and their sums taken apart only in steps that hold keys, 160 -> 110 a step
// forward and 215 -> 155 backward, where they were 66 % of the time: 217 -> 193 us
// (5.4 TB/s; forward 116, 6.0 TB/s).  The next two steps' loads in flight under
// each step, over the ends of rows, measured the same 193.
constexpr int kQkFwdE = 4, kQkBwdE = 4;
constexpr int kQkStep = 4;  // head steps whose loads are issued together

// Sum over the P2 lanes of a head, in all of them.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int P2>
__device__ __forceinline__ float head_sum(float v) {
  if constexpr (P2 >= 2) v = add_dpp<0xB1>(v);   // lane ^ 1
  if constexpr (P2 >= 4) v = add_dpp<0x4E>(v);   // lane ^ 2
  if constexpr (P2 >= 8) v = add_dpp<0x141>(v);  // the other quad of 8 lanes
  if constexpr (P2 >= 16) v = add_dpp<0x140>(v); // the other 8 of 16
  if constexpr (P2 >= 32) v = sum_xor16(v);
  return v;
}

// Sines and cosines of a row's pairs into the wave's line [2][128]: cosines, sines.
__device__ __forceinline__ void row_turns(const QkShape& a, int64_t row, int lane, float* line) {
  const int half = a.hd >> 1;
  __builtin_amdgcn_wave_barrier();  // the line's last readers are done (a wave's LDS operations stay in order)
  for (int i = lane; i < half; i += 64) {
    const double t = (double)a.pos[row * a.axes + a.axis[i]] * a.freq[i];
    float sn, cs;
    sincospif((float)(2.0 * (t - rint(t))), &sn, &cs);
    line[i] = cs;
    line[128 + i] = sn;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// E values of a bf16 row, as loaded.
template <int E>
struct QkRaw {
  uint32_t w[E / 2];
};
template <int E>
__device__ __forceinline__ QkRaw<E> raw(const uint16_t* p) {
  if constexpr (E == 8)
    return __builtin_bit_cast(QkRaw<E>, *reinterpret_cast<const uint4*>(p));
  else
    return __builtin_bit_cast(QkRaw<E>, *reinterpret_cast<const uint2*>(p));
}
template <int E>
__device__ __forceinline__ void widen(const QkRaw<E>& q, float* v) {
#pragma unroll
  for (int k = 0; k < E / 2; ++k) {
    v[2 * k] = __uint_as_float(q.w[k] << 16);
    v[2 * k + 1] = __uint_as_float(q.w[k] & 0xffff0000u);
  }
}

// Results beyond the last-level cache are stored non-temporally (kStreamBytes):
// 75,923 rows of 18 heads of 128 forward 123.7 -> 116.9 us (6.0 TB/s), gradients
// 222.8 -> 216.3.
template <int E, bool ONCE>
__device__ __forceinline__ void put_bf(uint16_t* p, const float* v) {
  typedef uint32_t V __attribute__((ext_vector_type(E / 2)));
  V r;
#pragma unroll
  for (int k = 0; k < E / 2; ++k) r[k] = pack_bf2_cvt(v[2 * k], v[2 * k + 1]);
  if constexpr (ONCE)
    __builtin_nontemporal_store(r, reinterpret_cast<V*>(p));
  else
    *reinterpret_cast<V*>(p) = r;
}

// The gains of a lane's elements, queries' and keys'.
template <int E>
struct QkGains {
  QkRaw<E> q[2], k[2];  // both halves
  __device__ __forceinline__ void load(const QkShape& a, int at) {
    const int half = a.hd >> 1;
    q[0] = raw<E>(a.gq + at);
    q[1] = raw<E>(a.gq + at + half);
    k[0] = raw<E>(a.gk + at);
    k[1] = raw<E>(a.gk + at + half);
  }
  // any: whether a head of the step is a key (for the whole wavefront)
  __device__ __forceinline__ void get(bool any, bool key, float* v) const {
    if (!any) {
      widen<E>(q[0], v);
      widen<E>(q[1], v + E);
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        QkRaw<E> r;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) r.w[i] = key ? k[s].w[i] : q[s].w[i];
        widen<E>(r, v + E * s);
      }
    }
  }
};

// x and y may be the same rows: a lane reads what it writes before it does.
template <int E, int P2, bool NORM, bool ROPE, bool ONCE>
__global__ __launch_bounds__(256) void qk_fwd_kernel(QkShape a, const uint16_t* x, uint16_t* y, int32_t parts) {
  __shared__ __attribute__((aligned(16))) float lines[4][256];
  constexpr int PER = 64 / P2;  // heads per step
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane % P2, slot = lane / P2;
  const int64_t item = (int64_t)blockIdx.x * 4 + w;
  const int64_t row = item / parts;
  if (row >= a.rows) return;
  const int heads = a.heads + a.kv, half = a.hd >> 1;
  const int steps = (heads + PER - 1) / PER, part = (int)(item - row * parts);
  const int s0 = steps * part / parts, s1 = steps * (part + 1) / parts;
  const bool live = E * q < half;
  const uint32_t mine = slot * a.hd + E * q;
  const uint16_t* const xr = x + row * a.ldx;
  uint16_t* const yr = y + row * a.ldy;
  QkRaw<E> v[kQkStep][2];
  auto fetch = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kQkStep; ++j) {
      const int h = (s + j) * PER + slot;
      v[j][0] = v[j][1] = QkRaw<E>{};
      if (s + j < s1 && live && h < heads) {
        const uint16_t* const at = xr + (s + j) * PER * a.hd;
        v[j][0] = raw<E>(at + mine);
        v[j][1] = raw<E>(at + half + mine);
      }
    }
  };
  fetch(s0);  // in flight under the sines
  QkGains<E> g;
  if constexpr (NORM) g.load(a, live ? E * q : 0);
  const float* const line = lines[w] + (live ? E * q : 0);
  const float part_of = 1.f / (float)a.hd;
  if constexpr (ROPE) row_turns(a, row, lane, lines[w]);
  for (int s = s0; s < s1; s += kQkStep) {
    if (s > s0) fetch(s);
#pragma unroll
    for (int j = 0; j < kQkStep; ++j) {
      if (s + j >= s1) break;
      const int h = (s + j) * PER + slot;
      float u[2 * E];
      widen<E>(v[j][0], u);
      widen<E>(v[j][1], u + E);
      if constexpr (NORM) {
        float ss = 0.f, gv[2 * E];
#pragma unroll
        for (int k = 0; k < 2 * E; ++k) ss = fmaf(u[k], u[k], ss);
        const float r = rsqrtf(fmaf(head_sum<P2>(ss), part_of, a.eps));
        g.get((s + j + 1) * PER > a.heads, h >= a.heads, gv);
#pragma unroll
        for (int k = 0; k < 2 * E; ++k) u[k] = u[k] * r * gv[k];
      }
      if constexpr (ROPE) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const float p = u[k], o = u[E + k], cs = line[k], sn = line[128 + k];
          u[k] = p * cs - o * sn;
          u[E + k] = o * cs + p * sn;
        }
      }
      if (live && h < heads) {
        uint16_t* const at = yr + (s + j) * PER * a.hd;
        put_bf<E, ONCE>(at + mine, u);
        put_bf<E, ONCE>(at + half + mine, u + E);
      }
    }
  }
}

// Workgroups walk rows in steps of the grid; each leaves its sums of du xh in
// part [workgroup][2][hd], queries then keys, which qk_gain_kernel adds in
// order.  dx may be the rows of x or of dy.  With few rows (qk_one) one
// workgroup of 16 wavefronts takes them all, and its sums are the gradients.
template <int E, int P2, bool NORM, bool ROPE, bool ONCE, int W>
__global__ __launch_bounds__(64 * W, 4) void qk_bwd_kernel(QkShape a, const uint16_t* x, const uint16_t* dy,
                                                        uint16_t* dx, float* __restrict__ part,
                                                        float* __restrict__ dgq, float* __restrict__ dgk) {
  __shared__ __attribute__((aligned(16))) float lines[W][256];
  __shared__ float sums[NORM ? W : 1][2][256];
  constexpr int PER = 64 / P2, STEP = 2;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane % P2, slot = lane / P2;
  const int heads = a.heads + a.kv, half = a.hd >> 1, steps = (heads + PER - 1) / PER;
  const bool live = E * q < half;
  QkGains<E> g;
  float dg[2][2 * E];
  if constexpr (NORM) {
    g.load(a, live ? E * q : 0);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) dg[k][i] = 0.f;
  }
  const float* const line = lines[w] + (live ? E * q : 0);
  const uint32_t mine = slot * a.hd + E * q;
  const float part_of = 1.f / (float)a.hd;
  for (int64_t row = (int64_t)blockIdx.x * W + w; row < a.rows; row += (int64_t)gridDim.x * W) {
    const uint16_t* const xr = x + row * a.ldx;
    const uint16_t* const yr = dy + row * a.ldy;
    uint16_t* const dr = dx + row * a.ldd;
    QkRaw<E> v[STEP][4];
    auto fetch = [&](int s) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < STEP; ++j) {
        const int h = (s + j) * PER + slot;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j][k] = QkRaw<E>{};
        if (live && h < heads) {
          const int at = (s + j) * PER * a.hd;
          if constexpr (NORM) {
            v[j][0] = raw<E>(xr + at + mine);
            v[j][1] = raw<E>(xr + at + half + mine);
          }
          v[j][2] = raw<E>(yr + at + mine);
          v[j][3] = raw<E>(yr + at + half + mine);
        }
      }
    };
    fetch(0);
    if constexpr (ROPE) row_turns(a, row, lane, lines[w]);
    for (int s = 0; s < steps; s += STEP) {
      if (s > 0) fetch(s);
#pragma unroll
      for (int j = 0; j < STEP; ++j) {
        if (s + j >= steps) break;
        const int h = (s + j) * PER + slot;
        float du[2 * E];
        widen<E>(v[j][2], du);
        widen<E>(v[j][3], du + E);
        if constexpr (ROPE) {
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const float p = du[k], o = du[E + k], cs = line[k], sn = line[128 + k];
            du[k] = p * cs + o * sn;
            du[E + k] = o * cs - p * sn;
          }
        }
        if constexpr (NORM) {
          // with t = g du: mean(xh t) = r mean(x t), dx = r (t - x r mean(xh t))
          float xv[2 * E], gv[2 * E], ss = 0.f, dot = 0.f;
          widen<E>(v[j][0], xv);
          widen<E>(v[j][1], xv + E);
          const bool any = (s + j + 1) * PER > a.heads, key = h >= a.heads;
          g.get(any, key, gv);
#pragma unroll
          for (int k = 0; k < 2 * E; ++k) {
            ss = fmaf(xv[k], xv[k], ss);
            gv[k] *= du[k];
            dot = fmaf(xv[k], gv[k], dot);
          }
          const float r = rsqrtf(fmaf(head_sum<P2>(ss), part_of, a.eps));
          if (!any) {
#pragma unroll
            for (int k = 0; k < 2 * E; ++k) dg[0][k] = fmaf(du[k], xv[k] * r, dg[0][k]);
          } else {
#pragma unroll
            for (int k = 0; k < 2 * E; ++k) {
              const float t = du[k] * (xv[k] * r);
              dg[0][k] += key ? 0.f : t;  // (lanes without a head hold zeros)
              dg[1][k] += key ? t : 0.f;
            }
          }
          const float c = r * (r * head_sum<P2>(dot) * part_of);
#pragma unroll
          for (int k = 0; k < 2 * E; ++k) du[k] = r * fmaf(-xv[k], c, gv[k]);
        }
        if (live && h < heads) {
          uint16_t* const at = dr + (s + j) * PER * a.hd;
          put_bf<E, ONCE>(at + mine, du);
          put_bf<E, ONCE>(at + half + mine, du + E);
        }
      }
    }
  }
  if constexpr (NORM) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) {
        float v = dg[k][i];
#pragma unroll
        for (int o = P2; o < 64; o <<= 1) v += __shfl_xor(v, o, kWave);
        if (slot == 0 && live) sums[w][k][E * q + (i < E ? i : half + i - E)] = v;
      }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * a.hd; e += 64 * W) {
      const int k = e >= a.hd, c = e - k * a.hd;
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < W; i += 4)
        v += (sums[i][k][c] + sums[i + 1][k][c]) + (sums[i + 2][k][c] + sums[i + 3][k][c]);
      if constexpr (W == 4)
        part[(int64_t)blockIdx.x * 2 * a.hd + e] = v;
      else
        (k ? dgk : dgq)[c] = v;
    }
  }
}

// dgq | dgk = the sums of `blocks` workgroups, 16 columns per workgroup here, 64
// of the sums at a time.
__global__ __launch_bounds__(1024) void qk_gain_kernel(const float* __restrict__ part, int32_t blocks, int32_t hd,
                                                       float* __restrict__ dgq, float* __restrict__ dgk) {
  __shared__ float lds[16][17];
  const int c = threadIdx.x & 15, k = threadIdx.x >> 4, e = blockIdx.x * 16 + c;
  float v = 0.f;
#pragma unroll 8
  for (int32_t b = k; b < blocks; b += 64) v += part[(int64_t)b * 2 * hd + e];
  v = sum_xor16(v);  // the four of a wavefront
  v = sum_xor32(v);
  if ((threadIdx.x & 63) < 16) lds[threadIdx.x >> 6][c] = v;
  __syncthreads();
  if (k == 0) {
    v = lds[0][c];
#pragma unroll
    for (int i = 1; i < 16; ++i) v += lds[i][c];
    if (e < hd) dgq[e] = v; else dgk[e - hd] = v;
  }
}

// Whether the rows written are past the last-level cache.
static bool qk_streams(const QkShape& a) { return (int64_t)a.rows * (a.heads + a.kv) * a.hd * 2 > kStreamBytes; }

// Gradients of few rows by one workgroup: one launch instead of two, on one CU.  18
// heads of 128: 1 and 8 rows 9.4 -> 6.9 us a call, 16 (37 k elements) 9.3 -> 8.7,
// 24 9.4 -> 10.5; 16 heads of 256: 8 rows (33 k) 10.1 -> 9.1, 16 10.1 -> 12.4.
static bool qk_one(const QkShape& a) { return (int64_t)a.rows * (a.heads + a.kv) * a.hd <= 1 << 15; }

// Calls f<P2, NORM, ROPE, ONCE>() for the shape, with E elements of both halves a lane.
template <int E, typename F>
static hipError_t with_qk(const QkShape& a, F&& f) {
  auto kind = [&](auto p2, auto once) {
    const bool norm = a.gq != nullptr, rope = a.pos != nullptr;
    if (norm && rope) return f(p2, std::true_type(), std::true_type(), once);
    if (norm) return f(p2, std::true_type(), std::false_type(), once);
    return f(p2, std::false_type(), std::true_type(), once);
  };
  auto go = [&](auto p2) {
    return qk_streams(a) ? kind(p2, std::true_type()) : kind(p2, std::false_type());
  };
  constexpr int M = 16 / E;  // lanes of 32 elements
  if (a.hd <= 32) return go(std::integral_constant<int, M>());
  if (a.hd <= 64) return go(std::integral_constant<int, 2 * M>());
  if (a.hd <= 128) return go(std::integral_constant<int, 4 * M>());
  return go(std::integral_constant<int, 8 * M>());
}

static bool qk_ok(const QkShape& a) {
  return a.rows >= 1 && a.hd >= 16 && a.hd <= 256 && a.hd % 16 == 0 && (a.gq || a.pos) && !a.gq == !a.gk;
}

hipError_t launch_qk_fwd(hipStream_t s, const QkShape& a, const uint16_t* x, uint16_t* y) {
  if (!qk_ok(a)) return hipErrorInvalidValue;
  return with_qk<kQkFwdE>(a, [&](auto p2, auto norm, auto rope, auto once) {
    constexpr int PER = 64 / decltype(p2)::value;
    const int32_t steps = (a.heads + a.kv + PER - 1) / PER;
    const int32_t parts = a.rows < kQkFewRows ? steps : 1;
    const int64_t blocks = ((int64_t)a.rows * parts + 3) / 4;
    qk_fwd_kernel<kQkFwdE, p2(), norm(), rope(), once()><<<(unsigned)blocks, 256, 0, s>>>(a, x, y, parts);
    return hipGetLastError();
  });
}

int32_t qk_bwd_blocks(int32_t rows) {
  return (int32_t)std::min<int64_t>(((int64_t)rows + 3) / 4, kQkBwdBlocks);
}

hipError_t launch_qk_bwd(hipStream_t s, const QkShape& a, const uint16_t* x, const uint16_t* dy, uint16_t* dx,
                         float* part, float* dgq, float* dgk) {
  const int32_t blocks = qk_bwd_blocks(a.rows);
  if (a.rows > 0) {
    if (!qk_ok(a)) return hipErrorInvalidValue;
    const hipError_t e = with_qk<kQkBwdE>(a, [&](auto p2, auto norm, auto rope, auto once) {
      if constexpr (norm() && !once()) {
        if (qk_one(a)) {
          qk_bwd_kernel<kQkBwdE, p2(), norm(), rope(), once(), 16><<<1, 1024, 0, s>>>(a, x, dy, dx, part, dgq, dgk);
          return hipGetLastError();
        }
      }
      qk_bwd_kernel<kQkBwdE, p2(), norm(), rope(), once(), 4><<<blocks, 256, 0, s>>>(a, x, dy, dx, part, dgq, dgk);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (a.gq && qk_one(a)) return hipSuccess;
  }
  if (!a.gq) return hipSuccess;
  qk_gain_kernel<<<2 * a.hd / 16, 1024, 0, s>>>(part, blocks, a.hd, dgq, dgk);
  return hipGetLastError();
}

}  // namespace jnx
