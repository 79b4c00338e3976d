// Segment-masked varlen attention over the packed batch (forward), gfx950,
// and the rotary position embedding applied to q and k before it.
//
// Every sample attends over its own valid rows only -- bidirectionally, or
// causally (row j sees rows 0..j) -- nothing crosses a sample (hence a
// tenant) boundary and alignment rows are neither keys nor queries (their
// output rows are written as zero).  With fewer key/value heads than query
// heads, query head h reads key/value head h / (H / Hkv).
//
// Work item = (sample, head, 128-query tile); a workgroup = 4 wavefronts x 32
// query rows.  (sample, head) groups are dealt round-robin to the 8 XCDs
// (hardware places workgroup b on XCD b % 8) with all query tiles of a group
// on one XCD: they share its L2 for the group's keys and values, and a run of
// long samples (one tenant's) is spread over every XCD.
//
// Per step of KB keys, the K and V tiles ([KB][HD] bf16, row-major) are
// moved global -> LDS by direct DMA (global_load_lds_dwordx4), double
// buffered: the DMA of step j+1 runs under the compute of step j, one
// workgroup barrier per step.  Each LDS row is a permutation of its 16-byte
// chunks (chunk c stored at c ^ swz(row)), chosen per head width so that
// both reads below touch every LDS bank once per 256 bytes.
//
// Scores: S^T = K Q^T with v_mfma_f32_32x32x16_bf16, K the "A" operand
// (16-byte LDS reads), Q held in registers as "B", so each lane owns one
// query row's scores for 16 of every 32 keys and the online-softmax row
// max / sum need only its registers plus one exchange with lane ^ 32
// (v_permlane32_swap, no LDS round trip).  Both products run their
// contraction chunks outermost, so independent accumulators alternate, and
// read the next chunk's fragments before the current chunk's MFMAs.  The
// probabilities then sit in the operand layout of O^T += V^T P^T (keys
// contracted in the permuted order the score layout gives), so P stays in
// registers.  The V^T operand is read from the row-major V tile with
// ds_read_b64_tr_b16: in each 16-lane group, lane j addresses 4 elements of
// key row k0 + j/4 at column n0 + 4(j%4) and receives, transposed, the
// column n0 + (lane % 16) of rows k0..k0+3 -- 4 consecutive keys of one
// head-dim row, as the MFMA wants.  Statistics in fp32, P rounded to bf16.
// Head width 256 runs attn16_fwd_kernel: the same algorithm with 8 waves x 16
// query rows and v_mfma_f32_16x16x32_bf16 (two waves per SIMD).
#include <algorithm>
#include <type_traits>

#include "jn_device.h"
#include "jn_internal.h"
#include "jn_kv.h"

namespace jnx {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

#define JN_GPTR(p) ((__attribute__((address_space(1))) void*)(p))
#define JN_LPTR(p) ((__attribute__((address_space(3))) void*)(p))

constexpr int kQRows = 128;  // query rows per workgroup (4 waves x 32, or 8 x 16 at head width 256)
constexpr float kRescale = 8.0f;  // log2 headroom before the running max is moved
constexpr int kKeys = 64;    // keys per step (64 measured best for head widths 64 and 256)

// Chunk permutation of LDS row r (HD/8 chunks of 16 bytes per row).  K
// fragment reads touch 16 consecutive rows (one chunk each) per 16 lanes;
// transposed V reads touch rows k0..k0+3 (k0 % 4 == 0) x 4 adjacent chunks
// per 16 lanes.  Both cover 16 distinct 16-byte bank slots with:
//   HD 32  (4 rows per 256-byte bank row): (r >> 2) & 3
//   HD 64  (2 rows per bank row):          bit-reversed ((r >> 1) & 7)
//   HD 128:                                4 * (r & 3) + ((r >> 2) & 3)
//   HD 256 (r = 4 q + e):                  2 * (e + 4 * ((q ^ q / 2) & 1)) + q / 2
// At head width 256 a transposed read (16 lanes = 4 rows x 2 chunks) is
// served together with a second 16-lane group, and the bank-conflict
// counter located the pairs: groups q and q ^ 1 and groups q and q ^ 2.
// The HD 128 rule puts rows r and r ^ 4 on one bank slot pair (19% of the
// kernel's cycles in conflicts), 2 * (r & 7) + r / 8 rows r and r ^ 8 (9.5%);
// this rule pairs rows r and r ^ 12 only, which no served pair holds
// together (0 conflict cycles, and still 16 distinct slots for the 16 rows of
// a K fragment read).
template <int HD>
__device__ __forceinline__ int attn_swz(int r) {
  if constexpr (HD == 32) {
    return (r >> 2) & 3;
  } else if constexpr (HD == 64) {
    const int x = (r >> 1) & 7;
    return ((x & 1) << 2) | (x & 2) | (x >> 2);
  } else if constexpr (HD == 128) {
    return ((r & 3) << 2) | ((r >> 2) & 3);
  } else {
    const int q = (r >> 2) & 3, e = r & 3;
    return ((e | (((q ^ (q >> 1)) & 1) << 2)) << 1) | ((q >> 1) & 1);
  }
}

template <int N>
__device__ __forceinline__ void attn_wait_vmcnt() {
  static_assert(N >= 0 && N < 16, "vmcnt range");
  __builtin_amdgcn_s_waitcnt(N | (7 << 4) | (15 << 8) | (0 << 14));
}

struct AttnShape {
  int32_t d;        // output row width = H * hd
  int32_t ld;       // qkv row width = (H + 2 Hkv) * hd
  int32_t kv_col;   // first key column (H * hd)
  int32_t v_col;    // first value column ((H + Hkv) * hd)
  int32_t n_kv;     // key/value heads
  int32_t group;    // query heads per key/value head
  int32_t qtiles;   // 128-query tiles per sample (of the longest sample)
  int32_t total;    // (sample, key/value head) groups
  int32_t nblocks;  // work-item slots (blocks of the one-item-per-workgroup mapping)
  float scale_log2;
};

template <int HD, int KB, bool CAUSAL>
__global__ __launch_bounds__(256, (HD >= 256 && KB >= 64) ? 1 : 2) void attn_fwd_kernel(
    const uint16_t* __restrict__ qkv, uint16_t* __restrict__ out, const int32_t* __restrict__ seqlens,
    const int32_t* __restrict__ cu_seqlens, AttnShape sh) {
  constexpr int CPR = HD / 8;            // 16-byte chunks per row
  constexpr int TILE = KB * HD;          // elements of one K (or V) tile
  constexpr int NDMA = 2 * TILE / 512;   // 1 KB DMA instructions per stage (K tile, then V tile)
  constexpr int DPW = NDMA / 4;          // per wavefront
  constexpr int RPI = 512 / HD;          // rows per DMA instruction
  constexpr int NQC = HD / 16;           // 16-wide head-dim chunks (score contraction)
  constexpr int NOT = HD / 32;           // 32-row tiles of O^T
  constexpr int NKT = KB / 32;           // 32-key score tiles per step
  constexpr int NKC = KB / 16;           // 16-key P^T operands per step
  static_assert(NDMA % 4 == 0 && KB % 32 == 0, "tile shape");
  __shared__ __attribute__((aligned(1024))) uint16_t lds[2][2 * TILE];

  // XCD-aware work mapping: (sample, key/value head) group g goes to XCD
  // g % 8, and the query tiles of all its query heads to consecutive slots of
  // that XCD (block b runs on XCD b % 8, slot b / 8).  Groups interleave
  // across XCDs, so samples of very different lengths spread evenly, while
  // each group's keys and values are read by one XCD only.
  const int32_t b = blockIdx.x;
  const int32_t slot = b >> 3;
  const int32_t units = sh.group * sh.qtiles;
  const int32_t kg = (slot / units) * 8 + (b & 7);
  if (kg >= sh.total) return;
  const int32_t r_in = slot % units;
  const int32_t qt = r_in % sh.qtiles;
  const int32_t i = kg / sh.n_kv, kvh = kg % sh.n_kv;
  const int32_t h = kvh * sh.group + r_in / sh.qtiles;
  const int32_t d = sh.d;
  const int32_t L = seqlens[i];
  const int32_t base = cu_seqlens[i];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  if (qt == 0) {  // alignment rows of this sample: zero output
    const int32_t pad = cu_seqlens[i + 1] - base - L;
    for (int32_t e = tid; e < pad * (HD / 8); e += 256) {
      const int32_t row = base + L + e / (HD / 8);
      *reinterpret_cast<uint4*>(out + (int64_t)row * d + h * HD + (e % (HD / 8)) * 8) = make_uint4(0, 0, 0, 0);
    }
  }
  const int32_t q0 = qt * kQRows;
  if (q0 >= L) return;

  const int64_t ld = sh.ld;
  const float scale_log2 = sh.scale_log2;
  const uint16_t* Qg = qkv + h * HD;
  const uint16_t* Kg = qkv + sh.kv_col + kvh * HD;
  const uint16_t* Vg = qkv + sh.v_col + kvh * HD;

  // this wave's DMA instructions u = wave*DPW + k fill 1 KB each; lane ->
  // row (v*RPI + lane / CPR) of the K or V tile, physical chunk lane % CPR,
  // which holds logical chunk (lane % CPR) ^ swz(row)
  auto issue_stage = [&](int32_t kb, int stage) {
#pragma unroll
    for (int k = 0; k < DPW; ++k) {
      const int u = wave * DPW + k;
      const bool isv = u >= NDMA / 2;
      const int v = isv ? u - NDMA / 2 : u;
      const int r = v * RPI + lane / CPR;
      const int c = (lane % CPR) ^ attn_swz<HD>(r);
      const int32_t key = min(kb + r, L - 1);
      const uint16_t* src = (isv ? Vg : Kg) + (int64_t)(base + key) * ld + c * 8;
      __builtin_amdgcn_global_load_lds(JN_GPTR(src), JN_LPTR(&lds[stage][u * 512]), 16, 0, 0);
    }
  };

  const int32_t qw = q0 + wave * 32;  // this wave's first query row
  const bool active = qw < L;
  const int32_t qrow = min(qw + (lane & 31), L - 1);
  const int half = lane >> 5;
  bf16x8 qf[NQC];
#pragma unroll
  for (int c = 0; c < NQC; ++c)
    qf[c] = *reinterpret_cast<const bf16x8*>(Qg + (int64_t)(base + qrow) * ld + c * 16 + half * 8);

  // per-lane LDS offsets: K fragment rows kt*32 + lane%32 (swizzle period 16)
  const int krow = lane & 31;
  const int kswz = attn_swz<HD>(krow);
  // transposed V reads: 16-lane group gq = lane / 16, j = lane % 16
  const int j16 = lane & 15;
  const int vrow0 = 4 * half + (j16 >> 2);                           // + kc*16 (+8)
  const int vcol = ((lane >> 4) & 1) * 16 + 4 * (j16 & 3);           // + t*32
  const int vswz0 = attn_swz<HD>(vrow0), vswz1 = attn_swz<HD>(vrow0 + 8);

  f32x16 o[NOT];
#pragma unroll
  for (int t = 0; t < NOT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const int hi4 = half * 4;

  issue_stage(0, 0);
  // causal: keys past the tile's last query are never needed
  const int32_t kend = CAUSAL ? min(L, q0 + kQRows) : L;
  const int32_t nsteps = (kend + KB - 1) / KB;
  for (int32_t jstep = 0; jstep < nsteps; ++jstep) {
    const int32_t kb = jstep * KB;
    attn_wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();  // step j's tiles landed; step j-1's buffer is free
    if (jstep + 1 < nsteps) issue_stage(kb + KB, (jstep + 1) & 1);
    if (!active) continue;
    if (CAUSAL && kb > qw + 31) continue;  // every key of the step is later than the wave's queries
    const uint16_t* Ks = &lds[jstep & 1][0];
    const uint16_t* Vs = &lds[jstep & 1][TILE];

    // S^T for NKT 32-key tiles: dim chunk c outer, so the tiles' accumulators
    // alternate, with the K fragments of chunk c+1 read before the MFMAs of
    // chunk c (each accumulator still sums c = 0..NQC-1 in order)
    f32x16 s[NKT];
    bf16x8 kf[2][NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
      kf[0][kt] = *reinterpret_cast<const bf16x8*>(Ks + (kt * 32 + krow) * HD + ((half ^ kswz) * 8));
    }
#pragma unroll
    for (int c = 0; c < NQC; ++c) {
      if (c + 1 < NQC) {
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
          kf[(c + 1) & 1][kt] =
              *reinterpret_cast<const bf16x8*>(Ks + (kt * 32 + krow) * HD + (((2 * (c + 1) + half) ^ kswz) * 8));
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c & 1][kt], qf[c], s[kt], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    // Online softmax in the log2 domain (scores scaled by log2(e)/sqrt(hd)).
    // The running max m only moves when some query of the wave gains more
    // than kRescale (2^8 headroom for p = 2^(s - m) in fp32 and bf16); O and
    // the running sum l always share the same m, so the final O / l is exact
    // whichever m was used.  Keys past the sample are masked in the last step
    // only (wave-uniform branch).  The probabilities use the hardware exp2
    // (v_exp_f32; results below 2^-126 flush to zero, far below P's bf16
    // rounding): the library exp2f adds a denormal-range fix-up of about four
    // instructions per score, which measured 7-21% of this kernel's time.
    float mloc = -INFINITY;
    if (kb + KB > L || (CAUSAL && kb + KB - 1 > qw)) {
      const int32_t qlane = qw + (lane & 31);
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int32_t key = kb + kt * 32 + (r >> 2) * 8 + hi4 + (r & 3);
          if (key >= L || (CAUSAL && key > qlane)) s[kt][r] = -INFINITY;
        }
    }
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) mloc = fmaxf(mloc, s[kt][r]);
    mloc = max_xor32(mloc) * scale_log2;
    if (__any(mloc > m_run + kRescale)) {
      const float m_new = fmaxf(m_run, mloc);
      if (__all(m_run == -INFINITY)) {
        m_run = m_new;  // first update: O and l are still zero
      } else {
        const float alpha = exp2f(m_run - m_new);
        l_run *= alpha;
        m_run = m_new;
#pragma unroll
        for (int t = 0; t < NOT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
      }
    }
    float lsum = 0.f;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[kt][r], scale_log2, -m_run));
        s[kt][r] = p;
        lsum += p;
      }
    lsum = sum_xor32(lsum);
    l_run += lsum;

    // P^T operands: 16-key chunk kc holds registers 8*(kc&1) .. +7 of tile kc>>1,
    // i.e. keys kc*16 + 4*half + 0..3 and kc*16 + 8 + 4*half + 0..3
    bf16x8 pf[NKC];
#pragma unroll
    for (int kc = 0; kc < NKC; ++kc)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[kc][e] = (__bf16)s[kc >> 1][(kc & 1) * 8 + e];
    // O^T += V^T P^T: key chunk kc outer, so the head-dim blocks'
    // accumulators alternate, with the V^T fragments of chunk kc+1 read
    // before the MFMAs of chunk kc (each o[t] still sums kc = 0..NKC-1 in order)
    auto read_v = [&](int kc, bf16x8 (&vf)[NOT]) {
      const int r0 = kc * 16 + vrow0;
#pragma unroll
      for (int t = 0; t < NOT; ++t) {
        const int col = t * 32 + vcol;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (__attribute__((address_space(3))) bf16x4*)(Vs + r0 * HD + (((col >> 3) ^ vswz0) * 8) + (col & 7)));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (__attribute__((address_space(3))) bf16x4*)(Vs + (r0 + 8) * HD + (((col >> 3) ^ vswz1) * 8) + (col & 7)));
        vf[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
    bf16x8 vb[2][NOT];
    read_v(0, vb[0]);
#pragma unroll
    for (int kc = 0; kc < NKC; ++kc) {
      if (kc + 1 < NKC) read_v(kc + 1, vb[(kc + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < NOT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[kc & 1][t], pf[kc], o[t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  if (!active) return;
  const int32_t q = qw + (lane & 31);
  if constexpr (HD <= 64) {
    const float inv = 1.0f / l_run;
    // lane (query l % 32, half l / 32) holds head-dim columns 32 t + 8 rr +
    // 4 (l / 32) .. +3; swapping the packed blocks rr+1 of the low half with
    // the blocks rr of the high half (rr even) leaves each lane 8 consecutive
    // columns, 32 t + 8 rr + 8 (l / 32), for one 16-byte store (at head width
    // 128 the causal kernel then spilled registers, so it keeps 8-byte stores)
    uint16_t* orow = out + (int64_t)(base + q) * d + h * HD + 2 * hi4;
#pragma unroll
    for (int t = 0; t < NOT; ++t)
#pragma unroll
      for (int rr = 0; rr < 4; rr += 2) {
        const auto a = __builtin_amdgcn_permlane32_swap(pack_bf2(o[t][rr * 4] * inv, o[t][rr * 4 + 1] * inv),
                                                        pack_bf2(o[t][rr * 4 + 4] * inv, o[t][rr * 4 + 5] * inv),
                                                        false, false);
        const auto c = __builtin_amdgcn_permlane32_swap(pack_bf2(o[t][rr * 4 + 2] * inv, o[t][rr * 4 + 3] * inv),
                                                        pack_bf2(o[t][rr * 4 + 6] * inv, o[t][rr * 4 + 7] * inv),
                                                        false, false);
        if (q < L) *reinterpret_cast<uint4*>(orow + t * 32 + rr * 8) = make_uint4(a[0], c[0], a[1], c[1]);
      }
  } else {
    if (q >= L) return;
    const float inv = 1.0f / l_run;
    uint16_t* orow = out + (int64_t)(base + q) * d + h * HD;
#pragma unroll
    for (int t = 0; t < NOT; ++t)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        *reinterpret_cast<uint2*>(orow + t * 32 + rr * 8 + hi4) =
            make_uint2(pack_bf2(o[t][rr * 4] * inv, o[t][rr * 4 + 1] * inv),
                       pack_bf2(o[t][rr * 4 + 2] * inv, o[t][rr * 4 + 3] * inv));
  }
}


// Head width 256: 8 wavefronts x 16 query rows with v_mfma_f32_16x16x32_bf16,
// so that two waves share each SIMD and one wave's softmax and LDS reads run
// under the other's matrix products (4 waves x 32 rows need ~480 registers
// per lane: one wave per SIMD, whose MFMA, VALU and LDS work then run one
// after another).  Per wave: O^T 16 x 256 in 64 registers, Q in 32, scores of
// a 64-key step in 16.  Measured: 0.56 -> 0.45 ms on the 2B-shaped batch,
// 15-23% faster on 300-3000-token samples; at head width 128 the same layout
// was no faster on 300-token samples and 9% slower on 1000-token ones, so
// that width keeps attn_fwd_kernel.
// Its 128 KB of K/V stages leave room for one workgroup per compute unit, so
// a workgroup that fetched its Q rows and first stage only after starting
// left the compute unit idle for that fetch, and between workgroups: timer
// stamps on the 2B-shaped batch put ~13K of a work item's ~38K cycles
// outside the key loop.  The grid is therefore one workgroup per compute
// unit, each running a fixed list of work items, with the next item's first
// K/V stage and Q rows fetched under the current item's last key step
// (8.1 -> 7.1 ms per 18-layer step).  The output is written 16 bytes per
// lane after a lane swap (8.1 -> 6.5 ms with both).  The work of an item,
// hence every output bit, is unchanged.
//   S^T = K Q^T: A = K (16 keys x 32 dims), B = Q (32 dims x 16 queries);
//     lane l holds query l % 16 and keys 4 (l / 16) .. +3 of each 16-key block.
//   O^T += V^T P^T over a 32-key chunk (blocks 2c, 2c+1): B slot 8 q + e of
//     lane l (q = l / 16) is key 4 q + e of block 2c for e < 4 and key
//     4 q + e - 4 of block 2c+1 otherwise -- the scores' own layout -- and the
//     A operand (16 head-dim rows) takes the same key order from two
//     transposed reads of 4 keys each.
template <int HD, bool CAUSAL>
__global__ __launch_bounds__(512, 1) void attn16_fwd_kernel(const uint16_t* __restrict__ qkv, uint16_t* __restrict__ out,
                                                          const int32_t* __restrict__ seqlens,
                                                          const int32_t* __restrict__ cu_seqlens, AttnShape sh) {
  constexpr int KB = 64;                 // keys per step
  constexpr int NW = 8;                  // wavefronts
  constexpr int CPR = HD / 8;            // 16-byte chunks per row
  constexpr int TILE = KB * HD;          // elements of one K (or V) tile
  constexpr int NDMA = 2 * TILE / 512;   // 1 KB DMA instructions per stage (K tile, then V tile)
  constexpr int DPW = NDMA / NW;         // per wavefront
  constexpr int RPI = 512 / HD;          // rows per DMA instruction
  constexpr int NQC = HD / 32;           // 32-wide head-dim chunks (score contraction)
  constexpr int NOT = HD / 16;           // 16-row blocks of O^T
  static_assert(HD == 256, "head width");
  static_assert(NDMA % NW == 0, "tile shape");
  __shared__ __attribute__((aligned(1024))) uint16_t lds[2][2 * TILE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j16 = lane & 15, quad = lane >> 4;
  const int32_t d = sh.d;
  const int64_t ld = sh.ld;
  const float scale_log2 = sh.scale_log2;
  const int32_t units = sh.group * sh.qtiles;

  // A workgroup runs the work items of blocks blockIdx.x, + gridDim.x, ...
  // (block b: the mapping of attn_fwd_kernel, so b % 8 still names the XCD
  // when gridDim.x % 8 == 0).  The first K/V stage and the Q rows of the
  // next item are fetched under the last key step of the current one.
  struct Item {
    int32_t h, kvh, L, base, q0, nsteps;
  };
  auto decode = [&](int32_t b, Item& it) -> bool {  // false: the block has no work
    const int32_t slot = b >> 3;
    const int32_t kg = (slot / units) * 8 + (b & 7);
    if (kg >= sh.total) return false;
    const int32_t r_in = slot % units;
    const int32_t qt = r_in % sh.qtiles;
    const int32_t i = kg / sh.n_kv;
    it.kvh = kg % sh.n_kv;
    it.h = it.kvh * sh.group + r_in / sh.qtiles;
    it.L = seqlens[i];
    it.base = cu_seqlens[i];
    if (qt == 0) {  // alignment rows of this sample: zero output
      const int32_t pad = cu_seqlens[i + 1] - it.base - it.L;
      for (int32_t e = tid; e < pad * (HD / 8); e += 512) {
        const int32_t row = it.base + it.L + e / (HD / 8);
        *reinterpret_cast<uint4*>(out + (int64_t)row * d + it.h * HD + (e % (HD / 8)) * 8) = make_uint4(0, 0, 0, 0);
      }
    }
    it.q0 = qt * kQRows;
    if (it.q0 >= it.L) return false;
    const int32_t kend = CAUSAL ? min(it.L, it.q0 + kQRows) : it.L;
    it.nsteps = (kend + KB - 1) / KB;
    return true;
  };
  auto next_item = [&](int32_t b, Item& it) -> int32_t {  // first block >= b (same residue) with work
    for (; b < sh.nblocks; b += gridDim.x)
      if (decode(b, it)) return b;
    return sh.nblocks;
  };
  auto issue_stage = [&](const Item& it, int32_t kb, int stage) {
    const uint16_t* Kg = qkv + sh.kv_col + it.kvh * HD;
    const uint16_t* Vg = qkv + sh.v_col + it.kvh * HD;
#pragma unroll
    for (int k = 0; k < DPW; ++k) {
      const int u = wave * DPW + k;
      const bool isv = u >= NDMA / 2;
      const int v = isv ? u - NDMA / 2 : u;
      const int r = v * RPI + lane / CPR;
      const int c = (lane % CPR) ^ attn_swz<HD>(r);
      const int32_t key = min(kb + r, it.L - 1);
      const uint16_t* src = (isv ? Vg : Kg) + (int64_t)(it.base + key) * ld + c * 8;
      __builtin_amdgcn_global_load_lds(JN_GPTR(src), JN_LPTR(&lds[stage][u * 512]), 16, 0, 0);
    }
  };
  bf16x8 qf[NQC];
  auto load_q = [&](const Item& it) {
    const int32_t qrow = min(it.q0 + wave * 16 + j16, it.L - 1);
    const uint16_t* Qg = qkv + it.h * HD + (int64_t)(it.base + qrow) * ld + quad * 8;
#pragma unroll
    for (int c = 0; c < NQC; ++c) qf[c] = *reinterpret_cast<const bf16x8*>(Qg + c * 32);
  };

  Item cur, nxt;
  int32_t b = next_item(blockIdx.x, cur);
  if (b >= sh.nblocks) return;
  load_q(cur);
  issue_stage(cur, 0, 0);

  // K fragment of 16-key block kb16, dim chunk c: row 16 kb16 + j16, logical
  // 16-byte chunk 4 c + quad; rows 16 kb16 + j share the swizzle of row j
  const int kswz = attn_swz<HD>(j16);
  // V^T reads: group quad, lane j16 addresses key row 4 quad + j16 / 4 (+ 32 c,
  // + 16 for the second half) at head-dim column 16 t + 4 (j16 % 4); those rows
  // share one swizzle
  const int vrow = 4 * quad + (j16 >> 2);
  const int vswz = attn_swz<HD>(vrow);

  int par = 0;  // buffer of the current item's first step
  while (true) {
    const int32_t qw = cur.q0 + wave * 16;  // this wave's first query row
    const bool active = qw < cur.L;
    f32x4 o[NOT];
#pragma unroll
    for (int t = 0; t < NOT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    int32_t bn = sh.nblocks;  // next block with work, found in the last step
    for (int32_t jstep = 0; jstep < cur.nsteps; ++jstep) {
      const int32_t kb = jstep * KB;
      const int stage = (par + jstep) & 1;
      attn_wait_vmcnt<0>();
      __builtin_amdgcn_s_barrier();  // step j's tiles landed; step j-1's buffer is free
      const bool last = jstep + 1 == cur.nsteps;
      if (!last) {
        issue_stage(cur, kb + KB, stage ^ 1);
      } else {
        bn = next_item(b + gridDim.x, nxt);
        if (bn < sh.nblocks) issue_stage(nxt, 0, stage ^ 1);
      }
      // every key of the step later than the wave's queries: nothing to do
      const bool work = active && !(CAUSAL && kb > qw + 15);
      const uint16_t* Ks = &lds[stage][0];
      const uint16_t* Vs = &lds[stage][TILE];

      // scores: dim chunk c outer, so the four 16-key blocks' accumulators
      // alternate; the K fragments of chunk c+1 are read before the MFMAs of
      // chunk c (each accumulator still sums c = 0..NQC-1 in order)
      f32x4 s[4];
      if (work) {
        bf16x8 kf[2][4];
#pragma unroll
        for (int kb16 = 0; kb16 < 4; ++kb16) {
          s[kb16] = f32x4{0.f, 0.f, 0.f, 0.f};
          kf[0][kb16] = *reinterpret_cast<const bf16x8*>(Ks + (kb16 * 16 + j16) * HD + ((quad ^ kswz) * 8));
        }
#pragma unroll
        for (int c = 0; c < NQC; ++c) {
          if (c + 1 < NQC) {
#pragma unroll
            for (int kb16 = 0; kb16 < 4; ++kb16)
              kf[(c + 1) & 1][kb16] = *reinterpret_cast<const bf16x8*>(Ks + (kb16 * 16 + j16) * HD +
                                                                       (((4 * (c + 1) + quad) ^ kswz) * 8));
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int kb16 = 0; kb16 < 4; ++kb16)
            s[kb16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c & 1][kb16], qf[c], s[kb16], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (last && bn < sh.nblocks) load_q(nxt);  // Q is not read again in this item
      if (!work) continue;
      // online softmax (see attn_fwd_kernel); the four lanes of a query are
      // lane ^ 16 and lane ^ 32 apart
      float mloc = -INFINITY;
      if (kb + KB > cur.L || (CAUSAL && kb + KB - 1 > qw)) {
        const int32_t qlane = qw + j16;
#pragma unroll
        for (int kb16 = 0; kb16 < 4; ++kb16)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int32_t key = kb + kb16 * 16 + quad * 4 + e;
            if (key >= cur.L || (CAUSAL && key > qlane)) s[kb16][e] = -INFINITY;
          }
      }
#pragma unroll
      for (int kb16 = 0; kb16 < 4; ++kb16)
#pragma unroll
        for (int e = 0; e < 4; ++e) mloc = fmaxf(mloc, s[kb16][e]);
      mloc = max_xor32(max_xor16(mloc)) * scale_log2;
      if (__any(mloc > m_run + kRescale)) {
        const float m_new = fmaxf(m_run, mloc);
        if (__all(m_run == -INFINITY)) {
          m_run = m_new;  // first update: O and l are still zero
        } else {
          const float alpha = exp2f(m_run - m_new);
          l_run *= alpha;
          m_run = m_new;
#pragma unroll
          for (int t = 0; t < NOT; ++t) o[t] *= alpha;
        }
      }
      float lsum = 0.f;
#pragma unroll
      for (int kb16 = 0; kb16 < 4; ++kb16)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[kb16][e], scale_log2, -m_run));
          s[kb16][e] = p;
          lsum += p;
        }
      lsum = sum_xor32(sum_xor16(lsum));
      l_run += lsum;

      bf16x8 pf[2];
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pf[c][e] = (__bf16)s[2 * c][e];
          pf[c][4 + e] = (__bf16)s[2 * c + 1][e];
        }
      // P.V: the V^T fragments of head-dim block t+2 are read before the
      // MFMAs of block t
      auto read_v = [&](int t, bf16x8 (&vf)[2]) {
        const int col = t * 16 + 4 * (j16 & 3);
        const int pos = (((col >> 3) ^ vswz) * 8) + (col & 7);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int r0 = c * 32 + vrow;
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4*)(Vs + r0 * HD + pos));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4*)(Vs + (r0 + 16) * HD + pos));
          vf[c] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
      };
      bf16x8 vb[2][2];
      read_v(0, vb[0]);
#pragma unroll
      for (int t = 0; t < NOT; ++t) {
        if (t + 1 < NOT) read_v(t + 1, vb[(t + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 2; ++c) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb[t & 1][c], pf[c], o[t], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }

    if (active) {
      // lane (j16, quad) holds head-dim columns 16 t + 4 quad .. +3 of query
      // j16; swapping the packed blocks t+1 of quads 0, 2 with the blocks t
      // of quads 1, 3 leaves each lane 8 consecutive columns: 16 t (quad 0),
      // 16 t + 16 (1), 16 t + 8 (2), 16 t + 24 (3), one 16-byte store each
      const int32_t q = qw + j16;
      const float inv = 1.0f / l_run;
      uint16_t* orow = out + (int64_t)(cur.base + q) * d + cur.h * HD + 16 * (quad & 1) + 8 * (quad >> 1);
#pragma unroll
      for (int t = 0; t < NOT; t += 2) {
        const auto a = __builtin_amdgcn_permlane16_swap(pack_bf2(o[t][0] * inv, o[t][1] * inv),
                                                        pack_bf2(o[t + 1][0] * inv, o[t + 1][1] * inv), false, false);
        const auto c = __builtin_amdgcn_permlane16_swap(pack_bf2(o[t][2] * inv, o[t][3] * inv),
                                                        pack_bf2(o[t + 1][2] * inv, o[t + 1][3] * inv), false, false);
        if (q < cur.L) *reinterpret_cast<uint4*>(orow + t * 16) = make_uint4(a[0], c[0], a[1], c[1]);
      }
    }
    if (bn >= sh.nblocks) break;
    par = (par + cur.nsteps) & 1;
    cur = nxt;
    b = bn;
  }
}

// compute units of the current device (cached per device)
static int attn_compute_units() {
  static int cached[64] = {};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
  if (cached[dev] == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
    cached[dev] = n;
  }
  return cached[dev];
}

hipError_t launch_attention(hipStream_t s, const void* qkv, void* out, const int32_t* seqlens,
                            const int32_t* cu_seqlens, int32_t N, int32_t d, int32_t n_heads, int32_t n_kv_heads,
                            bool causal, int32_t max_seqlen, int32_t align) {
  (void)align;
  const int hd = d / n_heads;
  const int32_t kv = n_kv_heads > 0 ? n_kv_heads : n_heads;
  if (kv < 1 || n_heads % kv != 0) return hipErrorInvalidValue;
  AttnShape sh;
  sh.d = d;
  sh.ld = (n_heads + 2 * kv) * hd;
  sh.kv_col = n_heads * hd;
  sh.v_col = (n_heads + kv) * hd;
  sh.n_kv = kv;
  sh.group = n_heads / kv;
  sh.qtiles = (max_seqlen + kQRows - 1) / kQRows;
  const int64_t total = (int64_t)N * kv;
  const int64_t blocks = (total + 7) / 8 * 8 * sh.group * sh.qtiles;
  if (total <= 0 || blocks > (1LL << 30)) return hipErrorInvalidValue;
  sh.total = (int32_t)total;
  sh.nblocks = (int32_t)blocks;
  sh.scale_log2 = 1.4426950408889634f / sqrtf((float)hd);
  const dim3 grid((unsigned)blocks);
  // head width 256: one workgroup per compute unit (its LDS and registers
  // allow no second), each running every gridDim.x-th block
  int cus = attn_compute_units();
  cus -= cus % 8;
  const dim3 grid16((unsigned)(cus >= 8 && blocks > cus ? cus : blocks));
  auto Q = reinterpret_cast<const uint16_t*>(qkv);
  auto O = reinterpret_cast<uint16_t*>(out);
#define JN_ATTN(HDV)                                                                        \
  case HDV:                                                                                 \
    if (causal)                                                                             \
      attn_fwd_kernel<HDV, kKeys, true><<<grid, 256, 0, s>>>(Q, O, seqlens, cu_seqlens, sh);  \
    else                                                                                    \
      attn_fwd_kernel<HDV, kKeys, false><<<grid, 256, 0, s>>>(Q, O, seqlens, cu_seqlens, sh); \
    break;
#define JN_ATTN16(HDV)                                                                          \
  case HDV:                                                                                     \
    if (causal)                                                                                 \
      attn16_fwd_kernel<HDV, true><<<grid16, 512, 0, s>>>(Q, O, seqlens, cu_seqlens, sh);        \
    else                                                                                        \
      attn16_fwd_kernel<HDV, false><<<grid16, 512, 0, s>>>(Q, O, seqlens, cu_seqlens, sh);       \
    break;
  switch (hd) {
    JN_ATTN(32)
    JN_ATTN(64)
    JN_ATTN(128)
    JN_ATTN16(256)
    default:
      return hipErrorInvalidValue;
  }
#undef JN_ATTN
#undef JN_ATTN16
  return hipGetLastError();
}

// ------------------------------------------------------------------ rope ---
// Rotary embedding in place on the q and k head slices of qkv (bf16).  One
// block per row; a thread owns two adjacent pairs (2j, 2j+1) of the row's
// rotation and applies them to a strided subset of its heads, so each sine /
// cosine is computed once per row.  Angles in fp32: p * theta^(-2i/hd).
__global__ __launch_bounds__(256) void rope_kernel(uint16_t* __restrict__ qkv, int32_t ld,
                                                   const int32_t* __restrict__ token_pos, int32_t heads,
                                                   int32_t hd, float log2_theta) {
  const int32_t t = blockIdx.x;
  const int32_t pos = token_pos[t];
  if (pos < 0) return;  // alignment row
  const int32_t half = hd >> 1, q4 = hd >> 2;
  const int32_t j = threadIdx.x % q4, hg = threadIdx.x / q4, hstep = 256 / q4;
  if (hg >= hstep) return;
  float c[2], sn[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float inv_freq = exp2f(-(float)(2 * (2 * j + e)) / (float)hd * log2_theta);
    sincosf((float)pos * inv_freq, &sn[e], &c[e]);
  }
  uint16_t* row = qkv + (int64_t)t * ld;
  for (int32_t h = hg; h < heads; h += hstep) {
    uint32_t* pa = reinterpret_cast<uint32_t*>(row + h * hd + 2 * j);
    uint32_t* pb = reinterpret_cast<uint32_t*>(row + h * hd + half + 2 * j);
    const uint32_t wa = *pa, wb = *pb;
    const float a0 = __uint_as_float(wa << 16), a1 = __uint_as_float(wa & 0xffff0000u);
    const float b0 = __uint_as_float(wb << 16), b1 = __uint_as_float(wb & 0xffff0000u);
    *pa = pack_bf2(a0 * c[0] - b0 * sn[0], a1 * c[1] - b1 * sn[1]);
    *pb = pack_bf2(b0 * c[0] + a0 * sn[0], b1 * c[1] + a1 * sn[1]);
  }
}

hipError_t launch_rope(hipStream_t s, void* qkv, int32_t ld, const int32_t* token_pos, int32_t T, int32_t heads,
                       int32_t hd, float theta) {
  if (T < 1 || heads < 1 || hd % 4 != 0 || hd / 4 > 256 || !(theta > 0.f)) return hipErrorInvalidValue;
  rope_kernel<<<T, 256, 0, s>>>(reinterpret_cast<uint16_t*>(qkv), ld, token_pos, heads, hd, log2f(theta));
  return hipGetLastError();
}

// ------------------------------------------- attention over a paged cache ---
// A sequence's new rows j and the query heads g of one key head h are the query rows
// r = j G + g of a unit (sequence, key head); all of them read the same keys and
// values, the cached rows and (as the mask says) the new ones. How many keys each unit
// has is known on the device only, so the units' key tiles are laid end to end and
// every workgroup takes an equal run of them: whatever the lengths, all finish
// together. A unit that several workgroups hold is left as partial results (O, m, l)
// which kv_join_kernel adds. A workgroup finds its run from the sequences' lengths by
// itself (KvWalk), so there is no planning launch; at most two of its units are
// not whole, the first (slot 0) and the last (slot 1).
struct KvDesc {                // of a slot of a workgroup: its part of a unit
  int32_t seq, h, qt, wa, wb;  // held by workgroups wa .. wb; wb < 0: nothing
};
constexpr int32_t kKvJoinMany = 16;
struct KvWork {
  KvDesc* desc;          // [P][2]
  float2* ml;            // [P][2][rows]
  float* o;              // [P][2][rows][HD]
  int32_t P;             // workgroups, a multiple of 8
  int32_t group;         // query heads of a key head
  int32_t least;         // tiles of a workgroup, where there are so many
};

// x * P / total and the like for x, P <= total * 1024: in 32 bits where it fits.
__device__ __forceinline__ int64_t kv_div(int64_t a, int64_t b) {
  if (a < (1ll << 32) && b < (1ll << 32)) return (int64_t)((uint32_t)a / (uint32_t)b);
  return a / b;
}

__device__ __forceinline__ int64_t wave_scan64(int64_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o, kWave);
    if (lane >= o) v += u;
  }
  return v;
}

// Lane l's value, known to be the same for all lanes (in scalar registers).
__device__ __forceinline__ int64_t wave_get64(int64_t v, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane((int32_t)v, l), hi = __builtin_amdgcn_readlane((int32_t)(v >> 32), l);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// The same value in all lanes, said so.
__device__ __forceinline__ int32_t wave_same(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t wave_same64(int64_t v) { return wave_get64(v, 0); }

// The run of tiles [pos, end) of a workgroup, walked unit by unit. KT keys a tile; R
// query rows a tile of a unit (0: a unit has one tile of rows), a unit is then
// (sequence, key head, row tile), and a chain's row tiles end at their last row's keys.
template <int KT, int R>
struct KvWalk {
  int64_t total, pos, end, unit0;  // unit0: first tile of the current unit
  int32_t P, p;                    // workgroups with work, and this one's place in their order
  int32_t seq, h, qt, tiles;       // the current unit, and its tiles
  int32_t group;
  KvSeq sq;
  int32_t kend;                    // keys of the unit

  static __device__ __forceinline__ int32_t row_tiles(const KvSeq& q, int32_t G) {
    return R ? (int32_t)(((int64_t)q.n * G + R - 1) / R) : q.n > 0;
  }
  static __device__ __forceinline__ int32_t keys(const KvBatch& b, const KvSeq& q, int32_t G, int32_t qt) {
    int32_t n = q.n;
    if constexpr (R != 0)
      if (!b.whole && !b.parents) n = min(n, (int32_t)(((int64_t)qt * R + R - 1) / G) + 1);
    return min(q.past + n, b.places);
  }
  static __device__ __forceinline__ int32_t tiles_of(int32_t keys) { return (keys + KT - 1) / KT; }
  // Tiles of the first k <= row_tiles row tiles of a key head. A chain's row tile i has
  // min(floor((R i + B) / (KT G)), C) tiles, B = R - 1 + G (past + KT), C those of its last
  // row: those below C are summed as the steps of the Euclidean algorithm (count, modulus,
  // slope and offset below), the rest are C each. All in 32 bits but the sum: G n <= 2^26,
  // and past is taken modulo KT. (Row tile after row tile instead, the search made two
  // pieces of 2,048 and 1,792 rows take 329 us, with this 312.)
  static __device__ __forceinline__ int64_t upto(const KvBatch& b, const KvSeq& q, int32_t G, int32_t k) {
    const int32_t last = tiles_of(min(q.past + q.n, b.places));
    if constexpr (R == 0) return (int64_t)k * last;
    if (b.whole || b.parents || k <= 1) {
      return (int64_t)k * tiles_of(keys(b, q, G, 0));
    } else {
      const int32_t x = q.past / KT, y = q.past % KT, rise = G * KT * (last - x - 1) - G * y - (R - 1);
      const int32_t below = rise <= 0 ? 0 : min(k, (rise + R - 1) / R);
      int64_t sum = (int64_t)(k - below) * last + (int64_t)below * (x + 1);
      uint32_t t = below, m = KT * G, a = R, o = R - 1 + G * y;
      while (true) {
        const uint32_t qa = a / m, qo = o / m;
        sum += (int64_t)t * (t - 1) / 2 * qa + (int64_t)t * qo;
        a -= qa * m;
        o -= qo * m;
        const uint32_t top = a * t + o;
        if (top < m) return sum;
        t = top / m;
        o = top - t * m;
        const uint32_t was = m;
        m = a;
        a = was;
      }
    }
  }
  // Tiles of a key head of sequence s, which is q.
  static __device__ __forceinline__ int64_t of_seq(const KvBatch& b, const KvSeq& q, int32_t G, int32_t s) {
    return s < b.n_seqs ? upto(b, q, G, row_tiles(q, G)) : 0;
  }

  // At most `most` workgroups, of `least` tiles each where there are so many. Runs that
  // follow each other go to one XCD, whose workgroups are every eighth.
  __device__ __forceinline__ bool start(const KvBatch& b, int32_t kv, int32_t G, int32_t most, int32_t least, int lane) {
    group = G;
    int64_t all = 0, mine = 0;
    KvSeq q{};
#pragma unroll 4
    for (int32_t s0 = 0; s0 < b.n_seqs; s0 += 64) {
      if (s0 + lane < b.n_seqs) q = kv_seq(b, s0 + lane);
      mine = of_seq(b, q, G, s0 + lane);
      all += mine;
    }
    int64_t scan = wave_scan64(all, lane);
    total = wave_get64(scan, 63) * kv;
    total = wave_same64(total);
    const bool all_run = total >= (int64_t)most * least;
    p = all_run ? (blockIdx.x & 7) * (most >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    P = all_run ? most : (int32_t)((total + least - 1) / least);
    if (p >= P) return false;
    pos = wave_same64(kv_div(total * p, P));
    end = wave_same64(kv_div(total * (p + 1), P));
    int64_t before = 0;
    seq = 0;
    for (int32_t s0 = 0;; s0 += 64) {
      if (b.n_seqs > 64) {
        if (s0 + lane < b.n_seqs) q = kv_seq(b, s0 + lane);
        mine = of_seq(b, q, G, s0 + lane);
        scan = wave_scan64(mine, lane);
      }
      const int32_t c = __builtin_popcountll(__ballot((before + scan) * kv <= pos));
      if (c < 64) {
        seq = s0 + c;
        before += wave_get64(scan - mine, c);
        mine = wave_get64(mine, c);
        sq = KvSeq{__builtin_amdgcn_readlane(q.past, c), __builtin_amdgcn_readlane(q.row0, c),
                   __builtin_amdgcn_readlane(q.n, c)};
        break;
      }
      before += wave_get64(scan, 63);
    }
    qt = 0;
    unit(b);
    int64_t rest = pos - before * kv;
    h = wave_same((int32_t)kv_div(rest, mine));
    rest -= h * mine;
    unit0 = wave_same64(pos - rest);
    if constexpr (R != 0) {
      // the last row tile that begins at or before `rest`, 64 of them at a time
      int32_t len = row_tiles(sq, G);
      while (len > 0) {
        const int32_t stride = (len + 63) >> 6, k = (lane + 1) * stride;
        const bool before = k <= len && upto(b, sq, G, qt + k) <= rest;
        const int32_t c = __builtin_popcountll(__ballot(before)) * stride;
        qt += c;
        len = min(len - c, stride - 1);
      }
      qt = wave_same(qt);
      unit0 += wave_same64(upto(b, sq, G, qt));
      unit(b);
    }
    return true;
  }
  __device__ __forceinline__ void unit(const KvBatch& b) {
    kend = wave_same(keys(b, sq, group, qt));
    tiles = tiles_of(kend);
  }
  __device__ __forceinline__ void take(const KvBatch& b) {
    const KvSeq q = kv_seq(b, seq);
    sq = KvSeq{__builtin_amdgcn_readfirstlane(q.past), __builtin_amdgcn_readfirstlane(q.row0),
               __builtin_amdgcn_readfirstlane(q.n)};
    qt = 0;
    unit(b);
  }
  // To the unit behind the current one (pos < end: there is one).
  __device__ __forceinline__ void next(const KvBatch& b, int32_t kv) {
    unit0 += tiles;
    if (R != 0 && ++qt < row_tiles(sq, group)) return unit(b);
    if (++h < kv) {
      qt = 0;
      return unit(b);
    }
    h = 0;
    do {
      ++seq;
      take(b);
    } while (sq.n == 0);
  }
  __device__ __forceinline__ int32_t holder(int64_t x) const { return (int32_t)kv_div((x + 1) * P - 1, total); }
};

// s_waitcnt vmcnt(N) alone.
template <int N>
__device__ __forceinline__ void kv_wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// 16 bytes a lane from `src` to 1 KB of LDS at `dst` (the same for all lanes), which only
// this wavefront reads: it waits by kv_wait_vmcnt, and no barrier stands between.
__device__ __forceinline__ void kv_dma(const uint16_t* src, uint16_t* dst) {
  __builtin_amdgcn_global_load_lds(JN_GPTR(src), JN_LPTR(dst), 16, 0, 0);
}

// Four (two) V^T fragments of 16 columns x 32 keys of a V tile: rows a and a + 16 of
// two transposed reads each, at LDS byte addresses at[t] + off. The wait stands in the
// same statement: a read in flight never outlives it (and the compiler's own form would
// wait for every prefetch in flight).
template <int HD>
__device__ __forceinline__ void kv_read_v(const uint32_t* at, uint32_t off, bf16x8 (&v)[4]) {
  uint64_t r[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(at[0] + off), "v"(at[1] + off), "v"(at[2] + off), "v"(at[3] + off), "n"(16 * HD * 2)
      : "memory");
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const bf16x4 lo = __builtin_bit_cast(bf16x4, r[2 * t]), hi = __builtin_bit_cast(bf16x4, r[2 * t + 1]);
    v[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}
template <int HD>
__device__ __forceinline__ void kv_read_v(const uint32_t* at, uint32_t off, bf16x8 (&v)[2]) {
  uint64_t r[4];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4\n\t"
      "ds_read_b64_tr_b16 %1, %4 offset:%6\n\t"
      "ds_read_b64_tr_b16 %2, %5\n\t"
      "ds_read_b64_tr_b16 %3, %5 offset:%6\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(at[0] + off), "v"(at[1] + off), "n"(16 * HD * 2)
      : "memory");
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bf16x4 lo = __builtin_bit_cast(bf16x4, r[2 * t]), hi = __builtin_bit_cast(bf16x4, r[2 * t + 1]);
    v[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// x, as a value that the compiler knows nothing of: what is made of it is made where it
// is used and not kept in registers through the loops around (the masks' bits, the
// ends of units: 60 registers of the loops below).
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

__device__ __forceinline__ uint32_t kv_lds(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// What the new rows of a tree see, as bits of the new rows: row j itself and its
// ancestors. All threads of the workgroup; rows j0 .. j0 + rows - 1.
struct KvTree {
  uint16_t up[JN_KV_TREE_ROWS];
  uint64_t seen[128][JN_KV_TREE_ROWS / 64];
};
template <int THREADS>
__device__ __forceinline__ void kv_tree(KvTree& t, const KvBatch& b, const KvSeq& sq, int32_t j0, int32_t rows) {
  for (int32_t j = threadIdx.x; j < sq.n; j += THREADS) t.up[j] = (uint16_t)kv_parent(b.parents + sq.row0, j);
  __syncthreads();
  for (int32_t i = threadIdx.x; i < rows && j0 + i < sq.n; i += THREADS) {
    uint64_t w[4] = {0, 0, 0, 0};
    for (uint32_t j = j0 + i; j != 0xffffu; j = t.up[j]) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if ((j >> 6) == (uint32_t)k) w[k] |= 1ull << (j & 63);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) t.seen[i][k] = w[k];
  }
  __syncthreads();
}
// Bits of new rows k .. k + 31 (k may be below 0 or beyond the last).
__device__ __forceinline__ uint32_t kv_seen(const uint64_t* w, int32_t k) {
  if (k <= -32 || k >= JN_KV_TREE_ROWS) return 0;
  if (k < 0) return (uint32_t)w[0] << -k;
  const int i = k >> 6, s = k & 63;
  uint64_t v = w[i] >> s;
  if (s > 32 && i + 1 < JN_KV_TREE_ROWS / 64) v |= w[i + 1] << (64 - s);
  return (uint32_t)v;
}

// Values that are not finite in rows that only some query rows see: 0 * inf is NaN, so
// the products take them as zeros, and here they are added to the query rows that see
// them, whose probability p of the key is not zero. Keys t0 .. t1 - 1, a key after the
// other: such values are rare, and the products' loop stays free of them.
template <int HD, int NB, typename See>
__device__ __forceinline__ void kv_add_odd(const KvBatch& b, const KvCache& c, KvTable pages, int32_t h, int32_t t0,
                                           int32_t t1, const bf16x8 (&qf)[HD / 32][NB], const float (&m)[NB], float scale,
                                           f32x4 (&o)[HD / 16][NB], int lane, See&& sees) {
  const int quad = lane >> 4;
#pragma unroll 1
  for (int32_t t = t0; t < t1; ++t) {
    const int32_t g = pages[t >> c.page_log2];
    if ((uint32_t)g >= (uint32_t)c.n_pages) continue;
    const int64_t at = kv_at(c, g, h, t);
    bool bad = false;
    for (int e = lane; e < HD; e += 64) bad |= (c.v[at + e] & 0x7f80) == 0x7f80;
    if (!__any(bad)) continue;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float z = 0.f;
#pragma unroll
      for (int n = 0; n < HD / 32; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) z = fmaf((float)qf[n][nb][e], bf2f(c.k[at + n * 32 + quad * 8 + e]), z);
      z = sum_xor32(sum_xor16(z));
      const float p = sees(nb, t) ? __builtin_amdgcn_exp2f(fmaf(z, scale, -m[nb])) : 0.f;
#pragma unroll
      for (int x = 0; x < HD / 16; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint16_t v = c.v[at + x * 16 + quad * 4 + e];
          if ((v & 0x7f80) == 0x7f80 && p != 0.f) o[x][nb][e] = fmaf(p, bf2f(v), o[x][nb][e]);
        }
    }
  }
}
// v with zeros for its elements that are not finite, and whether there are any.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bool kv_finite(u32x4& v) {
  uint32_t any = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t odd = ((v[k] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;  // (no carry: 0x7fff + 0x80 < 2^16)
    any |= odd;
    v[k] &= ~((odd >> 15) * 0xffffu);
  }
  return any != 0;
}

// Chunk permutation of LDS row r for the products below: 16 rows read at one chunk (K)
// and 4 rows x 2 chunks a 16-lane group (V^T), where groups q and q ^ 1, and q and q ^ 2, are
// served together. attn_swz has that at head width 256; at 128 its rule is for 32 x 32
// products and puts rows r and r ^ 4 on one slot pair.
template <int HD>
__device__ __forceinline__ int kv_swz(int r) {
  const int q = (r >> 2) & 3, e = r & 3, pair = (q ^ (q >> 1)) & 1, low = q >> 1;
  if constexpr (HD == 32) return pair << 1 | low;
  if constexpr (HD == 64) return ((e >> 1) << 1 | pair) << 1 | low;
  return (e | pair << 2) << 1 | low;
}

// ---- few query rows (a unit has at most 16 NB) ----
// The time is the reading of keys and values, each read once: four wavefronts, each
// with 32 keys of a 128-key tile and all query rows. Keys go from the cache to
// registers in the layout that the product takes (16 keys a fragment: 16 bytes a
// lane of a row), values by DMA to the wavefront's own LDS tile, from which
// transposed reads make V^T; the next step's are in flight under each step, and
// nothing waits for another wavefront before the unit's end, where their O, m and l are
// added in LDS.
//   S^T = K Q^T, O^T += V^T P^T as in attn16_fwd_kernel.
// P is rounded to bf16 for its product, here and in kv_many_kernel (l sums it before that):
// results are 1.9e-3 to 2.3e-3 from 64 bits, relative, where rounding them alone gives 1.7e-3;
// P as two bf16 would double the second product.
// A key's page is the same for the 16 keys of a fragment (pages are multiples of 16),
// so page numbers are read once for all lanes, a step ahead. Values of places that no row
// sees are set to zero in LDS (0 * NaN is NaN).
// Bound by HBM: one token of 64 streams over 535,814 rows of 2 key heads of 128 takes
// 103 us, 5.3 TB/s. Few registers let two workgroups of head width 128 share a CU (128
// KB in flight); up to 32 query rows (16 at 256), beyond which O and Q leave room for one
// wavefront a SIMD and kv_many_kernel is faster (61 rows over 131,070 200 us here, 106 there).
template <int HD, int NB>
__global__ __launch_bounds__(256, HD == 256 ? 1 : 2) void kv_few_kernel(KvCache c, KvBatch b, KvAttn a, KvWork wk) {
  constexpr int R = 16 * NB, KT = 128;
  constexpr int NC = HD / 32, NT = HD / 16, CPR = HD / 8, RPI = 512 / HD;
  constexpr int NV = 32 / RPI, NK = 2 * NC;  // DMA instructions and key loads of a step
  constexpr int TG = NT < 4 ? NT : 4;        // V^T fragments read together
  constexpr int LD = HD + 4;
  __shared__ __attribute__((aligned(1024))) uint16_t vt[4][2][32 * HD];
  __shared__ KvTree tree;
  __shared__ float sm[4][R], sl[4][R];
  static_assert(4 * 16 * LD * 4 <= sizeof(vt), "the sums use the tiles' memory");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j16 = lane & 15, quad = lane >> 4;
  KvWalk<KT, 0> run;
  const bool any = run.start(b, c.kv, wk.group, wk.P, wk.least, lane);
  const int32_t p = run.p;
  if (tid < 2) wk.desc[2 * p + tid].wb = -1;
  if (!any) return;
  const int32_t G = wk.group;

  const int vrow = 4 * quad + (j16 >> 2), vswz = kv_swz<HD>(vrow);
  uint32_t vat[NT];  // the lane's transposed reads of the first tile
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int col = t * 16 + 4 * (j16 & 3);
    vat[t] = kv_lds(&vt[wave][0][vrow * HD + (((col >> 3) ^ vswz) * 8) + (col & 7)]);
  }
  const int drow = lane / CPR;  // of a DMA instruction
  int32_t doff[RPI >= 16 ? 1 : 16 / RPI];
#pragma unroll
  for (int v = 0; v < 16 / RPI; ++v) {
    const int r = v * RPI + drow;
    doff[v] = r * HD + (((lane % CPR) ^ kv_swz<HD>(r)) * 8);
  }
  const int32_t koff = j16 * HD + quad * 8;

  while (true) {
    const KvSeq sq = run.sq;
    const int32_t M = sq.n * G, kend = run.kend;
    const int32_t ta = wave_same((int32_t)(run.pos - run.unit0));
    const int32_t tb = wave_same((int32_t)min((int64_t)run.tiles, run.end - run.unit0));
    const KvTable pages = kv_table(b.pages) + (int64_t)wave_same(run.seq) * b.max_pages;
    const bool masks = tb * KT > sq.past;
    if (b.parents && masks) kv_tree<256>(tree, b, sq, 0, R);

    bf16x8 qf[NC][NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int32_t r = nb * 16 + j16, j = r / G;
      const uint16_t* const qr = a.q + (int64_t)(sq.row0 + (r < M ? j : 0)) * a.ldq +
                                 ((int64_t)run.h * G + (r < M ? r - j * G : 0)) * HD + quad * 8;
#pragma unroll
      for (int k = 0; k < NC; ++k) qf[k][nb] = *reinterpret_cast<const bf16x8*>(qr + k * 32);
    }
    f32x4 o[NT][NB];
    float m_run[NB], l_run[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m_run[nb] = -INFINITY;
      l_run[nb] = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t steps = tb - ta;
    // of a step: its keys' page numbers, read a step before they are needed, and their
    // heads' offsets
    struct Pages {
      int32_t page[2];
      int64_t at[2];
    };
    auto page_id = [&](int32_t i, int e) __attribute__((always_inline)) {
      return pages[min(((ta + i) * KT + wave * 32 + 16 * e) >> c.page_log2, b.max_pages - 1)];
    };
    auto pages_of = [&](int32_t i, int32_t id0, int32_t id1) __attribute__((always_inline)) {
      Pages x;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int32_t t = (ta + i) * KT + wave * 32 + 16 * e, id = e ? id1 : id0;
        x.page[e] = t < kend && (uint32_t)id < (uint32_t)c.n_pages ? id : -1;
        x.at[e] = x.page[e] >= 0 ? kv_at(c, x.page[e], run.h, t) : 0;
      }
      return x;
    };
    auto fetch_v = [&](const Pages& x, int stage) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int v = 0; v < 16 / RPI; ++v)
          kv_dma(c.v + x.at[e] + doff[v], &vt[wave][stage][e * 16 * HD + v * 512]);
    };
    bf16x8 kf[2][NC];
    auto fetch_k = [&](const Pages& x) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int n = 0; n < NC; ++n) kf[e][n] = *reinterpret_cast<const bf16x8*>(c.k + x.at[e] + koff + n * 32);
    };
    Pages use = pages_of(0, page_id(0, 0), page_id(0, 1)), next = use;
    int32_t id0 = page_id(1, 0), id1 = page_id(1, 1);
    bool odd = false;
    fetch_v(use, 0);
    fetch_k(use);
    for (int32_t i = 0; i < steps; ++i) {
      const int32_t t = (ta + i) * KT + wave * 32;
      const bool more = i + 1 < steps;
      const uint32_t stage = (i & 1) * (32 * HD * 2);
      if (more) {
        next = pages_of(i + 1, id0, id1);
        id0 = page_id(i + 2, 0);
        id1 = page_id(i + 2, 1);
        fetch_v(next, (i + 1) & 1);
      }
      f32x4 s[2][NB];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[e][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            s[e][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e][n], qf[n][nb], s[e][nb], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (more) fetch_k(next);  // into the registers that the product has read
      __builtin_amdgcn_sched_barrier(0);
      const bool hole = use.page[0] < 0 || use.page[1] < 0 || t + 32 > kend;  // places that no row sees
      const bool mask = t + 32 > sq.past;                                   // or not every row
      if (hole || mask) {
        const int l = here(lane), q4 = (l >> 4) * 4;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int32_t j = (nb * 16 + (l & 15)) / G;
          uint32_t bits = 0xffffffffu;  // of keys t .. t + 31
          if (mask && !b.whole) {
            const int32_t seen = sq.past + j + 1 - t;  // a chain's row sees keys below this
            bits = seen >= 32 ? 0xffffffffu : seen <= 0 ? 0u : (1u << seen) - 1;
            if (b.parents) {
              const int32_t old = sq.past - t;  // keys below this are cached rows
              bits = (old >= 32 ? 0xffffffffu : old <= 0 ? 0u : (1u << old) - 1) |
                     kv_seen(tree.seen[min(j, sq.n - 1)], t - sq.past);
            }
          }
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int32_t x = e * 16 + q4 + k;
              if (use.page[e] < 0 || t + x >= kend || !((bits >> x) & 1)) s[e][nb][k] = -INFINITY;
            }
        }
      }
      bf16x8 pf[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) top = fmaxf(top, s[e][nb][k]);
        top = max_xor32(max_xor16(top)) * a.scale_log2;
        if (__any(top > m_run[nb] + kRescale)) {
          const float m_new = fmaxf(m_run[nb], top);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[nb] - m_new);
          l_run[nb] *= alpha;
          m_run[nb] = m_new;
#pragma unroll
          for (int t2 = 0; t2 < NT; ++t2) o[t2][nb] *= alpha;
        }
        const float m = m_run[nb] == -INFINITY ? 0.f : m_run[nb];  // (a row that has seen nothing yet)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[e][nb][k], a.scale_log2, -m));
            l_run[nb] += x;
            pf[nb][4 * e + k] = (__bf16)x;
          }
      }
      if (more)
        kv_wait_vmcnt<NK + NV>();  // this step's values have landed; the next step's loads may be in flight
      else
        kv_wait_vmcnt<0>();
      if (hole || mask) {
        // rows of the tile that nobody sees become zeros, and, where not every query row sees
        // all of it, values that are not finite
        const int l = here(lane);
        const int32_t r = l >> 1;
        const bool none = (r < 16 ? use.page[0] : use.page[1]) < 0 || t + r >= kend;
        uint16_t* const row = &vt[wave][i & 1][r * HD + (l & 1) * (HD / 2)];
        bool bad = false;
#pragma unroll 1
        for (int e = 0; e < HD / 2; e += 8) {
          u32x4 v = *reinterpret_cast<const u32x4*>(row + e);
          if (mask) bad |= kv_finite(v);
          *reinterpret_cast<u32x4*>(row + e) = none ? u32x4{0, 0, 0, 0} : v;
        }
        odd |= __any(bad && !none);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
#pragma unroll
      for (int t0 = 0; t0 < NT; t0 += TG) {
        bf16x8 vf[TG];
        kv_read_v<HD>(vat + t0, stage, vf);
#pragma unroll
        for (int k = 0; k < TG; ++k)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            o[t0 + k][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[k], pf[nb], o[t0 + k][nb], 0, 0, 0);
      }
      use = next;
    }
    if (odd)
      for (int32_t i = 0; i < steps; ++i) {
        const int32_t t = (ta + i) * KT + wave * 32;
        if (t + 32 <= sq.past) continue;  // (as they are in the product: every row sees them)
        kv_add_odd<HD, NB>(b, c, pages, run.h, t, min(t + 32, kend), qf, m_run, a.scale_log2, o, here(lane), [&](int nb, int32_t x) {
          const int32_t j = (nb * 16 + (here(lane) & 15)) / G, k = x - sq.past;
          if (k < 0 || b.whole) return true;
          return b.parents ? (kv_seen(tree.seen[min(j, sq.n - 1)], k) & 1) != 0 : k <= j;
        });
      }

    // the wavefronts' results, added
    const int el = here(lane), ej = el & 15, eq = el >> 4, et = wave * 64 + el;
    const bool whole = ta == 0 && tb == run.tiles;
    const int slot = ta > 0 ? 0 : 1;
    if (!whole && tid == 0) {
      KvDesc d{run.seq, run.h, 0, run.holder(run.unit0), run.holder(run.unit0 + run.tiles - 1)};
      wk.desc[2 * p + slot] = d;
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float l = sum_xor32(sum_xor16(l_run[nb]));
      if (eq == 0) {
        sm[wave][nb * 16 + ej] = m_run[nb];
        sl[wave][nb * 16 + ej] = l;
      }
    }
    float* const sums = reinterpret_cast<float*>(&vt[0][0][0]);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb * 16 >= M) break;
      __syncthreads();  // m and l are there; the tiles, or the last rows' sums, are read
      const int r = nb * 16 + ej;
      const float top = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
      const float f = m_run[nb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[nb] - top);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        *reinterpret_cast<f32x4*>(&sums[(wave * 16 + ej) * LD + t * 16 + eq * 4]) = o[t][nb] * f;
      __syncthreads();
      for (int i = et; i < 16 * CPR; i += 256) {
        const int row = i / CPR, col = (i % CPR) * 8, rr = nb * 16 + row;
        if (rr >= M) break;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += sums[(w * 16 + row) * LD + col + e];
        const float mt = fmaxf(fmaxf(sm[0][rr], sm[1][rr]), fmaxf(sm[2][rr], sm[3][rr]));
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) l += sm[w][rr] == -INFINITY ? 0.f : sl[w][rr] * __builtin_amdgcn_exp2f(sm[w][rr] - mt);
        if (whole) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          uint4 x;
          x.x = pack_bf2(v[0] * inv, v[1] * inv);
          x.y = pack_bf2(v[2] * inv, v[3] * inv);
          x.z = pack_bf2(v[4] * inv, v[5] * inv);
          x.w = pack_bf2(v[6] * inv, v[7] * inv);
          const int32_t j = rr / G;
          *reinterpret_cast<uint4*>(a.out + (int64_t)(sq.row0 + j) * a.ldo + ((int64_t)run.h * G + rr - j * G) * HD + col) = x;
        } else {
          const int64_t at = (int64_t)(2 * p + slot) * R + rr;
          float4* const to = reinterpret_cast<float4*>(wk.o + at * HD + col);
          to[0] = make_float4(v[0], v[1], v[2], v[3]);
          to[1] = make_float4(v[4], v[5], v[6], v[7]);
          if (col == 0) wk.ml[at] = make_float2(mt, l);
        }
      }
    }
    run.pos = run.unit0 + tb;
    if (run.pos >= run.end) break;
    __syncthreads();  // the sums are read before the next unit's tiles overwrite them
    run.next(b, c.kv);
  }
}

// ---- many query rows ----
// W wavefronts of 16 NB rows each share tiles of 64 keys in LDS: the next tile's rows
// are loaded to registers a whole tile ahead and written to the other buffer as the
// current one is multiplied, one barrier a tile. LDS rows as in attn16_fwd_kernel
// (16-byte chunks permuted), and its products. Values of places that nobody sees are written
// as zeros, as are those of masked tiles that are not finite (kv_add_odd).
// 32 rows a wavefront (head width 256: 16, whose registers leave two wavefronts a SIMD;
// 32 there took twice as long), 128 rows a workgroup, which halves the LDS reads of a
// product against 16 rows; 64 rows where a unit has no more. Pieces of 2,048 rows behind 6,001 and of
// 1,792 behind 3,563, 16 query heads of 128: 286 us, 0.64 PFLOP/s (312 and 0.59 with the join), the matrix
// cores 30 % busy beside 200 other vector instructions a tile and wavefront; where all rows see each other
// 369 with the join, 0.58. 61 rows over 131,070 of 8 heads: 105 us, 5.1 TB/s.
template <int HD, int NB, int W>
__global__ __launch_bounds__(64 * W, 2) void kv_many_kernel(KvCache c, KvBatch b, KvAttn a, KvWork wk) {
  constexpr int R = 16 * NB * W, KT = 64, THREADS = 64 * W;
  constexpr int NC = HD / 32, NT = HD / 16, CPR = HD / 8;
  constexpr int NL = KT * CPR / THREADS;  // 16-byte loads of a thread for a tile of keys, and of values
  constexpr int RPL = THREADS / CPR;      // rows of one
  static_assert(NL * THREADS == KT * CPR && (64 / CPR <= 16 || CPR == 4), "a wavefront's load lies in 16 rows");
  __shared__ __attribute__((aligned(1024))) uint16_t kt[2][KT * HD], vt[2][KT * HD];
  __shared__ KvTree tree;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j16 = lane & 15, quad = lane >> 4;
  const int32_t G = wk.group;
  KvWalk<KT, R> run;
  const bool any = run.start(b, c.kv, G, wk.P, wk.least, lane);
  const int32_t p = run.p;
  if (tid < 2) wk.desc[2 * p + tid].wb = -1;
  if (!any) return;

  const int lrow = tid / CPR, lchunk = tid % CPR;
  const int kswz = kv_swz<HD>(j16);
  const int vrow = 4 * quad + (j16 >> 2), vswz = kv_swz<HD>(vrow);

  while (true) {
    const KvSeq sq = run.sq;
    const int64_t all = (int64_t)sq.n * G;
    const int32_t r0 = run.qt * R, M = (int32_t)min(all - r0, (int64_t)R);  // the unit's rows r0 .. r0 + M - 1
    const int32_t kend = run.kend;
    const int32_t ta = wave_same((int32_t)(run.pos - run.unit0));
    const int32_t tb = wave_same((int32_t)min((int64_t)run.tiles, run.end - run.unit0));
    const KvTable pages = kv_table(b.pages) + (int64_t)wave_same(run.seq) * b.max_pages;
    const int32_t jfirst = r0 / G;
    const int32_t rw = wave * 16 * NB;  // the wavefront's first row of the tile
    const bool active = rw < M;
    const int32_t jw = (r0 + rw) / G;   // and its place behind the cached rows, the lowest of its rows'
    bf16x8 qf[NC][NB];
    int32_t jr[NB];
    auto load_q = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int32_t r = min(rw + nb * 16 + j16, M - 1) + r0;
        jr[nb] = r / G;
        const uint16_t* const qr = a.q + (int64_t)(sq.row0 + jr[nb]) * a.ldq + ((int64_t)run.h * G + r - jr[nb] * G) * HD + quad * 8;
#pragma unroll
        for (int k = 0; k < NC; ++k) qf[k][nb] = *reinterpret_cast<const bf16x8*>(qr + k * 32);
      }
    };
    f32x4 o[NT][NB];
    float m_run[NB], l_run[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m_run[nb] = -INFINITY;
      l_run[nb] = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4 kr[NL], vr[NL];
    // of a tile: its four 16-key blocks' page numbers, read a tile before they are needed,
    // and as bits which blocks have one
    int32_t id[4];
    auto ids = [&](int32_t i) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) id[e] = pages[min(((ta + i) * KT + 16 * e) >> c.page_log2, b.max_pages - 1)];
    };
    uint32_t on[3] = {0, 0, 0};  // of the current tile and the next two
    bool odd = false;
    auto load = [&](int32_t i) __attribute__((always_inline)) {
      on[0] = on[1];
      on[1] = on[2];
      on[2] = 0;
      int64_t at[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int32_t t = (ta + i) * KT + 16 * e;
        const bool ok = t < kend && (uint32_t)id[e] < (uint32_t)c.n_pages;
        on[2] |= (uint32_t)ok << e;
        at[e] = ok ? kv_at(c, id[e], run.h, t) : 0;
      }
#pragma unroll
      for (int k = 0; k < NL; ++k) {
        int e = (k * RPL) >> 4;  // the wavefront's block of this load
        int64_t from = at[e & 3];
        if constexpr (RPL > 16) {
          const int w = wave * (64 / CPR) >> 4;
#pragma unroll
          for (int x = 1; x < RPL / 16; ++x) from = w == x ? at[(e + x) & 3] : from;
          e += w;
        }
        const int32_t off = ((k * RPL + lrow) & 15) * HD + lchunk * 8;
        kr[k] = *reinterpret_cast<const u32x4*>(c.k + from + off);
        vr[k] = *reinterpret_cast<const u32x4*>(c.v + from + off);
      }
    };
    // tile i, whose blocks `on` says, from the registers to its buffer
    auto store = [&](int32_t i, uint32_t has) __attribute__((always_inline)) {
      const int st = i & 1;
      const int32_t t = (ta + i) * KT;
      const bool edge = has != 0xfu || t + KT > kend, mask = t + KT > sq.past;
      if (edge || mask) {
#pragma unroll
        for (int k = 0; k < NL; ++k) {
          const int row = k * RPL + lrow;
          const bool none = !((has >> (row >> 4)) & 1) || t + row >= kend;
          const bool bad = mask && kv_finite(vr[k]);
          odd |= bad && !none;
          if (none) vr[k] = u32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int k = 0; k < NL; ++k) {
        const int row = k * RPL + lrow;
        const int at = row * HD + ((lchunk ^ kv_swz<HD>(row & 15)) * 8);
        *reinterpret_cast<u32x4*>(&kt[st][at]) = kr[k];
        *reinterpret_cast<u32x4*>(&vt[st][at]) = vr[k];
      }
    };
    const int32_t steps = tb - ta;
    ids(0);
    load(0);
    ids(1);
    load_q();  // (under the first tile's loads, as the tree's bits)
    if (b.parents && tb * KT > sq.past) kv_tree<THREADS>(tree, b, sq, jfirst, min(R, 128));
    store(0, on[2]);
    if (steps > 1) {
      load(1);
      ids(2);
    } else {
      on[1] = on[2];
    }
    __syncthreads();
    // on[1], on[2]: of tiles i and i + 1 at the top of step i
    for (int32_t i = 0; i < steps; ++i) {
      const uint32_t has = i + 1 < steps ? on[1] : (steps > 1 ? on[2] : on[1]);
      if (i + 1 < steps) store(i + 1, on[2]);
      if (i + 2 < steps) {
        load(i + 2);
        ids(i + 3);
      }
      const int32_t t = (ta + i) * KT;
      const bool mask = t + KT > sq.past;
      // (a chain's rows before all keys of the tile have nothing to do)
      if (active && (b.whole || b.parents || t <= sq.past + (r0 + min(rw + 16 * NB, M) - 1) / G)) {
        const uint16_t* const Ks = kt[i & 1];
        const uint16_t* const Vs = vt[i & 1];
        f32x4 s[4][NB];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) s[e][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        // (a chunk's fragments are read under the products of the chunk before)
        auto read_k = [&](int n, bf16x8 (&kf)[4]) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            kf[e] = *reinterpret_cast<const bf16x8*>(Ks + (e * 16 + j16) * HD + (((4 * n + quad) ^ kswz) * 8));
        };
        bf16x8 kf[2][4];
        read_k(0, kf[0]);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          if (n + 1 < NC) read_k(n + 1, kf[(n + 1) & 1]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              s[e][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n & 1][e], qf[n][nb], s[e][nb], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (mask || has != 0xfu || t + KT > kend) {
          const int q4 = (here(lane) >> 4) * 4;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            uint64_t bits = ~0ull;  // of keys t .. t + 63
            auto below = [](int32_t x) { return x >= 64 ? ~0ull : x <= 0 ? 0ull : (1ull << x) - 1; };
            if (mask && b.parents) {
              const uint64_t* const w = tree.seen[jr[nb] - jfirst];
              bits = below(sq.past - t) | kv_seen(w, t - sq.past) | (uint64_t)kv_seen(w, t + 32 - sq.past) << 32;
            } else if (mask && !b.whole) {
              bits = below(sq.past + jr[nb] + 1 - t);
            }
            bits &= below(kend - t);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (!((has >> e) & 1) || !((bits >> (e * 16 + q4 + k)) & 1)) s[e][nb][k] = -INFINITY;
          }
        }
        bf16x8 pf[2][NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float top = -INFINITY;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, s[e][nb][k]);
          top = max_xor32(max_xor16(top)) * a.scale_log2;
          if (__any(top > m_run[nb] + kRescale)) {
            const float m_new = fmaxf(m_run[nb], top);
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[nb] - m_new);
            l_run[nb] *= alpha;
            m_run[nb] = m_new;
#pragma unroll
            for (int t2 = 0; t2 < NT; ++t2) o[t2][nb] *= alpha;
          }
          const float m = m_run[nb] == -INFINITY ? 0.f : m_run[nb];  // (a row that has seen nothing yet)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float x = __builtin_amdgcn_exp2f(fmaf(s[e][nb][k], a.scale_log2, -m));
              l_run[nb] += x;
              pf[e >> 1][nb][4 * (e & 1) + k] = (__bf16)x;
            }
        }
        auto read_v = [&](int t2, int x) __attribute__((always_inline)) {
          const int col = t2 * 16 + 4 * (j16 & 3), r = x * 32 + vrow;
          const int at = (((col >> 3) ^ vswz) * 8) + (col & 7);
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4*)(Vs + r * HD + at));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4*)(Vs + (r + 16) * HD + at));
          return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        bf16x8 vf[2][2];
        vf[0][0] = read_v(0, 0);
        vf[0][1] = read_v(0, 1);
#pragma unroll
        for (int t2 = 0; t2 < NT; ++t2) {
          if (t2 + 1 < NT) {
            vf[(t2 + 1) & 1][0] = read_v(t2 + 1, 0);
            vf[(t2 + 1) & 1][1] = read_v(t2 + 1, 1);
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              o[t2][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[t2 & 1][x], pf[x][nb], o[t2][nb], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      __syncthreads();  // the tile is read, the next one written
    }
    if (__syncthreads_or(odd) && active)
      kv_add_odd<HD, NB>(b, c, pages, run.h, max(ta * KT, sq.past / KT * KT), min(tb * KT, kend), qf, m_run, a.scale_log2, o,
                         here(lane), [&](int nb, int32_t x) {
                           const int32_t k = x - sq.past;
                           if (k < 0 || b.whole) return true;
                           return b.parents ? (kv_seen(tree.seen[jr[nb] - jfirst], k) & 1) != 0 : k <= jr[nb];
                         });

    const bool whole = ta == 0 && tb == run.tiles;
    const int slot = ta > 0 ? 0 : 1;
    const int el = here(lane), ej = el & 15, eq = el >> 4;
    if (!whole && tid == 0) {
      KvDesc d{run.seq, run.h, run.qt, run.holder(run.unit0), run.holder(run.unit0 + run.tiles - 1)};
      wk.desc[2 * p + slot] = d;
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float l = sum_xor32(sum_xor16(l_run[nb]));
      const int32_t r = rw + nb * 16 + ej;
      if (whole) {
        // 16 bytes a lane after a lane swap, as in attn16_fwd_kernel
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint16_t* const to = a.out + (int64_t)(sq.row0 + jr[nb]) * a.ldo +
                             ((int64_t)run.h * G + r0 + r - jr[nb] * G) * HD + 16 * (eq & 1) + 8 * (eq >> 1);
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          const auto x = __builtin_amdgcn_permlane16_swap(pack_bf2(o[t][nb][0] * inv, o[t][nb][1] * inv),
                                                          pack_bf2(o[t + 1][nb][0] * inv, o[t + 1][nb][1] * inv), false, false);
          const auto y = __builtin_amdgcn_permlane16_swap(pack_bf2(o[t][nb][2] * inv, o[t][nb][3] * inv),
                                                          pack_bf2(o[t + 1][nb][2] * inv, o[t + 1][nb][3] * inv), false, false);
          if (r < M) *reinterpret_cast<uint4*>(to + t * 16) = make_uint4(x[0], y[0], x[1], y[1]);
        }
      } else if (r < M) {
        const int64_t at = (int64_t)(2 * p + slot) * R + r;
#pragma unroll
        for (int t = 0; t < NT; ++t)
          *reinterpret_cast<f32x4*>(wk.o + at * HD + t * 16 + eq * 4) = o[t][nb];
        if (eq == 0) wk.ml[at] = make_float2(m_run[nb], l);
      }
    }
    run.pos = run.unit0 + tb;
    if (run.pos >= run.end) break;
    run.next(b, c.kv);
  }
}

// Partial results of units that several workgroups hold: workgroup p adds rows of the
// units of its two slots, which all that took part in a unit share. A row is a
// wavefront's (HD / 4 lanes, and what lanes are left share the parts), of units in many parts the
// whole workgroup's (from 16 parts on). `rows`: of a slot. The parts come from other XCDs'
// workgroups, through memory: 64 streams 7 us, 26 MB of 8 trees 10.6.
template <int HD>
__global__ __launch_bounds__(256) void kv_join_kernel(KvBatch b, KvAttn a, KvWork wk, int32_t rows) {
  constexpr int LN = HD / 4, GR = 64 / LN;  // lanes of a row, groups that share the parts
  __shared__ float4 so[4][LN];
  __shared__ float sl[4];
  const int lane = threadIdx.x & 63, ln = lane % LN, gr = lane / LN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t p = blockIdx.x, G = wk.group;
  for (int slot = 0; slot < 2; ++slot) {
    const KvDesc d = wk.desc[2 * p + slot];
    if (d.wb < 0) continue;
    const KvSeq sq = kv_seq(b, d.seq);
    const int32_t parts = d.wb - d.wa + 1, M = (int32_t)min((int64_t)sq.n * G - (int64_t)d.qt * rows, (int64_t)rows);
    const bool all = parts >= kKvJoinMany;  // four wavefronts a row
    const int32_t share = gridDim.y * (all ? 1 : 4), first = blockIdx.y * (all ? 1 : 4) + (all ? 0 : wave);
    auto part = [&](int32_t k) { return (int64_t)(2 * (d.wa + k) + (k == 0 ? 1 : 0)) * rows; };
    for (int32_t r = (p - d.wa) * share + first; r < M; r += parts * share) {
      float top = -INFINITY;
      for (int32_t k = lane; k < parts; k += 64) top = fmaxf(top, wk.ml[part(k) + r].x);
      top = wave_max(top);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
      const int32_t step = all ? 4 * GR : GR;
#pragma unroll 8
      for (int32_t k = all ? wave * GR + gr : gr; k < parts; k += step) {
        const int64_t at = part(k) + r;
        const float2 ml = wk.ml[at];
        const float4 x = *reinterpret_cast<const float4*>(wk.o + at * HD + 4 * ln);
        const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
        l = fmaf(f, ml.y, l);
        v.x = fmaf(f, x.x, v.x);
        v.y = fmaf(f, x.y, v.y);
        v.z = fmaf(f, x.z, v.z);
        v.w = fmaf(f, x.w, v.w);
      }
#pragma unroll
      for (int e = LN; e < 64; e <<= 1) {
        v.x += __shfl_xor(v.x, e, kWave);
        v.y += __shfl_xor(v.y, e, kWave);
        v.z += __shfl_xor(v.z, e, kWave);
        v.w += __shfl_xor(v.w, e, kWave);
        l += __shfl_xor(l, e, kWave);
      }
      if (all) {
        __syncthreads();  // the last row's sums are read
        if (gr == 0) so[wave][ln] = v;
        if (lane == 0) sl[wave] = l;
        __syncthreads();
        if (wave > 0) continue;
#pragma unroll
        for (int k = 1; k < 4; ++k) {
          const float4 x = so[k][ln];
          v.x += x.x;
          v.y += x.y;
          v.z += x.z;
          v.w += x.w;
          l += sl[k];
        }
      }
      if (gr == 0) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int32_t rr = d.qt * rows + r, j = rr / G;
        *reinterpret_cast<uint2*>(a.out + (int64_t)(sq.row0 + j) * a.ldo + ((int64_t)d.h * G + rr - j * G) * HD + 4 * ln) =
            make_uint2(pack_bf2(v.x * inv, v.y * inv), pack_bf2(v.z * inv, v.w * inv));
      }
    }
    __syncthreads();  // so and sl are read
  }
}

// Query rows of a unit's tile, and workgroups: as many as are resident together, and no
// more than the batch can have tiles.
// (Tiles of a workgroup, where there are so many: with one tile of 64 keys each of 128
// rows leaves as much as partial results as it reads of keys and values. 8 trees of 25
// rows over 2,000 rows: 1, 2, 4, 8 tiles 40.4, 38.2, 40.4, 53 us. One row: 1 tile.)
constexpr int32_t kKvLeastMany = 2, kKvLeastFew = 1;
struct KvPlan {
  bool many;
  int32_t rows, P;
  size_t desc, ml, total;
};
static KvPlan kv_plan(const KvCache& c, const KvBatch& b, int32_t heads) {
  const int32_t G = heads / c.kv;
  const int64_t M = (int64_t)std::min(b.max_new, b.rows) * G;
  KvPlan k{};
  k.many = M > (c.hd == 256 ? 16 : 32);
  k.rows = M <= 16 ? 16 : M <= 32 && !k.many ? 32 : M <= 64 ? 64 : 128;
  const int32_t keys = k.many ? 64 : 128;
  const int64_t units = (int64_t)b.n_seqs * c.kv * ((M + k.rows - 1) / k.rows);
  const int64_t tiles = std::min<int64_t>(units * ((b.places + keys - 1) / keys), 1 << 20);
  const int64_t P = 256 * (c.hd == 256 ? 1 : 2);
  k.P = (int32_t)std::min((tiles + 7) / 8 * 8, P);
  k.desc = ((size_t)k.P * 2 * sizeof(KvDesc) + 255) / 256 * 256;
  k.ml = ((size_t)k.P * 2 * k.rows * sizeof(float2) + 255) / 256 * 256;
  k.total = k.desc + k.ml + (size_t)k.P * 2 * k.rows * c.hd * sizeof(float);
  return k;
}

size_t kv_attention_bytes(const KvCache& c, const KvBatch& b, int32_t heads) { return kv_plan(c, b, heads).total; }

hipError_t launch_kv_attention(hipStream_t s, const KvCache& c, const KvBatch& b, const KvAttn& a, void* ws) {
  const KvPlan k = kv_plan(c, b, a.heads);
  KvWork w{};
  w.desc = (KvDesc*)ws;
  w.ml = (float2*)((char*)ws + k.desc);
  w.o = (float*)((char*)ws + k.desc + k.ml);
  w.P = k.P;
  w.group = a.heads / c.kv;
  w.least = k.many ? kKvLeastMany : kKvLeastFew;
  auto rows = [&](auto hd) {
    constexpr int HD = decltype(hd)::value, NB = HD == 256 ? 1 : 2, W = HD == 256 ? 8 : 4;
    static_assert(16 * NB * W == 128, "rows of the largest tile");
    if (k.rows == 128)
      kv_many_kernel<HD, NB, W><<<k.P, 64 * W, 0, s>>>(c, b, a, w);
    else if (k.many)
      kv_many_kernel<HD, 1, 4><<<k.P, 256, 0, s>>>(c, b, a, w);
    else if (k.rows == 16)
      kv_few_kernel<HD, 1><<<k.P, 256, 0, s>>>(c, b, a, w);
    else if constexpr (HD < 256)
      kv_few_kernel<HD, 2><<<k.P, 256, 0, s>>>(c, b, a, w);
    kv_join_kernel<HD><<<dim3(k.P, (k.rows + 31) / 32), 256, 0, s>>>(b, a, w, k.rows);
    return hipGetLastError();
  };
  switch (c.hd) {
    case 32: return rows(std::integral_constant<int, 32>());
    case 64: return rows(std::integral_constant<int, 64>());
    case 128: return rows(std::integral_constant<int, 128>());
    case 256: return rows(std::integral_constant<int, 256>());
  }
  return hipErrorInvalidValue;
}

}  // namespace jnx
