// egmla_decode_q8.cu - split-KV decode over the ungated latent in 8 bits, on its codes as
// they are cached, for the latent widths 256 and 512.
//
// With the gate off nothing is done to a latent but the two products, so the tensor cores
// take the e4m3 codes themselves (tcgen05 kind::f8f6f4): no warp widens them, a page's
// latents fill half the shared memory they would as bf16, and a tile is a whole page also
// at width 512.  What meets them is in 8 bits too, split so that it keeps its precision:
//   queries   q^ 2^-k = q1 + q2 / 16 (k per head, the largest magnitude between 224 and 448;
//             q^ is bf16, whose eight significant bits two codes of four hold exactly down
//             to 2^-13 of the head's largest entry, and to 2^-22 of that below).  One product of N = 32 columns
//             (16 heads x 2 parts), summed by the softmax warps:
//               s_j = scale (2^e_j 2^k (S1 + S2 / 16) + q^R . k^R_j),  2^e_j token j's scale,
//             with a 2^k below 1 before 2^e_j (up to 2^119, the sums up to 2^27) and one above
//             behind it, so that no product is infinite where the score is not
//   weights   P'_j = 2^(s'_j - m + 11), s'_j = s_j log2(e) + e_j: the token's scale goes into
//             its weight, whose reference m is the largest s'.  P' = p1 + p2 / 8 + p3 / 64 in
//             e5m2, whose three significant bits reach far down: to half a step of nine bits
//             (2^-9, bf16's) for weights down to 2^-25 of the largest, four bits at 2^-30,
//             nothing below 2^-34.  (In e4m3 with p2 / 16 and p3 / 2^16 it was eight bits of
//             large weights and four of small ones: a head whose largest weight falls on
//             values that W_UV takes to zero was off by 2.5 %.)  N = 48 columns, added when
//             the output is read:  O^T += Z^T P'
//   l = sum_j P'_j 2^-e_j with the rounded P', so that the rounding cancels in O / l (with P'
//             itself below 2^-25 of the largest).
// The RoPE part stays bf16 (kind::f16) in columns of its own.
//
// 128 ragged sequences of 128 to 16K tokens (337 MB) at d_c 512: 76 us a call, 62 to 65 of them
// this kernel (5.2 to 5.4 TB/s, 77 to 80 % of the copy rate), with the codes widened to bf16 as
// for the gate 130, over a bf16 cache 113.  It is bound by the page copies: half the score and
// output MMAs left out, 75 (a fifth slot and two P' buffers instead of four: 78).  8 x 32K at
// d_c 256: 33.1 us (over bf16 35.4), where no unit is full.
//
// Roles as in egmla_decode_tc.cu, but for the gate warps: the softmax, here the longest of
// all roles, has two groups of four warps, eight heads each, which need nothing of one
// another; four query warps make each segment's query block from the absorbed bf16
// queries, and clear the rows behind a sequence's end in its last page (whose codes may be
// anything, NaN too).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "egmla_common.cuh"
#include "egmla_decode_tc.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"
#include "egmla_q8.cuh"

namespace egmla {

namespace {

constexpr int kPlainThreads = 512;
constexpr int kGroupHeads = 8;                       // heads of a softmax group
constexpr int kSoft2Warp0 = 8;                       // warps 8-11: the second group (a warp reads the TMEM lanes of warp % 4)
constexpr int kQueryWarp0 = 12, kQueryWarps = 4;
constexpr int kQParts = 2, kPParts = 3;
constexpr float kQPart2 = 1.f / 16, kPPart2 = 1.f / 8, kPPart3 = 1.f / 64;
// weights of at most 2^(11 + 4): below e5m2's 57344, and as far above its smallest numbers
// as that allows; what a partial result holds is 2^-11 of its sums over them (l with 2^100
// for latents of zero would come near fp32's end)
constexpr float kWeightLog2 = 11.f, kPlainLazy = 4.f, kWeightUnit = 1.f / 2048;

template <int D_C>
struct PlainCfg {
  static constexpr int NCH = D_C / 128;                 // 128-feature swizzle-atom columns
  static constexpr uint32_t PCHUNK = kPage * 128;       // one of a page; also the RoPE keys
  static constexpr uint32_t KR_OFF = NCH * PCHUNK;
  static constexpr uint32_t SLOT = KR_OFF + PCHUNK;
  static constexpr uint32_t META = kPage * 4;           // the page's scales
  // query block: codes [n = 16 part + head][feature] in 8 x 16-byte core matrices, 16
  // features a K core of 512 bytes; q^R as the absorption wrote it; per head 2^min(k, 0) and
  // scale_log2 2^max(k, 0)
  static constexpr uint32_t QCORE = kQParts * kHeads * 16;
  static constexpr uint32_t Q_ROPE = D_C / 16 * QCORE;
  static constexpr uint32_t Q_SCALE = Q_ROPE + qprep_rope_bytes(kRope);
  static constexpr uint32_t QBUF = Q_SCALE + 128;
  // P' [n = 16 part + head][token], MN-major: 16 n x 8 tokens of 128 bytes
  static constexpr uint32_t PGROUP = kPParts * 128;     // eight tokens
  static constexpr uint32_t PBUF = kPage / 8 * PGROUP;
  static constexpr uint32_t XCH = 1024, MISC = 512;
  static constexpr uint32_t FIXED = QBUF + kNP * PBUF + XCH + MISC + 1024;
  static constexpr int NS_FIT = (int)((kSmemLimit - FIXED) / (SLOT + META));
  static constexpr int NS = NS_FIT > 6 ? 6 : NS_FIT;
  static constexpr uint32_t OFF_QBUF = NS * SLOT;
  static constexpr uint32_t OFF_PBUF = OFF_QBUF + QBUF;
  static constexpr uint32_t OFF_META = OFF_PBUF + kNP * PBUF;
  static constexpr uint32_t OFF_XCH = OFF_META + NS * META;
  static constexpr uint32_t OFF_MISC = OFF_XCH + XCH;
  static constexpr uint32_t SMEM = OFF_MISC + MISC + 1024;
  // TMEM: kNB score buffers of 32 latent and 16 RoPE columns, then O^T, 48 columns per
  // chunk of 128 features
  static constexpr int NMC = D_C / 128;
  static constexpr uint32_t S_ROPE = kQParts * kHeads, S_COLS = S_ROPE + kHeads;
  static constexpr uint32_t O_COLS = kPParts * kHeads;
  static constexpr uint32_t COL_S = 0, COL_O = kNB * S_COLS;
  static constexpr uint32_t TMEM_COLS = 512;
  static_assert(NS >= 3 && SMEM <= kSmemLimit && COL_O + NMC * O_COLS <= TMEM_COLS, "fits");
  static_assert(QBUF % 128 == 0 && PBUF % 128 == 0 && Q_ROPE % 16 == 0, "operands");
};

// the barriers in MISC
struct PlainBars : Bars {
  uint64_t zfix;   // the rows behind a sequence's end are cleared, once for every such page
};
static_assert(sizeof(PlainBars) <= 512, "barriers");

// kind::f8f6f4 with e4m3 A, e4m3 or e5m2 B, fp32 D
__host__ __device__ constexpr uint32_t idesc_f8(int M, int N, int a_mn, int b_mn, bool b_e5m2) {
  return (idesc_bf16(M, N, a_mn, b_mn) & ~((7u << 7) | (7u << 10))) | (b_e5m2 ? 1u << 10 : 0u);
}
__device__ __forceinline__ void mma_f8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// 32 lanes x 8 columns: thread i of the warp gets (or writes) its lane's 8 values
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
               "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
               "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
               : "memory");
}

// two codes as fp32 values
__device__ __forceinline__ float2 decode2(uint32_t c, __nv_fp8_interpretation_t type) {
  return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(c), type)));
}
// two values as e5m2 codes, the first in the low byte
__device__ __forceinline__ uint32_t encode2_e5m2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E5M2);
}

template <int D_C>
__global__ void __launch_bounds__(kPlainThreads, 1)
    decode_plain_q8_kernel(const __grid_constant__ CUtensorMap cmap, const __grid_constant__ CUtensorMap krmap,
                           const TcParams p) {
  using C = PlainCfg<D_C>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  PlainBars& bars = *reinterpret_cast<PlainBars*>(smem + C::OFF_MISC);
  volatile int* abort_flag = &bars.abort;
  const uint64_t wait_ns = p.wait_ns;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::NS; ++s) {
      mbar_init(smem_u32(&bars.full[s]), 1);
      // the page's output MMAs (commit) and the query warps, which look at every page
      mbar_init(smem_u32(&bars.empty[s]), 1 + kQueryWarps);
    }
    mbar_init(smem_u32(&bars.qfull[0]), kQueryWarps);
    // the last score MMA of the segment (commit) and the softmax warps' read of its scales
    mbar_init(smem_u32(&bars.qempty[0]), 1 + 2 * kSoftWarps);
    for (int s = 0; s < kNB; ++s) {
      mbar_init(smem_u32(&bars.sready[s]), 1);
      mbar_init(smem_u32(&bars.sfree[s]), 2 * kSoftWarps);
    }
    for (int s = 0; s < kNP; ++s) {
      mbar_init(smem_u32(&bars.spdone[s]), 2 * kSoftWarps);
      mbar_init(smem_u32(&bars.pfree[s]), 1);
    }
    mbar_init(smem_u32(&bars.zfix), kQueryWarps);
    mbar_init(smem_u32(&bars.drain_s), 1);
    mbar_init(smem_u32(&bars.drain_o), 1);
    bars.abort = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(&bars.tmem_base), C::TMEM_COLS);
    tmem_relinquish();
  }
  if (warp == kTmaWarp && lane == 0) {
    prefetch_tensormap(&cmap);
    prefetch_tensormap(&krmap);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem_base;
  grid_dependency_wait();

  if (warp == kTmaWarp) {
    // ---------------------------------------------------------------- TMA producer
    const uint64_t pol_stream = policy_evict_first();
    Walker<kPage> w;
    w.start(p);
    PageWindow pw;
    pw.init(p, lane);
    Tile t;
    int it = 0;
    int last_it[6] = {-1, -1, -1, -1, -1, -1};
    bool ok_loop = true;
    while (ok_loop && w.next(t)) {
      const int pg = pw.page(p, t, lane);
      const int slot = it % C::NS;
      if (lane == 0) {
        if (!mbar_wait(smem_u32(&bars.empty[slot]), ((it / C::NS) & 1) ^ 1, abort_flag, wait_ns)) ok_loop = false;
        if (ok_loop) {
          const bool ok = pg >= 0 && pg < p.num_pages;
          if (!ok) report_status(p.status, kStatusOutOfRange);
          // (test entry) a withheld page: no copy and no arrival
          const bool withheld = static_cast<int>(blockIdx.x) == p.stall_cta && it == p.stall_tile;
          if (!withheld) {
            const uint32_t fb = smem_u32(&bars.full[slot]);
            mbar_arrive_expect_tx(fb, ok ? C::SLOT + C::META : 0u);
            if (ok) {
              const uint32_t dst = sbase + slot * C::SLOT;
              tma_load_3d(dst, &cmap, 0, pg * kPage, 0, fb, pol_stream);
              tma_load_3d(dst + C::KR_OFF, &krmap, 0, pg * kPage, 0, fb, pol_stream);
              bulk_load_hint(sbase + C::OFF_META + slot * C::META, p.scales + static_cast<size_t>(pg) * kPage, C::META, fb,
                             pol_stream);
            }
            last_it[slot] = it;
          }
        }
      }
      // the first page alone, as in egmla_decode_tc.cu
      if (it == 0 && lane == 0 && ok_loop && last_it[0] == 0 &&
          !mbar_wait(smem_u32(&bars.full[0]), 0, abort_flag, wait_ns))
        ok_loop = false;
      ok_loop = __shfl_sync(0xffffffffu, ok_loop, 0);
      ++it;
    }
    if (lane == 0) {
      if (!p.fuse) grid_launch_dependents();
      volatile int own = 0;
      for (int s = 0; s < C::NS; ++s)
        if (last_it[s] >= 0 && !mbar_wait(smem_u32(&bars.full[s]), (last_it[s] / C::NS) & 1, &own, wait_ns)) *abort_flag = 1;
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- score MMAs
    if (elect_one()) {
      constexpr uint32_t IDESC_S = idesc_f8(64, kQParts * kHeads, 0, 0, false), IDESC_R = idesc_bf16(64, kHeads, 0, 0);
      const uint64_t zdesc = smem_desc(sbase, 16, 1024, kSwizzle128B);
      const uint64_t qdesc = smem_desc(sbase + C::OFF_QBUF, C::QCORE, 128, kSwizzleNone);
      const uint64_t rdesc = smem_desc(sbase + C::OFF_QBUF + C::Q_ROPE, kQGroupBytes, kQRowGroupBytes, kSwizzleNone);
      Walker<kPage> w;
      w.start(p);
      Tile t;
      int seg = -1, fixed = 0;
      bool issued = false;
      for (int js = 0; w.next(t); ++js) {
        const int slot = js % C::NS, sb = js % kNB;
        bool ok = true;
        if (t.first) {
          ++seg;
          ok = mbar_wait(smem_u32(&bars.qfull[0]), seg & 1, abort_flag, wait_ns);
        }
        ok = ok && mbar_wait(smem_u32(&bars.sfree[sb]), ((js / kNB) & 1) ^ 1, abort_flag, wait_ns);
        ok = ok && mbar_wait(smem_u32(&bars.full[slot]), (js / C::NS) & 1, abort_flag, wait_ns);
        if (t.ntok < kPage) ok = ok && mbar_wait(smem_u32(&bars.zfix), fixed++ & 1, abort_flag, wait_ns);
        if (!ok) break;
        tc_fence_after();
        const uint64_t za = zdesc + ((slot * C::SLOT) >> 4);
        const uint32_t ds = tmem + C::COL_S + sb * C::S_COLS;
#pragma unroll
        for (int kk = 0; kk < D_C / 32; ++kk)
          mma_f8_ss(ds, za + (((kk >> 2) * C::PCHUNK + (kk & 3) * 32) >> 4), qdesc + ((kk * 2 * C::QCORE) >> 4), IDESC_S,
                      kk > 0);
#pragma unroll
        for (int kk = 0; kk < kRope / 16; ++kk)
          mma_bf16_ss(ds + C::S_ROPE, za + ((C::KR_OFF + kk * 32) >> 4), rdesc + ((kk * 2 * kQGroupBytes) >> 4), IDESC_R,
                      kk > 0);
        mma_commit(smem_u32(&bars.sready[sb]));
        if (t.last) mma_commit(smem_u32(&bars.qempty[0]));
        issued = true;
      }
      if (issued) {
        volatile int own = 0;
        mma_commit(smem_u32(&bars.drain_s));
        if (!mbar_wait(smem_u32(&bars.drain_s), 0, &own, wait_ns)) *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp == kOutWarp) {
    // ---------------------------------------------------------------- output MMAs
    // A: the page's codes read MN-major (128 features of a column along M, eight tokens
    // 1 KB apart along K); B: P' MN-major.
    if (elect_one()) {
      constexpr uint32_t IDESC_O = idesc_f8(128, kPParts * kHeads, 1, 1, true);
      const uint64_t zdesc = smem_desc(sbase, C::PCHUNK, 1024, kSwizzle128B);
      const uint64_t pdesc = smem_desc(sbase + C::OFF_PBUF, C::PGROUP, 128, kSwizzleNone);
      Walker<kPage> w;
      w.start(p);
      Tile t;
      bool issued = false;
      for (int jo = 0; w.next(t); ++jo) {
        if (!mbar_wait(smem_u32(&bars.spdone[jo % kNP]), (jo / kNP) & 1, abort_flag, wait_ns)) break;
        tc_fence_after();
        const int slot = jo % C::NS;
        const uint64_t za = zdesc + ((slot * C::SLOT) >> 4), pb = pdesc + (((jo % kNP) * C::PBUF) >> 4);
        const uint32_t keep = t.first ? 0u : 1u;   // a segment's first MMAs overwrite O^T
#pragma unroll
        for (int ks = 0; ks < kPage / 32; ++ks)
#pragma unroll
          for (int mc = 0; mc < C::NMC; ++mc)
            mma_f8_ss(tmem + C::COL_O + C::O_COLS * mc, za + ((mc * C::PCHUNK + ks * 4096) >> 4),
                        pb + ((ks * 4 * C::PGROUP) >> 4), IDESC_O, ks > 0 ? 1u : keep);
        mma_commit(smem_u32(&bars.empty[slot]));
        mma_commit(smem_u32(&bars.pfree[jo % kNP]));
        issued = true;
      }
      if (issued) {
        volatile int own = 0;
        mma_commit(smem_u32(&bars.drain_o));
        if (!mbar_wait(smem_u32(&bars.drain_o), 0, &own, wait_ns)) *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp >= kQueryWarp0) {
    // ---------------------------------------------------------------- query blocks, rows behind the end
    // Warp w has heads 4w .. 4w + 3, eight lanes each; a lane every eighth block of 16
    // features of its head.
    constexpr int LANES = 32 * kQueryWarps / kHeads, BLOCKS = D_C / 16 / LANES;
    const int tid = (warp - kQueryWarp0) * 32 + lane;
    const int h = tid / LANES, l16 = tid % LANES;
    uint8_t* qb = smem + C::OFF_QBUF;
    Walker<kPage> w;
    w.start(p);
    Tile t;
    int seg = -1;
    for (int j = 0; w.next(t); ++j) {
      if (t.first) {
        ++seg;
        const uint8_t* src = p.qprep + static_cast<size_t>(t.b) * qprep_bytes_tc(D_C, kRope);
        uint4 raw[BLOCKS][2];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            raw[i][e] = __ldcg(reinterpret_cast<const uint4*>(src + qlat_offset(h, 16 * (l16 + LANES * i) + 8 * e, D_C)));
        static_assert(qprep_rope_bytes(kRope) == 16 * 32 * kQueryWarps, "a unit of q^R per thread");
        const uint4 rope = __ldcg(reinterpret_cast<const uint4*>(src + qprep_lat_bytes(D_C)) + tid);
        // the head's largest magnitude (two bf16 values at once: their bits order them)
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t v[4] = {raw[i][e].x, raw[i][e].y, raw[i][e].z, raw[i][e].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) most = max(most, max(v[k] << 16 & 0x7fff0000u, v[k] & 0x7fff0000u));
          }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        float scale, inverse;
        q8_scale(most, scale, inverse, -126);   // (queries of 2^-118 and less lose bits; their scores need latents of 2^110)
        // the block is free once the segment before has read it
        if (!warp_wait(smem_u32(&bars.qempty[0]), (seg & 1) ^ 1, abort_flag, wait_ns)) break;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          uint32_t part[kQParts][4];
#pragma unroll
          for (int k = 0; k < 8; ++k) {   // pairs
            const uint4& r4 = raw[i][k / 4];
            const uint32_t v = k % 4 == 0 ? r4.x : k % 4 == 1 ? r4.y : k % 4 == 2 ? r4.z : r4.w;
            const float2 x = unpack_bf16x2(v);
            const float x0 = x.x * inverse, x1 = x.y * inverse;
            const uint32_t c1 = q8_encode2(x0, x1);
            const float2 d = decode2(c1, __NV_E4M3);
            const uint32_t c2 = q8_encode2((x0 - d.x) * 16.f, (x1 - d.y) * 16.f);
            if (k % 2 == 0) {
              part[0][k / 2] = c1;
              part[1][k / 2] = c2;
            } else {
              part[0][k / 2] |= c1 << 16;
              part[1][k / 2] |= c2 << 16;
            }
          }
#pragma unroll
          for (int n = 0; n < kQParts; ++n)
            *reinterpret_cast<uint4*>(qb + (l16 + LANES * i) * C::QCORE + (2 * n + h / 8) * 128 + (h % 8) * 16) =
                make_uint4(part[n][0], part[n][1], part[n][2], part[n][3]);
        }
        reinterpret_cast<uint4*>(qb + C::Q_ROPE)[tid] = rope;
        if (l16 == 0) {
          float* hs = reinterpret_cast<float*>(qb + C::Q_SCALE);
          hs[h] = fminf(scale, 1.f);   // (a NaN is in the codes)
          hs[kHeads + h] = p.scale_log2 * fmaxf(scale, 1.f);
        }
        fence_proxy_async_smem();
        warp_arrive(smem_u32(&bars.qfull[0]));
      }
      // (every page is waited for and its slot given back, so that no phase of a slot's
      // barrier is taken for another)
      const int slot = j % C::NS;
      if (!warp_wait(smem_u32(&bars.full[slot]), (j / C::NS) & 1, abort_flag, wait_ns)) break;
      if (t.ntok < kPage) {
        for (int i = tid; i < (kPage - t.ntok) * 8; i += 32 * kQueryWarps)
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc)
            *reinterpret_cast<uint4*>(smem + slot * C::SLOT + fc * C::PCHUNK + (t.ntok + i / 8) * 128 + i % 8 * 16) =
                make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
        warp_arrive(smem_u32(&bars.zfix));
      }
      warp_arrive(smem_u32(&bars.empty[slot]));
    }
  } else if (warp < kSoftWarps || warp >= kSoft2Warp0) {
    // ---------------------------------------------------------------- softmax, output read-out
    // Group g has heads 8g .. 8g + 7; its warp w reads TMEM lane quadrant w: tokens 16w ..
    // 16w + 15 of a tile's scores, latent features 32w .. 32w + 31 of each 128-feature
    // chunk of O^T.  Thread t owns tokens r0 = 16w + t / 4 and r1 = r0 + 8 and heads 8g + 2q,
    // 8g + 2q + 1 (q = t % 4).  Lane i < 8 of every warp also keeps the reference of head 8g + i.
    const int g = warp >= kSoft2Warp0, quad = warp & 3, q = lane & 3;
    const int r0 = 16 * quad + (lane >> 2), r1 = r0 + 8;
    const int bar_tile = 1 + 2 * g, bar_xch = 2 + 2 * g;
    const uint32_t tq = tmem + (static_cast<uint32_t>(32 * quad) << 16);
    const float scale = p.scale_log2;
    float* xmax = reinterpret_cast<float*>(smem + C::OFF_XCH) + g * 64;   // [4 warps][8 heads]
    float* xsum = xmax + kSoftWarps * kGroupHeads;                        // [4 warps][8 heads]
    float m_ref[2], l_acc[2], qlow[2], qs[2];
    float m8 = -INFINITY;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      m_ref[k] = -INFINITY;
      l_acc[k] = 0.f;
      qlow[k] = 0.f;
      qs[k] = 0.f;
    }
    Walker<kPage> w;
    w.start(p);
    Tile t;
    int it = 0, seg = -1;
    while (w.next(t)) {
      const int slot = it % C::NS, sb = it % kNB, pb = it % kNP;
      bool ok = true;
      if (t.first) {
        ++seg;
        ok = warp_wait(smem_u32(&bars.qfull[0]), seg & 1, abort_flag, wait_ns);
        if (ok) {
          const float* hs = reinterpret_cast<const float*>(smem + C::OFF_QBUF + C::Q_SCALE) + kGroupHeads * g + 2 * q;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            qlow[k] = hs[k];
            qs[k] = hs[kHeads + k];
          }
          warp_arrive(smem_u32(&bars.qempty[0]));
        }
      }
      // the tokens' scales came with the page, long before its scores
      float ts[2] = {1.f, 1.f};
      ok = ok && warp_wait(smem_u32(&bars.full[slot]), (it / C::NS) & 1, abort_flag, wait_ns);
      if (ok) {
        const float* sc = reinterpret_cast<const float*>(smem + C::OFF_META + slot * C::META);
        if (r0 < t.ntok) ts[0] = sc[r0];   // (what lies behind the end is of no account)
        if (r1 < t.ntok) ts[1] = sc[r1];
      }
      ok = ok && warp_wait(smem_u32(&bars.sready[sb]), (it / kNB) & 1, abort_flag, wait_ns);
      float s[2][2];
      bool exceed = false;
      if (ok) {
        float v1[4], v2[4], vr[4];
        tc_fence_after();
        const uint32_t ds = tq + C::COL_S + sb * C::S_COLS + kGroupHeads * g;
        tmem_ld_16x256b_x1(ds, v1);
        tmem_ld_16x256b_x1(ds + kHeads, v2);
        tmem_ld_16x256b_x1(ds + C::S_ROPE, vr);
        tmem_wait_ld();
        tc_fence_before();
        warp_arrive(smem_u32(&bars.sfree[sb]));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool valid = (e ? r1 : r0) < t.ntok;
          const float lift = static_cast<float>(static_cast<int>(__float_as_uint(ts[e]) >> 23) - 127);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int i = 2 * e + k;
            const float lat = fmaf(v2[i], kQPart2, v1[i]) * qlow[k] * ts[e];
            const float x = fmaf(lat, qs[k], fmaf(vr[i], scale, lift));
            s[e][k] = valid ? x : -INFINITY;
            exceed = exceed || (x > m_ref[k] + kPlainLazy && valid);
          }
        }
      }
      if (soft_vote(bar_tile, exceed || !ok)) {
        if (soft_vote(bar_tile, !ok)) break;   // uniform: every warp of the group leaves
        // ---- slow path: tile maxima of the heads over the 64 tokens
        float tm[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) tm[k] = fmaxf(s[0][k], s[1][k]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
          for (int k = 0; k < 2; ++k) tm[k] = fmaxf(tm[k], __shfl_xor_sync(0xffffffffu, tm[k], o));
        if (lane < 4) {
#pragma unroll
          for (int k = 0; k < 2; ++k) xmax[quad * kGroupHeads + 2 * q + k] = tm[k];
        }
        soft_sync(bar_xch);
        float alpha = 1.f;
        if (lane < kGroupHeads) {
          const float tmax = fmaxf(fmaxf(xmax[lane], xmax[kGroupHeads + lane]),
                                   fmaxf(xmax[2 * kGroupHeads + lane], xmax[3 * kGroupHeads + lane]));
          if (m8 == -INFINITY) {
            m8 = tmax;
            alpha = 0.f;
          } else if (tmax > m8 + kPlainLazy) {
            alpha = ex2_approx(m8 - tmax);
            m8 = tmax;
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) m_ref[k] = __shfl_sync(0xffffffffu, m8, 2 * q + k);
        if (!t.first && __any_sync(0xffffffffu, lane < kGroupHeads && alpha != 1.f)) {
          // what was accumulated against the old reference, after the tile before
          const int pv = (it - 1) % kNP;
          ok = warp_wait(smem_u32(&bars.pfree[pv]), ((it - 1) / kNP) & 1, abort_flag, wait_ns);
          if (ok) {
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < kPParts * C::NMC; ++c) {
              float o[8];
              tmem_ld8(tq + C::COL_O + kHeads * c + kGroupHeads * g, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < kGroupHeads; ++i) o[i] *= __shfl_sync(0xffffffffu, alpha, i);
              tmem_st8(tq + C::COL_O + kHeads * c + kGroupHeads * g, o);
            }
            tmem_wait_st();
#pragma unroll
            for (int k = 0; k < 2; ++k) l_acc[k] *= __shfl_sync(0xffffffffu, alpha, 2 * q + k);
          }
        }
      }
      // the P' buffer of this tile is free once the output MMA kNP tiles back has read it
      ok = ok && warp_wait(smem_u32(&bars.pfree[pb]), ((it / kNP) & 1) ^ 1, abort_flag, wait_ns);
      if (ok) {
        uint8_t* pbuf = smem + C::OFF_PBUF + pb * C::PBUF;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = e ? r1 : r0;
          uint8_t* prow = pbuf + (r >> 3) * C::PGROUP + (r & 7) * 16 + kGroupHeads * g + 2 * q;
          // 2^-e of the token's scale (NaN: NaN)
          const float lower = ts[e] != ts[e] ? ts[e] : __uint_as_float((254u << 23) - __float_as_uint(ts[e]));
          const float p0 = ex2_approx(s[e][0] - (m_ref[0] - kWeightLog2));
          const float p1 = ex2_approx(s[e][1] - (m_ref[1] - kWeightLog2));
          const uint32_t c1 = encode2_e5m2(p0, p1);
          const float2 d1 = decode2(c1, __NV_E5M2);
          const float g0 = p0 - d1.x, g1 = p1 - d1.y;
          const uint32_t c2 = encode2_e5m2(g0 * (1.f / kPPart2), g1 * (1.f / kPPart2));
          const float2 d2 = decode2(c2, __NV_E5M2);
          const uint32_t c3 = encode2_e5m2(fmaf(d2.x, -kPPart2, g0) * (1.f / kPPart3), fmaf(d2.y, -kPPart2, g1) * (1.f / kPPart3));
          const float2 d3 = decode2(c3, __NV_E5M2);
          constexpr float u1 = kWeightUnit, u2 = kWeightUnit * kPPart2, u3 = kWeightUnit * kPPart3;
          // (a weight below the codes' nine bits counts in l as it is: a latent of zero has 2^-100
          // in P' and may have as much of l as any other)
          constexpr float kLeast = 1.f / 16384;
          const float t0 = p0 < kLeast ? p0 * u1 : fmaf(d3.x, u3, fmaf(d2.x, u2, d1.x * u1));
          const float t1 = p1 < kLeast ? p1 * u1 : fmaf(d3.y, u3, fmaf(d2.y, u2, d1.y * u1));
          l_acc[0] = fmaf(t0, lower, l_acc[0]);
          l_acc[1] = fmaf(t1, lower, l_acc[1]);
          *reinterpret_cast<uint16_t*>(prow) = static_cast<uint16_t>(c1);
          *reinterpret_cast<uint16_t*>(prow + 128) = static_cast<uint16_t>(c2);
          *reinterpret_cast<uint16_t*>(prow + 256) = static_cast<uint16_t>(c3);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        warp_arrive(smem_u32(&bars.spdone[pb]));
      }

      if (t.last) {
        // ---- segment end: l of every head over the 64 token rows, then O^T
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
          for (int k = 0; k < 2; ++k) l_acc[k] += __shfl_xor_sync(0xffffffffu, l_acc[k], o);
        if (lane < 4) {
#pragma unroll
          for (int k = 0; k < 2; ++k) xsum[quad * kGroupHeads + 2 * q + k] = l_acc[k];
        }
        if (soft_vote(bar_xch, !ok)) break;   // uniform
        ok = warp_wait(smem_u32(&bars.pfree[pb]), (it / kNP) & 1, abort_flag, wait_ns);
        if (ok) {
          tc_fence_after();
          const int slot_out = blockIdx.x + t.b;
          float* po = p.part_o + (static_cast<size_t>(slot_out) * kHeads + kGroupHeads * g) * D_C;
#pragma unroll
          for (int mc = 0; mc < C::NMC; ++mc) {
            float o[kPParts][8];
#pragma unroll
            for (int n = 0; n < kPParts; ++n) tmem_ld8(tq + C::COL_O + C::O_COLS * mc + kHeads * n + kGroupHeads * g, o[n]);
            tmem_wait_ld();
            const int f = 128 * mc + 32 * quad + lane;
#pragma unroll
            for (int i = 0; i < kGroupHeads; ++i)
              po[i * D_C + f] = kWeightUnit * fmaf(o[2][i], kPPart3, fmaf(o[1][i], kPPart2, o[0][i]));
          }
          tc_fence_before();
          if (quad == 0 && lane < kGroupHeads) {
            float lh = 0.f;
#pragma unroll
            for (int ww = 0; ww < kSoftWarps; ++ww) lh += xsum[ww * kGroupHeads + lane];
            float* ml = p.part_ml + (static_cast<size_t>(slot_out) * kHeads + kGroupHeads * g + lane) * 2;
            ml[0] = m8;
            ml[1] = lh;
          }
          if (p.fuse) {
            __syncwarp();
            if (lane == 0) {
              __threadfence();
              atomicAdd(p.seq_done + t.b, 1u);
            }
          }
        }
        m8 = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          m_ref[k] = -INFINITY;
          l_acc[k] = 0.f;
        }
      }
      ++it;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, C::TMEM_COLS);
  if (threadIdx.x == 0 && bars.abort) report_status(p.status, kStatusTimeout);
  if constexpr (D_C <= 256) {
    if (p.fuse) fused_combine<D_C, false, 2 * kSoftWarps>(p, smem, bars);
  }
}

template <int D_C>
cudaError_t launch_plain(const DecodeArgs& a, const CUtensorMap* maps, cudaStream_t st, bool* fused) {
  using C = PlainCfg<D_C>;
  auto kern = decode_plain_q8_kernel<D_C>;
  const cudaError_t e = allow_smem(kern, C::SMEM);
  if (e != cudaSuccess) return e;
  TcParams p = decode_params(a);
  // (the line between the two forms of the combine: see egmla_decode_tc.cu)
  p.fuse = !a.apart && D_C <= 256 && a.batch > 0 && kHeads * a.batch <= a.num_splits &&
           a.d_v <= kCombineRowsPerWarp * (kThreads / 32) &&
           a.num_splits <= resident_ctas<decode_plain_q8_kernel<D_C>, kPlainThreads>(C::SMEM);
  if (fused) *fused = p.fuse != 0;
  return launch_split_kernel<kPlainThreads>(kern, C::SMEM, a, maps, p, st);
}

}  // namespace

bool plain_q8_supported(int d_c) { return d_c == 256 || d_c == 512; }

cudaError_t launch_decode_plain_q8(const DecodeArgs& a, const CUtensorMap* maps, cudaStream_t st, bool* fused) {
  if (a.d_c == 256) return launch_plain<256>(a, maps, st, fused);
  if (a.d_c == 512) return launch_plain<512>(a, maps, st, fused);
  return cudaErrorInvalidValue;
}

}  // namespace egmla
