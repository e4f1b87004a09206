// egmla_shared.cu - decode attention of a batch of sequences over a prefix that
// they share (sm_103a).
//
// Every head of every sequence meets the same prefix tokens, so their absorbed
// queries are the rows of one matrix product per prefix page,
//   S = Q^ Z^T,  O += P Z   (Q^: 16 heads x 8 sequences = 128 rows),
// and the prefix is read once per 128 rows instead of once per sequence.  The
// sequences' own tokens go through the split-KV decode kernel; both leave
// partials (running maximum, denominator, un-normalised latent output), and the
// split combine merges the two lists.
//
//   shared_gate_kernel    z'_j = LN without its affine part of c_j (*) G[id_j] (the
//                         gate mode's form) for every prefix token, rounded once (to
//                         f16 after a LayerNorm, to bf16 otherwise), so that the
//                         tiles of all sequences read the gated latent instead of
//                         gating it each.  gamma is folded into q^
//                         as in the decode kernel, beta enters as the constant
//                         q^ . beta of a row's scores and as beta l in its output.
//   shared_attn_kernel    the two products above on tcgen05, one CTA per SM.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "egmla_common.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"
#include "egmla_rows.cuh"

namespace egmla {
namespace {

__device__ __forceinline__ float sh_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t sh_pack(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// two values in the operands' type (element 0 in the low half)
template <bool F16>
__device__ __forceinline__ uint32_t sh_pack_as(float lo, float hi) {
  if constexpr (F16) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    return sh_pack(lo, hi);
  }
}

__device__ __forceinline__ bool sh_warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                             uint64_t limit_ns) {
  __syncwarp();
  const bool ok = mbar_wait(bar, parity, abort_flag, limit_ns);
  return __all_sync(0xffffffffu, ok);
}

// ============================================================================ 1. the gated prefix
constexpr int kSgWarps = 8;
constexpr int kSgRows = 4;   // rows per warp, their loads in flight together

struct SharedGateParams {
  const __nv_bfloat16* c_pool;
  const int32_t* id_pool;
  const int32_t* table;
  const int32_t* prefix_len;
  const __nv_bfloat16* gate_table;
  uint16_t* z;
  int d_c, vocab, num_pages, max_len;
  float eps;
  int32_t* status;
};

// GM: the gate mode.  Rows of whole pages, those past the prefix zero (their weights are
// zero, and the cache may hold anything there).  With the gate off the attention reads
// the pool itself: only the last page, where it is not full, is copied.
// Bound by the latency of table - ids - rows and, at 32K tokens (50 MB read and written,
// 8 us of the call), by L2: four blocks per SM (five spill: 55.2 us the call against 53.0).
template <int GM>
__global__ void __launch_bounds__(32 * kSgWarps, 4) shared_gate_kernel(const SharedGateParams p) {
  constexpr bool GATE = GM != EG_MLA_GATE_NONE, GATE_ADD = GM == EG_MLA_GATE_ADD_LN;
  constexpr bool GATE_LN = GM == EG_MLA_GATE_MUL_LN || GM == EG_MLA_GATE_ADD_LN;
  using U = Unit<__nv_bfloat16>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // beside the query absorption (nothing here needs it): its wait comes at the end
  grid_launch_dependents();
  beside_acquire();
  const int len = min(max(__ldg(p.prefix_len), 0), p.max_len);   // (reported by the schedule)
  const int first = GATE ? 0 : len / kPage * kPage;   // the row that z begins with
  const int rows = (len + kPage - 1) / kPage * kPage - first;
  const int t0 = (blockIdx.x * kSgWarps + warp) * kSgRows;
  if (t0 < rows) {
    // four rows never straddle a page; rows past the prefix, and of a page that is out of
    // range, read the first row of the page (of the pool) and are written as zero
    const int page = __ldg(p.table + (first + t0) / kPage);
    const bool page_ok = static_cast<unsigned>(page) < static_cast<unsigned>(p.num_pages);
    const size_t base = static_cast<size_t>(page_ok ? page : 0) * kPage;
    const int off = (first + t0) % kPage, live_rows = page_ok ? len - (first + t0) : 0;
    const bool live = lane < p.d_c / 8;   // a lane holds eight features; the others repeat the last
    const int at = 8 * min(lane, p.d_c / 8 - 1);
    bool bad = !page_ok;
    uint4 c[kSgRows], g[kSgRows];
#pragma unroll
    for (int r = 0; r < kSgRows; ++r) {
      const size_t row = base + (r < live_rows ? off + r : 0);
      c[r] = __ldg(reinterpret_cast<const uint4*>(p.c_pool + row * p.d_c + at));
      if (GATE) {
        int id = __ldg(p.id_pool + row);
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(p.vocab)) {
          bad |= r < live_rows;
          id = 0;
        }
        g[r] = __ldg(reinterpret_cast<const uint4*>(p.gate_table + static_cast<size_t>(id) * p.d_c + at));
      }
    }
    uint16_t* z = p.z + static_cast<size_t>(t0) * p.d_c + at;
    if constexpr (GATE) {
      const float inv_n = 1.f / static_cast<float>(p.d_c);
      float2 x[kSgRows][4];
      float s[kSgRows];
#pragma unroll
      for (int r = 0; r < kSgRows; ++r) {
        if (GATE_ADD) {
          float2 t[4];
          U::widen(c[r], x[r]);
          U::widen(g[r], t);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[r][e] = __fadd2_rn(x[r][e], t[e]);
        } else {
          U::mul(c[r], g[r], x[r]);
        }
        const float2 sum = __fadd2_rn(__fadd2_rn(x[r][0], x[r][1]), __fadd2_rn(x[r][2], x[r][3]));
        s[r] = live ? sum.x + sum.y : 0.f;
      }
      if (GATE_LN) {
        warp_sums(s, lane);
#pragma unroll
        for (int r = 0; r < kSgRows; ++r) {
          const float2 mu = make_float2(-s[r] * inv_n, -s[r] * inv_n);
          float2 sq = make_float2(0.f, 0.f);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[r][e] = __fadd2_rn(x[r][e], mu);
            sq = __ffma2_rn(x[r][e], x[r][e], sq);
          }
          s[r] = live ? sq.x + sq.y : 0.f;
        }
        warp_sums(s, lane);
#pragma unroll
        for (int r = 0; r < kSgRows; ++r) {
          const float rstd = rsqrtf(fmaf(s[r], inv_n, p.eps));
#pragma unroll
          for (int e = 0; e < 4; ++e) x[r][e] = __fmul2_rn(x[r][e], make_float2(rstd, rstd));
        }
      }
#pragma unroll
      for (int r = 0; r < kSgRows; ++r)
        c[r] = make_uint4(sh_pack_as<GATE_LN>(x[r][0].x, x[r][0].y), sh_pack_as<GATE_LN>(x[r][1].x, x[r][1].y),
                          sh_pack_as<GATE_LN>(x[r][2].x, x[r][2].y), sh_pack_as<GATE_LN>(x[r][3].x, x[r][3].y));
    }
#pragma unroll
    for (int r = 0; r < kSgRows; ++r)
      if (live) *reinterpret_cast<uint4*>(z + r * p.d_c) = r < live_rows ? c[r] : make_uint4(0u, 0u, 0u, 0u);
    if (bad && lane == 0) report_status(p.status, kStatusOutOfRange);
  }
  grid_dependency_wait();
}

// ============================================================================ 2. attention over the prefix
// A unit is (row tile of 8 sequences, prefix page); a CTA takes a range of them
// (SharedSchedule) and leaves one partial per row tile that its range meets.
//
// Tensor memory (512 columns): O [128 x D_C] fp32, two score buffers [128 x 64]
// (P in bf16 written over the first half of each), and the latent part of the
// queries as the A operand of the score MMAs, D_C / 2 columns of bf16 pairs: with A
// in shared memory an M 128, N 64 MMA is paced by A's 4 KB, not by its arithmetic.
// The RoPE part of the queries stays in shared memory; the rest of it is a ring of
// pages (latent columns of 64 features, then the RoPE keys, 128-byte swizzle), each
// the K-major B operand of the scores and, its latent columns, the MN-major B
// operand of the output.
//
// One thread issues S(j + 1) before O += P(j) Z(j), so that the softmax of a page
// runs under the MMAs of its neighbours.  The MMAs of one thread run in order:
// S(j + 1) overwrites P(j - 1) after the MMA that reads it.
//
// Bound by the tensor pipe in steady state: 0.705 us for a page (9.4 MFLOP; over all SMs
// as fast as the measured bf16 peak).  64 sequences over 32K tokens at d_c 256: 37 us
// (cold, alone; tensor pipe 43 % of it), since the own tokens' kernel has a part of the
// SMs, and a CTA takes 7 us besides its pages: queries into tensor memory, the first
// pages and scores, the partial.
constexpr int kSaSoftWarps = 8;
constexpr int kSaThreads = 32 * (2 + kSaSoftWarps);
constexpr int kSaRows = 128;                    // rows of a tile: 8 sequences of 16 heads
constexpr int kSaSeqs = kSharedTile;
constexpr uint32_t kSaCol = kPage * 128;        // 8 KB: a page's rows x 64 features
constexpr float kSaLazyLog2 = 8.f;              // how far a row's maximum runs ahead of its reference

struct SaBars {
  uint64_t full[8], empty[8];
  uint64_t sfull[2], pfull[2], odone[2];
  uint64_t qfull, qfree, drain;
  uint32_t tmem_base;
  int abort;
};

template <int D_C>
struct SaCfg {
  static constexpr int kCols = D_C / 64;                          // latent columns of a page
  static constexpr uint32_t kSlot = (kCols + 1) * kSaCol;
  static constexpr int kSlots = D_C == 256 ? 5 : 6;
  static constexpr uint32_t kOffRing = kSaRows * 128;             // after q^R
  static constexpr uint32_t kOffAffine = kOffRing + kSlots * kSlot;   // gamma, beta
  static constexpr uint32_t kOffBars = kOffAffine + 2 * D_C * 4;
  static constexpr uint32_t kSmem = kOffBars + sizeof(SaBars) + 1024;
  static constexpr uint32_t kColS = 256, kColQ = 384;             // (O from column 0)
  static_assert(kSlots <= 8 && kSmem <= kSmemMost && kColQ + D_C / 2 <= 512, "shared and tensor memory");
};

struct SharedAttnParams {
  const uint8_t* qprep;   // the prepared query blocks: q^R, the sums of q^ . beta and (bf16) q^ gamma
  size_t qstride;
  const uint8_t* q16;     // q^ gamma in f16, q_scale times its value
  const int32_t* table;
  const int32_t* prefix_len;
  const SharedSchedule* sched;
  const float* gamma;   // null: 1
  const float* beta;    // null: 0
  float* part_ml;
  float* part_o;
  int batch, max_len, num_pages, gate;
  float scale_log2, q_scale;
  uint64_t wait_ns;
  int32_t* status;
};

// the range of one CTA: row tile by row tile
struct SaWalk {
  int pages, u, u1;   // pages of the prefix; the next unit and the range's end
  __device__ SaWalk(const SharedAttnParams& p) {
    const int4 v = *reinterpret_cast<const int4*>(p.sched);
    const SharedSchedule s = {v.x, v.y, v.z, v.w};
    pages = s.pages;
    s.range(p.batch, static_cast<int>(blockIdx.x), u, u1);
  }
  // row tile t, pages lp0 .. lp1 - 1; false at the end
  __device__ bool next(int& t, int& lp0, int& lp1) {
    if (u >= u1) return false;
    t = u / pages;
    lp0 = u - t * pages;
    lp1 = min(pages, lp0 + (u1 - u));
    u += lp1 - lp0;
    return true;
  }
};

// F16: the latent's products in f16 (q^ q_scale times its value, a power of two, q^R likewise),
// and the weights 2^kPShift times theirs, so that they reach from 2^-32 to 2^15 of the
// reference; otherwise in bf16 (a latent of any magnitude), unscaled.
template <int D_C, bool F16>
__global__ void __launch_bounds__(kSaThreads, 1)
    shared_attn_kernel(const __grid_constant__ CUtensorMap zmap, const __grid_constant__ CUtensorMap tailmap,
                       const __grid_constant__ CUtensorMap krmap, const SharedAttnParams p) {
  using C = SaCfg<D_C>;
  constexpr float kPShift = F16 ? 7.f : 0.f;
  extern __shared__ uint8_t sa_raw[];
  uint8_t* smem = sa_raw + ((1024u - (smem_u32(sa_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  SaBars& bars = *reinterpret_cast<SaBars*>(smem + C::kOffBars);
  volatile int* abort_flag = &bars.abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < C::kSlots; ++s) {
      mbar_init(smem_u32(&bars.full[s]), 1);
      mbar_init(smem_u32(&bars.empty[s]), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&bars.sfull[x]), 1);
      mbar_init(smem_u32(&bars.pfull[x]), kSaSoftWarps);
      mbar_init(smem_u32(&bars.odone[x]), 1);
    }
    mbar_init(smem_u32(&bars.qfull), kSaSoftWarps);
    mbar_init(smem_u32(&bars.qfree), kSaSoftWarps);
    mbar_init(smem_u32(&bars.drain), 1);
    bars.abort = 0;
    fence_mbar_init();
    prefetch_tensormap(&zmap);
    prefetch_tensormap(&tailmap);
    prefetch_tensormap(&krmap);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&bars.tmem_base), 512);
    tmem_relinquish();
  }
  beside_acquire();   // (inputs are read before the wait)
  float* affine = reinterpret_cast<float*>(smem + C::kOffAffine);
  for (int f = tid; f < D_C; f += kSaThreads) {   // (this kernel starts after all that comes before the call)
    affine[f] = p.gamma ? __ldg(p.gamma + f) : 1.f;
    affine[D_C + f] = p.beta ? __ldg(p.beta + f) : 0.f;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem_base;
  const int len = min(max(__ldg(p.prefix_len), 0), p.max_len);   // (an input too)
  grid_dependency_wait();
  grid_launch_dependents();   // the own tokens' split-KV kernel, beside this one
  SaWalk walk(p);
  int t, lp0, lp1;

  if (warp == 0) {
    // ---- pages
    if (elect_one()) {
      const uint64_t keep = policy_evict_last();   // other CTAs read the same pages
      int n = 0;
      bool ok = true;
      while (ok && walk.next(t, lp0, lp1)) {
        int next_page = __ldg(p.table + lp0);
        for (int lp = lp0; lp < lp1; ++lp, ++n) {
          const int page = next_page;
          if (lp + 1 < lp1) next_page = __ldg(p.table + lp + 1);
          const int s = n % C::kSlots;
          if (n >= C::kSlots &&
              !mbar_wait(smem_u32(&bars.empty[s]), ((n / C::kSlots) & 1) ^ 1, abort_flag, p.wait_ns)) {
            ok = false;
            break;
          }
          // rows past the pool read as zero: where a page id outside it points
          const bool bad = static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages);
          if (bad) report_status(p.status, kStatusOutOfRange);
          const int row = (bad ? p.num_pages : page) * kPage;
          const uint32_t dst = sbase + C::kOffRing + s * C::kSlot, fb = smem_u32(&bars.full[s]);
          mbar_arrive_expect_tx(fb, C::kSlot);
          if (p.gate)
            tma_load_3d(dst, &zmap, 0, lp * kPage, 0, fb, keep);
          else if ((lp + 1) * kPage > len)
            tma_load_3d(dst, &tailmap, 0, 0, 0, fb, keep);
          else
            tma_load_3d(dst, &zmap, 0, row, 0, fb, keep);
          tma_load_3d(dst + C::kCols * kSaCol, &krmap, 0, row, 0, fb, keep);
        }
      }
      // every copy issued lands before the CTA can leave (own flag: bounded, not cut short)
      volatile int own = 0;
      for (int q = n > C::kSlots ? n - C::kSlots : 0; q < n; ++q)
        if (!mbar_wait(smem_u32(&bars.full[q % C::kSlots]), (q / C::kSlots) & 1, &own, p.wait_ns)) *abort_flag = 1;
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- MMAs
    constexpr uint32_t idesc_r = idesc_bf16(kSaRows, kPage, 0, 0);   // RoPE part
    constexpr uint32_t idesc_s = F16 ? idesc_f16(kSaRows, kPage, 0, 0) : idesc_r;
    constexpr uint32_t idesc_o = F16 ? idesc_f16(kSaRows, D_C, 0, 1) : idesc_bf16(kSaRows, D_C, 0, 1);
    const uint64_t qrdesc = smem_desc(sbase, 16, 1024, kSwizzle128B);
    const uint64_t kdesc = smem_desc(sbase + C::kOffRing, 16, 1024, kSwizzle128B);
    // Z [keys x features] as the MN-major B operand: 64-feature columns 8 KB apart,
    // groups of 8 keys 1 KB apart
    const uint64_t vdesc = smem_desc(sbase + C::kOffRing, kSaCol, 1024, kSwizzle128B);
    if (elect_one()) {
      bool ok = true, issued = false;
      int n = 0, seg = 0;   // pages and row tiles before this row tile
      auto issue_s = [&](int i) {
        const int s = i % C::kSlots;
        ok = ok && mbar_wait(smem_u32(&bars.full[s]), (i / C::kSlots) & 1, abort_flag, p.wait_ns);
        if (!ok) return;
        tc_fence_after();
        const uint32_t d = tmem + C::kColS + kPage * (i & 1);
        const uint64_t kd = kdesc + ((s * C::kSlot) >> 4);
#pragma unroll
        for (int c = 0; c < C::kCols; ++c)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_bf16_ts(d, tmem + C::kColQ + 32 * c + 8 * kk, kd + ((c * kSaCol + kk * 32) >> 4), idesc_s,
                        (c > 0 || kk > 0) ? 1u : 0u);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          mma_bf16_ss(d, qrdesc + ((kk * 32) >> 4), kd + ((C::kCols * kSaCol + kk * 32) >> 4), idesc_r, 1u);
        mma_commit(smem_u32(&bars.sfull[i & 1]));
        issued = true;
      };
      auto issue_pv = [&](int i, bool first) {
        ok = ok && mbar_wait(smem_u32(&bars.pfull[i & 1]), (i >> 1) & 1, abort_flag, p.wait_ns);
        if (!ok) return;
        tc_fence_after();
        const int s = i % C::kSlots;
        const uint64_t vd = vdesc + ((s * C::kSlot) >> 4);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          mma_bf16_ts(tmem, tmem + C::kColS + kPage * (i & 1) + 8 * ks, vd + ((ks * 2048) >> 4), idesc_o,
                      (!first || ks > 0) ? 1u : 0u);
        mma_commit(smem_u32(&bars.empty[s]));
        mma_commit(smem_u32(&bars.odone[i & 1]));
      };
      while (ok && walk.next(t, lp0, lp1)) {
        ok = mbar_wait(smem_u32(&bars.qfull), seg & 1, abort_flag, p.wait_ns);
        const int m = lp1 - lp0;
        if (ok) issue_s(n);
        for (int j = 0; ok && j < m; ++j) {
          if (j + 1 < m) issue_s(n + j + 1);
          if (ok) issue_pv(n + j, j == 0);
        }
        n += m;
        ++seg;
      }
      if (issued) {
        mma_commit(smem_u32(&bars.drain));
        volatile int own = 0;
        if (!mbar_wait(smem_u32(&bars.drain), 0, &own, p.wait_ns)) *abort_flag = 1;
      }
    }
    __syncwarp();
  } else {
    // ---- queries, softmax, partials.  A warp has the 16 heads of one sequence: half
    // of its TMEM lane quadrant, four lanes per row (lane l: rows l / 4 and l / 4 + 8,
    // columns 2 (l % 4) and + 1 of every 8).
    const int quad = warp & 3, sub = (warp - 2) >> 2;
    const int seq = 2 * quad + sub;                         // of the tile
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(32 * quad + 16 * sub) << 16);
    const int r0 = lane >> 2, c2 = 2 * (lane & 3);
    const float sl2 = F16 ? p.scale_log2 / p.q_scale : p.scale_log2;
    // a partial leaves through the memory of q^R, which is read no more by then: 2 KB a warp
    uint8_t* stage = smem + (warp - 2) * 2048;
    int n = 0, seg = 0;
    bool ok = true;
    // O has taken page i, whose scores this warp has had.  Its scores came after O had page
    // i - 2, and O cannot have page i + 2 before this warp has given weights for it, so the
    // parity of every other page's barrier is that of page i; with one barrier for all, a
    // warp ahead of the others would take page i - 2's completion for it.
    auto o_has = [&](int i) {
      return sh_warp_wait(smem_u32(&bars.odone[i & 1]), (i >> 1) & 1, abort_flag, p.wait_ns);
    };
    while (ok && walk.next(t, lp0, lp1)) {
      // (the last partial has left that memory)
      if (seg > 0 && !sh_warp_wait(smem_u32(&bars.qfree), (seg - 1) & 1, abort_flag, p.wait_ns)) break;
      ++seg;
      // the tile's queries (every MMA that read the last tile's is complete).  A lane
      // takes its row of the quadrant, this warp one half of its latent features
      // (the A operand in tensor memory) and of its RoPE part (shared memory).  Plain
      // loads: this kernel may have started before the absorption had stored them.
      {
        const int row = 32 * quad + lane, h = row & 15, b = t * kSaSeqs + row / 16;
        const size_t bs = static_cast<size_t>(min(b, p.batch - 1));
        const uint8_t* src = p.qprep + bs * p.qstride;
        const uint8_t* lat = F16 ? p.q16 + bs * qprep_lat_bytes(D_C) : src;
        const bool live = b < p.batch;   // rows past the batch are zero
        constexpr int kHalf = D_C / 16;  // 16-byte units of half a row
        uint4 xr[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          xr[u] = make_uint4(0u, 0u, 0u, 0u);
          if (live)
            xr[u] = *reinterpret_cast<const uint4*>(src + qprep_lat_bytes(D_C) + qop_offset(h, 8 * (4 * sub + u)));
        }
#pragma unroll
        for (int u8 = 0; u8 < kHalf; u8 += 8) {
          uint4 x[8];   // eight loads in flight
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            x[u] = make_uint4(0u, 0u, 0u, 0u);
            if (live && u8 + u < kHalf)
              x[u] = *reinterpret_cast<const uint4*>(lat + qop_offset(h, 8 * (sub * kHalf + u8 + u)));
          }
#pragma unroll
          for (int u0 = 0; u0 < 8 && u8 + u0 < kHalf; u0 += 4) {
            uint32_t v[16];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              v[4 * u] = x[u0 + u].x;
              v[4 * u + 1] = x[u0 + u].y;
              v[4 * u + 2] = x[u0 + u].z;
              v[4 * u + 3] = x[u0 + u].w;
            }
            tmem_st16(tmem + (static_cast<uint32_t>(32 * quad) << 16) + C::kColQ + 4 * (sub * kHalf + u8 + u0), v);
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if constexpr (F16) {   // exact: the exponent alone changes
            const __nv_bfloat162 f = __float2bfloat162_rn(p.q_scale);
            __nv_bfloat162* w = reinterpret_cast<__nv_bfloat162*>(&xr[u]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __hmul2(w[i], f);
          }
          *reinterpret_cast<uint4*>(smem + row * 128 + (((4 * sub + u) ^ (row & 7)) << 4)) = xr[u];
        }
        tmem_wait_st();
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.qfull));
      }
      // the constant q^ . beta of a row's scores, from its per-chunk partials
      float bias[2] = {0.f, 0.f};
      if (p.beta != nullptr) {
        const float* sums = reinterpret_cast<const float*>(p.qprep + static_cast<size_t>(min(t * kSaSeqs + seq, p.batch - 1)) *
                                                                         p.qstride +
                                                           qprep_lat_bytes(D_C) + qprep_rope_bytes(64));
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int c = 0; c < D_C / kSumFeatures; ++c) bias[e] += sums[c * 32 + 16 + r0 + 8 * e];
      }
      float m_ref[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};
      for (int lp = lp0; ok && lp < lp1; ++lp, ++n) {
        ok = sh_warp_wait(smem_u32(&bars.sfull[n & 1]), (n >> 1) & 1, abort_flag, p.wait_ns);
        if (!ok) break;
        tc_fence_after();
        const uint32_t cs = C::kColS + kPage * (n & 1);
        float v[32];
        tmem_ld_16x256b_x8(lane_base + cs, v);
        tmem_wait_ld();
        const int lim = len - lp * kPage - c2;   // columns of the page in the prefix, from this lane's first
        if (lim + c2 < kPage) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (8 * k + (e & 1) >= lim) v[4 * k + e] = -INFINITY;
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) m4[e] = fmaxf(m4[e], v[4 * k + e]);
        float alpha[2] = {1.f, 1.f};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(m4[2 * e], m4[2 * e + 1]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) * sl2;
          if (lp == lp0) {
            m_ref[e] = mx;
          } else if (mx > m_ref[e] + kSaLazyLog2) {
            alpha[e] = sh_ex2(m_ref[e] - mx);
            m_ref[e] = mx;
          }
        }
        if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
          ok = o_has(n - 1);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int g = 0; g < C::kCols; ++g) {
            float o[32];
            tmem_ld_16x256b_x8(lane_base + 64 * g, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[4 * k + e] *= alpha[e >> 1];
            tmem_st_16x256b_x8(lane_base + 64 * g, o);
          }
        }
        const float2 sl2v = make_float2(sl2, sl2);
        float2 rs[2] = {{0.f, 0.f}, {0.f, 0.f}};
        uint32_t pk[16];
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 x = __ffma2_rn(make_float2(v[4 * k + 2 * e], v[4 * k + 2 * e + 1]), sl2v,
                                        make_float2(kPShift - m_ref[e], kPShift - m_ref[e]));
            const float2 pr = make_float2(sh_ex2(x.x), sh_ex2(x.y));
            rs[e] = __fadd2_rn(rs[e], pr);
            pk[2 * k + e] = sh_pack_as<F16>(pr.x, pr.y);
          }
        tmem_st_16x128b_x8(lane_base + cs, pk);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.pfull[n & 1]));
#pragma unroll
        for (int e = 0; e < 2; ++e) l[e] = fmaf(l[e], alpha[e], rs[e].x + rs[e].y);
      }
      // ---- the partial
      if (ok) ok = o_has(n - 1);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
      }
      const int b = t * kSaSeqs + seq;
      const size_t row = (static_cast<size_t>(blockIdx.x + t) * kSaSeqs + seq) * 16 + r0;   // and row + 8
      if (b < p.batch && (lane & 3) == 0) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float2*>(p.part_ml + (row + 8 * e) * 2) =
              make_float2(fmaf(bias[e], p.scale_log2, m_ref[e] - kPShift), l[e]);
      }
#pragma unroll
      for (int g = 0; g < C::kCols; ++g) {
        float o[32];
        tmem_ld_16x256b_x8(lane_base + 64 * g, o);
        tmem_wait_ld();
        if (b >= p.batch) continue;   // uniform in the warp
        // 32 columns at a time through shared memory, so that a store covers whole lines
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int k = 4 * half; k < 4 * half + 4; ++k) {
            const int f = 64 * g + 8 * k + c2;
            const float2 gm = *reinterpret_cast<const float2*>(affine + f);
            const float2 bt = *reinterpret_cast<const float2*>(affine + D_C + f);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int rr = r0 + 8 * e, u = ((8 * k + c2) & 31) >> 2;
              *reinterpret_cast<float2*>(stage + rr * 128 + ((u ^ (rr & 7)) << 4) + (c2 & 2) * 4) =
                  make_float2(fmaf(gm.x, o[4 * k + 2 * e], bt.x * l[e]), fmaf(gm.y, o[4 * k + 2 * e + 1], bt.y * l[e]));
            }
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int rr = 4 * i + (lane >> 3), u = lane & 7;
            const float4 x = *reinterpret_cast<const float4*>(stage + rr * 128 + ((u ^ (rr & 7)) << 4));
            *reinterpret_cast<float4*>(p.part_o + (row - r0 + rr) * D_C + 64 * g + 32 * half + 4 * u) = x;
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      if (lane == 0) mbar_arrive(smem_u32(&bars.qfree));
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
  if (tid == 0 && bars.abort) report_status(p.status, kStatusTimeout);
}

template <int D_C, bool F16>
cudaError_t launch_attn(const SharedArgs& a, const CUtensorMap* maps, const SharedAttnParams& p, cudaStream_t st) {
  const cudaError_t e = allow_smem(shared_attn_kernel<D_C, F16>, SaCfg<D_C>::kSmem);
  if (e != cudaSuccess) return e;
  return launch_chained(shared_attn_kernel<D_C, F16>, dim3(a.dec->num_splits), dim3(kSaThreads), SaCfg<D_C>::kSmem, st, maps[0],
                        maps[1], maps[2], p);
}

}  // namespace

bool shared_supported(int d_c) { return d_c == 192 || d_c == 256; }

cudaError_t launch_shared_gate(const SharedArgs& a, cudaStream_t st) {
  const DecodeArgs& d = *a.dec;
  uint8_t* ws = static_cast<uint8_t*>(d.workspace);
  SharedGateParams g;
  g.c_pool = static_cast<const __nv_bfloat16*>(d.c_pool);
  g.id_pool = d.id_pool;
  g.table = a.prefix_table;
  g.prefix_len = a.prefix_len;
  g.gate_table = static_cast<const __nv_bfloat16*>(d.gate_table);
  g.z = reinterpret_cast<uint16_t*>(ws + a.wl.off_z);
  g.d_c = d.d_c;
  g.vocab = d.vocab;
  g.num_pages = d.num_pages;
  g.max_len = a.max_prefix_len;
  g.eps = d.eps;
  g.status = d.status;
  const int rows = static_cast<int>(shared_z_rows(a.max_prefix_len, d.gate != 0));
  auto launch = [&](auto kernel) {
    return launch_chained(kernel, dim3((rows + kSgWarps * kSgRows - 1) / (kSgWarps * kSgRows)), dim3(32 * kSgWarps), 0, st,
                          g);
  };
  if (!d.gate) return launch(shared_gate_kernel<EG_MLA_GATE_NONE>);
  if (d.gate_add) return launch(shared_gate_kernel<EG_MLA_GATE_ADD_LN>);
  if (d.gate_ln) return launch(shared_gate_kernel<EG_MLA_GATE_MUL_LN>);
  return launch(shared_gate_kernel<EG_MLA_GATE_MUL>);
}

cudaError_t launch_shared_attn(const SharedArgs& a, const CUtensorMap* maps, cudaStream_t st) {
  const DecodeArgs& d = *a.dec;
  uint8_t* ws = static_cast<uint8_t*>(d.workspace);
  const WorkspaceLayout wl = workspace_layout(d.batch, d.num_splits, 16, d.d_c, d.d_rope, true);
  SharedAttnParams p;
  p.qprep = ws + wl.off_qprep;
  p.qstride = wl.qprep_stride;
  p.q16 = ws + a.wl.off_q;
  p.table = a.prefix_table;
  p.prefix_len = a.prefix_len;
  p.sched = reinterpret_cast<const SharedSchedule*>(ws + a.wl.off_sched);
  p.gamma = d.gate_ln ? d.ln_gamma : nullptr;
  p.beta = d.gate_ln ? d.ln_beta : nullptr;
  p.part_ml = reinterpret_cast<float*>(ws + a.wl.off_ml);
  p.part_o = reinterpret_cast<float*>(ws + a.wl.off_o);
  p.batch = d.batch;
  p.max_len = a.max_prefix_len;
  p.num_pages = d.num_pages;
  p.gate = d.gate;
  p.scale_log2 = d.scale_log2;
  p.q_scale = a.q_scale;
  p.wait_ns = d.wait_ns;
  p.status = d.status;
  if (d.gate_ln) return d.d_c == 256 ? launch_attn<256, true>(a, maps, p, st) : launch_attn<192, true>(a, maps, p, st);
  return d.d_c == 256 ? launch_attn<256, false>(a, maps, p, st) : launch_attn<192, false>(a, maps, p, st);
}

}  // namespace egmla
