// egmla_decode_tc.cuh - what the split-KV kernels on tensor cores share
// (egmla_decode_tc.cu, and egmla_decode_q8.cu for the ungated latent in 8 bits): roles, launch parameters,
// the walk over a split's pages, waits, votes and TMEM reads, the split combine at a
// kernel's end, and the launch.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "egmla_common.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"

namespace egmla {

namespace {

#ifndef EGMLA_GATE_WARPS
#define EGMLA_GATE_WARPS 8
#endif
constexpr int kHeads = 16;
constexpr int kRope = 64;
constexpr int kThreads = 32 * (7 + EGMLA_GATE_WARPS);
constexpr int kSoftWarps = 4;    // warps 0-3: TMEM lane quadrants 0-3
constexpr int kSoftThreads = 32 * kSoftWarps;
constexpr int kTmaWarp = 4;
constexpr int kMmaWarp = 5;      // score MMAs and query blocks; also allocates and frees TMEM
constexpr int kOutWarp = 6;      // output MMAs
constexpr int kGateWarp0 = 7;
constexpr int kGateWarps = EGMLA_GATE_WARPS;
// 16-byte units of each 64-feature column a gate thread takes (the 64 token
// rows of a page over the gate threads), and lanes per token row
constexpr int kGateUnits = 16 / kGateWarps;
constexpr int kGateLanesPerRow = 8 / kGateUnits;
static_assert(kGateWarps == 8 || kGateWarps == 16, "gate warps");
constexpr uint32_t kSmemLimit = 232448;
// named barriers of the softmax warps (0 is __syncthreads)
constexpr int kBarTile = 1;
constexpr int kBarXch = 2;
// W_UV,h rows per warp in the fused combine (the fused path needs d_v <= 9 x warps)
constexpr int kCombineRowsPerWarp = 9;
// a head's reference max moves only when a tile exceeds it by 2^8
constexpr float kLazyLog2 = 8.f;
// score buffers in TMEM and P' buffers in shared memory
constexpr int kNB = 4;
constexpr int kNP = 4;

struct TcParams {
  const uint8_t* c8;      // Q8: codes [num_pages, 64, d_c], scales [num_pages, 64]
  const float* scales;
  const int32_t* id_pool;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const __nv_bfloat16* gate_table;
  const float* gamma;
  const float* beta;
  const uint8_t* qprep;
  const int32_t* cu;
  const SplitStart* starts;
  float* part_ml;
  float* part_o;
  int32_t* status;
  int batch, max_pages, num_pages, vocab;
  float scale_log2, eps;
  __nv_bfloat16* dump_c;
  __nv_bfloat16* dump_kr;
  int32_t* dump_ids;
  __nv_bfloat16* dump_g;
  int dump_len;
  // optional event trace (eg_mla_debug_set_trace): per traced CTA and role a
  // run of (tag, clock64) pairs; tag = event << 24 | tile
  unsigned long long* trace;
  int trace_ctas, trace_cap;
  // fused split combine (cooperative launch only): W_UV and output
  const __nv_bfloat16* w_uv;
  __nv_bfloat16* out;
  uint32_t* seq_done;   // [b]: the split partials of sequence b stored
  int d_v;
  int fuse, early;
  // limit of every wait (ns); a test entry lowers it, together with a
  // withheld page copy (stall_cta, stall_tile; stall_cta < 0: none)
  uint64_t wait_ns;
  int stall_cta, stall_tile;
};

// Trace recorder of one role of one CTA.  Only the trace instantiation of the
// kernel records (ON); in the others every call compiles to nothing, since even
// untaken trace stores in the loops cost registers and instruction-cache room.
template <bool ON>
struct TracerT {
  unsigned long long* base;
  int n, cap;
  // part 0 of 1 is the role's whole run; part k of 2 is half of it (two writers)
  __device__ void init(const TcParams& p, int role, int part = 0, int parts = 1) {
    base = nullptr;
    n = 0;
    cap = p.trace_cap / parts;
    if (ON && p.trace != nullptr && static_cast<int>(blockIdx.x) < p.trace_ctas)
      base = p.trace + ((static_cast<size_t>(blockIdx.x) * kTraceRoles + role) * p.trace_cap + part * cap) * 2;
  }
  // (tag, SM clock); the phase marks carry the global timer that maps the
  // clock of each CTA to time
  __device__ __forceinline__ void mark(int event, int tile) {
    if (ON && base != nullptr && n < cap) {
      base[2 * n] = (static_cast<unsigned long long>(event) << 56) |
                    (static_cast<unsigned long long>(tile & 0xffffff) << 32);
      base[2 * n + 1] = clock64();
      ++n;
    }
  }
};

// Kernel phase `event` of this CTA into entry `event` of trace role 4 (thread 0;
// stateless, so that nothing stays live across the kernel for it).
template <bool ON>
__device__ __forceinline__ void phase_mark(const TcParams& p, int event) {
  if (ON && p.trace != nullptr && threadIdx.x == 0 && static_cast<int>(blockIdx.x) < p.trace_ctas && event < p.trace_cap) {
    unsigned long long* e = p.trace + ((static_cast<size_t>(blockIdx.x) * kTraceRoles + 4) * p.trace_cap + event) * 2;
    e[0] = (static_cast<unsigned long long>(event) << 56) | static_cast<uint32_t>(globaltimer());
    e[1] = clock64();
  }
}

// shared-memory barrier block (inside MISC)
struct Bars {
  uint64_t full[6], empty[6], zready[6], zfree[6];
  uint64_t qfull[2], qempty[2];
  uint64_t sready[kNB], sfree[kNB];
  uint64_t spdone[kNP], pfree[kNP];
  uint64_t drain_s, drain_o;   // all MMAs of the score / output issuer done
  uint32_t tmem_base;
  int abort;
};

struct Tile {
  int b, lp, ntok, tok0;
  bool first, last;
};

// Walks this CTA's tiles (TOK tokens: a page or half of one) one at a time,
// segment by segment (identically in every role, so no per-tile metadata needs
// to be exchanged).
template <int TOK>
struct Walker {
  const int32_t* cu;
  const int32_t* lens;
  int batch, g1, b, lp, lp_end, L;
  int part = 0;   // tile of the page
  bool first, done;

  // the split's start record (written by the prologue kernel): one round of loads
  __device__ void start(const TcParams& p) {
    cu = p.cu;
    lens = p.seq_lens;
    batch = p.batch;
    const int4* r = reinterpret_cast<const int4*>(p.starts + blockIdx.x);
    const int4 h0 = __ldg(r), h1 = __ldg(r + 1);
    b = h0.x;
    lp = h0.y;
    lp_end = h0.z;
    L = h0.w;
    g1 = h1.x;
    done = h1.y != 0;
    first = true;
  }
  __device__ void enter(int g) {
    const int base = __ldg(cu + b) + kSegCost;   // unit of the sequence's first page
    lp = max(g - base, 0);
    lp_end = min(g1, __ldg(cu + b + 1)) - base;
    L = __ldg(lens + b);
    first = true;
    if (lp_end <= lp) done = true;   // the range ends inside the sequence's start cost
  }
  __device__ bool next(Tile& t) {
    if (done) return false;
    t.b = b;
    t.lp = lp;
    t.tok0 = lp * kPage + part * TOK;
    t.ntok = min(TOK, L - t.tok0);
    t.first = first;
    first = false;
    if constexpr (TOK < kPage) {
      if (++part < kPage / TOK && t.tok0 + TOK < L) {
        t.last = false;
        return true;
      }
      part = 0;
    }
    lp += 1;
    t.last = lp >= lp_end;
    if (t.last) {
      const int g = __ldg(cu + b) + kSegCost + lp_end;
      if (g >= g1) {
        done = true;
      } else {
        ++b;
        while (b < batch - 1 && __ldg(cu + b + 1) <= g) ++b;
        enter(g);
      }
    }
    return true;
  }
};

// Page of tile t through a 32-entry window of the block table held one entry per
// lane (whole warp; the window moves when the tile leaves it).
// The window starts as the first pages of the split's start record.
struct PageWindow {
  int b = -1, base = 0, n = 0, reg = -1;
  __device__ __forceinline__ void init(const TcParams& p, int lane) {
    const SplitStart* r = p.starts + blockIdx.x;
    b = __ldg(&r->b);
    base = __ldg(&r->lp);
    n = __ldg(&r->npages);
    reg = lane < kStartPages ? __ldg(&r->page[lane]) : -1;
  }
  __device__ __forceinline__ int page(const TcParams& p, const Tile& t, int lane) {
    if (t.b != b || t.lp < base || t.lp >= base + n) {
      b = t.b;
      base = t.lp;
      n = 32;
      const int lp = t.lp + lane;
      reg = lp < p.max_pages ? __ldg(p.block_table + static_cast<size_t>(t.b) * p.max_pages + lp) : -1;
    }
    return __shfl_sync(0xffffffffu, reg, t.lp - base);
  }
};

// mbarrier wait taken by a whole warp: the warp first reconverges (a lane
// still on a divergent path would otherwise only resume after the others'
// suspended wait), every lane polls, then the warp agrees, so that a timeout
// never splits the warp before a .sync.aligned instruction
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint64_t limit_ns) {
  __syncwarp();
  const bool ok = mbar_wait(bar, parity, abort_flag, limit_ns);
  return __all_sync(0xffffffffu, ok);
}

// one arrival per warp: the warp barrier orders every lane's earlier writes
// before lane 0's release arrival
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// lane 0's non-blocking test of a phase, the same answer in every lane
__device__ __forceinline__ bool warp_test(uint32_t bar, uint32_t parity) {
  return __shfl_sync(0xffffffffu, mbar_test_now(bar, parity) ? 1 : 0, 0) != 0;
}

// Named barrier of the softmax warps that also ORs a predicate over them: every
// participant gets the same answer, so a branch on it is uniform.
__device__ __forceinline__ bool soft_vote(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "r"(id), "r"(kSoftThreads)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ void soft_sync(int id) {
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(kSoftThreads) : "memory");
}

__device__ __forceinline__ float2 unpack_bf16x2(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  __nv_bfloat162 x = *reinterpret_cast<__nv_bfloat162*>(&a);
  __nv_bfloat162 y = *reinterpret_cast<__nv_bfloat162*>(&b);
  __nv_bfloat162 z = __hmul2(x, y);
  return *reinterpret_cast<uint32_t*>(&z);
}

// a + b of a pair in fp32, with a straight from its bf16 values
__device__ __forceinline__ float2 add_bf16x2(uint32_t a, uint32_t b) {
  const float2 y = unpack_bf16x2(b);
  float2 z;
  asm("{\n\t.reg .b16 lo, hi, one;\n\t"
      "mov.b16 one, 0x3f80;\n\tmov.b32 {lo, hi}, %2;\n\t"
      "fma.rn.f32.bf16 %0, lo, one, %3;\n\tfma.rn.f32.bf16 %1, hi, one, %4;\n\t}"
      : "=f"(z.x), "=f"(z.y)
      : "r"(a), "f"(y.x), "f"(y.y));
  return z;
}

// s += z and q += z^2 of a pair, in fp32 straight from the bf16 values
__device__ __forceinline__ void sum_bf16x2(uint32_t z, float2& s, float2& q) {
  asm("{\n\t.reg .b16 lo, hi, one;\n\t"
      "mov.b16 one, 0x3f80;\n\tmov.b32 {lo, hi}, %4;\n\t"
      "fma.rn.f32.bf16 %0, lo, one, %0;\n\tfma.rn.f32.bf16 %1, hi, one, %1;\n\t"
      "fma.rn.f32.bf16 %2, lo, lo, %2;\n\tfma.rn.f32.bf16 %3, hi, hi, %3;\n\t}"
      : "+f"(s.x), "+f"(s.y), "+f"(q.x), "+f"(q.y)
      : "r"(z));
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  __nv_bfloat162 z = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&z);
}

// 2^x with the hardware approximation (max 2 ulp; the weights are rounded to
// bf16 right after, and -inf gives 0)
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 lanes x 32 columns of 32-bit (tcgen05.ld.16x256b.x4): thread t gets lanes
// t/4 and t/4 + 8 at columns 8k + 2(t%4) and 8k + 2(t%4) + 1 of every 8-column
// group k, as v[4k] = (t/4, 8k + 2(t%4)), v[4k + 1] = (t/4, +1),
// v[4k + 2] = (t/4 + 8, ...), v[4k + 3] = (t/4 + 8, +1)
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// 32 lanes x 32 columns of 32-bit: thread i of the warp gets its lane's 32 values
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
      "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// inverse of tmem_ld32 (same thread-to-element map)
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
      "%24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
      "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])),
      "r"(__float_as_uint(v[8])), "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])), "r"(__float_as_uint(v[11])),
      "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])), "r"(__float_as_uint(v[14])),
      "r"(__float_as_uint(v[15])), "r"(__float_as_uint(v[16])), "r"(__float_as_uint(v[17])),
      "r"(__float_as_uint(v[18])), "r"(__float_as_uint(v[19])), "r"(__float_as_uint(v[20])),
      "r"(__float_as_uint(v[21])), "r"(__float_as_uint(v[22])), "r"(__float_as_uint(v[23])),
      "r"(__float_as_uint(v[24])), "r"(__float_as_uint(v[25])), "r"(__float_as_uint(v[26])),
      "r"(__float_as_uint(v[27])), "r"(__float_as_uint(v[28])), "r"(__float_as_uint(v[29])),
      "r"(__float_as_uint(v[30])), "r"(__float_as_uint(v[31]))
      : "memory");
}

// 16 lanes x 8 columns, as tmem_ld_16x256b_x4 for one group of eight columns
__device__ __forceinline__ void tmem_ld_16x256b_x1(uint32_t taddr, float (&v)[4]) {
  uint32_t r[4];
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}

// two groups of eight columns
__device__ __forceinline__ void tmem_ld_16x256b_x2(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

// ---------------------------------------------------------------- fused split combine
// Eight bf16 of a 16-byte piece as floats.
__device__ __forceinline__ void bf16x8_to_float(const uint4& raw, float (&w)[8]) {
  const __nv_bfloat162* e = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __bfloat1622float2(e[i]);
    w[2 * i] = f.x;
    w[2 * i + 1] = f.y;
  }
}

// Sums of eight rows whose parts are spread over the warp (v[r] = this lane's
// part of row r): a transposing butterfly halves the rows a lane carries at
// each of the xor-16, -8 and -4 exchanges, then two plain steps finish; lane
// 4r + q (q < 4) ends with the sum of row r.
__device__ __forceinline__ float reduce8_rows(const float (&v)[8], int lane) {
  const bool b4 = (lane & 16) != 0, b3 = (lane & 8) != 0, b2 = (lane & 4) != 0;
  float a[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float send = b4 ? v[i] : v[i + 4];
    const float keep = b4 ? v[i + 4] : v[i];
    a[i] = keep + __shfl_xor_sync(0xffffffffu, send, 16);
  }
  float c[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float send = b3 ? a[i] : a[i + 2];
    const float keep = b3 ? a[i + 2] : a[i];
    c[i] = keep + __shfl_xor_sync(0xffffffffu, send, 8);
  }
  const float send = b2 ? c[0] : c[1];
  float s = (b2 ? c[1] : c[0]) + __shfl_xor_sync(0xffffffffu, send, 4);
  s += __shfl_xor_sync(0xffffffffu, s, 2);
  s += __shfl_xor_sync(0xffffffffu, s, 1);
  return s;
}

// Split-KV combine inside the decode kernel (cooperative launch: every CTA is
// resident, so a wait on other CTAs cannot starve).  A CTA merges its units
// (head h, sequence b) once the softmax warps of the splits that covered the
// sequence have counted their parts of its partials on its counter (zeroed by
// the prologue kernel of the same call).  Over the splits s that covered b,
//   o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s,  M = max_s m_s,
//   u_{b,h} = W_UV,h o
// (a sequence of length 0 gets u = 0).  Each warp loads its nine rows of
// W_UV,h (lane l holding features 8l .. 8l + 7) from global memory into
// registers before it waits, so that the loads overlap the wait.  Merge: a
// warp per 32 features, lane k loading (m, l) of slot k0 + k and
// every lane O of 32 slots at once (online rescaling across groups of 32),
// into shared memory.  u: the warp's first eight row sums
// reduced across the lanes by a transposing butterfly (9 shuffles, after
// which lane 4r holds row r) and the ninth by a plain warp sum.
// ARRIVALS: softmax warps that leave a part of each partial
template <int D_C, bool TRACE, int ARRIVALS = kSoftWarps>
__device__ void fused_combine(const TcParams& p, uint8_t* smem, Bars& bars) {
  constexpr int kWarps = kThreads / 32;
  constexpr int NFB = D_C / 32;      // 32-feature blocks of a row
  constexpr int LANES = D_C / 8;     // lanes holding 8 features each
  constexpr int kRows = kCombineRowsPerWarp;   // output rows of W_UV,h per warp
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int units = kHeads * p.batch;
  float* olat = reinterpret_cast<float*>(smem);   // [D_C], in the free page-slot area
  volatile int* abort_flag = &bars.abort;
  const uint64_t wait_ns = p.wait_ns;
  const uint64_t keep = policy_evict_last();
  const int v0 = warp * kRows;   // this warp's first output row
  const int total = p.cu[p.batch];
  const int chunk = split_chunk(total, gridDim.x);
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const int h = u % kHeads, b = u / kHeads;
    // this warp's W_UV,h rows, requested before the wait
    uint4 wraw[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int v = v0 + r;
      wraw[r] = make_uint4(0, 0, 0, 0);
      if (lane < LANES && v < p.d_v)
        wraw[r] = ldg_16_na_hint(p.w_uv + (static_cast<size_t>(h) * p.d_v + v) * D_C + 8 * lane, keep);
    }
    const int q0 = p.cu[b] + kSegCost, q1 = p.cu[b + 1];   // units of the sequence's pages
    const int c0 = q0 / chunk;
    const int n = q1 > q0 ? (q1 - 1) / chunk - c0 + 1 : 0;   // splits that covered it
    if (tid == 0 && !*abort_flag) {
      // every softmax warp's part of every split partial of the sequence stored
      const uint32_t want = static_cast<uint32_t>(ARRIVALS) * static_cast<uint32_t>(n);
      const uint64_t t0 = globaltimer();
      while (ld_acquire_gpu(p.seq_done + b) < want) {
        if (*abort_flag) break;
        if (globaltimer() - t0 > wait_ns) {
          report_status(p.status, kStatusTimeout);
          *abort_flag = 1;
          break;
        }
        __nanosleep(32);
      }
    }
    __syncthreads();
    if (u == static_cast<int>(blockIdx.x)) phase_mark<TRACE>(p, 4);
    if (*abort_flag) return;
    for (int w = warp; w < NFB; w += kWarps) {
      const int f = w * 32 + lane;
      const float* po = p.part_o + (static_cast<size_t>(c0 + b) * kHeads + h) * D_C + f;
      const float* pm = p.part_ml + (static_cast<size_t>(c0 + b) * kHeads + h) * 2;
      float M = -INFINITY, L = 0.f, acc = 0.f;
      for (int k0 = 0; k0 < n; k0 += 32) {
        const int kn = min(32, n - k0);
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < kn) ml = __ldcg(reinterpret_cast<const float2*>(pm + static_cast<size_t>(k0 + lane) * kHeads * 2));
        float ov[32];
#pragma unroll
        for (int kk = 0; kk < 32; ++kk)
          ov[kk] = kk < kn ? __ldcg(po + static_cast<size_t>(k0 + kk) * kHeads * D_C) : 0.f;
        float mc = ml.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mc = fmaxf(mc, __shfl_xor_sync(0xffffffffu, mc, o));
        const float Mn = fmaxf(M, mc);
        const float sc = exp2f(M - Mn);   // 0 on the first group (M = -inf)
        const float wk = lane < kn ? exp2f(ml.x - Mn) : 0.f;
        float lw = wk * ml.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lw += __shfl_xor_sync(0xffffffffu, lw, o);
        L = fmaf(L, sc, lw);
        // four independent sums over the slots (zero weight past kn)
        float a4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 32; ++kk) a4[kk & 3] = fmaf(__shfl_sync(0xffffffffu, wk, kk), ov[kk], a4[kk & 3]);
        acc = fmaf(acc, sc, (a4[0] + a4[1]) + (a4[2] + a4[3]));
        M = Mn;
      }
      olat[f] = n > 0 ? acc / L : 0.f;
    }
    __syncthreads();
    if (u == static_cast<int>(blockIdx.x)) phase_mark<TRACE>(p, 5);
    // u = W_UV,h o from the registers loaded above: rows v0 .. v0 + 7 by the
    // butterfly, the ninth by a plain reduction
    if (v0 < p.d_v) {   // uniform in the warp
      float o8[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (lane < LANES) {
        const float4 x0 = *reinterpret_cast<const float4*>(olat + 8 * lane);
        const float4 x1 = *reinterpret_cast<const float4*>(olat + 8 * lane + 4);
        o8[0] = x0.x; o8[1] = x0.y; o8[2] = x0.z; o8[3] = x0.w;
        o8[4] = x1.x; o8[5] = x1.y; o8[6] = x1.z; o8[7] = x1.w;
      }
      float part[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        float wv[8];
        bf16x8_to_float(wraw[r], wv);
        part[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) part[r] = fmaf(wv[e], o8[e], part[r]);
      }
      const float sum = reduce8_rows(reinterpret_cast<const float (&)[8]>(part), lane);
      float last = part[8];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) last += __shfl_xor_sync(0xffffffffu, last, o);
      __nv_bfloat16* orow = p.out + (static_cast<size_t>(b) * kHeads + h) * p.d_v;
      const int v = v0 + (lane >> 2);
      if ((lane & 3) == 0 && v < p.d_v) orow[v] = __float2bfloat16_rn(sum);
      if (lane == 0 && v0 + 8 < p.d_v) orow[v0 + 8] = __float2bfloat16_rn(last);
    }
    __syncthreads();   // olat is free for the next unit
    if (u == static_cast<int>(blockIdx.x)) phase_mark<TRACE>(p, 6);
  }
}

// CTAs of Kern (with its one shared-memory size) that the current device holds at
// once (1 per SM here), looked up once per kernel and device
template <auto Kern, int THREADS = kThreads>
int resident_ctas(uint32_t smem) {
  static std::atomic<int> cached[64];   // 0: not looked up yet
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    int per_sm = 0, sms = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, Kern, THREADS, smem) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    n = std::max(0, per_sm) * sms;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

inline TcParams decode_params(const DecodeArgs& a) {
  const WorkspaceLayout wl = workspace_layout(a.batch, a.num_splits, kHeads, a.d_c, kRope, true);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  TcParams p;
  p.c8 = static_cast<const uint8_t*>(a.c_pool);
  p.scales = a.scale_pool;
  p.id_pool = a.id_pool;
  p.block_table = a.block_table;
  p.seq_lens = a.seq_lens;
  p.gate_table = static_cast<const __nv_bfloat16*>(a.gate_table);
  // gamma and beta belong to the LayerNorm (none in the "remove LayerNorm" ablation)
  p.gamma = a.gate_ln ? a.ln_gamma : nullptr;
  p.beta = a.gate_ln ? a.ln_beta : nullptr;

  p.qprep = ws + wl.off_qprep;
  p.cu = reinterpret_cast<const int32_t*>(ws + wl.off_cu);
  p.starts = reinterpret_cast<const SplitStart*>(ws + wl.off_start);
  p.part_ml = reinterpret_cast<float*>(ws + wl.off_ml);
  p.part_o = reinterpret_cast<float*>(ws + wl.off_o);
  p.status = a.status;
  p.batch = a.batch;
  p.max_pages = a.max_pages;
  p.num_pages = a.num_pages;
  p.vocab = a.vocab;
  p.scale_log2 = a.scale_log2;
  p.eps = a.eps;
  p.dump_c = static_cast<__nv_bfloat16*>(a.dump_c);
  p.dump_kr = static_cast<__nv_bfloat16*>(a.dump_kr);
  p.dump_ids = a.dump_ids;
  p.dump_g = static_cast<__nv_bfloat16*>(a.dump_g);
  p.dump_len = a.max_seq_len;
  p.trace = static_cast<unsigned long long*>(a.trace);
  p.trace_ctas = a.trace_ctas;
  p.trace_cap = a.trace_cap;
  p.w_uv = static_cast<const __nv_bfloat16*>(a.w_uv);
  p.out = static_cast<__nv_bfloat16*>(a.out);
  p.seq_done = reinterpret_cast<uint32_t*>(ws + wl.off_done);
  p.d_v = a.d_v;
  p.early = a.early;
  p.wait_ns = a.wait_ns;
  p.stall_cta = a.stall_cta;
  p.stall_tile = a.stall_tile;
  return p;
}

template <int THREADS = kThreads, typename Kern>
cudaError_t launch_split_kernel(Kern* kern, uint32_t smem, const DecodeArgs& a, const CUtensorMap* maps, const TcParams& p,
                                cudaStream_t st) {
  // The kernel may start while the query-absorption kernel before it on the
  // stream still runs (programmatic stream serialisation): its setup then
  // overlaps that kernel's tail, and grid_dependency_wait orders the rest.
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.num_splits);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int na = 0;
  if (p.fuse) {
    attr[na].id = cudaLaunchAttributeCooperative;
    attr[na].val.cooperative = 1;
    ++na;
  }
  attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[na].val.programmaticStreamSerializationAllowed = 1;
  ++na;
  cfg.attrs = attr;
  cfg.numAttrs = na;
  return cudaLaunchKernelEx(&cfg, kern, maps[0], maps[1], p);
}

}  // namespace
}  // namespace egmla
