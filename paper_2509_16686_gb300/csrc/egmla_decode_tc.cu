// egmla_decode_tc.cu - split-KV EG-MLA decode on sm_103a tensor cores for the
// latent widths 192 and 256 (gated or plain) and 512 (plain).
//
// One CTA per split-KV work unit (see egmla_common.cuh for the schedule).  The
// CTA streams its cache pages, one 64-token page per tile (half a page at width
// 512), through a ring of shared-memory slots; the tiles are token rows of the
// tensor-core operations (M = 64 tokens), the 16 heads their columns (N = 16).  Roles:
//
//   TMA (warp 4)      latent page [64 tok x d_c] (one 3-D box: 64-feature
//                     columns x 64 rows) and RoPE-key page [64 x 64], both
//                     128-byte swizzled, and the page's token ids (a bulk copy
//                     into the slot's statistics area), as soon as the page
//                     slot is free; a CTA's first page is requested alone.
//                     The split's start comes from a record the
//                     query-absorption kernel wrote.
//   gate (warps 7-14; each quarter-warp owns two token rows, lane u the 16-byte
//                     units 2u, 2u + 1 of every 64-feature column of them)
//                     the gate rows g = G[id] (EG-MLA-A table, Section 5.2)
//                     of the next tile into registers, requested column by
//                     column between this tile's stores as soon as the next
//                     page (and so its ids) has landed, every quarter-warp
//                     load reading one whole 128-byte line from L2; z = c (*) g
//                     rounded to bf16 and written back in place, and the
//                     LayerNorm statistics mu, r = 1/sqrt(var + eps) of z
//                     (Eq. 5 over d_c).
//   scores (warp 5)   S = Z (q^ gamma)^T and S_rope = K^R q^R^T (M = 64 tokens,
//                     N = 16 heads, K = d_c and 64; fp32 in TMEM, four score
//                     buffers) as soon as a gated page and a score buffer are
//                     ready, and the query block of the next sequence segment.
//   output (warp 6)   O^T += Z^T P' (M = 128 latent features, N = 16 heads,
//                     K = 64 tokens; O^T stays in TMEM over a sequence
//                     segment).  An issuing thread stalls while the tensor
//                     pipe's queue is full, so the two MMA streams have a
//                     warp each (of which one thread does the waits; see
//                     WARP_ISSUE).
//   softmax (warps 0-3, one per TMEM lane quadrant: tokens 16w .. 16w + 15)
//                     thread t reads two tokens x four heads of S; the
//                     LayerNorm is applied after the MMA, since
//                       q^.LN(z) = r (q^ gamma).z - r mu sum(q^ gamma) + q^.beta,
//                     s = scale (r (S - mu w) + b + S_rope); an online softmax
//                     whose per-head reference max moves only when a tile
//                     exceeds it by 2^8 (one barrier vote of the four warps per
//                     tile decides; the maxima are exchanged only then), and
//                     P' = p r (bf16) as the B operand of the output MMA.
//
// At the end of each sequence segment the four softmax warps read O^T (latent
// features in TMEM lanes) and write the split's partial result: the
// un-normalised latent output gamma (*) (O - sum_j P'_j mu_j) + beta l, the
// reference max m and the denominator l = sum_j P'_j / r_j.  With heads as
// the MMA columns, no tensor-core work is spent on padding rows, tensor
// memory holds four score buffers and the whole output in 160 columns, and the
// query block takes 10 KB, which leaves room for five page slots at d_c = 256.
//
// The queries are absorbed before this kernel (q^ = W_UK^T q^C, with gamma
// folded in); the kernel may start while that kernel runs (programmatic
// stream serialisation) and waits for it after its set-up.  The split merge
// and W_UV run at its end when the grid is cooperative (fused_combine).
// Everything the kernel waits on has a time limit: on expiry it records
// EG_MLA_ERR_TIMEOUT, drains its own copies and MMAs, frees TMEM and exits.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "egmla_common.cuh"
#include "egmla_decode_tc.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"
#include "egmla_q8.cuh"

namespace egmla {

namespace {

// Q8: the cache holds the latent in 8 bits (egmla_q8.cuh).  The page's codes, scales and
// ids and its RoPE keys land in a ring of raw slots, from which the gate warps write the
// bf16 tile into a ring of latent slots: a raw slot is held until the tile's score MMAs
// are complete, a latent slot from the gate to its output MMAs.  (us for 8 x 32K at d_c 256
// and 128 ragged sequences at d_c 192, before ZZ: three latent slots and four raw ones 47.2
// and 75.7; four, and three and four raw ones, 48.5 and 73.9.)
//
// With 8 bits the copies bring 57 instead of 73 KB per page with its gate rows, and memory
// no longer counts: the gate warps do, which have to widen the codes (4.5 operations a
// pair of values beside the six of gate, sums and store), then the softmax.  44.5 us for 8
// x 32K tokens where a bf16 cache takes 45.7 and the bytes 17.9; without the gate's work,
// timed with its instructions left out, 40.  More warps for either role (twelve for the
// gate, eight for the softmax), at 96 registers each instead of 128, were slower: 57 and 54.
// ZZ (with Q8 and LN(c (*) g) at d_c 256): the LayerNorm's sums of a tile come from the tensor
// cores: Z [Z ; 1]^T, whose diagonal holds every row's sum of squares and whose last
// columns its sum.  Eight rows of ones behind the tile's 64 in each of its columns.  The
// tensor pipe was busy for 7 % of the time (24 with the sums), and the gate saves a third of its
// arithmetic and the row sums' shuffles: 8 x 32K 46.9 -> 45.0 us, 4 of 60 to 700 tokens 12.3
// -> 12.9.  At d_c 192, where the softmax takes longer than the gate, 128 ragged sequences
// went from 73.4 to 74.9.
template <int D_C, bool GATE, bool Q8 = false, bool ZZ = false>
struct Cfg {
  static constexpr int NCH = D_C / 64;                  // 64-feature swizzle-atom columns
  // tokens per tile: a page, or half a page for the widest latent, whose pages
  // are too large for a ring of three in shared memory: two slots of 72 KB took
  // about 150 us for 128 ragged sequences, five of 36 KB about 92 (562 MB: 3.7
  // and 6.1 TB/s; kernel alone, warm)
  static constexpr int TOK = D_C > 256 ? kPage / 2 : kPage;
  static constexpr uint32_t PCHUNK = TOK * 128;         // one atom column of a tile
  static constexpr uint32_t ZCHUNK = PCHUNK + (ZZ ? 1024 : 0);   // one of the latent's
  static constexpr uint32_t KR_OFF = NCH * ZCHUNK;
  static constexpr uint32_t SLOT = Q8 ? KR_OFF : KR_OFF + PCHUNK;   // latent (+ RoPE key) of one tile
  // raw slots: RoPE key, codes; apart from them the ids and the scales
  static constexpr uint32_t RSLOT = Q8 ? PCHUNK + TOK * D_C : 0;
  static constexpr uint32_t RMETA = Q8 ? (GATE ? 2 : 1) * kPage * 4 : 0;
  static constexpr uint32_t STAT_BYTES = GATE && !ZZ ? 2 * kPage * 4 : 0;   // per slot: mu[64], r[64]
  static constexpr uint32_t QB_LAT = qprep_lat_bytes(D_C);
  static constexpr uint32_t QPREP = qprep_bytes_tc(D_C, kRope);
  static constexpr uint32_t QBUF = (QPREP + 127) / 128 * 128;
  // P' [64 tokens x 16 heads] as the MN-major B operand of the output MMA
  static constexpr uint32_t PBUF = kPage * kHeads * 2;
  // LayerNorm gamma and beta of the segment read-out
  static constexpr uint32_t GB_BYTES = GATE ? 2 * D_C * 4 : 0;
  // softmax exchange: tile maxima [4 warps][16], segment sums [4 warps][16][2],
  // with half pages the odd latent columns' scores [32 tokens][16]
  static constexpr uint32_t XCH = 1024 + (TOK < kPage ? TOK * kHeads * 4 : 0);
  static constexpr uint32_t MISC = Q8 ? 512 : 1024;
  static constexpr int NP = ZZ && D_C == 256 ? 2 : kNP;   // P' buffers (two make room for the fourth raw slot)
  static constexpr uint32_t FIXED = NP * PBUF + GB_BYTES + XCH + MISC + 1024;
  // slots with two query buffers (the next segment's loaded while this one is
  // in use) or with one; one buffer when a second would cost a slot below five
  static constexpr int NS2 = (int)((kSmemLimit - FIXED - 2 * QBUF) / (SLOT + STAT_BYTES));
  static constexpr int NS1 = (int)((kSmemLimit - FIXED - QBUF) / (SLOT + STAT_BYTES));
  static constexpr int NQ = Q8 ? (D_C == 192 ? 2 : 1) : (NS2 < 5 && NS1 > NS2) ? 1 : 2;
  static constexpr int NS_FIT = NQ == 2 ? NS2 : NS1;
  static constexpr int NS = Q8 ? (D_C == 192 ? 4 : 3) : NS_FIT > 6 ? 6 : NS_FIT;
  // raw slots: what is left beside the latent slots
  static constexpr int NR_FIT =
      Q8 ? (int)((kSmemLimit - FIXED - NQ * QBUF - NS * (SLOT + STAT_BYTES)) / (RSLOT + RMETA + (Q8 ? 0 : 1))) : 0;
  static constexpr int NR = NR_FIT > 6 ? 6 : NR_FIT;
  static constexpr uint32_t OFF_RAW = NS * SLOT;
  static constexpr uint32_t OFF_QBUF = OFF_RAW + NR * RSLOT;
  static constexpr uint32_t OFF_PBUF = OFF_QBUF + NQ * QBUF;
  static constexpr uint32_t OFF_STAT = OFF_PBUF + NP * PBUF;
  static constexpr uint32_t OFF_META = OFF_STAT + NS * STAT_BYTES;
  static constexpr uint32_t OFF_GB = OFF_META + NR * RMETA;
  static constexpr uint32_t OFF_XCH = OFF_GB + GB_BYTES;
  static constexpr uint32_t OFF_MISC = OFF_XCH + XCH;
  static constexpr uint32_t SMEM = OFF_MISC + MISC + 1024;
  // TMEM columns: kNB score buffers of (latent 16 + RoPE 16) head columns,
  // then the latent output O^T (16 head columns per 128-feature M chunk)
  static constexpr int NMC = (D_C + 127) / 128;
  static constexpr uint32_t S_COLS = 32;
  static constexpr uint32_t COL_S = 0, COL_O = kNB * S_COLS;
  // Z [Z ; 1]^T: 64 columns of the tile's rows, 8 of the sums, a block per score buffer
  static constexpr uint32_t ZZ_COLS = kPage + 8, COL_ZZ = COL_O + kHeads * NMC;
  static constexpr uint32_t TMEM_COLS = ZZ ? 512 : 256;
  static constexpr uint32_t PAGE_TX = Q8 ? RSLOT + TOK * 4 : SLOT;
  static constexpr uint32_t ID_TX = GATE ? kPage * 4 : 0;   // the page's token ids
  static constexpr int RING = Q8 ? NR : NS;                 // slots that copies land in
  static_assert(NS >= 3 && RING >= 3, "the ring needs three page slots");
  static_assert(SLOT % 1024 == 0 && RSLOT % 1024 == 0, "swizzle atoms");
  static_assert(SMEM <= kSmemLimit, "shared memory");
  static_assert(D_C == 192 || D_C == 256 || (D_C == 512 && !GATE), "latent widths of this kernel");
  static_assert(COL_O + kHeads * NMC + (ZZ ? COL_ZZ - COL_O - kHeads * NMC + kNB * ZZ_COLS : 0) <= TMEM_COLS && NMC % 2 == 0, "tensor memory");
  // the score MMAs read 64 rows: at half pages two atom columns' 32, for the
  // RoPE key its 32 and what follows the slot, whose scores are not used
  static_assert(OFF_QBUF + 64 * 128 <= SMEM, "score operand");
  // first latent feature of output M chunk j (chunks of 128 rows); for
  // D_C = 192 the second chunk starts at 64 and overlaps the first, so that no
  // MMA reads past the latent part of a slot (its rows 64..127 are not read out)
  __host__ __device__ static constexpr int mc_start(int j) { return j == NMC - 1 ? D_C - 128 : 128 * j; }
};

// GM: gate mode (0 none, 1 LN(c (*) g), 2 c (*) g, 3 LN(c + g): eg_mla_gate_mode)
// DBG: 0 the decode, 1 the cache-read dump (raw pages and gate rows, no
// attention), 2 the decode with the pipeline trace, 3 the decode beside the attention
// over a shared prefix, 4 the decode over a cache in 8 bits
template <int D_C, int GM, int DBG>
__global__ void __launch_bounds__(kThreads, 1)
    decode_tc_kernel(const __grid_constant__ CUtensorMap cmap, const __grid_constant__ CUtensorMap krmap,
                     const TcParams p) {
  constexpr bool DUMP = DBG == 1, BESIDE = DBG == 3, Q8 = DBG == 4;
  using Tracer = TracerT<DBG == 2>;
  constexpr bool GATE = GM != 0;
  constexpr bool GATE_ADD = GM == 3;             // ablation: c + g
  constexpr bool GATE_LN = GM == 1 || GM == 3;   // LayerNorm after the gate
  constexpr bool ZZ = Q8 && GM == 1 && D_C == 256;
  using C = Cfg<D_C, GATE, Q8, ZZ>;
  // The MMA issuers: one thread of the warp, or (d_c 192 gated with a product) the
  // whole warp waiting together and electing a thread for each tile's MMAs.  Steps
  // replayed 24 to a graph, one thread / whole warp: d_c 192 with c (*) g 65.7 / 65.1
  // us for 16 x 32K, 114.1 / 112.9 for 31 x 32K, 65.9 / 65.2 for 128 ragged
  // sequences; with LN(c + g) 119.3 / 119.7 for 31 x 32K, and 79.9 / 84.2 at d_c 256
  // (ragged); ungated 52.8 / 55.0 and, at d_c 256, 59.0 / 61.3 (ragged; there the warps
  // also polled their queues); 124 / 135 at d_c 512, when its tiles had 36 short MMAs.
  constexpr bool WARP_ISSUE = D_C == 192 && GATE && !GATE_ADD;
  extern __shared__ uint8_t smem_raw[];
  // 1024-byte aligned base (128-byte swizzle atoms); derived by an offset from the
  // __shared__ array so that every access through it stays a shared-memory access
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  Bars& bars = *reinterpret_cast<Bars*>(smem + C::OFF_MISC);
  volatile int* abort_flag = &bars.abort;
  const uint64_t wait_ns = p.wait_ns;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  phase_mark<DBG == 2>(p, 0);
  // beside the attention over a shared prefix most of the grid has no work: out of the
  // way at once (what comes before that kernel, the schedule with it, is complete)
  if constexpr (BESIDE) {
    beside_acquire();
    if (p.starts[blockIdx.x].done) {
      grid_dependency_wait();
      return;
    }
  }
  // a fused launch inside a layer lets the output projection take each SM this
  // kernel leaves, so that its weights stream early
  if (p.early && p.fuse) grid_launch_dependents();

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::RING; ++s) {
      mbar_init(smem_u32(&bars.full[s]), 1);
      mbar_init(smem_u32(&bars.empty[s]), DUMP ? kGateWarps : 1);
    }
    for (int s = 0; s < C::NS; ++s) {
      mbar_init(smem_u32(&bars.zready[s]), kGateWarps);
      if (Q8) mbar_init(smem_u32(&bars.zfree[s]), 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&bars.qfull[s]), 1);
      // the last score MMA of the segment (commit) and the softmax warps' read of its sums
      mbar_init(smem_u32(&bars.qempty[s]), 1 + kSoftWarps);
    }
    for (int s = 0; s < kNB; ++s) {
      // the MMA commit plus a release arrival of the MMA warp after it saw the
      // gate's zready (so that the statistics are visible to the softmax warps)
      mbar_init(smem_u32(&bars.sready[s]), 2);
      mbar_init(smem_u32(&bars.sfree[s]), kSoftWarps);
    }
    for (int s = 0; s < C::NP; ++s) {
      mbar_init(smem_u32(&bars.spdone[s]), kSoftWarps);
      mbar_init(smem_u32(&bars.pfree[s]), 1);
    }
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
    if (!Q8) prefetch_tensormap(&cmap);
    prefetch_tensormap(&krmap);
  }
  if constexpr (ZZ) {
    constexpr uint32_t one2 = 0x3f803f80u;   // (no other write reaches these rows)
    for (int i = threadIdx.x; i < C::NS * C::NCH * 64; i += kThreads)
      *reinterpret_cast<uint4*>(smem + i / 64 * C::ZCHUNK + C::PCHUNK + i % 64 * 16) = make_uint4(one2, one2, one2, one2);
    fence_proxy_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  phase_mark<DBG == 2>(p, 1);
  const uint32_t tmem = bars.tmem_base;
  // Everything above touches only this CTA's shared and tensor memory; what
  // follows reads the query-absorption kernel's outputs (prepared queries,
  // split schedule, zeroed counters) and the cache it may have appended to.
  if constexpr (!BESIDE) grid_dependency_wait();

  // an issuer's wait, the choice of the thread that issues, and the warp's joining after it
  auto issuer_wait = [&](uint64_t& bar, uint32_t parity) {
    return WARP_ISSUE ? warp_wait(smem_u32(&bar), parity, abort_flag, wait_ns)
                      : mbar_wait(smem_u32(&bar), parity, abort_flag, wait_ns);
  };
  auto issuer_one = [] { return !WARP_ISSUE || elect_one(); };
  auto issuer_join = [] {
    if (WARP_ISSUE) __syncwarp();
  };

  if (warp == kTmaWarp) {
    // ---------------------------------------------------------------- TMA producer
    // The whole warp walks the tiles; lane 0 waits for the slot and issues the
    // copies.  A slot is free once the output MMA of the tile that held it is
    // complete.
    const uint64_t pol_stream = policy_evict_first();
    Walker<C::TOK> w;
    w.start(p);
    PageWindow pw;
    pw.init(p, lane);
    Tile t;
    int it = 0;
    int last_it[6] = {-1, -1, -1, -1, -1, -1};
    Tracer tr;
    tr.init(p, 0);
    if (lane != 0) tr.base = nullptr;
    bool ok_loop = true;
    while (ok_loop && w.next(t)) {
      const int pg = pw.page(p, t, lane);
      const int slot = it % C::RING;
      if (lane == 0) {
        tr.mark(0, it);
        if (!mbar_wait(smem_u32(&bars.empty[slot]), ((it / C::RING) & 1) ^ 1, abort_flag, wait_ns)) ok_loop = false;
        if (ok_loop) {
          tr.mark(1, it);
          const bool ok = pg >= 0 && pg < p.num_pages;
          if (!ok) report_status(p.status, kStatusOutOfRange);
          // (test entry) a withheld page: no copy and no arrival, so that the
          // gate's wait on this slot runs out
          const bool withheld = static_cast<int>(blockIdx.x) == p.stall_cta && it == p.stall_tile;
          if (!withheld) {
            const uint32_t fb = smem_u32(&bars.full[slot]);
            mbar_arrive_expect_tx(fb, ok ? C::PAGE_TX + C::ID_TX : 0u);
            const int y = pg * kPage + t.tok0 % kPage;
            if (Q8) {
              if (ok) {
                const uint32_t dst = sbase + C::OFF_RAW + slot * C::RSLOT, meta = sbase + C::OFF_META + slot * C::RMETA;
                bulk_load_hint(dst + C::PCHUNK, p.c8 + static_cast<size_t>(y) * D_C, C::TOK * D_C, fb, pol_stream);
                tma_load_3d(dst, &krmap, 0, y, 0, fb, pol_stream);
                bulk_load_hint(meta, p.scales + y, C::TOK * 4, fb, pol_stream);
                if (C::ID_TX)
                  bulk_load_hint(meta + kPage * 4, p.id_pool + static_cast<size_t>(pg) * kPage, C::ID_TX, fb, pol_stream);
              }
            } else if (ok) {
              const uint32_t dst = sbase + slot * C::SLOT;
              tma_load_3d(dst, &cmap, 0, y, 0, fb, pol_stream);
              tma_load_3d(dst + C::KR_OFF, &krmap, 0, y, 0, fb, pol_stream);
              // the page's token ids, into the half of the slot's statistics that
              // holds r once the gate has read them
              if (C::ID_TX)
                bulk_load_hint(sbase + C::OFF_STAT + slot * C::STAT_BYTES + kPage * 4,
                               p.id_pool + static_cast<size_t>(pg) * kPage, C::ID_TX, fb, pol_stream);
            }
            last_it[slot] = it;
          }
          tr.mark(2, it);
        }
      }
      // The first page alone: every CTA asks for one page, and the rest only
      // once it has landed, so that the first pages of all CTAs land early
      // (one page per SM) instead of in a burst of all their slots.
      if (it == 0 && lane == 0 && ok_loop && last_it[0] == 0 &&
          !mbar_wait(smem_u32(&bars.full[0]), 0, abort_flag, wait_ns))
        ok_loop = false;
      ok_loop = __shfl_sync(0xffffffffu, ok_loop, 0);
      ++it;
    }
    if (lane == 0) {
      // The split combine may take its place once every CTA's last page is
      // requested, a few microseconds before this kernel ends.  Never before the
      // kernel before the call, which may write W_UV, is complete: the combine copies
      // W_UV before its own wait.  This kernel's wait stands for that; beside the
      // attention over a shared prefix, where the wait comes at the end, the
      // absorption's does, after which alone it let the gate (and that the attention,
      // and that this kernel) start.  (At the start it
      // would crowd its blocks onto the first SMs to free up: 128 ragged
      // sequences 69.8 us against 68.2).  128 at d_c 512 119.7 -> 118.5 us, 32 x
      // 4K 37.7 -> 37.2, 64 x 8K layer 102.4 -> 101.5 (against a trigger at the
      // start), at d_c 192 91.3 -> 90.8; outside layers d_c 192 lost (67.7 ->
      // 67.9, 32 x 4K 33.7 -> 33.9).
      if (!p.fuse && (D_C > 192 || p.early)) grid_launch_dependents();
      // drain: every copy this thread issued must land before the CTA exits,
      // also after an abort (own flag: the wait is bounded but not cut short)
      volatile int own = 0;
      for (int s = 0; s < C::RING; ++s)
        if (last_it[s] >= 0 && !mbar_wait(smem_u32(&bars.full[s]), (last_it[s] / C::RING) & 1, &own, wait_ns)) *abort_flag = 1;
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- score MMAs, query blocks
    // Scores of tile js: at a segment start the segment's query block, a free score
    // buffer (the softmax warps read tile js - kNB's), and the gated page.  The
    // next segment's query block is requested once its buffer's previous segment
    // is done with it (last score MMA complete, sums read by the softmax warps),
    // tested after every tile.  Loops are unrolled with compile-time accumulate
    // flags.
    if (!DUMP && (WARP_ISSUE || elect_one())) {
      constexpr uint32_t IDESC_S = idesc_bf16(64, kHeads, 0, 0);
      // A operand: the page slot, 128-byte swizzled, K-major (tokens x
      // features); B: the query block in 8x8 core matrices, K cores 256 B
      // apart, head halves 128 B apart
      const uint64_t zdesc_k = smem_desc(sbase, 16, 1024, kSwizzle128B);
      const uint64_t qdesc0 = smem_desc(sbase + C::OFF_QBUF, kQGroupBytes, kQRowGroupBytes, kSwizzleNone);
      // half pages: two latent columns per MMA.  The 64 rows of the A operand at an
      // even column are its 32 tokens and the next column's 32, B's N = 32 the two
      // columns' query values; the scores are D's two diagonal blocks (the others
      // are not used), added by the softmax warps.  The MMAs are bound by the
      // operand bytes they read from shared memory, 59 KB per half page against 92
      // with a column at a time and half the rows unused: 128 ragged sequences at
      // d_c 512 118.4 -> 106.2 us.
      constexpr uint32_t IDESC_S2 = idesc_bf16(64, 2 * kHeads, 0, 0);
      const uint64_t qdesc2 = smem_desc(sbase + C::OFF_QBUF, 2 * kQGroupBytes, kQRowGroupBytes, kSwizzleNone);
      Walker<C::TOK> ws, wq;
      ws.start(p);
      wq.start(p);
      Tile ts, tq;
      bool q_more = wq.next(tq), q_walk = false;   // q_walk: tq's block is requested, the next segment not found yet
      int qn = 0, seg = -1;   // query blocks requested, segment of the scores
      bool issued = false;
      Tracer tr;
      tr.init(p, 1, 0, 2);
      if (WARP_ISSUE && lane != 0) tr.base = nullptr;
      auto find_query = [&]() {
        while (q_walk) {
          q_more = wq.next(tq);
          q_walk = q_more && !tq.first;
        }
      };
      // the next segment's query block (its buffer is free)
      auto load_query = [&]() {
        const int qb = qn % C::NQ;
        if (issuer_one()) {
          mbar_arrive_expect_tx(smem_u32(&bars.qfull[qb]), C::QPREP);
          bulk_load(sbase + C::OFF_QBUF + qb * C::QBUF, p.qprep + static_cast<size_t>(tq.b) * C::QPREP, C::QPREP,
                    smem_u32(&bars.qfull[qb]));
        }
        issuer_join();
        ++qn;
        q_walk = true;
      };
      auto query_free = [&]() {   // the next query block's buffer, tested without waiting
        const uint32_t bar = smem_u32(&bars.qempty[qn % C::NQ]), parity = ((qn / C::NQ) & 1) ^ 1;
        return WARP_ISSUE ? warp_test(bar, parity) : mbar_test_now(bar, parity);
      };
      for (int js = 0; ws.next(ts); ++js) {
        const int slot = js % C::NS, sb = js % kNB;
        bool ok = true;
        if (ts.first) {
          ++seg;
          if (qn <= seg) {
            find_query();
            ok = issuer_wait(bars.qempty[seg % C::NQ], ((seg / C::NQ) & 1) ^ 1);
            if (ok) load_query();
          }
        }
        if (ts.first) ok = ok && issuer_wait(bars.qfull[seg % C::NQ], (seg / C::NQ) & 1);
        ok = ok && issuer_wait(bars.sfree[sb], ((js / kNB) & 1) ^ 1);
        ok = ok && issuer_wait(bars.zready[slot], (js / C::NS) & 1);
        if (!ok) break;
        tr.mark(1, js);
        tc_fence_after();
        if (issuer_one()) {
          mbar_arrive(smem_u32(&bars.sready[sb]));
          const uint64_t za = zdesc_k + ((slot * C::SLOT) >> 4);
          const uint64_t ka = Q8 ? zdesc_k + ((C::OFF_RAW + js % C::RING * C::RSLOT) >> 4) : za + (C::KR_OFF >> 4);
          const uint64_t qb = qdesc0 + (((seg % C::NQ) * C::QBUF) >> 4);
          const uint32_t ds = tmem + C::COL_S + sb * C::S_COLS;
          if constexpr (C::TOK < kPage) {
            const uint64_t qb2 = qdesc2 + (((seg % C::NQ) * C::QBUF) >> 4);
#pragma unroll
            for (int kk = 0; kk < D_C / 32; ++kk)
              mma_bf16_ss(ds, za + (((kk >> 2) * 2 * C::PCHUNK + (kk & 3) * 32) >> 4),
                          qb2 + ((kk * 4 * kQGroupBytes) >> 4), IDESC_S2, kk > 0);
#pragma unroll
            for (int kk = 0; kk < kRope / 16; ++kk)
              mma_bf16_ss(ds, ka + ((kk * 32) >> 4),
                          qb + ((C::QB_LAT + kk * 2 * kQGroupBytes) >> 4), IDESC_S, 1);
          } else {
#pragma unroll
            for (int kk = 0; kk < D_C / 16; ++kk)
              mma_bf16_ss(ds, za + (((kk >> 2) * C::ZCHUNK + (kk & 3) * 32) >> 4),
                          qb + ((kk * 2 * kQGroupBytes) >> 4), IDESC_S, kk > 0);
#pragma unroll
            for (int kk = 0; kk < kRope / 16; ++kk)
              mma_bf16_ss(ds + kHeads, ka + ((kk * 32) >> 4),
                          qb + ((C::QB_LAT + kk * 2 * kQGroupBytes) >> 4), IDESC_S, kk > 0);
          }
          if constexpr (ZZ) {
            constexpr uint32_t IDESC_ZZ = idesc_bf16(64, C::ZZ_COLS, 0, 0);
#pragma unroll
            for (int kk = 0; kk < D_C / 16; ++kk) {
              const uint64_t zk = za + (((kk >> 2) * C::ZCHUNK + (kk & 3) * 32) >> 4);
              mma_bf16_ss(tmem + C::COL_ZZ + sb * C::ZZ_COLS, zk, zk, IDESC_ZZ, kk > 0);
            }
          }
          mma_commit(smem_u32(&bars.sready[sb]));
          if (Q8) mma_commit(smem_u32(&bars.empty[js % C::RING]));
          if (ts.last) mma_commit(smem_u32(&bars.qempty[seg % C::NQ]));
        }
        issuer_join();
        tr.mark(2, js);
        issued = true;
        // (after the tile's MMAs: finding the next segment takes global loads)
        find_query();
        if (q_more && query_free()) load_query();
      }
      // drain: the query-block copies land and every MMA finishes before the
      // CTA exits and TMEM is released (own flag: bounded but not cut short by
      // an abort)
      volatile int own = 0;
      for (int n = qn > C::NQ ? qn - C::NQ : 0; n < qn; ++n)
        if (!mbar_wait(smem_u32(&bars.qfull[n % C::NQ]), (n / C::NQ) & 1, &own, wait_ns)) *abort_flag = 1;
      if (issued) {
        if (issuer_one()) mma_commit(smem_u32(&bars.drain_s));
        issuer_join();
        if (!mbar_wait(smem_u32(&bars.drain_s), 0, &own, wait_ns)) *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp == kOutWarp) {
    // ---------------------------------------------------------------- output MMAs
    // O^T[feature, head] += Z^T P' for each tile in order, as soon as the
    // softmax warps wrote its P'; completion frees the page slot and the P'
    // buffer.  A operand: the page slot read MN-major (features along M,
    // 64-feature atoms ZCHUNK apart; tokens along K, 8-row groups 1 KB apart);
    // B: P' MN-major in 8x8 core matrices (token groups 256 B, head halves
    // 128 B).
    if (!DUMP && (WARP_ISSUE || elect_one())) {
      constexpr uint32_t IDESC_O = idesc_bf16(128, kHeads, 1, 1);
      const uint64_t zdesc_mn = smem_desc(sbase, C::ZCHUNK, 1024, kSwizzle128B);
      const uint64_t pdesc0 = smem_desc(sbase + C::OFF_PBUF, 256, 128, kSwizzleNone);
      Walker<C::TOK> wo;
      wo.start(p);
      Tile to;
      bool issued = false;
      Tracer tr;
      tr.init(p, 1, 1, 2);   // second half of the MMA role's run
      if (WARP_ISSUE && lane != 0) tr.base = nullptr;
      for (int jo = 0; wo.next(to); ++jo) {
        if (!issuer_wait(bars.spdone[jo % C::NP], (jo / C::NP) & 1)) break;
        tr.mark(3, jo);
        tc_fence_after();
        if (issuer_one()) {
          const int slot = jo % C::NS;
          const uint64_t za = zdesc_mn + ((slot * C::SLOT) >> 4);
          const uint64_t pb = pdesc0 + (((jo % C::NP) * C::PBUF) >> 4);
          const uint32_t keep = to.first ? 0u : 1u;   // a segment's first MMAs overwrite O^T
#pragma unroll
          for (int ks = 0; ks < C::TOK / 16; ++ks)
#pragma unroll
            for (int mc = 0; mc < C::NMC; ++mc)
              mma_bf16_ss(tmem + C::COL_O + kHeads * mc, za + (((C::mc_start(mc) / 64) * C::ZCHUNK + ks * 2048) >> 4),
                          pb + ((ks * 512) >> 4), IDESC_O, ks > 0 ? 1u : keep);
          mma_commit(smem_u32(Q8 ? &bars.zfree[slot] : &bars.empty[slot]));
          mma_commit(smem_u32(&bars.pfree[jo % C::NP]));
        }
        issuer_join();
        tr.mark(4, jo);
        issued = true;
      }
      if (issued) {
        if (issuer_one()) mma_commit(smem_u32(&bars.drain_o));
        issuer_join();
        volatile int own = 0;
        if (!mbar_wait(smem_u32(&bars.drain_o), 0, &own, wait_ns)) *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp >= kGateWarp0) {
    // ---------------------------------------------------------------- gate: z = c (*) g, LN statistics
    // Quarter-warp k = 4 (warp - 7) + lane / 8 owns token rows 2k (lanes 0-3)
    // and 2k + 1 (lanes 4-7); lane p = lane % 4 of a row takes the 16-byte
    // units 2p and 2p + 1 of every 64-feature column.  The gate-row load of a
    // column is then one 32-byte load per lane and a whole 128-byte line per
    // row (the load/store data path pays per instruction and per line, so
    // fewer, wider loads are cheaper), and a quarter-warp's shared-memory
    // accesses to the swizzled page still hit eight distinct bank groups (the
    // two rows differ in swizzle parity).  The gate rows come from L2 (the
    // table stays there under an evict-last hint while the cache stream is
    // evict-first).  The token ids come with the page (the producer copies them
    // into the slot), so the gate rows of the next tile are requested as soon
    // as its page has landed, while this tile is processed; no load sits on a
    // chain of dependent global accesses.
    const int gw = warp - kGateWarp0;
    const int pp = lane % kGateLanesPerRow;
    const int row = gw * (32 / kGateLanesPerRow) + lane / kGateLanesPerRow;
    const uint64_t pol_keep = policy_evict_last();
    constexpr bool gate_ln = GATE_LN;
    Walker<C::TOK> w;
    w.start(p);
    // id of this thread's row of tile jj, from the slot that holds its page (0
    // past the end of the page)
    auto slot_id = [&](int jj, const Tile& tt) -> int {
      const int32_t* ids = reinterpret_cast<const int32_t*>(
          smem + (Q8 ? C::OFF_META + (jj % C::RING) * C::RMETA : C::OFF_STAT + (jj % C::NS) * C::STAT_BYTES) + kPage * 4);
      return row < tt.ntok ? ids[row] : 0;
    };
    // this thread's part of the gate row of token id (row 0, reported, for an
    // id outside the vocabulary)
    auto g_row = [&](int id) -> const __nv_bfloat16* {
      if ((unsigned)id >= (unsigned)p.vocab) {
        report_status(p.status, kStatusOutOfRange);
        id = 0;
      }
      return p.gate_table + static_cast<size_t>(id) * D_C + pp * 8 * kGateUnits;
    };
    auto load_g = [&](int id, uint4 (&gv)[C::NCH][kGateUnits]) {
      const __nv_bfloat16* src = g_row(id);
#pragma unroll
      for (int fc = 0; fc < C::NCH; ++fc) {
        if constexpr (kGateUnits == 2)
          ldg_32_na_hint(src + fc * 64, pol_keep, gv[fc][0], gv[fc][1]);
        else
          gv[fc][0] = ldg_16_na_hint(src + fc * 64, pol_keep);
      }
    };
    // shared-memory offset of unit (kGateUnits pp + h) of column fc of this thread's row
    auto unit_off = [&](int fc, int h) -> uint32_t {
      return fc * C::ZCHUNK + row * 128 + (((kGateUnits * pp + h) ^ (row & 7)) << 4);
    };
    Tracer tr;
    tr.init(p, 2);
    if (threadIdx.x != kGateWarp0 * 32) tr.base = nullptr;
    // Q8: 16 codes of every 64-feature column of this thread's row, which are the units 2 pp
    // and the next of the column's bf16 values
    uint4 codes[Q8 ? C::NCH : 1];
    Q8Widen widen;
    static_assert(!Q8 || (kGateWarps == 8 && C::TOK == kPage), "rows of the codes");
    Tile t, t1;
    bool have = w.next(t);
    bool have1 = have && w.next(t1);
    if constexpr (Q8 && GATE) {
      // A cache in 8 bits: the gate warps take the longest of all roles here (widening a
      // code costs as much as gating and summing it), so nothing of theirs waits at a tile's
      // start: the next tile's codes and gate rows take the place of this tile's, column by
      // column, as soon as these are used (its copies have landed long before), its ids
      // and scales before that.  (Not with the additive gate at d_c 256, which keeps a tile's
      // values for a second pass and has no registers left: 8 x 32K 53.6 us, so loaded 77.  At
      // 192 128 ragged sequences took 88.0 us without it and take 84.5.)
      constexpr bool AHEAD = !GATE_ADD || D_C == 192;
      uint4 g[C::NCH][2];
      float scale = 0.f;
      auto raw_of = [&](int jj) { return smem + C::OFF_RAW + (jj % C::RING) * C::RSLOT + C::PCHUNK + row * D_C + 16 * pp; };
      auto scale_of = [&](int jj) {
        return reinterpret_cast<const float*>(smem + C::OFF_META + (jj % C::RING) * C::RMETA)[row];
      };
      if (have) have = warp_wait(smem_u32(&bars.full[0]), 0, abort_flag, wait_ns);
      bool loaded = false;
      for (int j = 0; have; ++j) {
        const int slot = j % C::NS;
        tr.mark(0, j);
        if (!loaded) {
          if (!warp_wait(smem_u32(&bars.full[j % C::RING]), (j / C::RING) & 1, abort_flag, wait_ns)) break;
          load_g(slot_id(j, t), g);
          scale = scale_of(j);
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc) codes[fc] = *reinterpret_cast<const uint4*>(raw_of(j) + fc * 64);
        }
        tr.mark(1, j);
        widen.set(scale);
        const bool more = widen.unfinished();
        loaded = AHEAD && have1 && warp_test(smem_u32(&bars.full[(j + 1) % C::RING]), ((j + 1) / C::RING) & 1);
        const uint8_t* raw_next = raw_of(j + 1);
        const __nv_bfloat16* g_next = p.gate_table;
        if (loaded) {
          g_next = g_row(slot_id(j + 1, t1));
          scale = scale_of(j + 1);
        }
        auto load_next = [&](int fc) {
          if (AHEAD && loaded) {
            ldg_32_na_hint(g_next + fc * 64, pol_keep, g[fc][0], g[fc][1]);
            codes[fc] = *reinterpret_cast<const uint4*>(raw_next + fc * 64);
          }
        };
        auto latent = [&](int fc, int h) {
          uint4 c = widen.unit(h ? codes[fc].z : codes[fc].x, h ? codes[fc].w : codes[fc].y);
          if (more) widen.finish(c);
          return c;
        };
        // the latent slot of the tile (output MMAs of the tile NS before it complete)
        if (!warp_wait(smem_u32(&bars.zfree[slot]), ((j / C::NS) & 1) ^ 1, abort_flag, wait_ns)) break;
        tr.mark(5, j);
        uint8_t* zpage = smem + slot * C::SLOT;
        float* st = reinterpret_cast<float*>(smem + C::OFF_STAT + slot * C::STAT_BYTES);
        const bool full_page = t.ntok == C::TOK, valid = row < t.ntok;
        float2 s1 = make_float2(0.f, 0.f), s2 = s1, a1 = s1, a2 = s1;
        auto row_sums = [&](float& sum1, float& sum2) {
          s1 = __fadd2_rn(s1, a1);
          s2 = __fadd2_rn(s2, a2);
          sum1 = s1.x + s1.y;
          sum2 = s2.x + s2.y;
#pragma unroll
          for (int o = 1; o < kGateLanesPerRow; o <<= 1) {
            sum1 += __shfl_xor_sync(0xffffffffu, sum1, o);
            sum2 += __shfl_xor_sync(0xffffffffu, sum2, o);
          }
        };
        constexpr float inv_dc = 1.f / D_C;
        if constexpr (GATE_ADD) {
          // (as below without the 8 bits: centred before the rounding; the same sums.  The codes are
          // widened once and kept for the second pass: 8 x 32K tokens 69.3 us, so 55.8, with the
          // sums from the bf16 values 53.6)
          uint4 wide[C::NCH][2];
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 c4 = latent(fc, h);
              wide[fc][h] = c4;
              const uint32_t* cw = reinterpret_cast<const uint32_t*>(&c4);
              const uint32_t* gw2 = reinterpret_cast<const uint32_t*>(&g[fc][h]);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 zf = add_bf16x2(cw[k], gw2[k]);
                s1 = __fadd2_rn(s1, zf);
                s2 = __ffma2_rn(zf, zf, s2);
              }
            }
          float sum1, sum2;
          row_sums(sum1, sum2);
          const float mu = sum1 * inv_dc;
          const float r = rsqrtf(fmaxf(sum2 * inv_dc - mu * mu, 0.f) + p.eps);
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 c4 = wide[fc][h];
              const uint32_t* cw = reinterpret_cast<const uint32_t*>(&c4);
              const uint32_t* gw2 = reinterpret_cast<const uint32_t*>(&g[fc][h]);
              uint4 z;
              uint32_t* zw = reinterpret_cast<uint32_t*>(&z);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 zf = __fadd2_rn(add_bf16x2(cw[k], gw2[k]), make_float2(-mu, -mu));
                zw[k] = pack_bf16x2(zf.x, zf.y);
              }
              if (!full_page && !valid) z = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(zpage + unit_off(fc, h)) = z;
            }
            load_next(fc);
          }
          if (pp == 0) {
            st[row] = 0.f;
            st[kPage + row] = valid ? r : 1.f;
          }
        } else {
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 c4 = latent(fc, h);
              uint4 z;
              z.x = mul_bf16x2(c4.x, g[fc][h].x);
              z.y = mul_bf16x2(c4.y, g[fc][h].y);
              z.z = mul_bf16x2(c4.z, g[fc][h].z);
              z.w = mul_bf16x2(c4.w, g[fc][h].w);
              if (!full_page && !valid) z = make_uint4(0, 0, 0, 0);
              if (GATE_LN && !ZZ) {
                sum_bf16x2(z.x, s1, s2);
                sum_bf16x2(z.y, a1, a2);
                sum_bf16x2(z.z, s1, s2);
                sum_bf16x2(z.w, a1, a2);
              }
              *reinterpret_cast<uint4*>(zpage + unit_off(fc, h)) = z;
            }
            // (the first column's with the second's: one task fewer among the first stores)
            if (fc == 1) load_next(0);
            if (fc > 0) load_next(fc);
          }
          tr.mark(6, j);
          if constexpr (!ZZ) {
            float mu = 0.f, r = 1.f;
            if (GATE_LN) {
              float sum1, sum2;
              row_sums(sum1, sum2);
              mu = sum1 * inv_dc;
              r = rsqrtf(fmaxf(sum2 * inv_dc - mu * mu, 0.f) + p.eps);
            }
            if (pp == 0) {
              st[row] = valid ? mu : 0.f;
              st[kPage + row] = valid ? r : 1.f;
            }
          }
        }
        tr.mark(2, j);
        fence_proxy_async_smem();
        warp_arrive(smem_u32(&bars.zready[slot]));
        tr.mark(3, j);
        t = t1;
        have = have1;
        have1 = have1 && w.next(t1);
      }
      have = false;
    }
    uint4 gcur[C::NCH][kGateUnits], gnext[C::NCH][kGateUnits];
    int id0 = 0;
    if (!Q8 && GATE && have) {
      // the first tile's rows: its page must land first
      if (warp_wait(smem_u32(&bars.full[0]), 0, abort_flag, wait_ns)) {
        id0 = slot_id(0, t);
        load_g(id0, gcur);
      } else {
        have = false;
      }
    }
    int j = 0;
    while (have) {
      const int slot = j % C::NS;
      tr.mark(0, j);
      // The next tile's gate rows: if its page has landed, requested column by
      // column between this tile's shared-memory stores (spreading the loads
      // over the tile instead of one burst), otherwise after this tile.
      bool next_issued = false;
      const __nv_bfloat16* gsrc_next = p.gate_table;
      if (GATE && have1 && warp_test(smem_u32(&bars.full[(j + 1) % C::RING]), ((j + 1) / C::RING) & 1)) {
        gsrc_next = g_row(slot_id(j + 1, t1));
        next_issued = true;
      }
      auto load_next_column = [&](int fc) {
        if (next_issued) {
          if constexpr (kGateUnits == 2)
            ldg_32_na_hint(gsrc_next + fc * 64, pol_keep, gnext[fc][0], gnext[fc][1]);
          else
            gnext[fc][0] = ldg_16_na_hint(gsrc_next + fc * 64, pol_keep);
        }
      };
      if (!warp_wait(smem_u32(&bars.full[j % C::RING]), (j / C::RING) & 1, abort_flag, wait_ns)) break;
      tr.mark(1, j);
      if (DUMP) id0 = slot_id(j, t);
      uint8_t* cpage = smem + slot * C::SLOT;
      if (DUMP) {
        if (row < t.ntok) {
          const size_t o = static_cast<size_t>(t.b) * p.dump_len + t.tok0 + row;
          uint4* dc = reinterpret_cast<uint4*>(p.dump_c + o * D_C);
          uint4* dg = reinterpret_cast<uint4*>(p.dump_g + o * D_C);
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
            for (int h = 0; h < kGateUnits; ++h) {
              dc[fc * 8 + kGateUnits * pp + h] = *reinterpret_cast<const uint4*>(cpage + unit_off(fc, h));
              dg[fc * 8 + kGateUnits * pp + h] = gcur[fc][h];
            }
          }
#pragma unroll
          for (int h = 0; h < kGateUnits; ++h)
            reinterpret_cast<uint4*>(p.dump_kr + o * kRope)[kGateUnits * pp + h] = *reinterpret_cast<const uint4*>(
                cpage + C::KR_OFF + row * 128 + (((kGateUnits * pp + h) ^ (row & 7)) << 4));
          if (pp == 0) p.dump_ids[o] = id0;
        }
#pragma unroll
        for (int fc = 0; fc < C::NCH; ++fc) load_next_column(fc);
        warp_arrive(smem_u32(&bars.empty[slot]));
      } else {
        const bool full_page = t.ntok == C::TOK;   // uniform: no token masking needed
        if constexpr (Q8) {
          // (ungated: the values alone)
          const uint8_t* raw = smem + C::OFF_RAW + (j % C::RING) * C::RSLOT + C::PCHUNK + row * D_C + 16 * pp;
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc) codes[fc] = *reinterpret_cast<const uint4*>(raw + fc * 64);
          widen.set(reinterpret_cast<const float*>(smem + C::OFF_META + (j % C::RING) * C::RMETA)[row]);
          const bool more = widen.unfinished();
          // the latent slot of the tile (output MMAs of the tile NS before it complete)
          if (!warp_wait(smem_u32(&bars.zfree[slot]), ((j / C::NS) & 1) ^ 1, abort_flag, wait_ns)) break;
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint4 z = widen.unit(h ? codes[fc].z : codes[fc].x, h ? codes[fc].w : codes[fc].y);
              if (more) widen.finish(z);
              if (row >= t.ntok) z = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(cpage + unit_off(fc, h)) = z;
            }
          }
        } else if (GATE) {
          float* st = reinterpret_cast<float*>(smem + C::OFF_STAT + slot * C::STAT_BYTES);
          // all shared-memory reads of this thread's units first (the in-place
          // stores below would otherwise order every later load behind them)
          uint4 cv[C::NCH][kGateUnits];
#pragma unroll
          for (int fc = 0; fc < C::NCH; ++fc)
#pragma unroll
            for (int h = 0; h < kGateUnits; ++h) cv[fc][h] = *reinterpret_cast<const uint4*>(cpage + unit_off(fc, h));
          tr.mark(5, j);
          const bool valid = row < t.ntok;
          if constexpr (GATE_ADD) {
            // ablation LN(c + g): c + g is exact in fp32; the row is centred by its
            // mean before the bf16 rounding (LN is shift-invariant), so the rounding
            // error is relative to the spread LN keeps, not to the gate's offset
            float2 s1 = make_float2(0.f, 0.f), s2 = make_float2(0.f, 0.f);
#pragma unroll
            for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
              for (int h = 0; h < kGateUnits; ++h) {
                const uint32_t* cw = reinterpret_cast<const uint32_t*>(&cv[fc][h]);
                const uint32_t* gw2 = reinterpret_cast<const uint32_t*>(&gcur[fc][h]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float2 zf = __fadd2_rn(unpack_bf16x2(cw[k]), unpack_bf16x2(gw2[k]));
                  s1 = __fadd2_rn(s1, zf);
                  s2 = __ffma2_rn(zf, zf, s2);
                }
              }
            }
            float sum1 = s1.x + s1.y, sum2 = s2.x + s2.y;
#pragma unroll
            for (int o = 1; o < kGateLanesPerRow; o <<= 1) {
              sum1 += __shfl_xor_sync(0xffffffffu, sum1, o);
              sum2 += __shfl_xor_sync(0xffffffffu, sum2, o);
            }
            constexpr float inv_dc = 1.f / D_C;
            const float mu = sum1 * inv_dc;
            const float var = fmaxf(sum2 * inv_dc - mu * mu, 0.f);
            const float r = rsqrtf(var + p.eps);
            const float2 mu2v = make_float2(mu, mu);
#pragma unroll
            for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
              for (int h = 0; h < kGateUnits; ++h) {
                const uint32_t* cw = reinterpret_cast<const uint32_t*>(&cv[fc][h]);
                const uint32_t* gw2 = reinterpret_cast<const uint32_t*>(&gcur[fc][h]);
                uint4 z;
                uint32_t* zw = reinterpret_cast<uint32_t*>(&z);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float2 zf = __fadd2_rn(__fadd2_rn(unpack_bf16x2(cw[k]), unpack_bf16x2(gw2[k])),
                                               make_float2(-mu2v.x, -mu2v.y));
                  zw[k] = pack_bf16x2(zf.x, zf.y);
                }
                if (!full_page && !valid) z = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(cpage + unit_off(fc, h)) = z;
              }
              load_next_column(fc);
            }
            tr.mark(6, j);
            if (pp == 0) {
              // the stored z is centred; rows past the page end get r = 1 (their
              // weight is 0, and l adds 0 / r)
              st[row] = 0.f;
              st[kPage + row] = valid ? r : 1.f;
            }
          } else {
            float2 s1 = make_float2(0.f, 0.f), s2 = make_float2(0.f, 0.f);
            float2 a1 = make_float2(0.f, 0.f), a2 = make_float2(0.f, 0.f);
#pragma unroll
            for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
              for (int h = 0; h < kGateUnits; ++h) {
                uint4 z;
                z.x = mul_bf16x2(cv[fc][h].x, gcur[fc][h].x);
                z.y = mul_bf16x2(cv[fc][h].y, gcur[fc][h].y);
                z.z = mul_bf16x2(cv[fc][h].z, gcur[fc][h].z);
                z.w = mul_bf16x2(cv[fc][h].w, gcur[fc][h].w);
                if (!full_page && !valid) z = make_uint4(0, 0, 0, 0);
                const float2 f0 = unpack_bf16x2(z.x), f1 = unpack_bf16x2(z.y);
                const float2 f2 = unpack_bf16x2(z.z), f3 = unpack_bf16x2(z.w);
                s1 = __fadd2_rn(s1, f0);
                a1 = __fadd2_rn(a1, f1);
                s1 = __fadd2_rn(s1, f2);
                a1 = __fadd2_rn(a1, f3);
                s2 = __ffma2_rn(f0, f0, s2);
                a2 = __ffma2_rn(f1, f1, a2);
                s2 = __ffma2_rn(f2, f2, s2);
                a2 = __ffma2_rn(f3, f3, a2);
                *reinterpret_cast<uint4*>(cpage + unit_off(fc, h)) = z;
              }
              load_next_column(fc);
            }
            s1 = __fadd2_rn(s1, a1);
            s2 = __fadd2_rn(s2, a2);
            float sum1 = s1.x + s1.y, sum2 = s2.x + s2.y;
            tr.mark(6, j);
            // row sums over the four lanes of the row (without the LayerNorm
            // ablation's norm: mu = 0, r = 1)
            if (gate_ln) {
#pragma unroll
              for (int o = 1; o < kGateLanesPerRow; o <<= 1) {
                sum1 += __shfl_xor_sync(0xffffffffu, sum1, o);
                sum2 += __shfl_xor_sync(0xffffffffu, sum2, o);
              }
            }
            if (pp == 0) {
              constexpr float inv_dc = 1.f / D_C;
              const float mu = gate_ln ? sum1 * inv_dc : 0.f;
              const float var = fmaxf(sum2 * inv_dc - mu * mu, 0.f);
              const float r = gate_ln ? rsqrtf(var + p.eps) : 1.f;
              // rows past the page end: mu = 0, r = 1 (their weight is 0, and l adds 0 / r)
              st[row] = valid ? mu : 0.f;
              st[kPage + row] = valid ? r : 1.f;
            }
          }
        } else if (!full_page) {
          if (row >= t.ntok && row < C::TOK) {
#pragma unroll
            for (int fc = 0; fc < C::NCH; ++fc)
#pragma unroll
              for (int h = 0; h < kGateUnits; ++h)
                *reinterpret_cast<uint4*>(cpage + unit_off(fc, h)) = make_uint4(0, 0, 0, 0);
          }
        }
        tr.mark(2, j);
        fence_proxy_async_smem();
        warp_arrive(smem_u32(&bars.zready[slot]));
      }
      tr.mark(3, j);
      if (GATE && have1 && !next_issued) {
        // the next page landed only now
        if (!warp_wait(smem_u32(&bars.full[(j + 1) % C::RING]), ((j + 1) / C::RING) & 1, abort_flag, wait_ns)) break;
        load_g(slot_id(j + 1, t1), gnext);
      }
      ++j;
      t = t1;
      have = have1;
      have1 = have1 && w.next(t1);
      if (GATE) {
#pragma unroll
        for (int fc = 0; fc < C::NCH; ++fc) {
#pragma unroll
          for (int h = 0; h < kGateUnits; ++h) gcur[fc][h] = gnext[fc][h];
        }
      }
    }
  } else if (warp < kSoftWarps && !DUMP) {
    // ---------------------------------------------------------------- softmax, output read-out
    // Warp w reads TMEM lane quadrant w: tokens 16w .. 16w + 15 of a tile's
    // scores (rows of the M = 64 accumulator) and latent features 32w .. 32w +
    // 31 of each 128-feature chunk of O^T.  Thread t owns tokens r0 = 16w + t/4
    // and r1 = r0 + 8 and heads hh(k) = 2q, 2q + 1, 8 + 2q, 9 + 2q (q = t % 4).
    // Lane h < 16 of every warp also keeps head h's reference max (the same in
    // all four warps), which the rare slow path of the max update uses.
    const int q = lane & 3;
    const int r0 = 16 * warp + (lane >> 2), r1 = r0 + 8;
    const uint32_t tq = tmem + (static_cast<uint32_t>(32 * warp) << 16);
    const float scale = p.scale_log2;
    float* xmax = reinterpret_cast<float*>(smem + C::OFF_XCH);        // [4 warps][16 heads]
    float* xsum = xmax + kSoftWarps * kHeads;                         // [4 warps][16 heads][2]
    float* xodd = xmax + 256;                                         // half pages: [32 tokens][16 heads]
    auto head_of = [&](int k) { return (k & 1) + 2 * q + 8 * (k >> 1); };
    // gamma and beta of the segment read-out in shared memory (written once by
    // the four warps; the first tile's barrier orders the writes before any read)
    float* gb = reinterpret_cast<float*>(smem + C::OFF_GB);
    if (GATE) {
      for (int f = threadIdx.x; f < D_C; f += kSoftThreads) {
        gb[f] = p.gamma ? __ldg(p.gamma + f) : 1.f;
        gb[D_C + f] = p.beta ? __ldg(p.beta + f) : 0.f;
      }
    }
    float m_ref[4], l_acc[4], bmu_acc[4], wq[4], bsc[4];
    float m16 = -INFINITY;   // head `lane` (lanes 0-15)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m_ref[k] = -INFINITY;
      l_acc[k] = 0.f;
      bmu_acc[k] = 0.f;
      wq[k] = 0.f;
      bsc[k] = 0.f;
    }
    Walker<C::TOK> w;
    w.start(p);
    Tile t;
    int it = 0, seg = -1;
    Tracer tr;
    tr.init(p, 3);
    if (threadIdx.x != 0) tr.base = nullptr;
    // A segment's reference maxima come from its whole first page: the second
    // half-page tile moves them exactly.  A head's largest weight is then more
    // often exactly 1, without the rounding of P' (mean error against 64 bits at
    // d_c 512, ten seeds: 2.311e-3 without, 2.261e-3 with; whole-page tiles 2.284e-3).
    float lazy = kLazyLog2;
    bool was_first = false;
    // ZZ: the softmax is the longest role beside the gate; the next tile is found, and the P'
    // buffer waited for, while the scores come out of TMEM (45.0 -> 44.6 us for 8 x 32K; at
    // d_c 192 without ZZ the same took 76.7 us instead of 73.4 for 128 ragged)
    Tile tn;
    bool next_tile = ZZ && w.next(t);
    while (ZZ ? next_tile : w.next(t)) {
      bool ok = true;
      if constexpr (C::TOK < kPage) {
        lazy = was_first && t.tok0 % kPage != 0 ? 0.f : kLazyLog2;
        was_first = t.first;
      }
      if (t.first) {
        ++seg;
        ok = warp_wait(smem_u32(&bars.qfull[seg % C::NQ]), (seg / C::NQ) & 1, abort_flag, wait_ns);
        if (ok && GATE) {
          // w_h = sum_f bf16(q^ gamma)_hf and b_h = q^_h . beta from their
          // per-chunk partials after the operands, added in chunk order
          const float* sums = reinterpret_cast<const float*>(smem + C::OFF_QBUF + (seg % C::NQ) * C::QBUF +
                                                             C::QB_LAT + qprep_rope_bytes(kRope));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int h = head_of(k);
            float wsum = 0.f, bsum = 0.f;
#pragma unroll
            for (int c = 0; c < D_C / kSumFeatures; ++c) {
              wsum += sums[c * 32 + h];
              bsum += sums[c * 32 + 16 + h];
            }
            wq[k] = wsum;
            bsc[k] = bsum * scale;
          }
        }
        if (ok) warp_arrive(smem_u32(&bars.qempty[seg % C::NQ]));
      }
      const int slot = it % C::NS, sb = it % kNB, pb = it % C::NP;
      tr.mark(0, it);
      // scores of this tile; the MMA warp's release arrival on the same barrier
      // orders the gate's statistics before them
      ok = ok && warp_wait(smem_u32(&bars.sready[sb]), (it / kNB) & 1, abort_flag, wait_ns);
      tr.mark(1, it);
      float s[2][4];
      float mu[2] = {0.f, 0.f}, rr[2] = {1.f, 1.f}, sd[2] = {1.f, 1.f};   // (ZZ: sd = 1 / rr)
      bool exceed = false;
      float v[16];
      if (ok) {
        tc_fence_after();
        tmem_ld_16x256b_x4(tq + C::COL_S + sb * C::S_COLS, v);
        float zz[8], zs[4];
        if constexpr (ZZ) {
          // the diagonal's 16 columns of this warp's rows, and the sums
          const uint32_t dz = tq + C::COL_ZZ + sb * C::ZZ_COLS;
          tmem_ld_16x256b_x2(dz + 16 * warp, zz);
          tmem_ld_16x256b_x1(dz + kPage, zs);
        } else if (GATE) {
          const float* st = reinterpret_cast<const float*>(smem + C::OFF_STAT + slot * C::STAT_BYTES);
          mu[0] = st[r0];
          mu[1] = st[r1];
          rr[0] = st[kPage + r0];
          rr[1] = st[kPage + r1];
        }
        if constexpr (ZZ) {
          tn = t;
          next_tile = w.next(tn);
          ok = warp_wait(smem_u32(&bars.pfree[pb]), ((it / C::NP) & 1) ^ 1, abort_flag, wait_ns);
        }
        tmem_wait_ld();
        if constexpr (ZZ) {
          // row i = lane / 4 of the warp's has its square sum in column i, held by lane 4 i +
          // i / 2, row i + 8 in column i + 8
          const int i = lane >> 2, owner = (lane & ~3) | (i >> 1);
          constexpr float inv_dc = 1.f / D_C;
          const float sq[2] = {__shfl_sync(0xffffffffu, i & 1 ? zz[1] : zz[0], owner),
                               __shfl_sync(0xffffffffu, i & 1 ? zz[7] : zz[6], owner)};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            mu[e] = zs[2 * e] * inv_dc;
            const float var = fmaxf(fmaf(sq[e], inv_dc, -mu[e] * mu[e]), 0.f) + p.eps;
            rr[e] = rsqrtf(var);
            sd[e] = var * rr[e];
          }
        }
        tc_fence_before();
        warp_arrive(smem_u32(&bars.sfree[sb]));   // score buffer read: tile it + kNB may overwrite it
        tr.mark(7, it);
        if constexpr (C::TOK < kPage) {
          // rows 32 .. 63 are the odd columns' part of tokens 0 .. 31: to their owners
          if (warp >= 2) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int hp = 0; hp < 2; ++hp)
                *reinterpret_cast<float2*>(xodd + ((e ? r1 : r0) - C::TOK) * kHeads + head_of(2 * hp)) =
                    make_float2(v[8 + hp * 4 + 2 * e], v[8 + hp * 4 + 2 * e + 1]);
          }
        }
      }
      if constexpr (C::TOK < kPage) soft_sync(kBarXch);   // (every warp, also after an error)
      if (ok) {
        const bool full_page = t.ntok == kPage;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool valid = full_page || (e ? r1 : r0) < t.ntok;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float lat = v[(k >> 1) * 4 + 2 * e + (k & 1)];
            const float rope = C::TOK == kPage ? v[8 + (k >> 1) * 4 + 2 * e + (k & 1)]
                               : warp < 2      ? xodd[(e ? r1 : r0) * kHeads + head_of(k)]
                                               : 0.f;
            float x;
            if (GATE) {
              x = fmaf(rr[e] * scale, fmaf(-mu[e], wq[k], lat), fmaf(rope, scale, bsc[k]));
            } else {
              x = (lat + rope) * scale;
            }
            s[e][k] = valid ? x : -INFINITY;
            exceed = exceed || (x > m_ref[k] + lazy && valid);
          }
        }
      }
      tr.mark(8, it);
      // one vote of the four warps: a head's reference max must move (or a
      // wait failed somewhere)
      if (soft_vote(kBarTile, exceed || !ok)) {
        if (soft_vote(kBarTile, !ok)) break;   // uniform: every warp leaves
        // ---- slow path: tile maxima of the heads over the 64 tokens
        float tm[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) tm[k] = fmaxf(s[0][k], s[1][k]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
          for (int k = 0; k < 4; ++k) tm[k] = fmaxf(tm[k], __shfl_xor_sync(0xffffffffu, tm[k], o));
        if (lane < 4) {
#pragma unroll
          for (int k = 0; k < 4; ++k) xmax[warp * kHeads + head_of(k)] = tm[k];
        }
        soft_sync(kBarXch);
        // lane h < 16: the new reference of head h and the factor for what was
        // accumulated against the old one (the same in every warp)
        float alpha = 1.f;
        if (lane < kHeads) {
          const float tmax = fmaxf(fmaxf(xmax[lane], xmax[kHeads + lane]),
                                   fmaxf(xmax[2 * kHeads + lane], xmax[3 * kHeads + lane]));
          if (m16 == -INFINITY) {
            m16 = tmax;
            alpha = 0.f;
          } else if (tmax > m16 + lazy) {
            alpha = ex2_approx(m16 - tmax);
            m16 = tmax;
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) m_ref[k] = __shfl_sync(0xffffffffu, m16, head_of(k));
        if (!t.first && __any_sync(0xffffffffu, lane < kHeads && alpha != 1.f)) {
          // O^T and the running sums were accumulated against the old
          // reference: the previous tile's output MMA must be complete first
          // (completion n of pfree[b] is output MMA n NP + b)
          const int pv = (it - 1) % C::NP;
          ok = warp_wait(smem_u32(&bars.pfree[pv]), ((it - 1) / C::NP) & 1, abort_flag, wait_ns);
          if (ok) {
            tc_fence_after();
#pragma unroll
            for (int m2 = 0; m2 < C::NMC / 2; ++m2) {   // two M chunks at a time
              float o[32];
              tmem_ld32(tq + C::COL_O + 32 * m2, o);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 32; ++c) o[c] *= __shfl_sync(0xffffffffu, alpha, c & 15);
              tmem_st32(tq + C::COL_O + 32 * m2, o);
            }
            tmem_wait_st();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float a = __shfl_sync(0xffffffffu, alpha, head_of(k));
              l_acc[k] *= a;
              bmu_acc[k] *= a;
            }
          }
        }
      }
      // the P' buffer of this tile is free once the output MMA NP tiles back
      // has read it
      if (!ZZ) ok = ok && warp_wait(smem_u32(&bars.pfree[pb]), ((it / C::NP) & 1) ^ 1, abort_flag, wait_ns);
      tr.mark(5, it);
      if (ok) {
        // The output MMA sees the bf16-rounded weights P'; the denominator and
        // the mean correction use the same rounded values (l = sum P'/r), so
        // the rounding of P' cancels in o = (sum P' z - sum P' mu) / l.
        // P'[token][head] as an MN-major B operand: element (head n, token k)
        // at (k / 8) 256 + (n / 8) 128 + (k % 8) 16 + (n % 8) 2.
        uint8_t* pbuf = smem + C::OFF_PBUF + pb * C::PBUF;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = e ? r1 : r0;
          const float ri = ZZ ? sd[e] : GATE ? 1.f / rr[e] : 1.f;
          float pq[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) pq[k] = ex2_approx(s[e][k] - m_ref[k]) * rr[e];
#pragma unroll
          for (int hp = 0; hp < 2; ++hp) {
            const uint32_t pw = pack_bf16x2(pq[2 * hp], pq[2 * hp + 1]);
            const float2 pr = unpack_bf16x2(pw);
            if (GATE) {
              l_acc[2 * hp] = fmaf(pr.x, ri, l_acc[2 * hp]);
              l_acc[2 * hp + 1] = fmaf(pr.y, ri, l_acc[2 * hp + 1]);
              bmu_acc[2 * hp] = fmaf(pr.x, mu[e], bmu_acc[2 * hp]);
              bmu_acc[2 * hp + 1] = fmaf(pr.y, mu[e], bmu_acc[2 * hp + 1]);
            } else {
              l_acc[2 * hp] += pr.x;
              l_acc[2 * hp + 1] += pr.y;
            }
            *reinterpret_cast<uint32_t*>(pbuf + (r >> 3) * 256 + hp * 128 + (r & 7) * 16 + 4 * q) = pw;
          }
        }
        tr.mark(6, it);
        fence_proxy_async_smem();
        tc_fence_before();
        warp_arrive(smem_u32(&bars.spdone[pb]));
      }
      tr.mark(3, it);

      if (t.last) {
        // ---- segment end: l and sum_j P'_j mu_j of every head over the 64 token rows
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            l_acc[k] += __shfl_xor_sync(0xffffffffu, l_acc[k], o);
            bmu_acc[k] += __shfl_xor_sync(0xffffffffu, bmu_acc[k], o);
          }
        if (lane < 4) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            xsum[(warp * kHeads + head_of(k)) * 2] = l_acc[k];
            xsum[(warp * kHeads + head_of(k)) * 2 + 1] = bmu_acc[k];
          }
        }
        if (soft_vote(kBarXch, !ok)) break;   // uniform
        float lh = 0.f, bh = 0.f;   // head `lane` (lanes 0-15)
        if (lane < kHeads) {
#pragma unroll
          for (int ww = 0; ww < kSoftWarps; ++ww) {
            lh += xsum[(ww * kHeads + lane) * 2];
            bh += xsum[(ww * kHeads + lane) * 2 + 1];
          }
        }
        // the segment's last output MMA (the earlier ones complete before it;
        // completion n of pfree[b] is output MMA n NP + b), then O^T
        ok = warp_wait(smem_u32(&bars.pfree[pb]), (it / C::NP) & 1, abort_flag, wait_ns);
        if (ok) {
          tc_fence_after();
          const int slot_out = blockIdx.x + t.b;
          float* po = p.part_o + static_cast<size_t>(slot_out) * kHeads * D_C;
#pragma unroll
          for (int m2 = 0; m2 < C::NMC / 2; ++m2) {   // two M chunks at a time
            float o[32];
            tmem_ld32(tq + C::COL_O + 32 * m2, o);
            tmem_wait_ld();
#pragma unroll
            for (int mc = 2 * m2; mc < 2 * m2 + 2; ++mc) {
              const int f = C::mc_start(mc) + 32 * warp + lane;
              if (C::mc_start(mc) + 32 * warp >= 128 * mc) {   // uniform in the warp
                float gm = 1.f, bt = 0.f;
                if (GATE) {
                  gm = gb[f];
                  bt = gb[D_C + f];
                }
#pragma unroll
                for (int h = 0; h < kHeads; ++h) {
                  float v = o[(mc & 1) * kHeads + h];
                  if (GATE) {
                    const float lhh = __shfl_sync(0xffffffffu, lh, h), bhh = __shfl_sync(0xffffffffu, bh, h);
                    v = fmaf(gm, v - bhh, bt * lhh);
                  }
                  po[h * D_C + f] = v;
                }
              }
            }
          }
          tc_fence_before();
          if (warp == 0 && lane < kHeads) {
            float* ml = p.part_ml + (static_cast<size_t>(slot_out) * kHeads + lane) * 2;
            ml[0] = m16;
            ml[1] = lh;
          }
          if (p.fuse) {
            // release this warp's part of the partial to the combine's wait on
            // its sequence (the warp barrier orders every lane's stores before
            // lane 0's fence)
            __syncwarp();
            if (lane == 0) {
              __threadfence();
              atomicAdd(p.seq_done + t.b, 1u);
            }
          }
        }
        tr.mark(4, it);
        // the next segment starts from scratch
        m16 = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          m_ref[k] = -INFINITY;
          l_acc[k] = 0.f;
          bmu_acc[k] = 0.f;
        }
      }
      if constexpr (ZZ) t = tn;
      ++it;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  phase_mark<DBG == 2>(p, 2);
  if (warp == kMmaWarp) tmem_dealloc(tmem, C::TMEM_COLS);
  if (threadIdx.x == 0 && bars.abort) report_status(p.status, kStatusTimeout);
  if constexpr (!DUMP && !BESIDE && D_C <= 256) {
    if (p.fuse) fused_combine<D_C, DBG == 2>(p, smem, bars);
  }
  if constexpr (BESIDE) grid_dependency_wait();
  phase_mark<DBG == 2>(p, 3);
}

template <int D_C, int GM, int DBG>
cudaError_t launch_one(const DecodeArgs& a, const CUtensorMap* maps, cudaStream_t st, bool* fused) {
  using C = Cfg<D_C, GM != 0, DBG == 4, DBG == 4 && GM == 1 && D_C == 256>;
  auto kern = decode_tc_kernel<D_C, GM, DBG>;
  cudaError_t e = allow_smem(kern, C::SMEM);
  if (e != cudaSuccess) return e;
  TcParams p = decode_params(a);
  // The split combine runs inside this kernel for the smallest batches, where a
  // step is mostly latency, when every CTA of the grid can be resident at once (a
  // cooperative launch guarantees it, or fails): a CTA for every sequence and head.
  // Beyond that, units share a wait, and the separate combine is faster.  us per
  // step, fused / apart: replayed 24 to a graph at d_c 256, 4 x 100 12.0 / 13.4, 9 x
  // 100 12.4 / 14.1, 8 x 32K 43.8 / 45.6, 9 x 32K 48.2 / 49.7, 10 x 100 14.7 / 13.9,
  // 10 x 32K 53.0 / 53.7, 12 x 8K 27.9 / 26.9, 32 x 8K 52.8 / 46.8; at d_c 192, 9 x 1K
  // 13.2 / 15.0, 10 x 1K 15.5 / 14.9, 10 x 32K 45.8 / 46.6, 12 x 32K 54.0 / 53.6.
  // Issued eagerly, where a cooperative launch cannot overlap the kernel before it,
  // the two are closer: 8 x 32K 46.9 / 46.5, 4 x 100 14.4 / 14.5, 4 x 8K 20.6 / 19.8.
  // (the fused combine holds kCombineRowsPerWarp rows of W_UV,h per warp)
  p.fuse = DBG != 1 && DBG != 3 && !a.apart && D_C <= 256 && a.batch > 0 && kHeads * a.batch <= a.num_splits &&
           a.d_v <= kCombineRowsPerWarp * (kThreads / 32) &&
           a.num_splits <= resident_ctas<decode_tc_kernel<D_C, GM, DBG>>(C::SMEM);
  if (fused) *fused = p.fuse != 0;
  return launch_split_kernel(kern, C::SMEM, a, maps, p, st);
}

}  // namespace

bool tc_supported(int d_c, int gate) {
  if (gate) return d_c == 192 || d_c == 256;
  return d_c == 192 || d_c == 256 || d_c == 512;
}

// d_c-dispatch of one gate mode; the trace instantiation exists for the modes
// none and mul_ln (the others run untraced)
template <int GM>
cudaError_t launch_mode(const DecodeArgs& a, const CUtensorMap* maps, cudaStream_t st, bool* fused) {
  if (a.scale_pool != nullptr) {   // (ungated, the other widths: egmla_decode_q8.cu)
    if (a.d_c == 192) return launch_one<192, GM, 4>(a, maps, st, fused);
    if constexpr (GM != 0) {
      if (a.d_c == 256) return launch_one<256, GM, 4>(a, maps, st, fused);
    }
    return cudaErrorInvalidValue;
  }
  if constexpr (GM <= 1) {
    if (a.trace != nullptr) {
      if (a.d_c == 192) return launch_one<192, GM, 2>(a, maps, st, fused);
      if (a.d_c == 256) return launch_one<256, GM, 2>(a, maps, st, fused);
      return cudaErrorInvalidValue;
    }
  }
  if (a.beside) {
    if (a.d_c == 192) return launch_one<192, GM, 3>(a, maps, st, fused);
    if (a.d_c == 256) return launch_one<256, GM, 3>(a, maps, st, fused);
    return cudaErrorInvalidValue;
  }
  if (a.d_c == 192) return launch_one<192, GM, 0>(a, maps, st, fused);
  if (a.d_c == 256) return launch_one<256, GM, 0>(a, maps, st, fused);
  return cudaErrorInvalidValue;
}

cudaError_t launch_decode_tc(const DecodeArgs& a, const CUtensorMap* maps, bool dump, cudaStream_t st,
                             bool* fused) {
  if (fused) *fused = false;
  if (dump) {   // cache-read test entry: the raw page and gate rows
    if (a.d_c == 192) return launch_one<192, 1, 1>(a, maps, st, nullptr);
    if (a.d_c == 256) return launch_one<256, 1, 1>(a, maps, st, nullptr);
    return cudaErrorInvalidValue;
  }
  if (!a.gate) {
    if (a.d_c == 512 && a.scale_pool == nullptr) return launch_one<512, 0, 0>(a, maps, st, fused);
    return launch_mode<0>(a, maps, st, fused);
  }
  if (a.gate_add) return launch_mode<3>(a, maps, st, fused);
  if (a.gate_ln) return launch_mode<1>(a, maps, st, fused);
  return launch_mode<2>(a, maps, st, fused);
}

}  // namespace egmla
