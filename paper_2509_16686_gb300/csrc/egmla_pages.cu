// egmla_pages.cu - the pages of a paged latent cache on the GPU (sm_103a):
//
//   page_plan_kernel     a serving step's pages from its requests' lengths: released
//                        pages onto the free stack, new ones from it into the block
//                        table, the packed offsets and the cache slot of every new
//                        token
//   page_summary_kernel  the mean key [c~ ; k^R] of every page that became full
//   select_pages_kernel  each sequence's pages by the largest logit that any head gives
//                        their mean key, the best of them as a block table
//
// The last two make the page-sparse decode: the split-KV kernels then attend over
// the selected pages alone (a cached RoPE key carries its position, so a page may
// stand anywhere in a block table).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "egmla_common.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"
#include "egmla_rows.cuh"

namespace egmla {
namespace {

__device__ __forceinline__ int pages_of(int n) { return (n + kPage - 1) / kPage; }

// inclusive sums of two values over the block's threads; `total`: of all.  ws: a pair per warp
__device__ __forceinline__ int2 block_scan2(int2 v, int2* ws, int2& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x / 32;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
    if (lane >= o) {
      v.x += x;
      v.y += y;
    }
  }
  if (lane == 31) ws[warp] = v;
  __syncthreads();
  int2 s = lane < nw ? ws[lane] : make_int2(0, 0);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, s.x, o), y = __shfl_up_sync(0xffffffffu, s.y, o);
    if (lane >= o) {
      s.x += x;
      s.y += y;
    }
  }
  total = make_int2(__shfl_sync(0xffffffffu, s.x, nw - 1), __shfl_sync(0xffffffffu, s.y, nw - 1));
  const int bw = warp > 0 ? warp - 1 : 0;
  const int bx = __shfl_sync(0xffffffffu, s.x, bw), by = __shfl_sync(0xffffffffu, s.y, bw);
  __syncthreads();   // ws is rewritten by the next scan
  return warp > 0 ? make_int2(v.x + bx, v.y + by) : v;
}

// inclusive sum over the block's threads; `total`: the sum of all.  ws: a word per warp
__device__ __forceinline__ int block_scan(int v, int* ws, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x / 32;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  if (lane == 31) ws[warp] = v;
  __syncthreads();
  int s = lane < nw ? ws[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += t;
  }
  total = __shfl_sync(0xffffffffu, s, nw - 1);
  const int before = __shfl_sync(0xffffffffu, s, warp > 0 ? warp - 1 : 0);
  __syncthreads();   // ws is rewritten by the next scan
  return v + (warp > 0 ? before : 0);
}

// the largest b in [0, n) with cum[b] <= x (cum non-decreasing, cum[0] <= x)
__device__ __forceinline__ int find_in(const int32_t* cum, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cum[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// ============================================================================ 1. page plan
// One cluster: every CTA computes the same sums over the batch (three words per
// sequence in its shared memory), and takes its share of the pages and slots.  The
// first cluster barrier lets outputs overwrite inputs (seq_lens, free_count), the
// second orders the pages pushed before those popped.
// A chain of latencies: lengths, sums, stack, stores.  3.1 us for 64 sequences of a token
// each; 9.2 for 1,024 requests, one in sixteen a prompt of up to 8K tokens, where the
// slots' searches and stores are shared by eight CTAs.
constexpr int kPlanThreads = 1024;   // 256 for small steps (fewer warps to wait for)

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanArgs p) {
  extern __shared__ int32_t plan_smem[];
  __shared__ int2 ws[32];
  int32_t* E = plan_smem;              // [batch + 1] exclusive sums of the pages asked for
  int32_t* len = E + p.batch + 1;      // [batch] lengths before the step
  int32_t* cum = len + p.batch;        // [batch + 1] of the pages released, then of the tokens granted
  const int tid = threadIdx.x, T = blockDim.x, C = static_cast<int>(gridDim.x), rank = static_cast<int>(blockIdx.x);
  const int first = rank * T + tid, step = C * T;   // this thread's share of a list
  const int64_t most = static_cast<int64_t>(p.max_pages) * kPage;
  grid_dependency_wait();
  const int given = __ldg(p.free_count);
  const int F = static_cast<unsigned>(given) <= static_cast<unsigned>(p.num_pages) ? given : 0;
  bool bad = given != F, refused = false;
  // a sequence's pages: released if n < 0, asked for otherwise
  auto request = [&](int b, int& L, int& back, int& need, int& ask, bool& fits) {
    L = p.seq_lens[b];
    const int n = __ldg(p.new_tokens + b);
    const bool sane = L >= 0 && L <= most;
    back = sane && n < 0 ? pages_of(L) : 0;
    ask = sane && n > 0 ? n : 0;
    fits = static_cast<int64_t>(L) + ask <= most;
    need = fits && ask > 0 ? static_cast<int>((static_cast<int64_t>(L) + ask + kPage - 1) / kPage) - pages_of(L) : 0;
    return sane;
  };
  int total_need = 0, R = 0;
  for (int b0 = 0; b0 < p.batch; b0 += T) {
    const int b = b0 + tid;
    int L = 0, back = 0, need = 0, ask = 0;
    bool fits = true;
    if (b < p.batch && !request(b, L, back, need, ask, fits)) bad = true;
    int2 sum;
    const int2 v = block_scan2(make_int2(need, back), ws, sum);
    if (b < p.batch) {
      E[b] = total_need + v.x - need;
      len[b] = L;
      cum[b] = R + v.y - back;
    }
    total_need += sum.x;
    R += sum.y;
  }
  if (tid == 0) {
    E[p.batch] = total_need;
    cum[p.batch] = R;
  }
  // more pages released than there is room for: the rest is dropped (R may be near 2^31, F + R above it)
  const int avail = F + min(R, p.num_pages - F);
  if (avail - F < R) bad = true;
  __syncthreads();
  cluster_sync();
  // pages released, in the order of the batch
  if (R > 0) {
    for (int i = first; i < avail - F; i += step) {
      const int b = find_in(cum, p.batch, i);
      const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + (i - cum[b])];
      if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) bad = true;
      p.free_pages[F + i] = page;
    }
    __syncthreads();   // cum is rewritten below
    cluster_sync();
  }
  // what is granted, first come first served
  int total = 0, granted_pages = 0;
  for (int b0 = 0; b0 < p.batch; b0 += T) {
    const int b = b0 + tid;
    int t = 0, g = 0, L = 0;
    if (b < p.batch) {
      L = len[b];
      const int n = __ldg(p.new_tokens + b), need = E[b + 1] - E[b];
      const bool sane = L >= 0 && L <= most;
      if (sane && n > 0) {
        const bool ok = static_cast<int64_t>(L) + n <= most && (need == 0 || E[b] + need <= avail);
        if (ok) {
          t = n;
          g = need;
        } else {
          refused = true;
        }
      }
      if (b % C == rank) {
        p.seq_lens_out[b] = sane && n < 0 ? 0 : L + t;
        if (p.positions) p.positions[b] = t > 0 ? L : -1;
      }
    }
    int2 sum;
    const int2 v = block_scan2(make_int2(t, g), ws, sum);
    if (b < p.batch) cum[b] = total + v.x - t;
    if (b < p.batch && b % C == rank) p.cu_seqlens[b] = total + v.x - t;
    total += sum.x;
    granted_pages += sum.y;
  }
  if (tid == 0) cum[p.batch] = total;
  if (tid == 0 && rank == 0) {
    p.cu_seqlens[p.batch] = total;
    *p.free_count_out = avail - granted_pages;
  }
  __syncthreads();
  // pages granted: those asked for first, since nothing is granted after a refusal
  for (int i = first; i < granted_pages; i += step) {
    const int b = find_in(E, p.batch, i);
    const int page = p.free_pages[avail - 1 - i];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) bad = true;
    p.block_table[static_cast<size_t>(b) * p.max_pages + pages_of(len[b]) + (i - E[b])] = page;
  }
  // the new tokens' slots
  if (p.slots != nullptr) {
    if (total > p.max_slots) bad = true;
    const bool vec = (reinterpret_cast<uintptr_t>(p.slots) & 15) == 0;
    // G slots of a thread in a row: one search for them
    auto fill = [&](auto g) {
      constexpr int G = decltype(g)::value;
      for (int k0 = first * G; k0 < p.max_slots; k0 += step * G) {
        int b = k0 < total ? find_in(cum, p.batch, k0) : 0;
        int page[G], off[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {   // (no load depends on another)
          const int k = k0 + i;
          page[i] = -1;
          off[i] = 0;
          if (k < total) {
            while (cum[b + 1] <= k) ++b;
            const int L = len[b], pos = L + (k - cum[b]), lp = pos / kPage, have = pages_of(L);
            const int32_t* src = lp < have ? p.block_table + static_cast<size_t>(b) * p.max_pages + lp
                                           : p.free_pages + (avail - 1 - (E[b] + lp - have));
            page[i] = *src;
            off[i] = pos % kPage;
          }
        }
        int slot[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const bool in = static_cast<unsigned>(page[i]) < static_cast<unsigned>(p.num_pages);
          slot[i] = in ? page[i] * kPage + off[i] : -1;
          if (!in && k0 + i < total) bad = true;
        }
        if (G >= 4 && vec && k0 + G <= p.max_slots)
#pragma unroll
          for (int i = 0; i < G; i += 4)
            *reinterpret_cast<int4*>(p.slots + k0 + i) =
                make_int4(slot[i], slot[(i + 1) % G], slot[(i + 2) % G], slot[(i + 3) % G]);
        else
#pragma unroll
          for (int i = 0; i < G; ++i)
            if (k0 + i < p.max_slots) p.slots[k0 + i] = slot[i];
      }
    };
    if (p.max_slots <= step)
      fill(std::integral_constant<int, 1>{});
    else
      fill(std::integral_constant<int, 8>{});
  }
  // a refusal (which every CTA has seen) is reported where nothing is out of range
  if (bad) report_status(p.status, kStatusOutOfRange);
  if (__syncthreads_or(refused)) {
    cluster_sync();
    if (rank == 0 && tid == 0) report_status(p.status, kStatusNoPages);
  }
}

// ============================================================================ 2. page summaries
constexpr int kSumWarps = 8;
constexpr int kSumRows = kPage / kSumWarps;   // rows of a page per warp
constexpr int kSumMaxDc = 512, kSumMaxDr = 64;

// A block takes a page, a warp eight of its rows, kFlight of them at a time with every
// load in flight; a lane has 16-byte units lane, lane + 32, .. of a row (NU of them).
// LayerNorm in two passes over the registers, the sums of the rows in flight reduced
// together.  The mean of gamma x_j + beta is gamma mean(x_j) + beta, so the affine part
// comes last.  k^R rows: a lane has one unit of every few rows.
// Bound by issue and latency: 44.7 us for 8 x 32K tokens at d_c 256, 6.8 TB/s of cache and
// gate rows; floor 28.  What it took (57.0 before): products straight from the bf16 pairs,
// idle lanes that repeat a unit instead of zeros and selects, 64 registers (four blocks
// per SM; with three 51.8, five 63.0; eight rows in flight 54.6, two 46.2).  Copies by TMA
// into a ring, or the next page's ids ahead in persistent blocks, gained nothing.  GM: the
// gate mode.
template <typename T, int NU, int GM>
__global__ void __launch_bounds__(32 * kSumWarps, NU == 1 ? 4 : NU == 2 ? 3 : 2) page_summary_kernel(const SummaryArgs p) {
  using U = Unit<T>;
  constexpr bool GATE = GM != EG_MLA_GATE_NONE, GATE_ADD = GM == EG_MLA_GATE_ADD_LN;
  constexpr bool GATE_LN = GM == EG_MLA_GATE_MUL_LN || GM == EG_MLA_GATE_ADD_LN;
  constexpr int VP = U::kPairs, VE = 2 * VP;   // pairs and elements of a unit
  constexpr int kFlight = NU == 1 ? 4 : 2;
  __shared__ float part[kSumWarps][kSumMaxDc + kSumMaxDr];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x / p.page_bound, i = blockIdx.x - b * p.page_bound;
  grid_dependency_wait();
  int L = __ldg(p.seq_lens + b);
  int n = p.new_tokens != nullptr ? __ldg(p.new_tokens + b) : L;
  bool bad = false;
  if (L < 0 || L > p.max_seq_len) {
    bad = true;
    L = L < 0 ? 0 : p.max_seq_len;
  }
  n = min(max(n, 0), L);
  if (n > p.max_new) {
    bad = true;
    n = p.max_new;
  }
  const int lp = (L - n) / kPage + i;
  if (bad && i == 0 && threadIdx.x == 0) report_status(p.status, kStatusOutOfRange);
  if (lp >= L / kPage) return;
  const int page = __ldg(p.block_table + static_cast<size_t>(b) * p.max_pages + lp);
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) {
    if (threadIdx.x == 0) report_status(p.status, kStatusOutOfRange);
    return;
  }
  const int units = p.d_c / VE, runits = p.d_r / VE;
  const size_t row0 = static_cast<size_t>(page) * kPage + warp * kSumRows;
  const T* kr = static_cast<const T*>(p.kr_pool) + row0 * p.d_r;
  // k^R: unit lane % rw of rows lane / rw, + 32 / rw, ..  (rw: the units of a row, padded)
  int rw = 1;
  while (rw < runits) rw *= 2;
  const int ru = lane & (rw - 1);
  float2 racc[VP];
#pragma unroll
  for (int e = 0; e < VP; ++e) racc[e] = make_float2(0.f, 0.f);
  for (int r = lane / rw; r < kSumRows; r += 32 / rw) {
    if (ru < runits) {
      float2 t[VP];
      U::widen(__ldg(reinterpret_cast<const uint4*>(kr + static_cast<size_t>(r) * p.d_r) + ru), t);
#pragma unroll
      for (int e = 0; e < VP; ++e) racc[e] = __fadd2_rn(racc[e], t[e]);
    }
  }
  int id_row = 0;   // lane r: row r's token
  if (GATE && lane < kSumRows) id_row = __ldg(p.id_pool + row0 + lane);
  if (GATE && static_cast<unsigned>(id_row) >= static_cast<unsigned>(p.vocab)) {
    report_status(p.status, kStatusOutOfRange);
    id_row = 0;
  }
  float2 acc[NU][VP];
  bool live[NU];   // lanes past a row's end repeat its last unit; their sums are left out
  int at[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    live[u] = lane + 32 * u < units;
    at[u] = min(lane + 32 * u, units - 1) * VE;
#pragma unroll
    for (int e = 0; e < VP; ++e) acc[u][e] = make_float2(0.f, 0.f);
  }
  const T* c = static_cast<const T*>(p.c_pool) + row0 * p.d_c;
  const T* table = static_cast<const T*>(p.gate_table);
  const float inv_n = 1.f / static_cast<float>(p.d_c);
#pragma unroll 1
  for (int r0 = 0; r0 < kSumRows; r0 += kFlight) {
    uint4 cw[kFlight][NU], gw[kFlight][NU];
#pragma unroll
    for (int r = 0; r < kFlight; ++r) {
      const int id = GATE ? __shfl_sync(0xffffffffu, id_row, r0 + r) : 0;
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        cw[r][u] = __ldg(reinterpret_cast<const uint4*>(c + (r0 + r) * p.d_c + at[u]));
        if (GATE) gw[r][u] = __ldg(reinterpret_cast<const uint4*>(table + static_cast<size_t>(id) * p.d_c + at[u]));
      }
    }
    float2 x[kFlight][NU][VP];
    float s[kFlight];
#pragma unroll
    for (int r = 0; r < kFlight; ++r) {
      s[r] = 0.f;
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        if (GATE && !GATE_ADD) {
          U::mul(cw[r][u], gw[r][u], x[r][u]);
        } else {
          U::widen(cw[r][u], x[r][u]);
          if (GATE) {
            float2 t[VP];
            U::widen(gw[r][u], t);
#pragma unroll
            for (int e = 0; e < VP; ++e) x[r][u][e] = __fadd2_rn(x[r][u][e], t[e]);
          }
        }
        if (GATE_LN) {
          float2 sum = x[r][u][0];
#pragma unroll
          for (int e = 1; e < VP; ++e) sum = __fadd2_rn(sum, x[r][u][e]);
          if (live[u]) s[r] += sum.x + sum.y;
        }
      }
    }
    if (GATE_LN) {
      warp_sums(s, lane);
#pragma unroll
      for (int r = 0; r < kFlight; ++r) {
        const float2 mu = make_float2(-s[r] * inv_n, -s[r] * inv_n);
        s[r] = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          float2 sq = make_float2(0.f, 0.f);
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            x[r][u][e] = __fadd2_rn(x[r][u][e], mu);
            sq = __ffma2_rn(x[r][u][e], x[r][u][e], sq);
          }
          if (live[u]) s[r] += sq.x + sq.y;
        }
      }
      warp_sums(s, lane);
#pragma unroll
      for (int r = 0; r < kFlight; ++r) {
        const float rstd = rsqrtf(fmaf(s[r], inv_n, p.eps));
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int e = 0; e < VP; ++e) acc[u][e] = __ffma2_rn(x[r][u][e], make_float2(rstd, rstd), acc[u][e]);
      }
    } else {
#pragma unroll
      for (int r = 0; r < kFlight; ++r)
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int e = 0; e < VP; ++e) acc[u][e] = __fadd2_rn(acc[u][e], x[r][u][e]);
    }
  }
#pragma unroll
  for (int u = 0; u < NU; ++u)
    if (lane + 32 * u < units)
#pragma unroll
      for (int e = 0; e < VP; ++e)
        *reinterpret_cast<float2*>(&part[warp][VE * (lane + 32 * u) + 2 * e]) = acc[u][e];
#pragma unroll
  for (int e = 0; e < VP; ++e)
    for (int o = rw; o < 32; o *= 2) {
      racc[e].x += __shfl_xor_sync(0xffffffffu, racc[e].x, o);
      racc[e].y += __shfl_xor_sync(0xffffffffu, racc[e].y, o);
    }
  if (lane < runits)
#pragma unroll
    for (int e = 0; e < VP; ++e) *reinterpret_cast<float2*>(&part[warp][p.d_c + VE * lane + 2 * e]) = racc[e];
  __syncthreads();
  float* out = p.summary + static_cast<size_t>(page) * (p.d_c + p.d_r);
  for (int f = threadIdx.x; f < p.d_c + p.d_r; f += blockDim.x) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kSumWarps; ++w) s += part[w][f];   // in row order
    s *= 1.f / kPage;
    if (GATE_LN && f < p.d_c) s = fmaf(s, p.gamma ? __ldg(p.gamma + f) : 1.f, p.beta ? __ldg(p.beta + f) : 0.f);
    out[f] = s;
  }
}

// ============================================================================ 3. page selection
// score(b, p) = max_h scale (q^_bh . m^c_p + q^R_bh . m^R_p), fp32 products and sums.
// One launch: a block scores groups of 32 pages of a sequence (its queries in shared
// memory, a warp four pages at a time, so that a query value read serves four products; lanes
// share a row, the heads' sums take one transposing reduction); the last block of a
// sequence to finish selects its pages.  The lengths that are left do not
// depend on the choice, so the split-KV schedule is already made (selected_lengths).
//
// The selection: scores as whole numbers of the same order (no number comes last); the
// want-th largest by up to four passes over a histogram of eight bits each; then, in
// order, the pages above it and the first of those equal to it, between the pages that
// are always kept.
//
// Bound by the products' reads of shared memory and FMAs in turn (2.0 us a group of pages)
// and by the chain after them: 32 sequences of 512 pages at d_c 256 have their scores
// 12.0 us after the kernel's start, 3.1 of it the wait for the queries, and their pages
// at 16.4; four of 128 pages at 5.1 and 9.3.
constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32, kScHeads = 16;
constexpr int kSelPages = 32;    // pages of a block at a time
constexpr int kSelRounds = 4;    // times, at most
constexpr int kWideRounds = 2;   // of rows in two parts
constexpr int kSelKeys = 4096;   // scores kept in shared memory; of more the rest is read again

// Pages and heads of a warp (32 sums): two warps share a group of four pages.  A row's
// 16-byte units go over the lanes, three of a lane at a time.
constexpr int kScPP = 4, kScHH = 8, kScShare = kScHeads / kScHH, kScUnits = 3;
static_assert(kSelWarps / kScShare * kScPP == kSelPages && kScPP * kScHH == 32, "pages of a block");

// v[i] summed over the warp's lanes, value t returned to lane t
__device__ __forceinline__ float sum32_transpose(float (&v)[32], int lane) {
#pragma unroll
  for (int o = 16, n = 32; o > 0; o >>= 1, n >>= 1) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i < n / 2) {
        const bool hi = lane & o;
        const float keep = hi ? v[i + n / 2] : v[i], give = hi ? v[i] : v[i + n / 2];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
  }
  return v[0];
}

// scores as whole numbers of the same order: no number last, +0 and -0 (a score that underflows) the same
__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = s == 0.f ? 0u : __float_as_uint(s);
  return s != s ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void copy16_async(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// one of the block's threads announces that the block is done (of `of`); true for the
// whole block if it is the last, which then sees what the others wrote
__device__ __forceinline__ bool last_to_finish(int32_t* count, int of, int* flag) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    *flag = atomicAdd(count, 1) == of - 1;
  }
  __syncthreads();
  const bool last = *flag != 0;
  if (last) __threadfence();
  return last;
}

// PARTS: of a row, three units of a lane each
template <int PARTS>
__global__ void __launch_bounds__(kSelThreads, 1) select_pages_kernel(const SelectArgs p) {
  constexpr int PP = kScPP, HH = kScHH, kShare = kScShare, NU = kScUnits;
  extern __shared__ __align__(16) uint8_t sel_smem[];
  __shared__ int hist[256];
  __shared__ int ws[32], flag, digit, above;
  __shared__ float bests[kSelRounds][kShare][kSelPages];
  float4* sq = reinterpret_cast<float4*>(sel_smem);            // [kScHeads][units]
  uint2* keys = reinterpret_cast<uint2*>(sel_smem);            // afterwards: (key, page id)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x / p.chunks, j = blockIdx.x - b * p.chunks;
  const int D = p.d_c + p.d_r, units = D / 4;
  // lengths, block table and summaries are no work of the absorption, beside which this
  // kernel starts: they are read before the wait for its queries
  beside_acquire();
  const int given = __ldg(p.seq_lens + b);
  const int L = min(max(given, 0), p.max_seq_len), np = (L + kPage - 1) / kPage;
  const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_pages;
  float* scores = p.scores + static_cast<size_t>(b) * p.max_pages;
  // of a longer sequence the pages lo .. hi - 1 are ranked, `want` of them taken
  const int lo = p.keep_first, hi = np - p.keep_last, want = p.budget - p.keep_first - p.keep_last;
  const bool ranked = np > p.budget && want > 0;
  // groups of pages j, j + chunks, .. are this block's: a short sequence's go to as many blocks
  const int groups = (hi - lo + kSelPages - 1) / kSelPages, blocks = ranked ? min(groups, p.chunks) : 1;
  if (j >= blocks) return;   // (without the wait: those that have work stay for it)
  if (given != L && j == 0 && tid == 0) report_status(p.status, kStatusOutOfRange);
  float4 m[PP][NU];
  bool bad = false;
  // part `part` of the mean keys of the warp's pages w0 .. w0 + PP - 1
  auto load_pages = [&](int w0, int part) {
#pragma unroll
    for (int k = 0; k < PP; ++k) {
      int page = __ldg(table + min(w0 + k, hi - 1));
      if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) {
        bad = true;
        page = 0;
      }
      const float4* row = reinterpret_cast<const float4*>(p.summary + static_cast<size_t>(page) * D);
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int u = lane + 32 * (NU * part + i);
        m[k][i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (u < units) m[k][i] = __ldg(row + u);
      }
    }
  };
  const int row0 = warp / kShare * PP, h0 = warp % kShare * HH;   // the warp's pages of a group, its heads
  if (ranked) load_pages(lo + j * kSelPages + row0, 0);
  grid_dependency_wait();
  grid_launch_dependents();   // (the split-KV kernel sets up where SMs are free: 64 ragged sequences 65.5 -> 64.7 us)
  if (ranked) {
    const float* q = p.q + static_cast<size_t>(b) * p.q_stride;
    for (int h = warp; h < kScHeads; h += kSelWarps)
      for (int u = lane; u < units; u += 32) {
        float4* dst = sq + h * units + u;
        if (h >= p.H)
          *dst = make_float4(0.f, 0.f, 0.f, 0.f);
        else if (4 * u < p.d_c)
          copy16_async(dst, q + h * p.d_c + 4 * u);
        else
          copy16_async(dst, q + p.H * p.d_c + h * p.d_r + 4 * u - p.d_c);
      }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int r = 0; r < kSelRounds; ++r) {
      const int w0 = lo + (j + r * p.chunks) * kSelPages + row0;
      if (w0 >= hi) break;
      float acc[32];   // [page][head]
#pragma unroll
      for (int e = 0; e < 32; ++e) acc[e] = 0.f;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        if (r > 0 || part > 0) load_pages(w0, part);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          const int u = lane + 32 * (NU * part + i);
          const bool in = u < units;   // (past the row both are zero)
#pragma unroll
          for (int h = 0; h < HH; ++h) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (in) x = sq[(h0 + h) * units + u];
#pragma unroll
            for (int k = 0; k < PP; ++k) {
              float& a = acc[k * HH + h];
              a = fmaf(x.x, m[k][i].x, a);
              a = fmaf(x.y, m[k][i].y, a);
              a = fmaf(x.z, m[k][i].z, a);
              a = fmaf(x.w, m[k][i].w, a);
            }
          }
        }
      }
      float best = sum32_transpose(acc, lane);   // lane l: of page l / HH
      if (h0 + lane % HH >= p.H) best = NAN;   // no head: left out, as a head without a number is
#pragma unroll
      for (int o = HH / 2; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
      if (lane % HH == 0) bests[r][warp % kShare][row0 + lane / HH] = best;
    }
    if (bad && lane == 0) report_status(p.status, kStatusOutOfRange);
    __syncthreads();
    for (int i = tid; i < kSelRounds * kSelPages; i += kSelThreads) {
      const int r = i / kSelPages, k = i % kSelPages, lp = lo + (j + r * p.chunks) * kSelPages + k;
      if (lp >= hi) continue;
      float s = bests[r][0][k];
#pragma unroll
      for (int e = 1; e < kShare; ++e) s = fmaxf(s, bests[r][e][k]);
      scores[lp] = s * p.scale;
    }
    if (blocks > 1 && !last_to_finish(p.counters + b, blocks, &flag)) return;
  }
  __syncthreads();   // (the scores of this block's warps; sq is read no more)

  // ---- the sequence's pages
  int32_t* out = p.sel_table + static_cast<size_t>(b) * p.width;
  int32_t* sel = p.selected != nullptr ? p.selected + static_cast<size_t>(b) * p.budget : nullptr;
  const int taken = min(np, p.budget);
  if (sel != nullptr)
    for (int i = taken + tid; i < p.budget; i += kSelThreads) sel[i] = -1;
  auto take_page = [&](int pos, int i) {
    out[pos] = __ldg(table + i);
    if (sel != nullptr) sel[pos] = i;
  };
  if (np <= p.budget) {
    for (int i = tid; i < np; i += kSelThreads) take_page(i, i);
  } else {
    for (int i = tid; i < lo; i += kSelThreads) take_page(i, i);
    for (int i = tid; i < p.keep_last; i += kSelThreads) take_page(p.budget - p.keep_last + i, hi + i);
  }
  if (ranked) {
    const int n = hi - lo;
    for (int i = tid; i < min(n, kSelKeys); i += kSelThreads)
      keys[i] = make_uint2(score_key(scores[lo + i]), static_cast<uint32_t>(__ldg(table + lo + i)));
    __syncthreads();
    auto key = [&](int i) { return i < kSelKeys ? keys[i].x : score_key(scores[lo + i]); };
    // the want-th largest key begins with the digits of `prefix` from `shift` up; `left` of
    // those that do are wanted
    uint32_t prefix = 0;
    int left = want, shift = 32;
    for (bool all = false; shift > 0 && !all;) {
      shift -= 8;
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i0 = 0; i0 < n; i0 += kSelThreads) {   // the equal digits of a warp counted once
        const uint32_t k = i0 + tid < n ? key(i0 + tid) : 0u;
        const bool in = i0 + tid < n && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)));
        const uint32_t d = in ? (k >> shift) & 255u : 256u, same = __match_any_sync(0xffffffffu, d);
        if (in && lane == __ffs(same) - 1) atomicAdd(&hist[d], __popc(same));
      }
      __syncthreads();
      if (warp == 0) {   // digits from the largest down: lane l has 255 - 8 l and the seven below
        int c[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] = hist[255 - 8 * lane - e];
          sum += c[e];
        }
        int before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int t = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += t;
        }
        before -= sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (before < left && before + c[e] >= left) {
            digit = 255 - 8 * lane - e;
            above = before;
            flag = before + c[e] == left;   // every one of them is wanted: no further digit matters
          }
          before += c[e];
        }
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(digit) << shift;
      left -= above;
      all = flag != 0;
    }
    // in order: a page's place is the number before it of pages above, and of the first
    // `left` equals
    int larger = 0, equal = 0;
    for (int i0 = 0; i0 < n; i0 += kSelThreads) {
      const int i = i0 + tid;
      const uint32_t k = i < n ? key(i) >> shift : 0u, t = prefix >> shift;
      const bool up = i < n && k > t, tie = i < n && k == t;
      int total;
      const int incl = block_scan((up ? 1 : 0) + (tie ? 1 << 16 : 0), ws, total);   // (512 of each at most)
      const int ups = larger + (incl & 0xffff) - (up ? 1 : 0), ties = equal + (incl >> 16) - (tie ? 1 : 0);
      if (up || (tie && ties < left)) {
        const int pos = lo + ups + min(ties, left);
        out[pos] = i < kSelKeys ? static_cast<int32_t>(keys[i].y) : __ldg(table + lo + i);
        if (sel != nullptr) sel[pos] = lo + i;
      }
      larger += total & 0xffff;
      equal += total >> 16;
    }
  }
}

}  // namespace

// ---------------------------------------------------------------- launchers
// A decode step's plan is a few words per sequence: one CTA.  Longer lists are shared by
// eight.
cudaError_t launch_page_plan(const PlanArgs& a, cudaStream_t st) {
  const size_t smem = (3 * static_cast<size_t>(a.batch) + 2) * 4;
  const cudaError_t e = allow_smem(page_plan_kernel, (3 * static_cast<size_t>(kPlanMaxBatch) + 2) * 4);
  if (e != cudaSuccess) return e;
  const int slots = a.slots != nullptr ? a.max_slots : 0;
  const int ctas = slots + a.batch > 4096 ? 8 : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(a.batch <= 256 && ctas == 1 ? 256 : kPlanThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, page_plan_kernel, a);
}

namespace {
template <typename T, int NU>
cudaError_t launch_summary(const SummaryArgs& a, cudaStream_t st) {
  auto launch = [&](auto kernel) {
    return launch_chained(kernel, dim3(static_cast<unsigned>(a.batch) * a.page_bound), dim3(32 * kSumWarps), 0, st, a);
  };
  switch (a.gate_mode) {
    case EG_MLA_GATE_MUL_LN: return launch(page_summary_kernel<T, NU, EG_MLA_GATE_MUL_LN>);
    case EG_MLA_GATE_MUL: return launch(page_summary_kernel<T, NU, EG_MLA_GATE_MUL>);
    case EG_MLA_GATE_ADD_LN: return launch(page_summary_kernel<T, NU, EG_MLA_GATE_ADD_LN>);
    default: return launch(page_summary_kernel<T, NU, EG_MLA_GATE_NONE>);
  }
}
}  // namespace

cudaError_t launch_page_summary(const SummaryArgs& a, cudaStream_t st) {
  const int units = a.d_c * (a.fp32 ? 4 : 2) / 16;
  if (a.fp32)
    return units <= 32 ? launch_summary<float, 1>(a, st)
                       : units <= 64 ? launch_summary<float, 2>(a, st) : launch_summary<float, 4>(a, st);
  return units <= 32 ? launch_summary<__nv_bfloat16, 1>(a, st) : launch_summary<__nv_bfloat16, 2>(a, st);
}

namespace {
int row_parts(int d_c, int d_r) { return ((d_c + d_r) / 4 + 32 * kScUnits - 1) / (32 * kScUnits); }

template <int PARTS>
cudaError_t launch_select(const SelectArgs& a, cudaStream_t st) {
  auto bytes = [](int D) {
    const size_t q = static_cast<size_t>(kScHeads) * D * 4, keys = kSelKeys * sizeof(uint2);
    return q > keys ? q : keys;
  };
  const cudaError_t e = allow_smem(select_pages_kernel<PARTS>, bytes(kSumMaxDc + kSumMaxDr));
  if (e != cudaSuccess) return e;
  return launch_chained(select_pages_kernel<PARTS>, dim3(static_cast<unsigned>(a.chunks) * a.batch), dim3(kSelThreads),
                        bytes(a.d_c + a.d_r), st, a);
}
}  // namespace

// Fewer blocks than groups of pages where those are more than SMs (one block fits on
// each): a block's further rounds find the queries in shared memory.
int select_chunks(int max_seq_len, int batch, int budget, int keep_first, int keep_last, int d_c, int d_r) {
  const int pages = (max_seq_len + kPage - 1) / kPage, ranked = pages - keep_first - keep_last;
  if (batch == 0 || pages <= budget || budget <= keep_first + keep_last) return 1;
  const int64_t groups = (ranked + kSelPages - 1) / kSelPages, all = groups * batch;
  const int most = row_parts(d_c, d_r) == 1 ? kSelRounds : kWideRounds;
  const int64_t rounds = all > most * kSms ? most : (all + kSms - 1) / kSms;
  return static_cast<int>((groups + rounds - 1) / rounds);
}

cudaError_t launch_select_pages(const SelectArgs& a, cudaStream_t st) {
  static_assert((kSumMaxDc + kSumMaxDr) / 4 <= 2 * kScUnits * 32, "a row's units over the lanes");
  return row_parts(a.d_c, a.d_r) == 1 ? launch_select<1>(a, st) : launch_select<2>(a, st);
}

}  // namespace egmla
