// egmla_pages.cu - the pages of a paged latent cache on the GPU (sm_103a):
//
//   page_plan_kernel     a serving step's pages from its requests' lengths: released
//                        pages onto the free stack, new ones from it into the block
//                        table, the packed offsets and the cache slot of every new
//                        token
//   page_summary_kernel  the mean key [c~ ; k^R] of every page that became full
//   page_scores_kernel   each sequence's pages by their mean keys: the largest
//                        logit that any head gives it
//   select_pages_kernel  the best pages of each sequence as a block table
//
// The last three make the page-sparse decode: the split-KV kernels then attend over
// the selected pages alone (a cached RoPE key carries its position, so a page may
// stand anywhere in a block table).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "egmla_common.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"

namespace egmla {
namespace {

__device__ __forceinline__ int pages_of(int n) { return (n + kPage - 1) / kPage; }

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
constexpr int kPlanThreads = 512;

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanArgs p) {
  extern __shared__ int32_t plan_smem[];
  __shared__ int ws[32];
  int32_t* E = plan_smem;              // [batch + 1] exclusive sums of the pages asked for
  int32_t* len = E + p.batch + 1;      // [batch] lengths before the step
  int32_t* cum = len + p.batch;        // [batch + 1] of the pages released, then of the tokens granted
  const int tid = threadIdx.x, C = static_cast<int>(gridDim.x), rank = static_cast<int>(blockIdx.x);
  const int first = rank * kPlanThreads + tid, step = C * kPlanThreads;   // this thread's share of a list
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
  for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int L = 0, back = 0, need = 0, ask = 0, sum;
    bool fits = true;
    if (b < p.batch && !request(b, L, back, need, ask, fits)) bad = true;
    const int e = block_scan(need, ws, sum);
    if (b < p.batch) {
      E[b] = total_need + e - need;
      len[b] = L;
    }
    total_need += sum;
    const int r = block_scan(back, ws, sum);
    if (b < p.batch) cum[b] = R + r - back;
    R += sum;
  }
  if (tid == 0) {
    E[p.batch] = total_need;
    cum[p.batch] = R;
  }
  const int avail = min(F + R, p.num_pages);
  if (avail < F + R) bad = true;   // more pages released than there are
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
  for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int t = 0, g = 0, L = 0, sum;
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
    const int c = block_scan(t, ws, sum);
    if (b < p.batch) cum[b] = total + c - t;
    if (b < p.batch && b % C == rank) p.cu_seqlens[b] = total + c - t;
    total += sum;
    block_scan(g, ws, sum);
    granted_pages += sum;
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
    for (int k = first; k < p.max_slots; k += step) {
      int slot = -1;
      if (k < total) {
        const int b = find_in(cum, p.batch, k);
        const int pos = len[b] + (k - cum[b]), lp = pos / kPage, have = pages_of(len[b]);
        const int page = lp < have ? p.block_table[static_cast<size_t>(b) * p.max_pages + lp]
                                   : p.free_pages[avail - 1 - (E[b] + lp - have)];
        if (static_cast<unsigned>(page) < static_cast<unsigned>(p.num_pages))
          slot = page * kPage + pos % kPage;
        else
          bad = true;
      }
      p.slots[k] = slot;
    }
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

// 16 bytes of a row as pairs of fp32 values
template <typename T>
struct Unit;
template <>
struct Unit<__nv_bfloat16> {
  static constexpr int kPairs = 4;
  static __device__ __forceinline__ void widen(const uint4& w, float2 (&x)[4]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
  }
};
template <>
struct Unit<float> {
  static constexpr int kPairs = 2;
  static __device__ __forceinline__ void widen(const uint4& w, float2 (&x)[2]) {
    x[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    x[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
  }
};

// v[r] summed over the warp's lanes, for every lane
__device__ __forceinline__ void warp_sums(float (&v)[2], int lane) {
  const bool h16 = lane & 16;
  float c = (h16 ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, h16 ? v[0] : v[1], 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
#pragma unroll
  for (int r = 0; r < 2; ++r) v[r] = __shfl_sync(0xffffffffu, c, 16 * r);
}
__device__ __forceinline__ void warp_sums(float (&v)[4], int lane) {
  const bool h16 = lane & 16, h8 = lane & 8;
  const float a = (h16 ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, h16 ? v[0] : v[2], 16);
  const float b = (h16 ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, h16 ? v[1] : v[3], 16);
  float c = (h8 ? b : a) + __shfl_xor_sync(0xffffffffu, h8 ? a : b, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = __shfl_sync(0xffffffffu, c, 16 * (r >> 1) + 8 * (r & 1));
}
// A block takes a page, a warp eight of its rows, kFlight of them at a time with every
// load in flight; a lane has 16-byte units lane, lane + 32, .. of a row (NU of them).  LayerNorm in two passes over the
// registers, the sums of the rows in flight reduced together.  The mean of gamma x_j +
// beta is gamma mean(x_j) + beta, so the affine part comes last.  k^R rows: a lane has one
// unit of every few rows.
// Bound by issue and latency (0.5 of the issue slots, 136 instructions a row, most of them
// widening, the two passes and the two reductions): 57.0 us for 8 x 32K tokens at d_c
// 256, 5.3 TB/s of cache and gate rows; floor 27.4.  GM, the gate mode, at compile time:
// 59.2 -> 57.0.  Forms that copy the pages by TMA into a ring or keep the next page's ids
// ahead in persistent blocks measured 57.1 and 73.2 and were not kept.
template <typename T, int NU, int GM>
__global__ void __launch_bounds__(32 * kSumWarps, NU == 4 ? 2 : 3) page_summary_kernel(const SummaryArgs p) {
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
#pragma unroll
  for (int u = 0; u < NU; ++u)
#pragma unroll
    for (int e = 0; e < VP; ++e) acc[u][e] = make_float2(0.f, 0.f);
  const T* c = static_cast<const T*>(p.c_pool) + row0 * p.d_c;
  const T* table = static_cast<const T*>(p.gate_table);
  const float inv_n = 1.f / static_cast<float>(p.d_c);
#pragma unroll 1
  for (int r0 = 0; r0 < kSumRows; r0 += kFlight) {
    uint4 cw[kFlight][NU], gw[kFlight][NU];
#pragma unroll
    for (int r = 0; r < kFlight; ++r) {
      const int id = __shfl_sync(0xffffffffu, id_row, r0 + r);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int at = lane + 32 * u;
        cw[r][u] = gw[r][u] = make_uint4(0u, 0u, 0u, 0u);
        if (at < units) {
          cw[r][u] = __ldg(reinterpret_cast<const uint4*>(c + static_cast<size_t>(r0 + r) * p.d_c) + at);
          if (GATE) gw[r][u] = __ldg(reinterpret_cast<const uint4*>(table + static_cast<size_t>(id) * p.d_c) + at);
        }
      }
    }
    float2 x[kFlight][NU][VP];
    float s[kFlight];
#pragma unroll
    for (int r = 0; r < kFlight; ++r) {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float2 t[VP];
        U::widen(cw[r][u], x[r][u]);
        if (GATE) U::widen(gw[r][u], t);
#pragma unroll
        for (int e = 0; e < VP; ++e) {
          if (GATE) x[r][u][e] = GATE_ADD ? __fadd2_rn(x[r][u][e], t[e]) : __fmul2_rn(x[r][u][e], t[e]);
          sum = __fadd2_rn(sum, x[r][u][e]);
        }
      }
      s[r] = sum.x + sum.y;
    }
    if (GATE_LN) {
      warp_sums(s, lane);
#pragma unroll
      for (int r = 0; r < kFlight; ++r) {
        const float2 mu = make_float2(-s[r] * inv_n, -s[r] * inv_n);
        float2 sq = make_float2(0.f, 0.f);
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const bool live = lane + 32 * u < units;
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            x[r][u][e] = live ? __fadd2_rn(x[r][u][e], mu) : make_float2(0.f, 0.f);
            sq = __ffma2_rn(x[r][u][e], x[r][u][e], sq);
          }
        }
        s[r] = sq.x + sq.y;
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

// ============================================================================ 3. page scores
// score(b, p) = max_h scale (q^_bh . m^c_p + q^R_bh . m^R_p) in exact fp32 products.
// A block takes a sequence's queries into shared memory and kScPages of its pages; a
// warp four pages at a time, so that a query value read serves four products.  Lanes
// share a row; the 16 heads' sums of two pages take one transposing reduction.
constexpr int kScWarps = 8, kScPages = 32, kScHeads = 16;

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

__global__ void __launch_bounds__(32 * kScWarps) page_scores_kernel(const SelectArgs p) {
  extern __shared__ float4 sc_q[];   // [kScHeads][units]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x / p.chunks, D = p.d_c + p.d_r, units = D / 4;
  grid_dependency_wait();
  const int np = pages_of(min(max(__ldg(p.seq_lens + b), 0), p.max_seq_len));
  if (np <= p.budget) return;   // every page is taken
  const int lo = p.keep_first, hi = np - p.keep_last;   // the pages that are ranked
  const int p0 = lo + (blockIdx.x - b * p.chunks) * kScPages;
  if (p0 >= hi) return;
  const float* q = p.q + static_cast<size_t>(b) * p.q_stride;
  for (int i = threadIdx.x; i < kScHeads * units; i += blockDim.x) {
    const int h = i / units, u = i - h * units;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (h < p.H)
      v = 4 * u < p.d_c ? *reinterpret_cast<const float4*>(q + h * p.d_c + 4 * u)
                        : *reinterpret_cast<const float4*>(q + p.H * p.d_c + h * p.d_r + 4 * u - p.d_c);
    sc_q[i] = v;
  }
  __syncthreads();
  const int w0 = p0 + 4 * warp;
  if (w0 >= hi) return;
  const float4* row[4];
  bool bad = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    int page = __ldg(p.block_table + static_cast<size_t>(b) * p.max_pages + min(w0 + k, hi - 1));
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) {
      bad = true;
      page = 0;
    }
    row[k] = reinterpret_cast<const float4*>(p.summary + static_cast<size_t>(page) * D);
  }
  float acc[2][32];   // pages 2 i and 2 i + 1: [page % 2][head]
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[0][i] = acc[1][i] = 0.f;
  for (int u = lane; u < units; u += 32) {
    float4 m[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = __ldg(row[k] + u);
#pragma unroll
    for (int h = 0; h < kScHeads; ++h) {
      const float4 x = sc_q[h * units + u];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float& a = acc[k / 2][16 * (k % 2) + h];
        a = fmaf(x.x, m[k].x, a);
        a = fmaf(x.y, m[k].y, a);
        a = fmaf(x.z, m[k].z, a);
        a = fmaf(x.w, m[k].w, a);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float s = sum32_transpose(acc[i], lane);
    if ((lane & 15) >= p.H) s = -INFINITY;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, o));
    const int lp = w0 + 2 * i + (lane >> 4);
    if ((lane & 15) == 0 && lp < hi) p.scores[static_cast<size_t>(b) * p.max_pages + lp] = s * p.scale;
  }
  if (bad && lane == 0) report_status(p.status, kStatusOutOfRange);
}

// ============================================================================ 4. page selection
// A block per sequence.  The ranked pages' scores as whole numbers of the same order
// (no number comes last); the count-th largest by four passes over a histogram of
// eight bits each; then the pages above it and the first of those equal to it, in
// order, between the pages that are always kept.
constexpr int kSelThreads = 256;

__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = __float_as_uint(s);
  return s != s ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelThreads) select_pages_kernel(const SelectArgs p) {
  __shared__ int hist[256];
  __shared__ int ws[32];
  __shared__ uint32_t sh_digit;
  __shared__ int sh_above;
  const int b = blockIdx.x, tid = threadIdx.x;
  grid_dependency_wait();
  const int given = __ldg(p.seq_lens + b);
  const int L = min(max(given, 0), p.max_seq_len);
  const int np = pages_of(L);
  if (given != L && tid == 0) report_status(p.status, kStatusOutOfRange);
  const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_pages;
  int32_t* out = p.sel_table + static_cast<size_t>(b) * p.width;
  int32_t* sel = p.selected != nullptr ? p.selected + static_cast<size_t>(b) * p.budget : nullptr;
  const int taken = min(np, p.budget);
  if (tid == 0) p.sel_lens[b] = L - (np - taken) * kPage;
  if (sel != nullptr)
    for (int i = taken + tid; i < p.budget; i += kSelThreads) sel[i] = -1;
  if (np <= p.budget) {
    for (int i = tid; i < np; i += kSelThreads) {
      out[i] = __ldg(table + i);
      if (sel != nullptr) sel[i] = i;
    }
    return;
  }
  const float* scores = p.scores + static_cast<size_t>(b) * p.max_pages;
  const int lo = p.keep_first, hi = np - p.keep_last, want = p.budget - p.keep_first - p.keep_last;
  // the want-th largest key (`prefix`) and how many of its equals are wanted (`left`)
  uint32_t prefix = 0;
  int left = want;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[tid] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kSelThreads) {
        const uint32_t k = score_key(scores[i]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1);
      }
      __syncthreads();
      // digits from the largest down: thread t has digit 255 - t
      int total;
      const int mine = hist[255 - tid], incl = block_scan(mine, ws, total);
      if (incl >= left && incl - mine < left) {
        sh_digit = static_cast<uint32_t>(255 - tid);
        sh_above = incl - mine;
      }
      __syncthreads();
      prefix |= sh_digit << shift;
      left -= sh_above;
    }
  }
  int at = lo, equal = 0;   // pages written, and equals met, before this round
  for (int i = tid; i < lo; i += kSelThreads) {
    out[i] = __ldg(table + i);
    if (sel != nullptr) sel[i] = i;
  }
  for (int i = tid; i < p.keep_last; i += kSelThreads) {
    out[p.budget - p.keep_last + i] = __ldg(table + hi + i);
    if (sel != nullptr) sel[p.budget - p.keep_last + i] = hi + i;
  }
  for (int i0 = lo; want > 0 && i0 < hi; i0 += kSelThreads) {
    const int i = i0 + tid;
    const uint32_t k = i < hi ? score_key(scores[i]) : 0u;
    const bool tie = i < hi && k == prefix;
    int total;
    const int t = block_scan(tie ? 1 : 0, ws, total) - (tie ? 1 : 0) + equal;   // equals before this page
    equal += total;
    const bool take = i < hi && (k > prefix || (tie && t < left));
    const int pos = block_scan(take ? 1 : 0, ws, total) - 1 + at;
    at += total;
    if (take) {
      out[pos] = __ldg(table + i);
      if (sel != nullptr) sel[pos] = i;
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
  const int ctas = (a.slots != nullptr ? a.max_slots : 0) + a.batch > 4096 ? 8 : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kPlanThreads);
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

int score_chunks(int max_seq_len, int keep_first, int keep_last) {
  const int ranked = (max_seq_len + kPage - 1) / kPage - keep_first - keep_last;
  return ranked > 0 ? (ranked + kScPages - 1) / kScPages : 0;
}

cudaError_t launch_select_pages(const SelectArgs& a, cudaStream_t st) {
  if ((a.max_seq_len + kPage - 1) / kPage > a.budget && a.budget > a.keep_first + a.keep_last) {
    const size_t smem = static_cast<size_t>(kScHeads) * (a.d_c + a.d_r) * 4;
    cudaError_t e = allow_smem(page_scores_kernel, static_cast<size_t>(kScHeads) * (kSumMaxDc + kSumMaxDr) * 4);
    if (e == cudaSuccess)
      e = launch_chained(page_scores_kernel, dim3(static_cast<unsigned>(a.chunks) * a.batch), dim3(32 * kScWarps), smem,
                         st, a);
    if (e != cudaSuccess) return e;
  }
  return launch_chained(select_pages_kernel, dim3(a.batch), dim3(kSelThreads), 0, st, a);
}

}  // namespace egmla
