// egmla_tokens.cu - packed tokens between the projections and the cache: the rotary
// embedding of their queries and keys, their rows written into a cache that holds the
// latent in 8 bits, and cached rows read back.  See include/egmla.h for the contract.
//
// Packed token k belongs to the sequence b with cu[b] <= k < cu[b + 1], as its token
// k - cu[b], at position positions[b] + k - cu[b] (cu null: to sequence k, at
// positions[k]).  A warp finds b for its token by ballots over 32 offsets at a time, which
// see some of the offsets only: those around b are looked at again, and all offsets once
// per call, so that a list that is not in order is reported and misplaces no token.
//
// All three calls are bound by memory: every row is read once and written once, in 16-byte
// units with several in flight per lane, by warps that need nothing of one another.
// Blocks of four warps, or of one where rope has many tokens: a block's slots free up
// together (32K tokens' rope with eight warps a block 69.2 us, four 63.9, one 63.1).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../../include/egmla.h"
#include "egmla_common.cuh"
#include "egmla_kernels.h"
#include "egmla_ptx.cuh"
#include "egmla_q8.cuh"

namespace egmla {
namespace {

constexpr int kTokThreads = 128, kTokWarps = kTokThreads / 32;

struct Packed {
  const int32_t* cu;          // [batch + 1], null: one token per sequence
  const int32_t* positions;   // [batch], null: 0
  int batch, tokens;
  int32_t* status;
};

// Sequence of packed token k, the same in every lane: how many of cu[1 .. batch] are <= k;
// `batch` behind the last one.
__device__ __forceinline__ int sequence_of(const Packed& p, int k, int lane) {
  int b = 0, n = p.batch;
  while (n > 0) {
    const int step = (n + 31) / 32, i = (lane + 1) * step;
    const bool below = i <= n && __ldg(p.cu + b + i) <= k;
    const int c = __popc(__ballot_sync(0xffffffffu, below));
    b += c * step;
    n = min(n - c * step, step - 1);
  }
  return b;
}

// First token of sequence b if token k is surely its: cu[b] <= k < cu[b + 1], and both in order
// with the offsets before and behind them (before the first 0).  A single offset that makes
// the list decrease is then none of b's two, and b is the sequence that the others say.
// -1: of no sequence, or in doubt.
__device__ __forceinline__ int first_of(const Packed& p, int b, int k) {
  const int before = b > 0 ? __ldg(p.cu + b - 1) : 0, first = __ldg(p.cu + b), end = __ldg(p.cu + b + 1);
  const int behind = b + 2 <= p.batch ? __ldg(p.cu + b + 2) : INT32_MAX;
  return before <= first && first <= k && k < end && end <= behind ? first : -1;
}

// Reports offsets that do not begin at 0 or that decrease; warp w of the grid's `warps` looks at
// its part of them, of which there are kOffsetsPerLane to a lane at most (offset_blocks).
// (Where the warp goes on to look for its tokens' sequences, it has brought the lines that
// this needs.)
constexpr int kOffsetsPerLane = 2;
__device__ __forceinline__ void check_offsets(const Packed& p, int w, int warps, int lane) {
  if (p.cu == nullptr) return;
  bool wrong = w == 0 && __ldg(p.cu) != 0;
#pragma unroll 1
  for (int64_t i = static_cast<int64_t>(w) * 32 + lane; i < p.batch; i += static_cast<int64_t>(warps) * 32)
    wrong |= __ldg(p.cu + i) > __ldg(p.cu + i + 1);
  if (wrong) report_status(p.status, kStatusOutOfRange);
}
// Blocks that this takes: more than the tokens' where there are many empty sequences.
int offset_blocks(const Packed& p, int warps_per_block) {
  const int64_t per_block = 32LL * kOffsetsPerLane * warps_per_block;
  return p.cu == nullptr ? 0 : static_cast<int>((p.batch + per_block - 1) / per_block);
}

// Position of packed token k, the same in every lane; false for a token of no sequence or of
// one with a negative position.
__device__ __forceinline__ bool find_position(const Packed& p, int k, int lane, int64_t& pos) {
  int first = k, b = k;   // the sequence's first packed token
  if (p.cu != nullptr) {
    b = sequence_of(p, k, lane);
    if (b >= p.batch) return false;   // a row behind the last sequence
    first = first_of(p, b, k);
    if (first < 0) return false;
  }
  const int start = p.positions != nullptr ? __ldg(p.positions + b) : 0;
  if (start < 0) return false;
  pos = static_cast<int64_t>(start) + k - first;
  return true;
}

// ------------------------------------------------------------------ rotary embedding
// pair i of a token at position t turns by t f_i: (x, y) -> m (x cos - y sin, x sin + y cos).
// The angle is a 64-bit fraction of a turn, t times f_i / (2 pi) (rounded to 2^-64 of a turn
// and, on the host, to a double): an integer product, whose low 64 bits are what is left
// after whole turns, so that far positions lose no more than the double's rounding and no
// double precision runs on the GPU.  Sine and cosine are taken in fp32 of what is left to the nearest quarter turn.
constexpr int kMaxPairs = 128;

struct RopeArgs {
  Packed tok;
  const uint8_t *q, *k;
  uint8_t *q_out, *k_out;
  int64_t q_stride, q_out_stride, k_stride, k_out_stride;   // bytes between tokens
  int H, dn, dr;
  int half, q_in_place;
  float magnitude;
  uint64_t turn[kMaxPairs];   // f_i / (2 pi) in 2^-64
};

// cos and sin of a 2^-64 fraction of a turn, times m
__device__ __forceinline__ float2 turn_cos_sin(uint64_t fraction, float m) {
  const uint32_t x = static_cast<uint32_t>(fraction >> 32);
  const uint32_t quarter = (x + 0x20000000u) >> 30;   // the nearest quarter turn, mod 4
  const int32_t rest = static_cast<int32_t>(x - (quarter << 30));
  float s, c;
  sincospif(static_cast<float>(rest) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
  const bool swap = quarter & 1;
  float cs = swap ? s : c, sn = swap ? c : s;
  if (quarter == 1 || quarter == 2) cs = -cs;
  if (quarter >= 2) sn = -sn;
  return make_float2(m * cs, m * sn);
}

// 16 bytes that are read once
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

template <typename T>
__device__ __forceinline__ float to_f32(T x) { return static_cast<float>(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// the values of a 16-byte unit
template <typename T>
union Vec {
  uint4 raw;
  T v[16 / sizeof(T)];
};

__device__ __forceinline__ float2 turned(float x, float y, float2 cs) {
  return make_float2(fmaf(x, cs.x, -(y * cs.y)), fmaf(x, cs.y, y * cs.x));
}

// One part of a head in registers: what is loaded before it is turned.
template <typename T, bool HALF>
struct RopeItem {
  static constexpr int N = 16 / sizeof(T);
  Vec<T> a, b;   // HALF: a unit of the first half and its partner in the second; else a alone
  __device__ __forceinline__ void load(const uint4* row, int r, int half_units) {
    a.raw = ld_stream(row + r);
    if (HALF) b.raw = ld_stream(row + r + half_units);
  }
  __device__ __forceinline__ void turn_and_store(uint4* row, int r, int half_units, const float2* cs) {
    if constexpr (HALF) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 t = turned(to_f32(a.v[i]), to_f32(b.v[i]), cs[r * N + i]);
        a.v[i] = from_f32<T>(t.x);
        b.v[i] = from_f32<T>(t.y);
      }
      row[r + half_units] = b.raw;
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float2 t = turned(to_f32(a.v[2 * i]), to_f32(a.v[2 * i + 1]), cs[r * (N / 2) + i]);
        a.v[2 * i] = from_f32<T>(t.x);
        a.v[2 * i + 1] = from_f32<T>(t.y);
      }
    }
    row[r] = a.raw;
  }
};

// The token's units of heads h0 .. h1 - 1 dealt to the lanes: item u is unit u % n of head
// h0 + u / n, kept up without divisions as u grows by 32.
struct Deal {
  int h, r, n, dh, dr;
  __device__ __forceinline__ Deal(int h0, int n, int lane) : h(h0 + lane / n), r(lane % n), n(n), dh(32 / n), dr(32 % n) {}
  __device__ __forceinline__ void next() {
    h += dh;
    r += dr;
    if (r >= n) {
      r -= n;
      ++h;
    }
  }
};

// A warp per token and part of its H + 1 heads (the last one is the key); blockIdx.y: the
// part.  Rows, heads and their rotated parts consist of 16-byte units, each read once,
// kUnroll of them in flight per lane, the first before the token's angles are known.  The
// angles are taken once per warp and token, a pair per lane, and shared by all heads.
// 32,768 tokens of 16 heads of 128 + 64 and a key, from projection rows to dense ones (411
// MB): 63.1 us, 6.5 TB/s, 96 % of the copy rate (in blocks of four warps with two units in
// flight 73.9, three 70.0, four 63.9; a pair of bf16 values at a time, as below, 229).  13 ragged
// prompts (13,271 tokens) in halves: 28.0 us, with the compiler's choice of 91 registers and
// blocks of four warps 29.9, blocks of one with 72 registers 28.4 (spills), with 106 29.1.
template <bool HALF, int WARPS>
constexpr int kRopeResident = WARPS == 1 ? 24 : HALF ? 5 : 7;   // blocks per SM
template <typename T, bool HALF, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, kRopeResident<HALF, WARPS>) rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int kUnroll = 4;
  __shared__ __align__(16) float2 table[WARPS][kMaxPairs];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = blockIdx.x * WARPS + warp;
  grid_dependency_wait();
  if (k >= a.tok.tokens) {
    if (blockIdx.y == 0) check_offsets(a.tok, k, gridDim.x * WARPS, lane);
    return;
  }
  constexpr int kBytes = sizeof(T);
  const int heads = a.H + 1, parts = gridDim.y, part = blockIdx.y;
  const int h0 = heads * part / parts, h1 = heads * (part + 1) / parts;
  const int units = a.dr * kBytes / 16, items = HALF ? units / 2 : units;   // of a head's rotated part
  const int nope = a.dn * kBytes / 16, stride = nope + units;
  const uint4* q = reinterpret_cast<const uint4*>(a.q + k * a.q_stride);
  const uint4* key = reinterpret_cast<const uint4*>(a.k + k * a.k_stride);
  uint4* q_out = reinterpret_cast<uint4*>(a.q_out + k * a.q_out_stride);
  uint4* key_out = reinterpret_cast<uint4*>(a.k_out + k * a.k_out_stride);
  const int hq = a.q == nullptr ? a.H : h0;                       // first head there is
  const int hend = a.k == nullptr ? min(h1, a.H) : h1;

  RopeItem<T, HALF> item[kUnroll];
  Deal first(hq, items, lane);
  {
    Deal d = first;
#pragma unroll
    for (int j = 0; j < kUnroll; ++j, d.next())
      if (d.h < hend) item[j].load(d.h < a.H ? q + d.h * stride + nope : key, d.r, items);
  }
  if (part == 0) check_offsets(a.tok, k, gridDim.x * WARPS, lane);
  int64_t pos;
  if (!find_position(a.tok, k, lane, pos)) return;
  if (nope > 0 && !a.q_in_place && a.q != nullptr) {
    Deal d(h0, nope, lane);
    const int end = min(h1, a.H);
    while (d.h < end) {
      uint4 v[kUnroll];
      Deal e = d;
#pragma unroll
      for (int j = 0; j < kUnroll; ++j, e.next())
        if (e.h < end) v[j] = ld_stream(q + e.h * stride + e.r);
#pragma unroll
      for (int j = 0; j < kUnroll; ++j, d.next())
        if (d.h < end) q_out[d.h * stride + d.r] = v[j];
    }
  }
  float2* cs = table[warp];
  for (int i = lane; i < a.dr / 2; i += 32) cs[i] = turn_cos_sin(static_cast<uint64_t>(pos) * a.turn[i], a.magnitude);
  __syncwarp();
  while (first.h < hend) {
    Deal d = first;
#pragma unroll
    for (int j = 0; j < kUnroll; ++j, d.next())
      if (d.h < hend) item[j].turn_and_store(d.h < a.H ? q_out + d.h * stride + nope : key_out, d.r, items, cs);
    first = d;
#pragma unroll
    for (int j = 0; j < kUnroll; ++j, d.next())
      if (d.h < hend) item[j].load(d.h < a.H ? q + d.h * stride + nope : key, d.r, items);
  }
}

// The same at any alignment and size, a pair per lane and turn: values of two or four bytes
// instead of sixteen (32,768 bf16 tokens as above, shifted by one entry: 151 us).
template <typename T>
__global__ void __launch_bounds__(kTokThreads) rope_any_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ float2 table[kTokWarps][kMaxPairs];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = blockIdx.x * kTokWarps + warp;
  grid_dependency_wait();
  if (blockIdx.y == 0) check_offsets(a.tok, k, gridDim.x * kTokWarps, lane);
  if (k >= a.tok.tokens) return;
  int64_t pos;
  if (!find_position(a.tok, k, lane, pos)) return;
  const int pairs = a.dr / 2, heads = a.H + 1, parts = gridDim.y, part = blockIdx.y;
  float2* cs = table[warp];
  for (int i = lane; i < pairs; i += 32) cs[i] = turn_cos_sin(static_cast<uint64_t>(pos) * a.turn[i], a.magnitude);
  __syncwarp();
  const T* q = reinterpret_cast<const T*>(a.q + k * a.q_stride);
  const T* key = reinterpret_cast<const T*>(a.k + k * a.k_stride);
  T* q_out = reinterpret_cast<T*>(a.q_out + k * a.q_out_stride);
  T* key_out = reinterpret_cast<T*>(a.k_out + k * a.k_out_stride);
  const int h0 = heads * part / parts, h1 = heads * (part + 1) / parts;
  const int dq = a.dn + a.dr, hend = a.k == nullptr ? min(h1, a.H) : h1;
  if (a.dn > 0 && !a.q_in_place && a.q != nullptr)
    for (Deal d(h0, a.dn, lane); d.h < min(h1, a.H); d.next()) q_out[d.h * dq + d.r] = q[d.h * dq + d.r];
  for (Deal d(a.q == nullptr ? a.H : h0, pairs, lane); d.h < hend; d.next()) {
    const int x = a.half ? d.r : 2 * d.r, y = a.half ? x + pairs : x + 1;
    const T* src = d.h < a.H ? q + d.h * dq + a.dn : key;
    T* dst = d.h < a.H ? q_out + d.h * dq + a.dn : key_out;
    const float2 t = turned(to_f32(src[x]), to_f32(src[y]), cs[d.r]);
    dst[x] = from_f32<T>(t.x);
    dst[y] = from_f32<T>(t.y);
  }
}

// Parts that a token's heads are cut into: as many as give every SM eight warps, and two while
// all of their warps are resident at once.  us with one part / with the rule (blocks of
// four warps): 1 token 3.1 / 2.5, 64 tokens 3.4 / 2.8, 256 3.4 / 2.9, 1024 4.0 / 3.6, 2048 5.6 /
// 4.8; as many as give sixteen: 256 tokens 3.4, 512 3.4 (rule 3.1).  One part comes in blocks of one
// warp: halves of 2048 tokens 5.3 us (two parts, whose last wave is nearly empty, 6.4), 4096
// 10.7 (11.3); 64 tokens in such blocks 2.9 (2.8), 1024 3.7 (3.6).
constexpr int kRopeWarps = 8;
template <typename T, int WARPS>
cudaError_t launch_rope_units(const RopeArgs& a, int parts, cudaStream_t st) {
  const dim3 grid(std::max((a.tok.tokens + WARPS - 1) / WARPS, offset_blocks(a.tok, WARPS)), parts), block(32 * WARPS);
  return a.half ? launch_chained(rope_kernel<T, true, WARPS>, grid, block, 0, st, a)
                : launch_chained(rope_kernel<T, false, WARPS>, grid, block, 0, st, a);
}
template <typename T>
cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  auto on = [](const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 16 == 0; };
  const int e = sizeof(T);
  const bool units = a.dn * e % 16 == 0 && a.dr * e % (a.half ? 32 : 16) == 0 && on(a.q, a.q_stride) &&
                     on(a.q_out, a.q_out_stride) && on(a.k, a.k_stride) && on(a.k_out, a.k_out_stride);
  int want = (kSms * kRopeWarps - 1) / a.tok.tokens + 1;
  const int resident = kSms * kTokWarps * (a.half ? kRopeResident<true, kTokWarps> : kRopeResident<false, kTokWarps>);
  if (want < 2 && a.tok.tokens <= resident / 2) want = 2;
  const int parts = want < a.H + 1 ? want : a.H + 1;
  if (!units)
    return launch_chained(rope_any_kernel<T>,
                          dim3(std::max((a.tok.tokens + kTokWarps - 1) / kTokWarps, offset_blocks(a.tok, kTokWarps)), parts),
                          dim3(kTokThreads), 0, st, a);
  return parts == 1 ? launch_rope_units<T, 1>(a, parts, st) : launch_rope_units<T, kTokWarps>(a, parts, st);
}

// ------------------------------------------------------------------ the cache in 8 bits
struct CacheArgs {
  Packed tok;
  uint8_t* c8;
  float* scale;
  uint8_t* kr;
  int32_t* ids;
  // packed rows: written by the read, read by the append (null: none)
  uint8_t *c_rows, *kr_rows;
  int32_t* id_rows;
  int64_t c_stride, kr_stride;   // bytes between tokens
  const int32_t* table;
  int max_pages, num_pages, d_c, kr_bytes;
};

// Rows of the pool of the packed tokens k0 .. k0 + T - 1: lane i < T gets token i's, -1 for none.
template <int T>
__device__ __forceinline__ int cache_rows(const CacheArgs& a, int k0, int lane) {
  int b = k0 + lane, first = b;
  if (a.tok.cu != nullptr && a.tok.batch <= 32) {
    // every offset in a lane: the tokens' sequences by a ballot each
    const bool held = lane < a.tok.batch;
    const int own = held ? __ldg(a.tok.cu + lane) : 0, end = held ? __ldg(a.tok.cu + lane + 1) : INT32_MAX;
#pragma unroll
    for (int i = 0; i < T; ++i) {
      const int n = __popc(__ballot_sync(0xffffffffu, end <= k0 + i && held));
      if (lane == i) b = n;
    }
    // (as first_of and check_offsets)
    const int at = min(b, 31), begin = __shfl_sync(0xffffffffu, own, at), last = __shfl_sync(0xffffffffu, end, at);
    const uint32_t falls = __ballot_sync(0xffffffffu, held && own > end);   // bit i: from offset i to i + 1
    if (falls != 0 || (lane == 0 && own != 0)) report_status(a.tok.status, kStatusOutOfRange);
    const bool doubt = (falls | falls << 1 | falls >> 1) >> at & 1;
    first = !doubt && begin <= k0 + lane && k0 + lane < last ? begin : -1;   // (below 0 too: of no sequence)
  } else if (a.tok.cu != nullptr) {
    // a search for the first token, and for another only where its sequence ends before it
    check_offsets(a.tok, k0 / T, gridDim.x * kTokWarps, lane);
    int found = 0, end = INT32_MIN;
#pragma unroll
    for (int i = 0; i < T; ++i) {
      if (k0 + i >= end) {
        found = sequence_of(a.tok, k0 + i, lane);
        end = found < a.tok.batch ? __ldg(a.tok.cu + found + 1) : INT32_MAX;
      }
      if (lane == i) b = found;
    }
  }
  int64_t pos = -1;
  if (lane < T && k0 + lane < a.tok.tokens && b < a.tok.batch) {
    const int start = a.tok.positions != nullptr ? __ldg(a.tok.positions + b) : 0;
    if (a.tok.cu != nullptr && a.tok.batch > 32) first = first_of(a.tok, b, k0 + lane);
    if (first >= 0 && start >= 0) pos = static_cast<int64_t>(start) + k0 + lane - first;
  }
  if (pos < 0) return -1;
  const int64_t lp = pos / kPage;
  const int page = lp < a.max_pages ? __ldg(a.table + static_cast<size_t>(b) * a.max_pages + lp) : -1;
  if (page < 0 || page >= a.num_pages) {
    report_status(a.tok.status, kStatusOutOfRange);
    return -1;
  }
  return page * kPage + static_cast<int>(pos % kPage);   // (num_pages x 64 rows fit 32 bits)
}

// eight values of a packed row as they are stored
template <typename T>
struct Packed8 {
  static constexpr int N = 16 / sizeof(T);
  Vec<T> v[8 / N];
  __device__ __forceinline__ void load(const uint8_t* row, int unit) {
#pragma unroll
    for (int j = 0; j < 8 / N; ++j) v[j].raw = ld_stream(reinterpret_cast<const uint4*>(row) + unit * (8 / N) + j);
  }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f32(v[i / N].v[i % N]);
  }
  // the fp32 bits of the largest magnitude (above those of infinity: a NaN)
  __device__ __forceinline__ uint32_t most() const {
    float x[8];
    widen(x);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
  }
};
template <typename T>
__device__ __forceinline__ void store8(uint8_t* row, int unit, const float (&x)[8]) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < 8 / N; ++j) {
    Vec<T> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.v[i] = from_f32<T>(x[j * N + i]);
    *reinterpret_cast<uint4*>(row + (unit * (8 / N) + j) * 16) = v.raw;
  }
}

// A warp per T tokens, eight features of the latent a lane and turn (TURNS of them).  The
// tokens' rows are requested before their places are looked up, a chain of three
// dependent loads that T tokens share.  32,768 tokens at d_c 256 (34 MB): 8.6 us from L2, 12.1
// cold (2.8 TB/s); from L2 with one token a warp 13.1, two 9.9, eight 10.8.  Ten blocks of
// four warps an SM: more than a wave, each of whose warps asks for its k^R rows last.
template <typename E, int T, int TURNS>
__global__ void __launch_bounds__(kTokThreads) append_q8_kernel(const __grid_constant__ CacheArgs a) {
  const int lane = threadIdx.x & 31, k0 = (blockIdx.x * kTokWarps + (threadIdx.x >> 5)) * T;
  grid_dependency_wait();
  const int units = a.d_c / 8, kru = a.kr_bytes / 16;
  Packed8<E> x[T][TURNS];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
      x[t][j] = Packed8<E>{};
      if (k0 + t < a.tok.tokens && lane + 32 * j < units) x[t][j].load(a.c_rows + (k0 + t) * a.c_stride, lane + 32 * j);
    }
  const int row = cache_rows<T>(a, k0, lane);
  if (k0 >= a.tok.tokens) return;   // (here for the offsets alone)
  float own_scale = 0.f;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < TURNS; ++j) most = max(most, x[t][j].most());
    most = __reduce_max_sync(0xffffffffu, most);
    const int r = __shfl_sync(0xffffffffu, row, t);
    if (r < 0) continue;
    float scale, inverse;
    q8_scale(most, scale, inverse);
    if (lane == t) own_scale = scale;
    uint2* dst = reinterpret_cast<uint2*>(a.c8 + static_cast<size_t>(r) * a.d_c);
#pragma unroll
    for (int j = 0; j < TURNS; ++j)
      if (lane + 32 * j < units) {
        float v[8];
        x[t][j].widen(v);
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
          w[i] = q8_encode2(v[4 * i] * inverse, v[4 * i + 1] * inverse) |
                 q8_encode2(v[4 * i + 2] * inverse, v[4 * i + 3] * inverse) << 16;
        dst[lane + 32 * j] = make_uint2(w[0], w[1]);
      }
  }
  if (lane < T && row >= 0) {
    a.scale[row] = own_scale;
    if (a.ids != nullptr && a.id_rows != nullptr) a.ids[row] = a.id_rows[k0 + lane];
  }
  Deal d(0, kru, lane);
  for (int u = 0; u < T * kru; u += 32, d.next()) {   // (every lane to the end, for the shuffle)
    const int r = __shfl_sync(0xffffffffu, row, d.h < T ? d.h : 0);
    if (d.h < T && r >= 0)
      reinterpret_cast<uint4*>(a.kr + static_cast<size_t>(r) * a.kr_bytes)[d.r] =
          ld_stream(reinterpret_cast<const uint4*>(a.kr_rows + (k0 + d.h) * a.kr_stride) + d.r);
  }
}

// A warp per T tokens, likewise.  85K tokens at d_c 256 (66 MB): 13.2 us, 5.0 TB/s, with one
// token a warp 21.1, two 16.1, eight 16.3 (their last wave is nearly empty).
template <typename E, int T, int TURNS>
__global__ void __launch_bounds__(kTokThreads) read_q8_kernel(const __grid_constant__ CacheArgs a) {
  const int lane = threadIdx.x & 31, k0 = (blockIdx.x * kTokWarps + (threadIdx.x >> 5)) * T;
  grid_dependency_wait();
  const int units = a.d_c / 8, kru = a.kr_bytes / 16;
  const int row = cache_rows<T>(a, k0, lane);
  if (k0 >= a.tok.tokens) return;   // (here for the offsets alone)
  const float own_scale = lane < T && row >= 0 ? __ldg(a.scale + row) : 0.f;
  uint2 w[T][TURNS];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int r = __shfl_sync(0xffffffffu, row, t);
#pragma unroll
    for (int j = 0; j < TURNS; ++j)
      if (r >= 0 && lane + 32 * j < units)
        w[t][j] = __ldg(reinterpret_cast<const uint2*>(a.c8 + static_cast<size_t>(r) * a.d_c) + lane + 32 * j);
  }
  if (a.kr_rows != nullptr) {
    Deal d(0, kru, lane);
    for (int u = 0; u < T * kru; u += 32, d.next()) {   // (every lane to the end, for the shuffle)
      const int r = __shfl_sync(0xffffffffu, row, d.h < T ? d.h : 0);
      if (d.h < T && r >= 0)
        reinterpret_cast<uint4*>(a.kr_rows + (k0 + d.h) * a.kr_stride)[d.r] =
            ld_stream(reinterpret_cast<const uint4*>(a.kr + static_cast<size_t>(r) * a.kr_bytes) + d.r);
    }
  }
  if (lane < T && row >= 0 && a.id_rows != nullptr) a.id_rows[k0 + lane] = a.ids[row];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int r = __shfl_sync(0xffffffffu, row, t);
    const float scale = __shfl_sync(0xffffffffu, own_scale, t);
#pragma unroll
    for (int j = 0; j < TURNS; ++j)
      if (r >= 0 && lane + 32 * j < units) {
        float x[8];
        q8_decode4(w[t][j].x, x);
        q8_decode4(w[t][j].y, x + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= scale;
        store8<E>(a.c_rows + (k0 + t) * a.c_stride, lane + 32 * j, x);
      }
  }
}

// Tokens per warp: one while that leaves every SM no more than kTokFew warps, so that the
// fewest tokens wait for one another; else T.  us to read, one / four a warp: 64 tokens 2.1
// / 2.6, 1024 2.3 / 2.7, 3000 2.5 / 2.9, 5000 3.0 / 3.0, 8000 3.5 / 3.2; to write 64 2.3 / 2.4,
// 3000 2.8 / 2.8, 8000 4.0 / 3.3.
constexpr int kTokFew = 32;
template <int T, typename F>
cudaError_t launch_tokens(const CacheArgs& a, cudaStream_t st, F&& kernel) {
  const bool few = a.tok.tokens <= kSms * kTokFew;
  const int per_block = kTokWarps * (few ? 1 : T);
  const int blocks = std::max((a.tok.tokens + per_block - 1) / per_block, offset_blocks(a.tok, kTokWarps));
  return launch_chained(kernel(few), dim3(blocks), dim3(kTokThreads), 0, st, a);
}
template <typename E>
cudaError_t launch_append_q8(const CacheArgs& a, cudaStream_t st) {
  if (a.d_c <= 256)
    return launch_tokens<4>(a, st, [](bool few) { return few ? append_q8_kernel<E, 1, 1> : append_q8_kernel<E, 4, 1>; });
  return launch_tokens<4>(a, st, [](bool few) { return few ? append_q8_kernel<E, 1, 2> : append_q8_kernel<E, 4, 2>; });
}
template <typename E>
cudaError_t launch_read_q8(const CacheArgs& a, cudaStream_t st) {
  if (a.d_c <= 256)
    return launch_tokens<4>(a, st, [](bool few) { return few ? read_q8_kernel<E, 1, 1> : read_q8_kernel<E, 4, 1>; });
  return launch_tokens<4>(a, st, [](bool few) { return few ? read_q8_kernel<E, 1, 2> : read_q8_kernel<E, 4, 2>; });
}

// ------------------------------------------------------------------ arguments
bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// the common part of the three calls; EG_MLA_OK or the error code
int check_packed(const int32_t* cu, const int32_t* positions, int32_t batch, int32_t tokens) {
  if (batch < 0 || tokens < 0) return EG_MLA_ERR_INVALID_ARG;
  if (tokens > INT32_MAX - 256) return EG_MLA_ERR_UNSUPPORTED;   // (a block's tokens are counted in 32 bits)
  if (cu == nullptr && (tokens != batch || (positions == nullptr && tokens > 0))) return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

int to_status(cudaError_t e) { return e == cudaSuccess ? EG_MLA_OK : EG_MLA_ERR_CUDA; }

// frequencies of a rotary embedding, in turns per position, and its magnitude;
// EG_MLA_OK or the error code
int rope_frequencies(const eg_mla_rope_dims& r, int d, RopeArgs& a) {
  const double theta0 = r.theta > 0.f ? r.theta : 10000.0;
  const double s = r.scaling == EG_MLA_ROPE_UNSCALED ? 1.0 : r.factor;
  if (!std::isfinite(r.theta) || theta0 < 1.0 || !std::isfinite(s) || s < 1.0 || !std::isfinite(r.magnitude))
    return EG_MLA_ERR_INVALID_ARG;
  const bool yarn = r.scaling == EG_MLA_ROPE_YARN;
  const double fast = r.beta_fast > 0.f ? r.beta_fast : 32.0, slow = r.beta_slow > 0.f ? r.beta_slow : 1.0;
  if (yarn && (r.original_len <= 0 || !std::isfinite(fast) || !std::isfinite(slow) || !(fast > slow)))
    return EG_MLA_ERR_INVALID_ARG;
  if (r.scaling == EG_MLA_ROPE_NTK && d <= 2) return EG_MLA_ERR_INVALID_ARG;
  const double theta = r.scaling == EG_MLA_ROPE_NTK ? theta0 * std::pow(s, static_cast<double>(d) / (d - 2)) : theta0;
  constexpr double kInvTwoPi = 0.15915494309189533577;
  for (int i = 0; i < d / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / d);
    if (r.scaling == EG_MLA_ROPE_LINEAR) f /= s;
    if (yarn) {
      const double turns = r.original_len * f * kInvTwoPi;
      const double kept = std::fmin(1.0, std::fmax(0.0, (turns - slow) / (fast - slow)));
      f *= (1.0 - kept) / s + kept;
    }
    // the inverse turns by the negative fraction
    const uint64_t t = static_cast<uint64_t>(std::ldexp(f * kInvTwoPi, 64));
    a.turn[i] = r.inverse ? 0 - t : t;
  }
  a.magnitude = r.magnitude > 0.f ? r.magnitude : yarn ? static_cast<float>(0.1 * std::log(s) + 1.0) : 1.f;
  return EG_MLA_OK;
}

// the shapes of the cache in 8 bits, and the rows' strides and alignments; EG_MLA_OK or the error code
int fill_cache(CacheArgs& a, const eg_mla_dims* d, const void* c8, const float* scale, const void* kr,
               const int32_t* ids, const void* c_rows, int64_t c_stride, const void* kr_rows, int64_t kr_stride,
               const int32_t* id_rows, const int32_t* cu, const int32_t* positions, const int32_t* table,
               int32_t max_pages, int32_t batch, int32_t tokens, int32_t num_pages, int32_t* status) {
  int rc = q8_check_dims(d);
  if (rc != EG_MLA_OK) return rc;
  rc = check_packed(cu, positions, batch, tokens);
  if (rc != EG_MLA_OK) return rc;
  if (num_pages <= 0 || max_pages <= 0) return EG_MLA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(num_pages) * kPage > INT32_MAX) return EG_MLA_ERR_UNSUPPORTED;
  std::memset(&a, 0, sizeof(a));
  a.tok = {cu, positions, batch, tokens, status};
  if (tokens == 0 || batch == 0) return EG_MLA_OK;
  const int e = d->dtype == EG_MLA_BF16 ? 2 : 4;
  if (c8 == nullptr || scale == nullptr || kr == nullptr || c_rows == nullptr || table == nullptr)
    return EG_MLA_ERR_INVALID_ARG;
  if (c_stride < d->d_c || (kr_rows != nullptr && kr_stride < d->d_rope)) return EG_MLA_ERR_INVALID_ARG;
  if (!on16(c8) || !on16(kr) || !on16(c_rows) || !on16(kr_rows) || c_stride * e % 16 != 0 ||
      (kr_rows != nullptr && kr_stride * e % 16 != 0))
    return EG_MLA_ERR_INVALID_ARG;
  a.c8 = static_cast<uint8_t*>(const_cast<void*>(c8));
  a.scale = const_cast<float*>(scale);
  a.kr = static_cast<uint8_t*>(const_cast<void*>(kr));
  a.ids = const_cast<int32_t*>(ids);
  a.c_rows = static_cast<uint8_t*>(const_cast<void*>(c_rows));
  a.kr_rows = static_cast<uint8_t*>(const_cast<void*>(kr_rows));
  a.id_rows = const_cast<int32_t*>(id_rows);
  a.c_stride = c_stride * e;
  a.kr_stride = kr_stride * e;
  a.table = table;
  a.max_pages = max_pages;
  a.num_pages = num_pages;
  a.d_c = d->d_c;
  a.kr_bytes = d->d_rope * e;
  return EG_MLA_OK;
}

}  // namespace

int q8_check_dims(const eg_mla_dims* d) {
  if (d == nullptr || d->d_rope <= 0 || d->d_c <= 0 || d->page_size <= 0) return EG_MLA_ERR_INVALID_ARG;
  if (d->dtype != EG_MLA_BF16 && d->dtype != EG_MLA_FP32) return EG_MLA_ERR_INVALID_ARG;
  if (d->page_size != kPage || d->d_c % 16 != 0 || d->d_c > 512 || d->d_rope > 256 ||
      d->d_rope % (d->dtype == EG_MLA_BF16 ? 8 : 4) != 0)
    return EG_MLA_ERR_UNSUPPORTED;
  return EG_MLA_OK;
}

}  // namespace egmla

using namespace egmla;

extern "C" {

int eg_mla_rope(const eg_mla_dims* dims, const eg_mla_rope_dims* rope, const void* q, int64_t q_stride, void* q_out,
                int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out, int64_t k_out_stride,
                const int32_t* cu_seqlens, const int32_t* positions, int32_t batch, int32_t tokens,
                int32_t* dev_status, void* stream) {
  if (dims == nullptr || rope == nullptr) return EG_MLA_ERR_INVALID_ARG;
  if (dims->dtype != EG_MLA_BF16 && dims->dtype != EG_MLA_FP32) return EG_MLA_ERR_INVALID_ARG;
  if (dims->num_heads <= 0 || dims->d_nope < 0 || dims->d_rope <= 0) return EG_MLA_ERR_INVALID_ARG;
  if (rope->layout != EG_MLA_ROPE_INTERLEAVED && rope->layout != EG_MLA_ROPE_HALF) return EG_MLA_ERR_INVALID_ARG;
  if (rope->scaling < EG_MLA_ROPE_UNSCALED || rope->scaling > EG_MLA_ROPE_YARN) return EG_MLA_ERR_INVALID_ARG;
  if (dims->d_rope % 2 != 0 || dims->d_rope > 2 * kMaxPairs) return EG_MLA_ERR_UNSUPPORTED;
  const int64_t width = static_cast<int64_t>(dims->num_heads) * (static_cast<int64_t>(dims->d_nope) + dims->d_rope);
  if (width > INT32_MAX / 4 || dims->num_heads > 65534) return EG_MLA_ERR_UNSUPPORTED;
  int rc = check_packed(cu_seqlens, positions, batch, tokens);
  if (rc != EG_MLA_OK) return rc;
  RopeArgs a;
  std::memset(&a, 0, sizeof(a));
  rc = rope_frequencies(*rope, dims->d_rope, a);
  if (rc != EG_MLA_OK) return rc;
  if (tokens == 0 || batch == 0) return EG_MLA_OK;
  if ((q == nullptr && k == nullptr) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr))
    return EG_MLA_ERR_INVALID_ARG;
  if (q != nullptr && (q_stride < width || q_out_stride < width || (q == q_out && q_stride != q_out_stride)))
    return EG_MLA_ERR_INVALID_ARG;
  if (k != nullptr && (k_stride < dims->d_rope || k_out_stride < dims->d_rope || (k == k_out && k_stride != k_out_stride)))
    return EG_MLA_ERR_INVALID_ARG;
  const int e = dims->dtype == EG_MLA_BF16 ? 2 : 4;
  for (const void* p : {q, static_cast<const void*>(q_out), k, static_cast<const void*>(k_out)})
    if (reinterpret_cast<uintptr_t>(p) % e != 0) return EG_MLA_ERR_INVALID_ARG;
  a.tok = {cu_seqlens, positions, batch, tokens, dev_status};
  a.q = static_cast<const uint8_t*>(q);
  a.k = static_cast<const uint8_t*>(k);
  a.q_out = static_cast<uint8_t*>(q_out);
  a.k_out = static_cast<uint8_t*>(k_out);
  a.q_stride = q_stride * e;
  a.q_out_stride = q_out_stride * e;
  a.k_stride = k_stride * e;
  a.k_out_stride = k_out_stride * e;
  a.H = dims->num_heads;
  a.dn = dims->d_nope;
  a.dr = dims->d_rope;
  a.half = rope->layout == EG_MLA_ROPE_HALF;
  a.q_in_place = q == q_out;
  auto* st = static_cast<cudaStream_t>(stream);
  return to_status(dims->dtype == EG_MLA_BF16 ? launch_rope<__nv_bfloat16>(a, st) : launch_rope<float>(a, st));
}

int eg_mla_append_latent_q8(const eg_mla_dims* dims, void* c8_pool, float* scale_pool, void* krope_pool,
                            int32_t* id_pool, const void* c_new, int64_t c_stride, const void* krope_new,
                            int64_t krope_stride, const int32_t* ids_new, const int32_t* cu_seqlens,
                            const int32_t* positions, const int32_t* block_table, int32_t max_pages_per_seq,
                            int32_t batch, int32_t tokens, int32_t num_pages, int32_t* dev_status, void* stream) {
  CacheArgs a;
  const int rc = fill_cache(a, dims, c8_pool, scale_pool, krope_pool, id_pool, c_new, c_stride, krope_new, krope_stride,
                            ids_new, cu_seqlens, positions, block_table, max_pages_per_seq, batch, tokens, num_pages,
                            dev_status);
  if (rc != EG_MLA_OK || tokens == 0 || batch == 0) return rc;
  if (krope_new == nullptr) return EG_MLA_ERR_INVALID_ARG;
  auto* st = static_cast<cudaStream_t>(stream);
  return to_status(dims->dtype == EG_MLA_BF16 ? launch_append_q8<__nv_bfloat16>(a, st) : launch_append_q8<float>(a, st));
}

int eg_mla_read_latent_q8(const eg_mla_dims* dims, const void* c8_pool, const float* scale_pool,
                          const void* krope_pool, const int32_t* id_pool, const int32_t* cu_seqlens,
                          const int32_t* positions, const int32_t* block_table, int32_t max_pages_per_seq,
                          void* c_out, int64_t c_stride, void* krope_out, int64_t krope_stride, int32_t* ids_out,
                          int32_t batch, int32_t tokens, int32_t num_pages, int32_t* dev_status, void* stream) {
  CacheArgs a;
  const int rc = fill_cache(a, dims, c8_pool, scale_pool, krope_pool, id_pool, c_out, c_stride, krope_out, krope_stride,
                            ids_out, cu_seqlens, positions, block_table, max_pages_per_seq, batch, tokens, num_pages,
                            dev_status);
  if (rc != EG_MLA_OK || tokens == 0 || batch == 0) return rc;
  if (ids_out != nullptr && id_pool == nullptr) return EG_MLA_ERR_INVALID_ARG;
  auto* st = static_cast<cudaStream_t>(stream);
  return to_status(dims->dtype == EG_MLA_BF16 ? launch_read_q8<__nv_bfloat16>(a, st) : launch_read_q8<float>(a, st));
}

}  // extern "C"
