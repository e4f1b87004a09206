// egmla_tokens.cu - packed tokens between the projections and the cache: the rotary
// embedding of their queries and keys, their rows written into a cache that holds the
// latent in 8 bits, and cached rows read back.  See include/egmla.h for the contract.
//
// Packed token k belongs to the sequence b with cu[b] <= k < cu[b + 1], as its token
// k - cu[b], at position positions[b] + k - cu[b] (cu null: to sequence k, at
// positions[k]).  A warp finds b for its token by ballots over 32 offsets at a time.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

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

constexpr int kTokThreads = 256, kTokWarps = kTokThreads / 32;

struct Packed {
  const int32_t* cu;          // [batch + 1], null: one token per sequence
  const int32_t* positions;   // [batch], null: 0
  int batch, tokens;
  int32_t* status;
};

// Sequence and position of packed token k, the same in every lane; false for a token of
// no sequence or of one with a negative position.
__device__ __forceinline__ bool find_token(const Packed& p, int k, int lane, int& b, int64_t& pos) {
  int first = k;   // the sequence's first packed token
  b = k;
  if (p.cu != nullptr) {
    // how many of cu[1 .. batch] are <= k
    int n = p.batch;
    b = 0;
    while (n > 0) {
      const int step = (n + 31) / 32, i = (lane + 1) * step;
      const bool below = i <= n && __ldg(p.cu + b + i) <= k;
      const int c = __popc(__ballot_sync(0xffffffffu, below));
      b += c * step;
      n = min(n - c * step, step - 1);
    }
    if (b >= p.batch) return false;   // a row behind the last sequence
    first = __ldg(p.cu + b);
    if (first > k) {   // (no token of offsets that begin above 0 or decrease)
      if (lane == 0) report_status(p.status, kStatusOutOfRange);
      return false;
    }
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
// after whole turns, so that far positions lose nothing and no double precision runs on the
// GPU.  Sine and cosine are taken in fp32 of what is left to the nearest quarter turn.
constexpr int kMaxPairs = 128;

struct RopeArgs {
  Packed tok;
  const uint8_t *q, *k;
  uint8_t *q_out, *k_out;
  int64_t q_stride, q_out_stride, k_stride, k_out_stride;   // bytes between tokens
  int H, dn, dr;
  int half, q_in_place, k_in_place;
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

// A warp per token and part of its H + 1 heads (the last one is the key); blockIdx.y: the
// part.  VEC: rows and their parts in 16-byte units.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kTokThreads) rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ float2 table[kTokWarps][kMaxPairs];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = blockIdx.x * kTokWarps + warp;
  const int pairs = a.dr / 2;
  grid_dependency_wait();
  int b;
  int64_t pos;
  if (k >= a.tok.tokens || !find_token(a.tok, k, lane, b, pos)) return;
  for (int i = lane; i < pairs; i += 32)
    table[warp][i] = turn_cos_sin(static_cast<uint64_t>(pos) * a.turn[i], a.magnitude);
  __syncwarp();
  const float2* cs = table[warp];
  const int heads = a.H + 1;
  int h0 = heads * static_cast<int>(blockIdx.y) / static_cast<int>(gridDim.y);
  const int h1 = heads * (static_cast<int>(blockIdx.y) + 1) / static_cast<int>(gridDim.y);
  const int dq = a.dn + a.dr;
  for (int h = h0; h < h1; ++h) {
    const bool key = h == a.H;
    if ((key ? a.k : a.q) == nullptr) continue;
    const T* src = reinterpret_cast<const T*>(key ? a.k + k * a.k_stride : a.q + k * a.q_stride) + (key ? 0 : h * dq);
    T* dst = reinterpret_cast<T*>(key ? a.k_out + k * a.k_out_stride : a.q_out + k * a.q_out_stride) + (key ? 0 : h * dq);
    const int dn = key ? 0 : a.dn;
    if (dn > 0 && !a.q_in_place)
      for (int f = lane; f < dn; f += 32) dst[f] = src[f];
    for (int i = lane; i < pairs; i += 32) {
      const int x = dn + (a.half ? i : 2 * i), y = a.half ? x + pairs : x + 1;
      const float2 r = turned(to_f32(src[x]), to_f32(src[y]), cs[i]);
      dst[x] = from_f32<T>(r.x);
      dst[y] = from_f32<T>(r.y);
    }
  }
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

// Row of the pool of packed token k, the same in every lane; -1: none.
__device__ __forceinline__ int64_t cache_row(const CacheArgs& a, int k, int lane) {
  int b;
  int64_t pos;
  if (!find_token(a.tok, k, lane, b, pos)) return -1;
  const int64_t lp = pos / kPage;
  const int page = lp < a.max_pages ? __ldg(a.table + static_cast<size_t>(b) * a.max_pages + lp) : -1;
  if (page < 0 || page >= a.num_pages) {
    if (lane == 0) report_status(a.tok.status, kStatusOutOfRange);
    return -1;
  }
  return static_cast<int64_t>(page) * kPage + pos % kPage;
}

// eight values of a packed row
template <typename T>
__device__ __forceinline__ void load8(const uint8_t* row, int unit, float (&x)[8]) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < 8 / N; ++j) {
    Vec<T> v;
    v.raw = *reinterpret_cast<const uint4*>(row + (unit * (8 / N) + j) * 16);
#pragma unroll
    for (int i = 0; i < N; ++i) x[j * N + i] = to_f32(v.v[i]);
  }
}
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

// A warp per token, eight features of the latent a lane and turn.
template <typename T>
__global__ void __launch_bounds__(kTokThreads) append_q8_kernel(const __grid_constant__ CacheArgs a) {
  const int lane = threadIdx.x & 31, k = blockIdx.x * kTokWarps + (threadIdx.x >> 5);
  grid_dependency_wait();
  if (k >= a.tok.tokens) return;
  const int units = a.d_c / 8;   // at most 64
  const uint8_t* src = a.c_rows + k * a.c_stride;
  float x[2][8] = {};
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (lane + 32 * j < units) load8<T>(src, lane + 32 * j, x[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[j][i]) & 0x7fffffffu);
  }
  const int64_t row = cache_row(a, k, lane);
  if (row < 0) return;
  most = __reduce_max_sync(0xffffffffu, most);
  float scale, inverse;
  q8_scale(most, scale, inverse);
  uint2* dst = reinterpret_cast<uint2*>(a.c8 + row * a.d_c);
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (lane + 32 * j < units) {
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = q8_encode2(x[j][4 * i] * inverse, x[j][4 * i + 1] * inverse) |
               q8_encode2(x[j][4 * i + 2] * inverse, x[j][4 * i + 3] * inverse) << 16;
      dst[lane + 32 * j] = make_uint2(w[0], w[1]);
    }
  for (int u = lane; u < a.kr_bytes / 16; u += 32)
    reinterpret_cast<uint4*>(a.kr + row * a.kr_bytes)[u] = reinterpret_cast<const uint4*>(a.kr_rows + k * a.kr_stride)[u];
  if (lane == 0) {
    a.scale[row] = scale;
    if (a.ids != nullptr && a.id_rows != nullptr) a.ids[row] = a.id_rows[k];
  }
}

template <typename T>
__global__ void __launch_bounds__(kTokThreads) read_q8_kernel(const __grid_constant__ CacheArgs a) {
  const int lane = threadIdx.x & 31, k = blockIdx.x * kTokWarps + (threadIdx.x >> 5);
  grid_dependency_wait();
  if (k >= a.tok.tokens) return;
  const int64_t row = cache_row(a, k, lane);
  if (row < 0) return;
  const float scale = __ldg(a.scale + row);
  const uint2* src = reinterpret_cast<const uint2*>(a.c8 + row * a.d_c);
  for (int u = lane; u < a.d_c / 8; u += 32) {
    const uint2 w = src[u];
    float x[8];
    q8_decode4(w.x, x);
    q8_decode4(w.y, x + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= scale;
    store8<T>(a.c_rows + k * a.c_stride, u, x);
  }
  if (a.kr_rows != nullptr)
    for (int u = lane; u < a.kr_bytes / 16; u += 32)
      reinterpret_cast<uint4*>(a.kr_rows + k * a.kr_stride)[u] = reinterpret_cast<const uint4*>(a.kr + row * a.kr_bytes)[u];
  if (lane == 0 && a.id_rows != nullptr) a.id_rows[k] = a.ids[row];
}

// ------------------------------------------------------------------ arguments
bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// the common part of the three calls; EG_MLA_OK or the error code
int check_packed(const int32_t* cu, const int32_t* positions, int32_t batch, int32_t tokens) {
  if (batch < 0 || tokens < 0) return EG_MLA_ERR_INVALID_ARG;
  if (cu == nullptr && (tokens != batch || (positions == nullptr && tokens > 0))) return EG_MLA_ERR_INVALID_ARG;
  return EG_MLA_OK;
}

unsigned token_blocks(int32_t tokens) { return static_cast<unsigned>((static_cast<int64_t>(tokens) + kTokWarps - 1) / kTokWarps); }

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
  a.k_in_place = k == k_out;
  const dim3 grid(token_blocks(tokens), 1);
  auto* st = static_cast<cudaStream_t>(stream);
  return to_status(dims->dtype == EG_MLA_BF16
                       ? launch_chained(rope_kernel<__nv_bfloat16, false>, grid, dim3(kTokThreads), 0, st, a)
                       : launch_chained(rope_kernel<float, false>, grid, dim3(kTokThreads), 0, st, a));
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
  const dim3 grid(token_blocks(tokens)), block(kTokThreads);
  auto* st = static_cast<cudaStream_t>(stream);
  return to_status(dims->dtype == EG_MLA_BF16 ? launch_chained(append_q8_kernel<__nv_bfloat16>, grid, block, 0, st, a)
                                              : launch_chained(append_q8_kernel<float>, grid, block, 0, st, a));
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
  const dim3 grid(token_blocks(tokens)), block(kTokThreads);
  auto* st = static_cast<cudaStream_t>(stream);
  return to_status(dims->dtype == EG_MLA_BF16 ? launch_chained(read_q8_kernel<__nv_bfloat16>, grid, block, 0, st, a)
                                              : launch_chained(read_q8_kernel<float>, grid, block, 0, st, a));
}

}  // extern "C"
