// egmla_kernels.h - internal launch interface between the C-ABI layer
// (egmla_api.cu) and the kernels.  Not part of the public ABI.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>
#include <mutex>

#include "../../include/egmla.h"
#include "egmla_common.cuh"

namespace egmla {

// Launch with programmatic stream serialisation: the grid is set up while the
// kernel before it on the stream drains, instead of after it has completed and
// flushed.  What holds the order:
//  - every block of a kernel launched this way executes grid_dependency_wait,
//    and before it touches nothing that a kernel before it writes, and writes
//    nothing, so that a completed kernel stands for everything before it;
//  - before the wait a kernel may read inputs that no kernel of the call writes:
//    the split combine copies W_UV, the fp32 one brings it to L2, the projection
//    GEMM copies its weights.  The caller's kernel before the call may write
//    W_UV: the combine must not start before that one is complete, so the bf16
//    split-KV kernel triggers a separate combine only after its own wait, or, beside
//    the attention over a shared prefix, knows it complete when it starts (below).  (An
//    L2 prefetch reads nothing that could be old.  The first projection's weights
//    must not be written by the kernel directly before the layer call.)
//  - a kernel may stand beside the one before it where it needs nothing of that one:
//    that one lets it start only after its own wait (so that all before it is
//    complete), and it waits at its end instead of its start (`beside`), so that its
//    completion stands for both.  In the shared-prefix decode the absorption triggers
//    after its wait, and gate, attention and split-KV kernel each start after the
//    trigger of the one before: whatever came before the call is complete when any of
//    them starts.  The combine's early copy of W_UV rests on that too.
// A kernel lets its successor start early (grid_launch_dependents) where that was
// measured to pay: mostly where the successor's blocks take a whole SM each, since
// smaller blocks, started early, crowd onto the first SMs to free up (the R0
// attention took 42 us instead of 33, the layer's query absorption 13 instead
// of 8); the figures stand at the triggers.  Whole calls against plain launches:
// one 777-token prefill 34.8 -> 26.8 us, the fp32 step 38.9 -> 32.6, 8 x 32K decode
// step 51.2 -> 48.9, 128 ragged sequences 84.2 -> 81.7, the d_c 512 step 188 -> 186,
// a layer of 64 x 8K 119.6 -> 115.1, R0 at 8 x 4K 169.6 -> 164.0.
template <typename... P, typename... A>
cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// SMs of a GB300: what the tile sizes of the small kernels aim at (their results do
// not depend on it; grids that must cover the device ask it)
constexpr int kSms = 152;

// cuTensorMapEncodeTiled through the runtime's driver entry point (no libcuda link)
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                              const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                              CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encode_fn() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(p);
  });
  return fn;
}

// Map of a bf16 tensor of R dimensions (innermost first) with the strides of the
// outer ones in elements; 128-byte swizzle, elements past an end read as zero and
// are not written.
template <size_t R>
bool encode_map(CUtensorMap* map, const void* base, const uint64_t (&dims)[R], const uint64_t (&strides)[R - 1],
                const uint32_t (&box)[R]) {
  const EncodeFn enc = encode_fn();
  if (enc == nullptr) return false;
  cuuint64_t d[R], s[R - 1];
  cuuint32_t b[R], step[R];
  for (size_t i = 0; i < R; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    step[i] = 1;
    if (i + 1 < R) s[i] = strides[i] * 2;
  }
  auto encode = [&] {
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, R, const_cast<void*>(base), d, s, b, step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  };
  CUresult r = encode();
  if (r == CUDA_ERROR_INVALID_CONTEXT) {
    // a host thread that has made no call on the device yet has no current context,
    // which the encoder needs: cudaSetDevice makes the device's own current
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) return false;
    r = encode();
  }
  return r == CUDA_SUCCESS;
}

// Lets `kernel` be launched with up to `most` bytes of dynamic shared memory.  The
// limit belongs to the function, not to the calling thread, so every call of a
// kernel sets the same one, the most that any supported shape needs: a call that
// set its own smaller need would take the launch of another thread's larger call
// from under it.
constexpr size_t kSmemMost = 227 * 1024;   // of a block, on this GPU
template <typename K>
cudaError_t allow_smem(K* kernel, size_t most) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
}

struct AppendArgs {
  void* c_pool;
  void* kr_pool;
  int32_t* id_pool;
  const void* c_new;
  const void* kr_new;
  const int32_t* ids_new;
  const int32_t* block_table;
  int max_pages;
  const int32_t* positions;
  int batch, num_pages, page_size;
  int c_row_bytes, kr_row_bytes;
  int32_t* status;
};

// roles recorded by the decode kernel's event trace (eg_mla_debug_set_trace)
constexpr int kTraceRoles = 5;

struct DecodeArgs {
  // shapes
  int H, d_nope, d_rope, d_v, d_c, page_size, vocab;
  int dtype;  // 0 bf16, 1 fp32
  int gate;      // 0 none, 1 gated (the three gate modes below)
  int gate_add;  // gate by c + g (EG_MLA_GATE_ADD_LN) instead of c (*) g
  int gate_ln;   // LayerNorm after the gate (EG_MLA_GATE_MUL_LN, EG_MLA_GATE_ADD_LN)
  float scale_log2;  // softmax scale * log2(e)
  float eps;
  // tensors
  const void* q;
  const void* c_pool;
  const float* scale_pool;  // non-null: c_pool holds the latent in 8 bits (egmla_q8.cuh)
  const void* kr_pool;
  const int32_t* id_pool;
  const int32_t* block_table;
  int max_pages;
  const int32_t* seq_lens;
  int max_seq_len;
  int batch, num_pages;
  const void* gate_table;
  const float* ln_gamma;
  const float* ln_beta;
  const void* w_uk;
  const void* w_uv;
  void* out;
  int num_splits;
  int apart;   // the split combine always as a kernel of its own
  int beside;  // the split-KV kernel runs beside the kernel before it (see launch_chained)
  int early;   // let the kernel after the split-KV kernel start early (it streams weights of its own)
  void* workspace;
  int32_t* status;
  // cache-read test entry outputs (eg_mla_debug_gather)
  void* dump_c;
  void* dump_kr;
  int32_t* dump_ids;
  void* dump_g;
  // pipeline event trace of the decode kernel (eg_mla_debug_set_trace)
  void* trace;
  int trace_ctas, trace_cap;
  // limit of every pipeline wait (ns), and a withheld page copy of the
  // tensor-core decode kernel (eg_mla_debug_set_fault; stall_cta < 0: none)
  uint64_t wait_ns;
  int stall_cta, stall_tile;
};

cudaError_t launch_append(const AppendArgs& a, cudaStream_t st);
// query absorption and split schedule; with `app` non-null its blocks also
// append the new token of every sequence (the pools are read by no block of it)
// `maps`: W_UK as {d_c, d_nope, H} in boxes of {64, 64, 1} and q^C as {d_nope, H,
// batch} in boxes of {64, 1, absorb_tile}
// the page-sparse decode: the schedule is for these lengths, which are made from
// seq_lens, before the pages are known (lens null: not that)
struct SparseLens {
  int32_t* lens;       // [batch]
  int32_t* counters;   // [batch], zeroed
  int budget, max_seq_len;
};
// `extra`: the absorbed queries in other forms too.  a.q null: the schedule only
struct AbsorbExtra {
  uint8_t* q16;     // q^ gamma in f16, for the attention over a shared prefix (null: none)
  float q_scale;    // times this (shared_q_scale)
  float* q32;       // per sequence q^ [H, d_c], then q^R [H, d_rope], in fp32, for the page scores (null: none)
  SparseLens sparse;
  int chain;        // the kernel after this one runs beside it (see launch_chained)
  // a shared prefix, whose attention takes a part of the SMs (null: none): its length,
  // and where the schedule of both is written
  const int32_t* prefix_len;
  int max_prefix_len, gate;
  SharedSchedule* sched;
};
cudaError_t launch_prologue_tc(const DecodeArgs& a, const AppendArgs* app, const CUtensorMap* maps, cudaStream_t st,
                               const AbsorbExtra& extra = AbsorbExtra{});
// sequences per block of the absorption
int absorb_tile(int d_c, int batch);
// fp32: absorption (with the append blocks of `app` when it is non-null; q^ [H, d_c],
// then q^R [H, d_rope] per sequence) and page prefix sums
cudaError_t launch_prologue_f32(const DecodeArgs& a, const AppendArgs* app, cudaStream_t st,
                                const SparseLens& sparse = SparseLens{});
// the split-KV kernel after it
cudaError_t launch_decode_f32(const DecodeArgs& a, cudaStream_t st);
// The partials of a prefix that the batch shares, merged with the sequences' own
// (combine of the tensor-core path); how they lie: see SharedSchedule.
struct SharedParts {
  const float* ml;
  const float* o;
  const SharedSchedule* sched;
};
// `wmap` (tensor-core path): W_UV as {d_c, d_v, H} in boxes of {64, 128, 1};
// `shared` (may be null; tensor-core path): a second list of partials
cudaError_t launch_combine(const DecodeArgs& a, bool tc_path, const CUtensorMap* wmap, cudaStream_t st,
                           const SharedParts* shared = nullptr);
// tensor-core split-KV kernel; `maps` = {c_pool map (3-D box of a tile), kr_pool map}.
// *fused (may be null) is set when the split combine ran inside the kernel
// (cooperative launch); otherwise launch_combine must follow.
cudaError_t launch_decode_tc(const DecodeArgs& a, const CUtensorMap* maps, bool dump, cudaStream_t st,
                             bool* fused);
// the same over the ungated latent in 8 bits (scale_pool); `maps` = {codes as 16-bit pairs
// in boxes of a page's 128-feature columns, kr_pool map of whole pages}
cudaError_t launch_decode_plain_q8(const DecodeArgs& a, const CUtensorMap* maps, cudaStream_t st, bool* fused);
bool plain_q8_supported(int d_c);
// true if the bf16 tensor-core path has a kernel for these shapes
bool tc_supported(int d_c, int gate);

// Attention over a shared prefix (egmla_shared.cu): the gated prefix (runs beside the
// absorption), and the partials of every sequence over it (the kernel after it may run
// beside it), into the workspace parts `wl` of `dec`.
// `maps`: the gated prefix (gate off: the latent pool), its last page (gate off),
// the RoPE keys, each in boxes of one page.
struct SharedArgs {
  const DecodeArgs* dec;
  SharedLayout wl;
  float q_scale = 1.f;   // of q^ gamma in f16 (AbsorbExtra)
  const int32_t* prefix_table;
  const int32_t* prefix_len;
  int max_prefix_len;
};
bool shared_supported(int d_c);
cudaError_t launch_shared_gate(const SharedArgs& a, cudaStream_t st);
cudaError_t launch_shared_attn(const SharedArgs& a, const CUtensorMap* maps, cudaStream_t st);

// Pages of the cache (egmla_pages.cu); see include/egmla.h for what they compute.
constexpr int kPlanMaxBatch = 16384;   // three words per sequence in shared memory
constexpr int kStatusNoPages = -8;
struct PlanArgs {
  const int32_t* new_tokens;
  const int32_t* seq_lens;
  int32_t* seq_lens_out;
  int32_t* block_table;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* free_count_out;
  int32_t* cu_seqlens;
  int32_t* positions;   // may be null
  int32_t* slots;       // may be null
  int32_t* status;
  int batch, max_pages, num_pages, max_slots;
};
cudaError_t launch_page_plan(const PlanArgs& a, cudaStream_t st);

struct SummaryArgs {
  const void* c_pool;
  const void* kr_pool;
  const int32_t* id_pool;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* new_tokens;   // null: all tokens
  const void* gate_table;
  const float* gamma;          // null: 1
  const float* beta;           // null: 0
  float* summary;
  int32_t* status;
  int d_c, d_r, vocab, batch, max_pages, max_seq_len, num_pages;
  int max_new, page_bound;     // tokens and pages per sequence, at most
  int fp32, gate_mode;
  float eps;
};
cudaError_t launch_page_summary(const SummaryArgs& a, cudaStream_t st);

// scores of the pages, and the selected ones as a block table of `width` pages
struct SelectArgs {
  const float* q;         // per sequence q^ [H, d_c], then q^R [H, d_r]
  size_t q_stride;        // floats
  const float* summary;
  const int32_t* block_table;
  const int32_t* seq_lens;
  float* scores;          // [batch, max_pages]
  int32_t* sel_table;     // [batch, width]
  int32_t* selected;      // [batch, budget] logical pages, may be null
  int32_t* counters;      // [batch], zeroed by the absorption
  int32_t* status;
  int H, d_c, d_r, batch, max_pages, max_seq_len, num_pages;
  int budget, keep_first, keep_last, width;
  int chunks;             // select_chunks(): blocks per sequence
  float scale;
};
int select_chunks(int max_seq_len, int batch, int budget, int keep_first, int keep_last, int d_c, int d_r);
cudaError_t launch_select_pages(const SelectArgs& a, cudaStream_t st);

// R0 decode (egmla_r0.cu): bf16, 16 heads, d_n = d_v = 128, d_r = 64,
// d_c in {192, 256}
struct R0Args {
  const void* q;
  const void* c_pool;
  const void* kr_pool;
  const int32_t* id_pool;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const void* w_ukv;     // [16 * 256, d_c]: per head its 128 key rows, then its 128 value rows
  const void* gate_r0;   // [vocab, 4096]
  const float* ln_gamma;
  const float* ln_beta;
  void* out;
  void* workspace;
  int32_t* status;
  int d_c, vocab, batch, max_pages, num_pages;
  float eps, scale_log2;
};
size_t r0_workspace_bytes(int batch, int max_pages, int num_pages);
cudaError_t launch_decode_r0(const R0Args& a, cudaStream_t st);
// Prefill (egmla_prefill.cu): bf16, d_n = d_v = 128, d_r = 64, d_c a
// multiple of 64 up to 512, any head count.  Prompts packed row after row
// (cu_seqlens [batch + 1] on the device); the pool pointers may be null (no
// cache write).
struct PrefillArgs {
  const void* q;            // [total, H, d_n + d_r]
  const void* c;            // [total, d_c]
  const void* kr;           // [total, d_r]
  const int32_t* ids;       // [total]
  const int32_t* cu_seqlens;
  const void* gate_table;
  const float* ln_gamma;
  const float* ln_beta;
  const void* w_uk;
  const void* w_uv;
  void* out;                // [total, H, d_v]
  void* c_pool;
  void* kr_pool;
  int32_t* id_pool;
  const int32_t* block_table;
  void* workspace;
  int32_t* status;
  int H, d_c, vocab, batch, total, max_seq_len, max_pages, num_pages;
  int gate, gate_add, gate_ln;
  float eps, scale_log2;
};
size_t prefill_workspace_bytes(int batch, int total_tokens, int H, int d_c);
bool prefill_supported(int d_nope, int d_rope, int d_v, int d_c);
// `mark` (may be null) is called with (stream, true) just before the
// attention kernel's launch and (stream, false) just after it.
cudaError_t launch_prefill(const PrefillArgs& a, cudaStream_t st, void (*mark)(cudaStream_t, bool));
// The gate table G = E W^UE^T (Section 3 Eqs. 3-4 for every vocabulary
// entry): E [vocab, d_e], W^UE [d_c, d_e] bf16 row-major, G [vocab, d_c] bf16;
// d_e a multiple of 64 up to 512, d_c a multiple of 64 (egmla_prefill.cu).
cudaError_t launch_gate_table(const void* emb, const void* w_ue, int vocab, int d_e, int d_c, void* table,
                              int32_t* status, cudaStream_t st);
// out[b][n] = sum_k x[b][k] W[n][k] for b < batch, n < n_out: W [n_out, k] and
// x [batch, k] bf16 row-major (16-byte aligned, k % 8 == 0), out fp32 or
// bf16 with row stride ldo elements (egmla_linear.cu).  Launched with
// programmatic stream serialisation: the weight copies may start while the
// kernel before it on the stream still runs.
cudaError_t launch_linear_tc(const void* w, int n_out, int k, const void* x, int batch, void* out, int ldo,
                             bool out_f32, int32_t* status, cudaStream_t st);
// the launch shape launch_linear_tc picks: cluster size (CTAs splitting k),
// ring stages, and the clusters of that size the device holds at once
cudaError_t linear_tc_plan(int n_out, int k, int batch, int* cluster, int* stages, int* max_clusters);

}  // namespace egmla

// The step inside eg_mla_layer_decode (egmla_api.cu): eg_mla_step (`append`)
// or eg_mla_decode, whose split-KV kernel lets the output projection after it
// start early.  `launch` false: its arguments are checked and nothing is launched.
int egmla_layer_step(const eg_mla_dims* dims, bool append, void* c_pool, void* krope_pool, int32_t* id_pool,
                     const void* c_new, const void* krope_new, const int32_t* ids_new, const int32_t* positions,
                     const void* q, const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens,
                     int32_t max_seq_len, int32_t batch, int32_t num_pages, const void* gate_table,
                     const float* ln_gamma, const float* ln_beta, const void* w_uk, const void* w_uv, void* out,
                     int32_t num_splits, void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream,
                     bool launch);
