// egmla_common.cuh - launch-independent pieces shared by the decode kernels:
// the workspace layout and the split-KV work schedule.
//
// Split-KV schedule.  The work is counted in units: the cache pages of every
// sequence plus kSegCost per non-empty sequence (what a split pays to take in
// a sequence).  The units of all sequences are numbered globally in sequence
// order (prefix sums cu[b]) and cut into `num_splits` equal contiguous ranges
// of `chunk` units, one per CTA.  A
// CTA may therefore cover the tail of one sequence and the head of the next;
// it emits one partial result (running max m, denominator l, un-normalised
// latent output) per sequence it touches.  Partial slot of (CTA c, sequence b)
// is c + b: the CTA ranges of consecutive sequences overlap in at most one CTA,
// so these slots never collide and there are at most num_splits + batch of them.
#pragma once
#include <cmath>
#include <cstddef>
#include <cstdint>

namespace egmla {

constexpr int kPage = 64;

__host__ __device__ inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Per-sequence prepared query block of the tensor-core path: q^ (*) gamma
// [16 heads x d_c] and q^R [16 x d_rope] as bf16 MMA operands in 8x8 core
// matrices, then, per chunk of kSumFeatures latent features, the per-head fp32
// partial sums of w_h = sum_f bf16(q^ gamma)_hf and b_h = q^_h . beta
// ([d_c / kSumFeatures][2][16] floats; the consumer adds the chunks in order,
// so the result does not depend on launch order).  Every group of 8 columns
// (one K core of the operand, 256 bytes) holds heads 0-7 in its first 128
// bytes and heads 8-15 in its second: read as the N = 16 B operand of the
// score MMA (K-major, no swizzle) the K cores are 256 B apart and the two
// 8-head row groups 128 B apart.
constexpr int kQGroupBytes = 256;
constexpr int kQRowGroupBytes = 128;
__host__ __device__ constexpr size_t qop_offset(int h, int k) {
  return static_cast<size_t>(k / 8) * kQGroupBytes + (h / 8) * kQRowGroupBytes + (h % 8) * 16 + (k % 8) * 2;
}
// Latent widths walked in half pages: the K cores of two 64-feature columns
// alternate, so that the score MMA takes both as one operand of 32 rows (the row
// groups of the even column, then of the odd one, 128 B apart; K cores 512 B apart).
__host__ __device__ constexpr size_t qlat_offset(int h, int f, int d_c) {
  const int core = f / 8;
  return qop_offset(h, d_c <= 256 ? f : 8 * (core / 16 * 16 + core % 8 * 2 + core / 8 % 2) + f % 8);
}
__host__ __device__ constexpr size_t qprep_lat_bytes(int d_c) { return static_cast<size_t>(d_c / 8) * kQGroupBytes; }
__host__ __device__ constexpr size_t qprep_rope_bytes(int d_rope) {
  return static_cast<size_t>(d_rope / 8) * kQGroupBytes;
}
constexpr int kSumFeatures = 32;
__host__ __device__ constexpr size_t qprep_sums_bytes(int d_c) {
  return static_cast<size_t>(d_c / kSumFeatures) * 2 * 16 * 4;
}
__host__ __device__ constexpr size_t qprep_bytes_tc(int d_c, int d_rope) {
  return qprep_lat_bytes(d_c) + qprep_rope_bytes(d_rope) + qprep_sums_bytes(d_c);
}

// fp32 path: q^ [H, d_c] and q^R [H, d_rope] in fp32.
__host__ __device__ inline size_t qprep_bytes_f32(int H, int d_c, int d_rope) {
  return align_up(static_cast<size_t>(H) * (d_c + d_rope) * 4, 16);
}

// Where a split's page walk starts, written by the prologue kernel, so that
// each role of the decode kernel reads it with one round of loads instead of
// searching the prefix sums: the sequence b, the split's first page lp and
// end lp_end in it, the sequence length L, the split's end unit g1, whether
// the split is empty, and the physical ids of the first npages pages of the
// walk (at most kStartPages, all in sequence b).
constexpr int kStartPages = 8;
struct alignas(16) SplitStart {
  int32_t b, lp, lp_end, L, g1, done, npages, pad;
  int32_t page[kStartPages];
};
static_assert(sizeof(SplitStart) == 64, "split start record");

struct WorkspaceLayout {
  size_t off_cu, off_done, off_start, off_qprep, off_ml, off_o, total;
  size_t qprep_stride;
  int num_slots;
};

__host__ __device__ inline WorkspaceLayout workspace_layout(int batch, int num_splits, int H, int d_c,
                                                            int d_rope, bool tc_path) {
  WorkspaceLayout w;
  w.num_slots = num_splits + batch;
  w.qprep_stride = tc_path ? qprep_bytes_tc(d_c, d_rope) : qprep_bytes_f32(H, d_c, d_rope);
  size_t off = 0;
  w.off_cu = off;
  off = align_up(off + static_cast<size_t>(batch + 1) * 4, 256);
  // the fused combine's counters (zeroed by the prologue each call): the split
  // partials of each sequence stored (the area is as large as the prefix sums')
  w.off_done = off;
  off = align_up(off + static_cast<size_t>(batch + 1) * 4, 256);
  w.off_start = off;
  off = align_up(off + static_cast<size_t>(num_splits) * sizeof(SplitStart), 256);
  w.off_qprep = off;
  off = align_up(off + static_cast<size_t>(batch) * w.qprep_stride, 256);
  w.off_ml = off;
  off = align_up(off + static_cast<size_t>(w.num_slots) * H * 2 * 4, 256);
  w.off_o = off;
  off = align_up(off + static_cast<size_t>(w.num_slots) * H * d_c * 4, 256);
  w.total = off;
  return w;
}

// Split-KV schedule.  The splits share the work in units: one per cache page,
// plus kSegCost for the start of every non-empty sequence (the per-sequence cost
// of a split: loading the query block, reading out and storing the partial
// output), so that splits that take in more sequences get fewer pages.  cu[b]
// is the first unit of sequence b; its pages are units cu[b] + kSegCost + i,
// i < ceil(L_b / page); split c owns units [c chunk, (c + 1) chunk).
constexpr int kSegCost = 1;

// units per split for the total unit count
__host__ __device__ inline int split_chunk(int total_pages, int num_splits) {
  int c = (total_pages + num_splits - 1) / num_splits;
  return c < 1 ? 1 : c;
}

// first sequence whose page range contains global page g (cu has batch+1 entries,
// non-decreasing, cu[0] = 0, g < cu[batch])
__device__ inline int find_sequence(const int32_t* cu, int batch, int g) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    int mid = (lo + hi + 1) >> 1;
    if (__ldg(cu + mid) <= g) lo = mid; else hi = mid - 1;
  }
  // skip empty sequences that share the same start
  while (lo < batch - 1 && __ldg(cu + lo + 1) <= g) ++lo;
  return lo;
}

// Attention over a shared prefix (egmla_shared.cu).  A unit is (row tile of
// kSharedTile sequences, prefix page).  Each row tile's pages are cut into `parts`
// equal ranges, one per CTA, or (parts = 0) all units, row tiles outermost, into equal
// contiguous ranges; a range that meets two row tiles leaves two partials.  CTA c's
// partial of row tile t is slot c + t (as for the splits above), kSharedTile sequences x
// H heads per slot.
//
// The prefix's attention and the own tokens' split-KV kernel run beside each other, a
// CTA per SM: own_splits of the num_splits CTAs are for the own tokens (cut as above),
// the rest for the prefix; what is left of either grid has no work and leaves.  Of
// all such cuts the one whose longer side is shortest, by what was measured (in 10 ns):
// a prefix unit, a page of own tokens with and without a gate, and what a CTA of either
// kind takes besides (its queries, first scores and partial), the prefix's again for a
// second row tile.  64 sequences over 32K tokens took 59.5 us a call with the two one
// after the other on all SMs and 57.0 beside each other (53 with the later steps).
// A CTA takes two pages at least: the second costs 0.7 us, the partials that it saves the
// merge more (eight sequences over 2K tokens 21.2 us with one, 20.7 with two, 21.4 with
// three).
constexpr int kSharedTile = 8, kShMinPages = 2;
constexpr int kShUnitCost = 70, kShOwnGated = 137, kShOwnPlain = 93, kShFixed = 700, kShOwnFixed = 500;

struct alignas(16) SharedSchedule {
  int32_t pages, chunk, parts, own_splits;

  static __host__ __device__ int at_least(int x, int least) { return x > least ? x : least; }

  // for `own` of `splits` CTAs; cost: of the longer side.  own_units: of the own
  // tokens' schedule (its cu[batch])
  static __host__ __device__ SharedSchedule make(int batch, int prefix_len, int splits, int own, int own_units,
                                                 bool gate, int& cost) {
    SharedSchedule s;
    const int tiles = (batch + kSharedTile - 1) / kSharedTile;
    s.pages = (prefix_len + kPage - 1) / kPage;
    s.own_splits = own;
    const int ctas = splits > own ? splits - own : 1, units = tiles * s.pages;
    s.chunk = at_least(split_chunk(units, ctas), kShMinPages);
    s.parts = tiles > 0 ? ctas / tiles : 0;
    int64_t pre = static_cast<int64_t>(s.chunk) * kShUnitCost + kShFixed;
    if (s.pages % s.chunk != 0 && tiles > 1) pre += kShFixed;
    if (s.parts > 0) {
      const int chunk = at_least(split_chunk(s.pages, s.parts), kShMinPages);
      if (static_cast<int64_t>(chunk) * kShUnitCost + kShFixed <= pre) {
        s.chunk = chunk;
        pre = static_cast<int64_t>(chunk) * kShUnitCost + kShFixed;
      } else {
        s.parts = 0;
      }
    }
    int64_t most = own_units > 0 ? kShOwnFixed : 0;
    if (own_units > 0) most += static_cast<int64_t>(split_chunk(own_units, own)) * (gate ? kShOwnGated : kShOwnPlain);
    if (pre > most) most = pre;
    cost = static_cast<int>(most < INT32_MAX ? most : INT32_MAX);
    return s;
  }
  // the units of CTA c
  __host__ __device__ void range(int batch, int c, int& u0, int& u1) const {
    const int units = (batch + kSharedTile - 1) / kSharedTile * pages;
    if (parts > 0) {
      const int t = c / parts, lp = (c - t * parts) * chunk;
      u0 = t * pages + lp;
      u1 = t * pages + (lp + chunk < pages ? lp + chunk : pages);
      if (u0 >= u1 || u1 > units) u0 = u1 = units;
    } else {
      u0 = c * chunk < units ? c * chunk : units;
      u1 = u0 + chunk < units ? u0 + chunk : units;
    }
  }
  // the CTAs c0 .. c0 + n - 1 that leave a partial of row tile t
  __host__ __device__ int ctas_of(int t, int& c0) const {
    c0 = 0;
    if (pages == 0) return 0;
    if (parts > 0) {
      c0 = t * parts;
      return (pages + chunk - 1) / chunk;
    }
    c0 = t * pages / chunk;
    return ((t + 1) * pages - 1) / chunk - c0 + 1;
  }
};

// A normalised latent has |z'| <= sqrt(d_c), so the gate modes with a LayerNorm
// meet the prefix in f16, whose three more bits of significand than bf16's make the
// roundings of z', of the softmax weights and of q^ gamma small against the output's
// (rel-L2 against 64 bits of the emulated arithmetic, 8 and 17 sequences of a few
// tokens after 64: 3.0e-3 in bf16, 1.9e-3 in f16).  q^ gamma is kept 2^k times its
// value, with the k that puts softmax_scale 2^-k between 16 and 32 (-8 for the usual
// scale of 128 + 64 dimensions): f16's smallest step, 2^-24, then moves a score by
// about 1e-5 whatever the scale, and an element clamped to its largest value, 65504, is
// one that gives a score of 2^20 and more for each unit of z'.
inline float shared_q_scale(float softmax_scale) {
  const int k = std::ilogb(softmax_scale) - 4;
  return std::ldexp(1.f, k < -100 ? -100 : k > 100 ? 100 : k);
}

// rows of the gated prefix: whole pages; with the gate off only the last page
__host__ __device__ inline size_t shared_z_rows(int max_prefix_len, bool gate) {
  return gate ? align_up(static_cast<size_t>(max_prefix_len), kPage) : kPage;
}

// after the own tokens' decode workspace (`base` bytes)
struct SharedLayout {
  size_t off_sched, off_q, off_z, off_ml, off_o, total;
};

__host__ __device__ inline SharedLayout shared_layout(size_t base, int batch, int max_prefix_len, int ctas, int H,
                                                      int d_c, bool gate) {
  SharedLayout w;
  const size_t slots = static_cast<size_t>(ctas) + (batch + kSharedTile - 1) / kSharedTile;
  size_t off = align_up(base, 256);
  w.off_sched = off;
  off = align_up(off + sizeof(SharedSchedule), 256);
  w.off_q = off;   // q^ gamma in f16, laid out as in the prepared query blocks
  off = align_up(off + static_cast<size_t>(batch) * qprep_lat_bytes(d_c), 256);
  w.off_z = off;
  off = align_up(off + shared_z_rows(max_prefix_len, gate) * d_c * 2, 256);
  w.off_ml = off;
  off = align_up(off + slots * kSharedTile * H * 2 * 4, 256);
  w.off_o = off;
  off = align_up(off + slots * kSharedTile * H * d_c * 4, 256);
  w.total = off;
  return w;
}

// the page-sparse decode's own part of the workspace, after the decode workspace
// (`base` bytes) of the selected pages
struct SparseLayout {
  size_t off_q, off_scores, off_table, off_lens, off_counters, total;
  size_t q_stride;   // floats
  int width;         // pages of the selected block table
};

__host__ __device__ inline SparseLayout sparse_layout(size_t base, int batch, int max_pages, int budget, int H,
                                                      int d_c, int d_rope) {
  SparseLayout w;
  w.width = budget < max_pages ? budget : max_pages;
  w.q_stride = qprep_bytes_f32(H, d_c, d_rope) / 4;
  size_t off = align_up(base, 256);
  w.off_q = off;
  off = align_up(off + static_cast<size_t>(batch) * w.q_stride * 4, 256);
  w.off_scores = off;
  off = align_up(off + static_cast<size_t>(batch) * max_pages * 4, 256);
  w.off_table = off;
  off = align_up(off + static_cast<size_t>(batch) * w.width * 4, 256);
  w.off_lens = off;
  off = align_up(off + static_cast<size_t>(batch) * 4, 256);
  w.off_counters = off;
  off = align_up(off + static_cast<size_t>(batch) * 4, 256);
  w.total = off;
  return w;
}

}  // namespace egmla
