// Attention of a chunk of new rows over a paged cache (part of a prompt, one
// token, or a tree to verify): out_i = sum_s w_is v_s, w_is = softmax over the
// slots s that row i admits of scale q_i . k_s.
//
// Layout (bf16 or float16): q and out [T][Hq][D], pages [Hkv][page_size][D] (or of bytes
// with scales: pctree_held.h);
// query head h reads key/value head h / g, g = Hq / Hkv.  The g heads of a
// key/value head are rows of one matrix, row rho = i * g + (h mod g) of request
// row i, so that K and V are read once for all of them.
//
// Two kernels, by a request's rows (row count times g):
//
// * More than kFewRows: a workgroup takes 128 rows and a run of slots.  K and V of a
//   64-slot chunk go from their pages straight into LDS, one chunk ahead; every lane
//   holds the page of one slot of the chunk, read another chunk ahead, and the lanes
//   that load a slot's row fetch its page from that lane.  A wave computes S^T = K Q^T
//   and O^T += V^T P^T on MFMA 16x16x32 for its 32 rows, with an online softmax in base
//   2 (32-bit reference, sum and output); the two K tiles of a pair are arranged so that
//   a lane ends with 8 consecutive slots of its row, the B operand of the second
//   product.  The weights are rounded to 16 bits there, an operand of the matrix units.
// * Others (single tokens): bytes bound them.  A workgroup takes 16 rows and a run of
//   slots; each of its waves takes 32-slot chunks by itself, K straight into
//   registers, V into an LDS tile of its own, and 12 waves a compute unit keep 16 KB
//   each in flight (156 registers a lane; heads of 64: 16 waves, 8 KB).  The waves'
//   results are joined in LDS.
//
// Runs leave (maximum, sum, unnormalised output) per row for a merging kernel; a
// request short enough for one run is written at once.
//
// Masked slots: scores are replaced, not added to, so K may hold anything.  A
// weight of zero times an infinite or NaN value would still be NaN, so in chunks
// that some row sees only in part such values are replaced first, and the rows
// that do admit them are mended afterwards.
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pctree_held.h"
#include "pctree_lds.h"
#include "pctree_paged.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr int kChunk = 64;        // slots of an LDS stage, in halves of 32
constexpr int kHalves = kChunk / 32;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kColTiles = 2;
constexpr int kRowsPerWave = 16 * kColTiles;
constexpr int kRowsPerBlock = kWaves * kRowsPerWave;
constexpr int kMaxSplits = 32;
// Rows (times g) of a request that go 16 to a workgroup, which read K and V again for
// every 16.  (32 requests over 1000 to 4000 slots of 8 heads, us so and in blocks of 128
// rows: 32 rows 87, 88, 48 rows 108, 89, 64 rows 137, 90; 8 requests 32, 31, 38, 32, 42,
// 33; one 13.4, 14.3, 15.4, 14.7, 15.6, 15.2.)
constexpr int kFewRows = 32;
constexpr int kFewChunk = 32;        // slots of a wave's step there
constexpr int kFewRun = 4 * kFewChunk;  // the shortest run there, a chunk to each wave
constexpr int kFewChunk8 = 64;       // the same over pages in 8 bits
constexpr int kFewRun8 = 4 * kFewChunk8;
constexpr int kMergeThreads = 256;
constexpr int kMergeBatch = 8;
constexpr int kMatrix = 0x8, kReadLds = 0x100;  // instruction classes of the scheduler
// float16 weights are 2^12 times the softmax's (as is their sum): weights down
// to 2^-36 of the row's largest then stay above float16's smallest, 2^-24.  The weight
// of the reference is 4096, and the largest that kSlack lets past it 2^15.
constexpr float kHalfLift = 12.0f;
// The reference that scores are taken relative to follows a row's maximum only when
// that has grown past it by more than this many powers of two: until then weights are
// at most 2^8 (2^15 for a lifted float16), and the output so far need not be scaled (72
// products a chunk, in about half the chunks of a long row: a chunk of 2048 rows 280 us,
// 267 so).  It costs precision in the largest weight, which is exact only where it is the
// reference itself: 300 rows over 3000 slots are off by 2.30e-3 of float64 (root mean
// square), 2.17e-3 with a reference that follows at once; float16 2.86e-4, 2.72e-4.
template <bool H>
constexpr float kSlack = H ? 3.0f : 8.0f;

// Slots per run of a request whose rows end at slot `end`, at most `nsplit` runs of at
// least `least` slots (a multiple of 64).
__device__ __forceinline__ int run_slots(int end, int nsplit, int least) {
  const int units = (end + least - 1) / least;
  const int ns = min(nsplit, units);
  return (units + ns - 1) / ns * least;
}
__device__ __forceinline__ bool few_rows(const PagedAttnArgs& a, int cnt) {
  return cnt * a.g <= a.few;
}

// End of the slots that row i may admit.
__device__ __forceinline__ int row_end(const PagedAttnArgs& a, const PagedReq& q, int i) {
  return min(q.prefix + (a.mask ? q.cnt : i + 1), a.b.C);
}

__device__ __forceinline__ PagedReq attn_req(const PagedAttnArgs& a, int r) {
  PagedReq q = paged_req(a.b, r);
  if (a.mask) q.cnt = min(q.cnt, a.N);
  return q;
}

struct Work {
  PagedReq q;
  int r, kvh, split, qb;
  bool ok;
};
// What this workgroup does: row block qb of `rows` rows, a kv head and a run of a
// request.  Workgroups are dealt round-robin over the XCDs, each with its own L2; row
// blocks of one (kv head, run) read the same K and V, so each XCD has its own of
// these pairs, or, where there are fewer than eight, shares one with others (one long
// request of four heads ran on half of the chip before).
//
// Calls of up to 64 requests have workgroups for as many row blocks as their rows can
// fill, and find theirs from the counts, a request to a lane: the longest requests
// first, and of each the last rows, which see most, so that what starts last is short
// (64 single tokens: 161 to 148 us; a workgroup that finds nothing to do takes 1 to 2
// us of half a compute unit, and 24 requests of 1 to 700 rows had 15,000 of these).
__device__ __forceinline__ Work work_of(const PagedAttnArgs& a, int qblocks, int nsplit, int rows,
                                        bool few) {
  const int pairs = a.Hkv * nsplit;
  const int x = blockIdx.x % kXcds, j = blockIdx.x / kXcds;
  int pair, rb;
  if (pairs % kXcds == 0) {
    pair = kXcds * (j % (pairs / kXcds));  // (and one of eight, by the request)
    rb = j / (pairs / kXcds);
  } else if (kXcds % pairs == 0) {
    pair = x % pairs;
    rb = j * (kXcds / pairs) + x / pairs;
  } else {
    pair = blockIdx.x % pairs;
    rb = blockIdx.x / pairs;
  }
  Work w;
  const auto settle = [&]() {
    // (a short request has one run: rotated, or one or two XCDs would have all of them)
    if (pairs % kXcds == 0) pair += (x + w.r) % kXcds;
    w.split = pair % nsplit;
    w.kvh = pair / nsplit;
  };
  if (a.b.R > 64) {
    w.r = rb / qblocks;
    w.qb = qblocks - 1 - rb % qblocks;
    w.ok = w.r < a.b.R;
    if (!w.ok) return w;
    settle();
    w.q = attn_req(a, w.r);
    w.ok = few_rows(a, w.q.cnt) == few && w.qb * rows < w.q.cnt * a.g;
    return w;
  }
  const int lane = threadIdx.x & 63;
  PagedReq q = attn_req(a, min(lane, a.b.R - 1));
  if (lane >= a.b.R || few_rows(a, q.cnt) != few) q.cnt = 0;
  const int len = q.prefix + q.cnt, blocks = (q.cnt * a.g + rows - 1) / rows;
  // (equal lengths by lane, and those past 2^25 as equal; without branches: 64 rounds of
  // them were 5 us of every workgroup)
  const int key = min(len, (1 << 25) - 1) << 6 | (63 - lane);
  int before = 0;
  for (int i0 = 0; i0 < a.b.R; i0 += 8) {
#pragma unroll
    for (int i = i0; i < i0 + 8; ++i)
      before += __builtin_amdgcn_readlane(blocks, i) & -(int)(__builtin_amdgcn_readlane(key, i) > key);
  }
  const uint64_t mine = __ballot(rb >= before && rb - before < blocks);
  w.ok = mine != 0;
  if (!w.ok) return w;
  w.r = (int)__builtin_ctzll(mine);
  settle();
  w.q.start = __builtin_amdgcn_readlane(q.start, w.r);
  w.q.cnt = __builtin_amdgcn_readlane(q.cnt, w.r);
  w.q.prefix = __builtin_amdgcn_readlane(q.prefix, w.r);
  w.qb = __builtin_amdgcn_readlane(blocks, w.r) - 1 - (rb - __builtin_amdgcn_readlane(before, w.r));
  return w;
}

// Online softmax of one 16-row column tile over a chunk of NH halves of 32 slots:
// s[h][t] holds the raw scores of half h, tile t (slots 32 h + 8 grp + 4 t + e); bit 8 h
// + i of `adm` is set when slot 32 h + 8 grp + i is admitted (ignored when `all`).
// Writes the weights as B operands and returns the factor for the output so far.
// (Their sum is a product of its own, a row of ones with the weights: 32 clocks of the
// matrix unit for 64 of the vector unit, which is the busier one, and the sum is that
// of the rounded weights.)
template <bool H, int NH>
__device__ __forceinline__ float softmax_chunk(const f32x4 (&s)[NH][2], uint32_t adm, bool all,
                                               float c, float& m, u32x4 (&bp)[NH]) {
  float v[8 * NH];
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[8 * h + e] = s[h][0][e];
      v[8 * h + 4 + e] = s[h][1][e];
    }
  if (!all) {
#pragma unroll
    for (int i = 0; i < 8 * NH; ++i) v[i] = ((adm >> i) & 1u) ? v[i] : kNegInf;
  }
  float cmax = v[0];
#pragma unroll
  for (int i = 1; i < 8 * NH; ++i) cmax = fmaxf(cmax, v[i]);
  const float mx = row_max4(cmax);
  float alpha = 1.0f;
  if (__any((mx - m) * c > kSlack<H>)) {
    const float mn = fmaxf(m, mx);
    alpha = mn == m ? 1.0f : exp2_hw((m - mn) * c);  // m = -inf: 0
    m = mn;
  }
  const float off = (m == kNegInf ? 0.0f : m * c) - (H ? kHalfLift : 0.0f);
#pragma unroll
  for (int i = 0; i < 8 * NH; ++i) v[i] = exp2_hw(__builtin_fmaf(v[i], c, -off));
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) bp[h][i] = pack16<H>(v[8 * h + 2 * i], v[8 * h + 2 * i + 1]);
  return alpha;
}

// Admitted slots of the chunk at c0 for row i, the 16 bits of lane group grp
// (bits 8 h + j for slot 32 h + 8 grp + j).  mw: the row's mask words in LDS.
__device__ __forceinline__ uint32_t admitted(const PagedAttnArgs& a, const PagedReq& q,
                                             const uint32_t* mw, int i, int c0, int kend,
                                             uint64_t bad, int grp) {
  uint64_t win;
  if (a.mask) {
    const int j0 = c0 - q.prefix;
    const int wb = j0 >> 5, sh = j0 & 31;  // (floor)
    const uint32_t w0 = wb >= 0 && wb < a.NW ? mw[wb] : 0u;
    const uint32_t w1 = wb + 1 >= 0 && wb + 1 < a.NW ? mw[wb + 1] : 0u;
    const uint32_t w2 = wb + 2 >= 0 && wb + 2 < a.NW ? mw[wb + 2] : 0u;
    const uint64_t lo64 = ((uint64_t)w1 << 32) | w0;
    const uint64_t tree = sh ? (lo64 >> sh) | ((uint64_t)w2 << (64 - sh)) : lo64;
    const int np = min(max(-j0, 0), kChunk);
    win = low_bits(np) | (tree & ~low_bits(np));
  } else {
    win = low_bits(min(max(q.prefix + i + 1 - c0, 0), kChunk));
  }
  win &= low_bits(min(max(kend - c0, 0), kChunk)) & ~bad;
  return ((uint32_t)(win >> (8 * grp)) & 0xffu) | ((uint32_t)(win >> (32 + 8 * grp)) & 0xffu) << 8;
}

// Whether a 16-bit value is an infinity or NaN; a packed pair without such values.
template <bool H>
__device__ __forceinline__ bool odd16(uint32_t w) {
  constexpr uint32_t E = H ? 0x7c00u : 0x7f80u;
  return (w & E) == E;
}
template <bool H>
__device__ __forceinline__ uint32_t fine_pair(uint32_t w) {
  return (odd16<H>(w) ? 0u : w & 0xffffu) | (odd16<H>(w >> 16) ? 0u : w & 0xffff0000u);
}

// Four held values (pctree_held.h) times their scale, in 16 bits: exact, but for float16's
// range.
template <bool H>
__device__ __forceinline__ u32x2 held4(uint32_t w, float scale) {
  u32x2 r;
  if constexpr (H) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true));
  } else {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  }
  return r;
}
template <bool H>
__device__ __forceinline__ u32x4 held8(uint32_t w0, uint32_t w1, float scale) {
  const u32x2 a = held4<H>(w0, scale), b = held4<H>(w1, scale);
  return u32x4{a[0], a[1], b[0], b[1]};
}
// Where the scale of a slot at offset `off` of a page lies.
__device__ __forceinline__ size_t scale_place(const PagedAttnArgs& a, uint32_t page, int kvh,
                                              int off) {
  return page * (size_t)a.s.stride + ((size_t)kvh << (a.b.page_shift - a.s.block_shift)) +
         (uint32_t)(off >> a.s.block_shift);
}

// Where the run of a request of few rows leaves row rho.
__device__ __forceinline__ size_t few_part(const PagedAttnArgs& a, int split, int r, int kvh,
                                           int rho) {
  return (((size_t)split * a.b.R + r) * a.Hkv + kvh) * a.few_stride + rho;
}

// Infinite and NaN values that were set to zero: they make the outputs of the rows
// that do admit them NaN.  Rows ri[c] of a lane, their elements 16 t + d .. + 3 in
// o[c][t]; slots [first, kend).  Rare, so slot by slot from memory.
template <int D, bool H, bool Q8, int CT, int DT>
__device__ __forceinline__ void mend_odd(const PagedAttnArgs& a, const PagedReq& q, int r, int kvh,
                                         const int (&ri)[CT], int i_first, const uint32_t* mask,
                                         int first, int kend, int d, f32x4 (&o)[CT][DT]) {
  const int* table = a.b.page_table + (size_t)r * a.b.max_pages;
  const int pmask = (1 << a.b.page_shift) - 1;
#pragma unroll 1
  for (int s = first; s < kend; ++s) {
    const int p = table[s >> a.b.page_shift], j = s - q.prefix;
    if ((unsigned)p >= (unsigned)a.b.pages) continue;
    const size_t head = (size_t)p * a.b.page_units + (size_t)kvh * a.b.head_units;
    const uint16_t* vrow = a.v + head * 8 + (size_t)(s & pmask) * D + d;
    const uint8_t* held = (const uint8_t*)a.v + head * 16 + (size_t)(s & pmask) * D + d;
    float scale = 0.0f;
    if constexpr (Q8) scale = scale_up(scale_in(a.s.v[scale_place(a, p, kvh, s & pmask)]));
    bool sees[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
      sees[c] = j < 0 || (a.mask ? (mask[(ri[c] - i_first) * a.NW + (j >> 5)] >> (j & 31)) & 1
                                 : j <= ri[c]);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      u32x2 w;
      if constexpr (Q8) w = held4<H>(*(const uint32_t*)(held + 16 * t), scale);
      else w = *(const u32x2*)(vrow + 16 * t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool odd = odd16<H>(w[e / 2] >> (16 * (e & 1)));
#pragma unroll
        for (int c = 0; c < CT; ++c)
          if (odd && sees[c]) o[c][t][e] = __builtin_nanf("");
      }
    }
  }
}

// Where unit u of row `row` lies in a chunk that was converted (a further step on k_unit and
// v_unit, the same for every row of a fragment's read): lanes write every second unit of a
// row, and eight lanes' writes meet all banks only if half of them take the odd places.
template <int D, bool Q8>
__device__ __forceinline__ int staged(int u, int row) {
  return !Q8 ? 0 : D == 128 ? (u >> 3) & 1 : row & 1;
}

// 128 rows of one (request, kv head) to a workgroup.  Two products of 64 x 128 x D a chunk
// bound it, and the vector unit's softmax between them; over pages in 8 bits (Q8) also the
// conversion of every chunk, once for the workgroup (the chunk below: 252 us, 0.93 PFLOP/s;
// 373 with the conversion scheduled among the products, which costs registers).  (2048 rows over 6000 slots, 32
// and 8 heads of 128, 235 GFLOP: 228 to 238 us, 1.0 PFLOP/s, where a library product of
// 8192 runs at 1.2.  32-slot chunks 290, 48 rows a wave 445, for 267 at the time: registers.)
template <int D, bool H, bool Q8>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void paged_attn_kernel(
    PagedAttnArgs a) {
  constexpr int KS = D / 32, DT = D / 16, UPR = D / 8, CT = kColTiles;
  constexpr int TILE = kChunk * D;
  constexpr int IPW = kChunk * UPR / kThreads;  // load instructions per wave, chunk and tensor
  __shared__ __attribute__((aligned(16))) uint16_t sKV[2][2][TILE];
  __shared__ int sOdd;  // values were set to zero because some row may not admit them
  extern __shared__ uint32_t sMask[];

  const Work wk = work_of(a, a.qblocks, a.nsplit, kRowsPerBlock, false);
  if (!wk.ok) return;
  const PagedReq q = wk.q;
  const int cnt = q.cnt;
  const int rows = cnt * a.g, rho0 = wk.qb * kRowsPerBlock;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int i_first = rho0 / a.g;  // request rows of the block
  const int i_last = min((rho0 + kRowsPerBlock - 1) / a.g, cnt - 1);
  const int end = min(q.prefix + cnt, a.b.C);
  const int run = run_slots(end, a.nsplit, a.least);
  const bool direct = run >= end;  // one run: no merge
  const int kbeg = wk.split * run, kend = min(kbeg + run, row_end(a, q, i_last));
  if (kbeg >= kend) return;

  // this lane's rows and their Q^T fragments
  bool row_in[CT];
  int ri[CT], hq[CT];
  u32x4 bq[CT][KS];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int rho = rho0 + wave * kRowsPerWave + 16 * c + col;
    row_in[c] = rho < rows;
    const int rr = min(rho, rows - 1);
    ri[c] = rr / a.g;
    hq[c] = wk.kvh * a.g + rr % a.g;
    const uint16_t* qrow = a.q + ((size_t)(q.start + ri[c]) * a.Hq + hq[c]) * D + grp * 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) bq[c][s] = *(const u32x4*)(qrow + s * 32);
  }
  // the rows of the whole wave (uniform)
  const int w_first = min(rho0 + wave * kRowsPerWave, rows - 1) / a.g;
  const int w_last = min(rho0 + wave * kRowsPerWave + kRowsPerWave, rows) - 1;
  const int w_end = row_end(a, q, max(w_last, 0) / a.g);
  const bool w_live = rho0 + wave * kRowsPerWave < rows;

  // slots below it are admitted by every row of the block (where they have a page)
  const int all_see = min(kend, q.prefix + (a.mask ? 0 : i_first + 1));

  const int* table = a.b.page_table + (size_t)wk.r * a.b.max_pages;
  const int pmask = (1 << a.b.page_shift) - 1;
  constexpr int RPI = 64 / UPR;  // slots of a load instruction
  auto page_of = [&](int c0) __attribute__((always_inline)) {
    return table[min(c0 + lane, kend - 1) >> a.b.page_shift];
  };
  // The chunk's K and V into a buffer; returns the slots without a page.
  auto fetch = [&](int c0, int pg, int buf) __attribute__((always_inline)) -> uint64_t {
    const bool none = (unsigned)pg >= (unsigned)a.b.pages;
    const uint64_t bad = __ballot(none) & low_bits(kChunk);
    const uint32_t pgc = none ? 0u : (uint32_t)pg;
    const int last = kend - 1 - c0;
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
      const int row = (wave * IPW + i) * RPI + lane / UPR, pos = lane % UPR;
      const uint32_t p = __builtin_amdgcn_ds_bpermute(min(row, last) * 4, pgc);
      const size_t base = (size_t)p * a.b.page_units + (size_t)wk.kvh * a.b.head_units +
                          (uint32_t)((c0 + min(row, last)) & pmask) * UPR;
      load_lds16((const uint4*)a.k + base + (pos ^ k_unit<D>(row)),
                 &sKV[buf][0][(wave * IPW + i) * 512]);
      load_lds16((const uint4*)a.v + base + (pos ^ v_unit<D>(row)),
                 &sKV[buf][1][(wave * IPW + i) * 512]);
    }
    return bad;
  };
  // The same with scalar bases, for pages of at least 8 slots, where the slots of one
  // load instruction (4, or 8 of a smaller head) share a page; the lanes' offsets are
  // the same for every chunk.  (Slots past the run in its last page are loaded and
  // masked.)
  uint32_t koff[IPW], voff[IPW];
#pragma unroll
  for (int i = 0; i < IPW; ++i) {
    const int row = (wave * IPW + i) * RPI + lane / UPR, pos = lane % UPR;
    koff[i] = (uint32_t)(row * UPR + (pos ^ k_unit<D>(row))) * 16;
    voff[i] = (uint32_t)(row * UPR + (pos ^ v_unit<D>(row))) * 16;
  }
  const size_t head_base = (size_t)wk.kvh * a.b.head_units;
  auto fetch_scalar = [&](int c0, int pg, int buf) __attribute__((always_inline)) -> uint64_t {
    const bool none = (unsigned)pg >= (unsigned)a.b.pages;
    const uint64_t bad = __ballot(none) & low_bits(kChunk);
    const uint32_t pgc = none ? 0u : (uint32_t)pg;
    const bool one_page = (1 << a.b.page_shift) >= kChunk;
    if (one_page) {
      const size_t base = (size_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)pgc) * a.b.page_units +
                          head_base + (uint32_t)(c0 & pmask) * UPR;
#pragma unroll
      for (int i = 0; i < IPW; ++i) {
        load_lds16((const uint4*)a.k + base, koff[i], &sKV[buf][0][(wave * IPW + i) * 512]);
        load_lds16((const uint4*)a.v + base, voff[i], &sKV[buf][1][(wave * IPW + i) * 512]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < IPW; ++i) {
        const int row = (wave * IPW + i) * RPI;
        const size_t base = (size_t)(uint32_t)__builtin_amdgcn_readlane((int)pgc, row) * a.b.page_units +
                            head_base + (size_t)(((c0 + row) & pmask) - row) * UPR;
        load_lds16((const uint4*)a.k + base, koff[i], &sKV[buf][0][(wave * IPW + i) * 512]);
        load_lds16((const uint4*)a.v + base, voff[i], &sKV[buf][1][(wave * IPW + i) * 512]);
      }
    }
    return bad;
  };
  // Pages in 8 bits: a chunk goes through registers, loaded a chunk ahead and put into
  // LDS in 16 bits, scaled, after the products of the one before.
  constexpr int HU = D / 16, UPT = kChunk * HU / kThreads;  // 16-byte units of a row, of a thread
  u32x4 kx[UPT], vx[UPT];
  int ks[UPT], vs[UPT];
  auto fetch_held = [&](int c0, int pg) __attribute__((always_inline)) -> uint64_t {
    const bool none = (unsigned)pg >= (unsigned)a.b.pages;
    const uint64_t bad = __ballot(none) & low_bits(kChunk);
    const uint32_t pgc = none ? 0u : (uint32_t)pg;
    const int last = kend - 1 - c0;
#pragma unroll
    for (int i = 0; i < UPT; ++i) {
      const int row = min((i * kThreads + (int)threadIdx.x) / HU, last);
      const uint32_t p = __builtin_amdgcn_ds_bpermute(row * 4, pgc);
      const int off = (c0 + row) & pmask;
      const size_t at = (size_t)p * a.b.page_units + head_base + (uint32_t)off * HU + threadIdx.x % HU;
      const size_t sp = scale_place(a, p, wk.kvh, off);
      kx[i] = ((const u32x4*)a.k)[at];
      vx[i] = ((const u32x4*)a.v)[at];
      ks[i] = a.s.k[sp];
      vs[i] = a.s.v[sp];
    }
    return bad;
  };
  // (part: some row sees the chunk only in part, so infinite and NaN values become zeros;
  // bad: its slots without a page, whose values no row admits and nothing has to mend)
  auto stage = [&](int buf, bool part, uint64_t bad) __attribute__((always_inline)) {
    bool odd = false;
    if (bad) {
#pragma unroll
      for (int i = 0; i < UPT; ++i)
        if ((bad >> ((i * kThreads + threadIdx.x) / HU)) & 1) vx[i] = u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < UPT; ++i) {
      const int row = (i * kThreads + threadIdx.x) / HU, u = 2 * (threadIdx.x % HU);
      const float kf = scale_up(scale_in(ks[i])), vf = scale_up(scale_in(vs[i]));
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        *(u32x4*)(&sKV[buf][0][row * D + ((u + b) ^ k_unit<D>(row) ^ staged<D, Q8>(u, row)) * 8]) =
            held8<H>(kx[i][2 * b], kx[i][2 * b + 1], kf);
        u32x4 w = held8<H>(vx[i][2 * b], vx[i][2 * b + 1], vf);
        if (part) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f = fine_pair<H>(w[e]);
            odd |= f != w[e];
            w[e] = f;
          }
        }
        *(u32x4*)(&sKV[buf][1][row * D + ((u + b) ^ v_unit<D>(row) ^ staged<D, Q8>(u, row)) * 8]) = w;
      }
    }
    if (odd) sOdd = 1;
  };
  int pg = page_of(kbeg);
  uint64_t bad_next;
  if constexpr (Q8) bad_next = fetch_held(kbeg, pg);
  else bad_next = fetch(kbeg, pg, 0);
  pg = page_of(min(kbeg + kChunk, kend - 1));

  if (threadIdx.x == 0) sOdd = 0;
  if constexpr (Q8) {
    lds_barrier();
    stage(0, bad_next || kbeg + kChunk > all_see, bad_next);
  }
  if (a.mask) {
    const uint32_t* mg = a.mask + ((size_t)wk.r * a.N + i_first) * a.NW;
    for (int i = threadIdx.x; i < (i_last - i_first + 1) * a.NW; i += kThreads) sMask[i] = mg[i];
  }

  f32x4 o[CT][DT], l[CT];  // (the four elements of l are the same)
  float m[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    m[c] = kNegInf;
    l[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DT; ++t) o[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // A rows of a tile pair: tile 0 holds keys 8c + e, tile 1 keys 8c + 4 + e
  const int krow0 = 8 * (col >> 2) + (col & 3);
  constexpr uint32_t one = H ? 0x3c003c00u : 0x3f803f80u;
  const u32x4 ones = {one, one, one, one};
  const int vkey = 8 * grp + (col >> 2);  // the key this lane addresses (of the first four)

  // S^T of the chunk, both halves and column tiles: 8 independent chains.
  auto scores = [&](const uint16_t* sK, f32x4 (&sacc)[CT][kHalves][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int h = 0; h < kHalves; ++h) sacc[c][h][0] = sacc[c][h][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const int u = 4 * k + grp;
        const uint16_t* kr =
            sK + (32 * h + krow0) * D + (u ^ k_unit<D>(krow0) ^ staged<D, Q8>(4 * k, krow0)) * 8;
        const u32x4 a0 = *(const u32x4*)kr;
        const u32x4 a1 = *(const u32x4*)(kr + 4 * D);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          sacc[c][h][0] = mfma16<H>(a0, bq[c][k], sacc[c][h][0]);
          sacc[c][h][1] = mfma16<H>(a1, bq[c][k], sacc[c][h][1]);
        }
      }
    }
    // fragments six reads ahead of their two products (LDS answers after four)
    constexpr int READS = 2 * KS * kHalves, AHEAD = READS < 6 ? READS : 6;
    __builtin_amdgcn_sched_group_barrier(kReadLds, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < READS - AHEAD; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMatrix, CT, 0);
      __builtin_amdgcn_sched_group_barrier(kReadLds, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMatrix, CT * AHEAD, 0);
  };
  // O^T += V^T P^T of one half.
  auto weigh = [&](const uint16_t* sV, int h, const u32x4 (&bp)[CT]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const int u = (2 * t + ((col >> 1) & 1)) ^ v_unit<D>(vkey) ^ staged<D, Q8>(2 * t, vkey);
      const uint16_t* vr = sV + (32 * h + vkey) * D + u * 8 + (col & 1) * 4;
      const u32x2 lo = read_tr(vr), hi = read_tr(vr + 4 * D);
      const u32x4 av = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c][t] = mfma16<H>(av, bp[c], o[c][t]);
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) l[c] = mfma16<H>(ones, bp[c], l[c]);
    __builtin_amdgcn_sched_group_barrier(kReadLds, 8, 0);  // (four fragments ahead)
#pragma unroll
    for (int i = 0; i < DT - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMatrix, CT, 0);
      __builtin_amdgcn_sched_group_barrier(kReadLds, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMatrix, 5 * CT, 0);
  };

  int buf = 0, c0 = kbeg;
  bool some_bad = false;
  // Chunks that every row of the block sees whole: no masks, one test for both column
  // tiles' maxima, and the second half's weights computed beside the first half's
  // product.
  const int whole = a.b.page_shift >= 3 ? all_see : kbeg;
  auto stage_next = [&]() __attribute__((always_inline)) {
    if constexpr (Q8) {
      if (c0 + kChunk < kend) stage(buf ^ 1, bad_next || c0 + 2 * kChunk > all_see, bad_next);
    }
  };
  for (; c0 + kChunk <= whole && !bad_next; c0 += kChunk, buf ^= 1) {
    if constexpr (!Q8) wait_loads();
    lds_barrier();  // the chunk is complete; the other buffer is no longer read
    if (c0 + kChunk < kend) {
      if constexpr (Q8) bad_next = fetch_held(c0 + kChunk, pg);
      else bad_next = fetch_scalar(c0 + kChunk, pg, buf ^ 1);
      pg = page_of(min(c0 + 2 * kChunk, kend - 1));
    }
    if (!w_live) {
      stage_next();
      continue;
    }
    f32x4 sacc[CT][kHalves][2];
    scores(sKV[buf][0], sacc);
    float mx[CT];
    bool grows = false;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      mx[c] = sacc[c][0][0][0];
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[c] = fmaxf(mx[c], sacc[c][h][t][e]);
      mx[c] = row_max4(mx[c]);
      grows |= (mx[c] - m[c]) * a.scale_log2 > kSlack<H>;
    }
    if (__any(grows)) {
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const float mn = fmaxf(m[c], mx[c]);
        const float alpha = mn == m[c] ? 1.0f : exp2_hw((m[c] - mn) * a.scale_log2);
        m[c] = mn;
        l[c] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[c][t] *= alpha;
      }
    }
    float off[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
      off[c] = (m[c] == kNegInf ? 0.0f : m[c] * a.scale_log2) - (H ? kHalfLift : 0.0f);
    u32x4 bp[kHalves][CT];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          w[e] = exp2_hw(__builtin_fmaf(sacc[c][h][e / 4][e % 4], a.scale_log2, -off[c]));
#pragma unroll
        for (int e = 0; e < 4; ++e) bp[h][c][e] = pack16<H>(w[2 * e], w[2 * e + 1]);
      }
#pragma unroll
    for (int h = 0; h < kHalves; ++h) weigh(sKV[buf][1], h, bp[h]);
    // (one piece of code where the next chunk is whole too: 261 to 255 us)
    if (Q8 && c0 + 2 * kChunk <= all_see && !bad_next) stage(buf ^ 1, false, 0);
    else stage_next();
  }
  for (; c0 < kend; c0 += kChunk, buf ^= 1) {
    if constexpr (!Q8) wait_loads();
    lds_barrier();  // the chunk is complete; the other buffer is no longer read
    const uint64_t bad = bad_next;
    some_bad |= bad != 0;
    if (c0 + kChunk < kend) {
      if constexpr (Q8) bad_next = fetch_held(c0 + kChunk, pg);
      else bad_next = fetch(c0 + kChunk, pg, buf ^ 1);
      pg = page_of(min(c0 + 2 * kChunk, kend - 1));
    }
    uint16_t* sK = sKV[buf][0];
    uint16_t* sV = sKV[buf][1];
    // Chunks that some row of the block sees only in part (the same in every
    // wave): infinite and NaN values, and those of no page, become zeros.
    if (!Q8 && (bad || c0 + kChunk > all_see)) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < IPW; ++i) {
        const int u = i * kThreads + threadIdx.x;
        u32x4 w = *(const u32x4*)(sV + u * 8);
        const bool none = (bad >> (u / UPR)) & 1;
        bool any = none;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t f = none ? 0u : fine_pair<H>(w[e]);
          odd |= !none && f != w[e] && c0 + u / UPR < kend;
          any |= f != w[e];
          w[e] = f;
        }
        if (any) *(u32x4*)(sV + u * 8) = w;
      }
      if (odd) sOdd = 1;
      lds_barrier();
    }
    if (!w_live || c0 >= w_end) {  // (causal) no row of this wave sees the chunk
      stage_next();
      continue;
    }
    // every row of the wave admits every slot
    const bool full = !bad && c0 + kChunk <= min(kend, q.prefix + (a.mask ? 0 : w_first + 1));

    f32x4 sacc[CT][kHalves][2];
    scores(sK, sacc);
    u32x4 bp[kHalves][CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const uint32_t adm =
          full ? 0u : admitted(a, q, sMask + (ri[c] - i_first) * a.NW, ri[c], c0, kend, bad, grp);
      u32x4 w[kHalves];
      const float alpha = softmax_chunk<H, kHalves>(sacc[c], adm, full, a.scale_log2, m[c], w);
#pragma unroll
      for (int h = 0; h < kHalves; ++h) bp[h][c] = w[h];
      if (__any(alpha != 1.0f)) {
        l[c] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[c][t] *= alpha;
      }
    }
#pragma unroll
    for (int h = 0; h < kHalves; ++h) weigh(sV, h, bp[h]);
    stage_next();
  }
  // (every wave is past the loop's last barrier, and the last chunk's values were looked
  // at before it)
  if (sOdd) {
    const int first = some_bad ? kbeg : kbeg + max(all_see - kbeg, 0) / kChunk * kChunk;
    mend_odd<D, H, Q8, CT, DT>(a, q, wk.r, wk.kvh, ri, i_first, sMask, first, kend, 4 * grp, o);
  }

#pragma unroll
  for (int c = 0; c < CT; ++c) {
    if (!row_in[c]) continue;
    const size_t qidx = (size_t)(q.start + ri[c]) * a.Hq + hq[c];
    if (direct) {
      const float inv = l[c][0] == 0.0f ? 0.0f : 1.0f / l[c][0];  // (no admitted slot)
      uint16_t* orow = a.out + qidx * D;
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const f32x4 v = o[c][t] * inv;
        u32x2 w;
        w[0] = pack16<H>(v[0], v[1]);
        w[1] = pack16<H>(v[2], v[3]);
        *(u32x2*)(orow + t * 16 + 4 * grp) = w;
      }
    } else {
      const size_t prow = (size_t)wk.split * a.b.T * a.Hq + qidx;
      float* po = a.part_o + prow * D;
#pragma unroll
      for (int t = 0; t < DT; ++t) *(f32x4*)(po + t * 16 + 4 * grp) = o[c][t];
      if (grp == 0) {
        a.part_ml[2 * prow] = m[c];
        a.part_ml[2 * prow + 1] = l[c][0];
      }
    }
  }
}

// The results of a workgroup's waves, each in its own tile's place, joined.
template <int D, bool H, bool Q8, typename Tile>
__device__ __forceinline__ void few_join(const PagedAttnArgs& a, const Work& wk, Tile (&tiles)[kWaves],
                                         float2 (&sML)[kWaves][16], const int& sOdd,
                                         const uint32_t* mask, const f32x4 (&o)[D / 16], float m,
                                         float l, int kbeg, int kend, bool direct) {
  constexpr int DT = D / 16, PART = DT * 64;  // f32x4 of a wave's output
  static_assert(sizeof(Tile) >= PART * sizeof(f32x4), "an output fits a tile");
  const PagedReq& q = wk.q;
  const int rows = q.cnt * a.g, rho0 = wk.qb * 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int rho = min(rho0 + col, rows - 1), i_first = rho0 / a.g;
  const int ri = rho / a.g, hq = wk.kvh * a.g + rho % a.g;
  if (grp == 0) sML[wave][col] = make_float2(m, l);
  f32x4* sO = (f32x4*)tiles[wave];
#pragma unroll
  for (int t = 0; t < DT; ++t) sO[t * 64 + lane] = o[t];
  lds_barrier();
  const bool odd = sOdd != 0;
  for (int e = threadIdx.x; e < PART; e += kThreads) {  // (e % 64 == lane)
    if (rho0 + col >= rows) break;
    const int t = e / 64;
    float M = kNegInf;
    float2 ml[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      ml[w] = sML[w][col];
      M = fmaxf(M, ml[w].x);
    }
    float L = 0.0f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      // (equal maxima, -inf among them: factor 1)
      const float wt = ml[w].x == M ? 1.0f : exp2_hw((ml[w].x - M) * a.scale_log2);
      L += wt * ml[w].y;
      O += ((const f32x4*)tiles[w])[e] * wt;
    }
    const int d = t * 16 + 4 * grp;
    if (odd) {
      const int rows1[1] = {ri};
      f32x4 one[1][1] = {{O}};
      mend_odd<D, H, Q8, 1, 1>(a, q, wk.r, wk.kvh, rows1, i_first, mask, kbeg, kend, d, one);
      O = one[0][0];
    }
    if (direct) {
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
      u32x2 wv;
      wv[0] = pack16<H>(O[0] * inv, O[1] * inv);
      wv[1] = pack16<H>(O[2] * inv, O[3] * inv);
      *(u32x2*)(a.out + ((size_t)(q.start + ri) * a.Hq + hq) * D + d) = wv;
    } else {
      const size_t prow = few_part(a, wk.split, wk.r, wk.kvh, rho);
      *(f32x4*)(a.few_o + prow * D + d) = O;
      if (d == 0) {
        a.few_ml[2 * prow] = M;
        a.few_ml[2 * prow + 1] = L;
      }
    }
  }
}

// Requests of few rows: 16 of one (request, kv head) to a workgroup.  Bytes bound it: 64
// single tokens over 500 to 8000 slots, 711 MB, 142 us with the merge's 5, 5.0 TB/s; one
// token over 1000 slots is two launches' latency, 7.7 and 3.7 us.
template <int D, bool H>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void paged_few_kernel(
    PagedAttnArgs a) {
  constexpr int KS = D / 32, DT = D / 16, UPR = D / 8;
  constexpr int INS = kFewChunk * UPR / 64;  // load instructions of a chunk's V
  __shared__ __attribute__((aligned(16))) uint16_t sV[kWaves][kFewChunk * D];
  __shared__ float2 sML[kWaves][16];
  __shared__ int sOdd;
  extern __shared__ uint32_t sMask[];

  const Work wk = work_of(a, a.few_qblocks, a.few_nsplit, 16, true);
  if (!wk.ok) return;
  const PagedReq q = wk.q;
  const int rows = q.cnt * a.g, rho0 = wk.qb * 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int i_first = rho0 / a.g, i_last = (min(rho0 + 16, rows) - 1) / a.g;
  const int end = min(q.prefix + q.cnt, a.b.C);
  const int run = run_slots(end, a.few_nsplit, a.few_least);
  const bool direct = run >= end;
  const int kbeg = wk.split * run, kend = min(kbeg + run, row_end(a, q, i_last));
  if (kbeg >= kend) return;
  const int all_see = min(kend, q.prefix + (a.mask ? 0 : i_first + 1));
  const int* table = a.b.page_table + (size_t)wk.r * a.b.max_pages;
  const int pmask = (1 << a.b.page_shift) - 1;
  auto page_of = [&](int c0) __attribute__((always_inline)) {
    return table[min(c0 + (lane & 31), kend - 1) >> a.b.page_shift];
  };
  const int c_first = kbeg + wave * kFewChunk;
  int pg = page_of(min(c_first, kend - 1));

  const int rho = min(rho0 + col, rows - 1);
  const int ri = rho / a.g, hq = wk.kvh * a.g + rho % a.g;
  u32x4 bq[KS];
  {
    const uint16_t* qrow = a.q + ((size_t)(q.start + ri) * a.Hq + hq) * D + grp * 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) bq[s] = *(const u32x4*)(qrow + s * 32);
  }
  if (threadIdx.x == 0) sOdd = 0;
  if (a.mask) {
    const uint32_t* mg = a.mask + ((size_t)wk.r * a.N + i_first) * a.NW;
    for (int i = threadIdx.x; i < (i_last - i_first + 1) * a.NW; i += kThreads) sMask[i] = mg[i];
  }
  lds_barrier();
  const uint32_t* mw = sMask + (ri - i_first) * a.NW;

  f32x4 o[DT], l = {0.f, 0.f, 0.f, 0.f};
  float m = kNegInf;
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int krow0 = 8 * (col >> 2) + (col & 3);
  const int vkey = 8 * grp + (col >> 2);
  constexpr uint32_t one = H ? 0x3c003c00u : 0x3f803f80u;
  const u32x4 ones = {one, one, one, one};
  for (int c0 = c_first; c0 < kend; c0 += kWaves * kFewChunk) {
    const bool none = (unsigned)pg >= (unsigned)a.b.pages;
    const uint64_t bad = __ballot(none) & 0xffffffffu;
    const uint32_t pgc = none ? 0u : (uint32_t)pg;
    const int last = kend - 1 - c0;  // (slots past the run repeat its last one)
    auto at = [&](int row) __attribute__((always_inline)) {  // 16-byte units before the row
      const uint32_t p = __builtin_amdgcn_ds_bpermute(row * 4, pgc);
      return (size_t)p * a.b.page_units + (size_t)wk.kvh * a.b.head_units +
             (uint32_t)((c0 + min(row, last)) & pmask) * UPR;
    };
#pragma unroll
    for (int i = 0; i < INS; ++i) {
      const int u = i * 64 + lane, row = u / UPR, pos = u % UPR;
      load_lds16((const uint4*)a.v + at(row) + (pos ^ v_unit<D>(row)), &sV[wave][i * 512]);
    }
    u32x4 kf[2][KS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4* kr = (const u32x4*)a.k + at(krow0 + 4 * t) + grp;
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[t][k] = kr[4 * k];
    }
    pg = page_of(min(c0 + kWaves * kFewChunk, kend - 1));
    f32x4 sacc[1][2] = {{f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      sacc[0][0] = mfma16<H>(kf[0][k], bq[k], sacc[0][0]);
      sacc[0][1] = mfma16<H>(kf[1][k], bq[k], sacc[0][1]);
    }
    const bool full = !bad && c0 + kFewChunk <= all_see;
    const uint32_t adm = full ? 0u : admitted(a, q, mw, ri, c0, kend, bad, grp);
    u32x4 bp[1];
    const float alpha = softmax_chunk<H, 1>(sacc, adm, full, a.scale_log2, m, bp);
    if (__any(alpha != 1.0f)) {
      l *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
    }
    l = mfma16<H>(ones, bp[0], l);
    wait_loads();
    if (!full) {  // infinite and NaN values, and those of no page, become zeros
      bool odd = false;
#pragma unroll 1
      for (int i = 0; i < INS; ++i) {
        const int u = i * 64 + lane;
        u32x4 w = *(const u32x4*)(sV[wave] + u * 8);
        const bool gone = (bad >> (u / UPR)) & 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t f = gone ? 0u : fine_pair<H>(w[e]);
          odd |= !gone && f != w[e];
          w[e] = f;
        }
        *(u32x4*)(sV[wave] + u * 8) = w;
      }
      if (odd) sOdd = 1;
    }
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const uint16_t* vr = sV[wave] + vkey * D +
                           ((2 * t + ((col >> 1) & 1)) ^ v_unit<D>(vkey)) * 8 + (col & 1) * 4;
      const u32x2 lo = read_tr(vr), hi = read_tr(vr + 4 * D);
      o[t] = mfma16<H>(u32x4{lo[0], lo[1], hi[0], hi[1]}, bp[0], o[t]);
    }
    // (the tile's reads are back before the next chunk's loads overwrite it)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
  }
  few_join<D, H, false>(a, wk, sV, sML, sOdd, sMask, o, m, l[0], kbeg, kend, direct);
}

// The same over pages in 8 bits: a wave's step is 64 slots, as many bytes.  A lane takes
// 16 of a key's bytes at a time, two steps of the first product, and the queries lie in
// that order; values cross LDS in 8 bits, and a transposing read gives a lane 8 slots of
// one element, whose scale is one (a block holds 8 slots at least).  Both are converted,
// with their scales, right before the matrix instructions, 128 conversions of a pair a step.
// Bytes bound it: 64 single tokens over 500 to 8000 slots, 364 MB, 81 us with the merge's 5,
// 4.8 TB/s besides it; one token over 1000 slots 8.7 and 3.4 us.
template <int D, bool H>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void paged_few8_kernel(
    PagedAttnArgs a) {
  constexpr int DT = D / 16, HU = D / 16, KU = HU / 4;  // 16-byte units of a row, of a lane's keys
  constexpr int INS = kFewChunk8 * HU / 64;             // load instructions of a chunk's V
  constexpr int RPI = 64 / HU;                          // slots of one of these
  constexpr int BANKS = 16 / HU;                        // rows of 256 bytes
  __shared__ __attribute__((aligned(16))) uint8_t sV[kWaves][kFewChunk8 * D];
  __shared__ float2 sML[kWaves][16];
  __shared__ int sOdd;
  extern __shared__ uint32_t sMask[];

  const Work wk = work_of(a, a.few_qblocks, a.few_nsplit, 16, true);
  if (!wk.ok) return;
  const PagedReq q = wk.q;
  const int rows = q.cnt * a.g, rho0 = wk.qb * 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int i_first = rho0 / a.g, i_last = (min(rho0 + 16, rows) - 1) / a.g;
  const int end = min(q.prefix + q.cnt, a.b.C);
  const int run = run_slots(end, a.few_nsplit, a.few_least);
  const bool direct = run >= end;
  const int kbeg = wk.split * run, kend = min(kbeg + run, row_end(a, q, i_last));
  if (kbeg >= kend) return;
  const int all_see = min(kend, q.prefix + (a.mask ? 0 : i_first + 1));
  const int* table = a.b.page_table + (size_t)wk.r * a.b.max_pages;
  const int pmask = (1 << a.b.page_shift) - 1;
  auto page_of = [&](int c0) __attribute__((always_inline)) {
    return table[min(c0 + lane, kend - 1) >> a.b.page_shift];
  };
  const int c_first = kbeg + wave * kFewChunk8;
  int pg = page_of(min(c_first, kend - 1));

  const int rho = min(rho0 + col, rows - 1);
  const int ri = rho / a.g, hq = wk.kvh * a.g + rho % a.g;
  u32x4 bq[2 * KU];
  {
    const uint16_t* qrow = a.q + ((size_t)(q.start + ri) * a.Hq + hq) * D + grp * 16;
#pragma unroll
    for (int u = 0; u < KU; ++u) {
      bq[2 * u] = *(const u32x4*)(qrow + u * 64);
      bq[2 * u + 1] = *(const u32x4*)(qrow + u * 64 + 8);
    }
  }
  if (threadIdx.x == 0) sOdd = 0;
  if (a.mask) {
    const uint32_t* mg = a.mask + ((size_t)wk.r * a.N + i_first) * a.NW;
    for (int i = threadIdx.x; i < (i_last - i_first + 1) * a.NW; i += kThreads) sMask[i] = mg[i];
  }
  lds_barrier();
  const uint32_t* mw = sMask + (ri - i_first) * a.NW;

  f32x4 o[DT], l = {0.f, 0.f, 0.f, 0.f};
  float m = kNegInf;
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int vkey = 8 * grp + (col >> 1);  // the slot whose values this lane addresses
  constexpr uint32_t one = H ? 0x3c003c00u : 0x3f803f80u;
  const u32x4 ones = {one, one, one, one};
  // The lane's place in a chunk: of its keys (slots 8 c + e and, 4 further, 8 c + 4 + e of a
  // half; the same eight, so the same page and scale) and of the values it loads, the
  // units of a row permuted so that 16 rows' reads of one unit meet all banks.
  const int kgroup = col >> 2, krow = 8 * kgroup + (col & 3);
  const uint32_t koff = (uint32_t)(krow * HU + grp) * 16;
  uint32_t voff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = i * RPI + lane / HU;
    voff[i] = (uint32_t)(lane / HU * HU + (lane % HU ^ (row / BANKS % HU))) * 16;
  }
  const size_t head_bytes = (size_t)wk.kvh * a.b.head_units * 16;
  const size_t page_bytes = (size_t)a.b.page_units * 16;
  for (int c0 = c_first; c0 < kend; c0 += kWaves * kFewChunk8) {
    const bool none = (unsigned)pg >= (unsigned)a.b.pages;
    const uint64_t bad = __ballot(none);
    const uint32_t pgc = none ? 0u : (uint32_t)pg;
    const int last = kend - 1 - c0;  // (slots past the run: others of its last page)
    u32x4 kx[2][2][KU];
    if (a.b.page_shift >= 6) {  // the chunk lies in one page
      const size_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)pgc) * page_bytes + head_bytes +
                        (uint32_t)(c0 & pmask) * D;
      const uint8_t *kb = (const uint8_t*)a.k + at, *vb = (const uint8_t*)a.v + at;
#pragma unroll
      for (int i = 0; i < INS; ++i) load_lds16(vb + i * 1024, voff[i & 1], &sV[wave][i * 1024]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int u = 0; u < KU; ++u)
            kx[h][t][u] = *(const u32x4*)(kb + (32 * h + 4 * t) * D + u * 64 + koff);
    } else {
#pragma unroll
      for (int i = 0; i < INS; ++i) {
        const int row = i * RPI + lane / HU;
        const uint32_t p = __builtin_amdgcn_ds_bpermute(row * 4, pgc);
        load_lds16((const uint8_t*)a.v + p * page_bytes + head_bytes +
                       (uint32_t)((c0 + row) & pmask) * D + (voff[i & 1] % D),
                   &sV[wave][i * 1024]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 32 * h + krow;
        const uint32_t p = __builtin_amdgcn_ds_bpermute(row * 4, pgc);
        const uint8_t* kb = (const uint8_t*)a.k + p * page_bytes + head_bytes +
                            (uint32_t)((c0 + row) & pmask) * D + grp * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int u = 0; u < KU; ++u) kx[h][t][u] = *(const u32x4*)(kb + 4 * t * D + u * 64);
      }
    }
    // the scales of the chunk's groups of eight slots: keys in lanes 0 to 7, values in 8 to 15
    const int srow = 8 * (lane & 7);
    const size_t sp = scale_place(a, __builtin_amdgcn_ds_bpermute(srow * 4, pgc), wk.kvh,
                                  (c0 + srow) & pmask);
    const int sbyte = scale_in((lane & 8 ? a.s.v : a.s.k)[sp]);
    pg = page_of(min(c0 + kWaves * kFewChunk8, kend - 1));
    f32x4 sacc[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float kf = scale_up(__builtin_amdgcn_ds_bpermute((4 * h + kgroup) * 4, sbyte));
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sacc[h][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < KU; ++u) {
          const u32x4 w = kx[h][t][u];
          sacc[h][t] = mfma16<H>(held8<H>(w[0], w[1], kf), bq[2 * u], sacc[h][t]);
          sacc[h][t] = mfma16<H>(held8<H>(w[2], w[3], kf), bq[2 * u + 1], sacc[h][t]);
        }
      }
    }
    const bool full = !bad && c0 + kFewChunk8 <= all_see;
    const uint32_t adm = full ? 0u : admitted(a, q, mw, ri, c0, kend, bad, grp);
    u32x4 bp[2];
    const float alpha = softmax_chunk<H, 2>(sacc, adm, full, a.scale_log2, m, bp);
    if (__any(alpha != 1.0f)) {
      l *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
    }
    l = mfma16<H>(ones, bp[0], l);
    l = mfma16<H>(ones, bp[1], l);
    wait_loads();
    if (!full) {  // infinite and NaN values become zeros
      uint32_t odd = 0;  // a bit for each of the lane's 16 bytes
#pragma unroll 1
      for (int i = 0; i < INS; ++i) {
        u32x4 w = *(const u32x4*)(sV[wave] + i * 1024 + lane * 16);
        const float f = scale_up(__builtin_amdgcn_ds_bpermute((8 + (i * RPI + lane / HU) / 8) * 4, sbyte));
        uint32_t all = 0xffffffffu;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const u32x2 v = held4<H>(w[e], f);
          uint32_t keep = 0xffffffffu;
          if (odd16<H>(v[0])) keep &= 0xffffff00u;
          if (odd16<H>(v[0] >> 16)) keep &= 0xffff00ffu;
          if (odd16<H>(v[1])) keep &= 0xff00ffffu;
          if (odd16<H>(v[1] >> 16)) keep &= 0x00ffffffu;
          all &= keep;
          w[e] &= keep;
        }
        odd |= (uint32_t)(all != 0xffffffffu) << i;
        *(u32x4*)(sV[wave] + i * 1024 + lane * 16) = w;
      }
      for (; odd; odd &= odd - 1) {  // (a slot that no row admits leaves nothing to mend)
        const int row = __builtin_ctz(odd) * RPI + lane / HU;
        if (row <= last && !((bad >> row) & 1)) sOdd = 1;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float vf = scale_up(__builtin_amdgcn_ds_bpermute((8 + 4 * h + grp) * 4, sbyte));
      const int key = 32 * h + vkey;
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const u32x2 w = read_tr8(sV[wave] + key * D + (t ^ (key / BANKS % HU)) * 16 + (col & 1) * 8);
        o[t] = mfma16<H>(held8<H>(w[0], w[1], vf), bp[h], o[t]);
      }
    }
    // (the tile's reads are back before the next chunk's loads overwrite it)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
  }
  few_join<D, H, true>(a, wk, sV, sML, sOdd, sMask, o, m, l[0], kbeg, kend, direct);
}
// Merge of the runs: a wave takes 256 / D heads of one row, D / 4 threads each,
// 4 consecutive elements apiece.  Requests of one run are already written.
template <int D, bool H>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int TPR = D / 4, HPW = 64 / TPR;
  const int per_row = (a.Hq + HPW - 1) / HPW;
  const int wave =
      __builtin_amdgcn_readfirstlane(blockIdx.x * (kMergeThreads / 64) + threadIdx.x / 64);
  const int lane = threadIdx.x & 63;
  const int t = wave / per_row;
  if (t >= a.b.T) return;
  const int r = request_of_row(a.b, t);
  if (r < 0) return;
  const PagedReq q = attn_req(a, r);
  const int i = t - q.start, h = wave % per_row * HPW + lane / TPR, d = lane % TPR * 4;
  if (i >= q.cnt || h >= a.Hq) return;
  const int end = min(q.prefix + q.cnt, a.b.C);
  const bool few = few_rows(a, q.cnt);
  const int run = few ? run_slots(end, a.few_nsplit, a.few_least) : run_slots(end, a.nsplit, a.least);
  if (run >= end) return;
  const int ns = (row_end(a, q, i) + run - 1) / run;
  const size_t qidx = (size_t)t * a.Hq + h;
  // the row's parts, `rows` apart
  const size_t first = few ? few_part(a, 0, r, h / a.g, i * a.g + h % a.g) : qidx;
  const size_t rows = few ? (size_t)a.b.R * a.Hkv * a.few_stride : (size_t)a.b.T * a.Hq;
  const float* part_o = few ? a.few_o : a.part_o;
  const float* part_ml = few ? a.few_ml : a.part_ml;
  float M = kNegInf, L = 0.0f;
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < ns; s0 += kMergeBatch) {
    float ms[kMergeBatch], ls[kMergeBatch];
    f32x4 os[kMergeBatch];
#pragma unroll
    for (int j = 0; j < kMergeBatch; ++j) {
      const size_t prow = (size_t)min(s0 + j, ns - 1) * rows + first;
      ms[j] = part_ml[2 * prow];
      ls[j] = part_ml[2 * prow + 1];
      os[j] = *(const f32x4*)(part_o + prow * D + d);
    }
    float Mn = M;
#pragma unroll
    for (int j = 0; j < kMergeBatch; ++j)
      if (s0 + j < ns) Mn = fmaxf(Mn, ms[j]);
    // (equal maxima, -inf among them: factor 1; a run that admits nothing holds zeros)
    const float sc = M == Mn ? 1.0f : exp2_hw((M - Mn) * a.scale_log2);
    L *= sc;
    O *= sc;
#pragma unroll
    for (int j = 0; j < kMergeBatch; ++j) {
      if (s0 + j < ns) {
        const float w = ms[j] == Mn ? 1.0f : exp2_hw((ms[j] - Mn) * a.scale_log2);
        L += w * ls[j];
        O += os[j] * w;
      }
    }
    M = Mn;
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  u32x2 w;
  w[0] = pack16<H>(O[0] * inv, O[1] * inv);
  w[1] = pack16<H>(O[2] * inv, O[3] * inv);
  *(u32x2*)(a.out + qidx * D + d) = w;
}

// The mask rows of a workgroup of `rows` rows: at most (rows - 1) / g + 2 request rows.
unsigned mask_bytes(const PagedAttnArgs& a, int rows) {
  if (!a.mask) return 0;
  const int nodes = (rows - 1) / a.g + 2;
  return (unsigned)((nodes < a.N ? nodes : a.N) * a.NW * sizeof(uint32_t));
}

template <int D, bool H>
hipError_t launch(const PagedAttnArgs& a, const PagedPlan& p, bool held, hipStream_t stream) {
  if (p.blocks) {
    const unsigned blocks = (unsigned)p.blocks, lds = mask_bytes(a, kRowsPerBlock);
    if (held) paged_attn_kernel<D, H, true><<<blocks, kThreads, lds, stream>>>(a);
    else paged_attn_kernel<D, H, false><<<blocks, kThreads, lds, stream>>>(a);
  }
  if (p.few_blocks) {
    const unsigned blocks = (unsigned)p.few_blocks, lds = mask_bytes(a, 16);
    if (held) paged_few8_kernel<D, H><<<blocks, kThreads, lds, stream>>>(a);
    else paged_few_kernel<D, H><<<blocks, kThreads, lds, stream>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (p.nsplit == 1 && p.few_nsplit == 1)) return e;
  constexpr int HPW = 256 / D;
  const long long waves = (long long)a.b.T * ((a.Hq + HPW - 1) / HPW);
  paged_merge_kernel<D, H><<<(unsigned)((waves + 3) / 4), kMergeThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

PagedPlan plan_paged_attention(int R, int T, int max_rows, int Hq, int Hkv, int D, int C, bool held,
                               int cus) {
  PagedPlan p;
  p.few_least = held ? kFewRun8 : kFewRun;
  const int g = Hq / Hkv;
  const long long most = (long long)max_rows * g;  // rows of a request
  // Which kernels: requests of few rows have their own, unless none can have few (one
  // request of more) or nearly all must have many (a padded batch of trees).
  p.few = most <= kFewRows || (R > 1 && (long long)T * 2 < (long long)R * max_rows) ? kFewRows : 0;
  const bool many = most > kFewRows;
  p.few_stride = (int)(most < kFewRows ? most : kFewRows);
  p.few_qblocks = (p.few_stride + 15) / 16;
  const long long pairs = (long long)R * Hkv;
  const auto runs = [&](long long base, int target, int least) {
    const int units = (C + least - 1) / least;
    long long ns = base < target ? (target + base - 1) / base : 1;
    ns = ns < units ? ns : units;
    return (int)(ns < kMaxSplits ? ns : kMaxSplits);
  };
  // Runs for six workgroups a compute unit, at most 12 of a request, which the merge
  // reads in two steps (us at 32, 16, 12, 8 runs at most: 8 single tokens of 500 to 4000
  // slots 31, 25, 25, 23; 40 of one kv head and up to 8000 slots 30, 22, 25, 27; 64 tokens
  // of eight heads have 3 runs each, 150, and 165 with 2).  Long contexts of one or two
  // requests would want more: one request of eight heads is 96 workgroups, which take 95 us
  // for 131,072 slots in 8 bits, three requests 155 (in 16 bits 201 and 332).
  p.few_nsplit = p.few ? std::min(runs(pairs * p.few_qblocks, 6 * cus, p.few_least), 12) : 1;
  // workgroups for n row blocks of every (kv head, run) (work_of)
  const auto blocks = [&](long long n, int nsplit) {
    const long long pairs = (long long)Hkv * nsplit;
    return pairs < kXcds && kXcds % pairs == 0 ? (n * pairs + kXcds - 1) / kXcds * kXcds : n * pairs;
  };
  // row blocks that can hold rows: all of a request's, or by the rows there are
  const auto some = [&](long long each, int rows) {
    const long long by_rows = (long long)T * g / rows + R;
    return R <= 64 && by_rows < each * R ? by_rows : each * R;
  };
  p.few_blocks = p.few ? blocks(some(p.few_qblocks, 16), p.few_nsplit) : 0;
  const long long qb = (most + kRowsPerBlock - 1) / kRowsPerBlock;
  p.qblocks = (int)qb;
  const long long base = Hkv * some(qb, kRowsPerBlock);
  p.least = 2 * kChunk;
  // (a workgroup for each compute unit: 4 trees of 64 nodes, 1000 to 4000 slots, 57 us
  // with half of that, 40; a chunk of 512 rows over 4000 slots 95, 66)
  // Over 8-bit pages, whose chunks take as long and whose partial outputs weigh the same,
  // two workgroups where one would leave units idle, but no more runs than the page table's
  // capacity has 256 slots (us with one, with two, with two and shorter runs: the 4 trees 52, 44, 44; the chunk 74, 61,
  // 62; 8 trees of 128 nodes, 28 heads over 4 of 64, up to 3000 slots 45, 36, 37; 128 rows
  // over 1000 slots 20.4, 21.5, 24.0; 64 19.4, 20.3, 19.3).
  const bool twice = held && base < cus;
  p.nsplit = many ? runs(base, twice ? 2 * cus : cus, p.least) : 1;
  if (twice) p.nsplit = std::max(1, std::min(p.nsplit, C / (2 * p.least)));
  // Long and short requests side by side: the long ones' chains of chunks last longest,
  // so those of more than 1024 slots are cut (24 requests of 1 to 700 rows, one of 3000
  // slots, heads of 64: 71 us uncut, 60 with runs of 512, 48; 12 requests of 1 to 500
  // rows, 2000 slots, heads of 128: 39, 55, 42).
  if (many && p.few && base < 4 * cus && p.nsplit < 4) {
    p.least = 1024;
    p.nsplit = runs(1, 4, p.least);
  }
  p.blocks = many ? blocks(some(qb, kRowsPerBlock), p.nsplit) : 0;
  p.parts = p.nsplit > 1 ? (size_t)p.nsplit * T * Hq : 0;
  p.few_parts = p.few_nsplit > 1 ? (size_t)p.few_nsplit * pairs * p.few_stride : 0;
  const size_t parts = p.parts + p.few_parts;
  p.ws_bytes = parts ? parts * (D + 2) * sizeof(float) + 256 : 0;
  return p;
}

hipError_t launch_paged_attention(PagedAttnArgs a, const PagedPlan& p, int D, bool f16, bool held,
                                  void* workspace, hipStream_t stream) {
  a.qblocks = p.qblocks;
  a.nsplit = p.nsplit;
  a.least = p.least;
  a.few = p.few;
  a.few_qblocks = p.few_qblocks;
  a.few_nsplit = p.few_nsplit;
  a.few_least = p.few_least;
  a.few_stride = p.few_stride;
  a.part_o = (float*)workspace;
  a.few_o = a.part_o + p.parts * D;
  a.part_ml = a.few_o + p.few_parts * D;
  a.few_ml = a.part_ml + p.parts * 2;
  if (D == 128)
    return f16 ? launch<128, true>(a, p, held, stream) : launch<128, false>(a, p, held, stream);
  return f16 ? launch<64, true>(a, p, held, stream) : launch<64, false>(a, p, held, stream);
}

}  // namespace pctree
