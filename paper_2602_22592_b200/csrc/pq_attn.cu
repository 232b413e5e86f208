// Attention of one new token per sequence over the paged key-value cache:
//     o = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale (q . k_j) - m),   m = max_j scale (q . k_j),   j < length of the sequence.
//
// A pass reads every cached row and multiplies it with the group x head_dim query values that share its head: one to
// sixteen multiplications per byte, far below what the tensor cores need to be the limit, so that the memory is.  (Rows are read once for
// each column block: of sixteen query heads, or of eight above head_dim 128.  More query heads to a cache head than that read them again.)
// What follows from that:
//   * A warp works alone while it reads: it walks tiles of sixteen positions, copies them asynchronously in whole lines (a copy of a
//     warp is 512 neighbouring bytes; 16 bytes here and there in eight rows at once reached 4.5 TB/s, lines reach 5.9) into a ring
//     of its own, and meets no barrier.  The ring, 200 KB per SM, covers the latency.  Its 16-byte pieces are swizzled, so that
//     ldmatrix reads them without bank conflicts.
//   * The work is cut into equal shares of tiles per CTA, and within it per warp, over ALL sequences and heads (lengths live on the
//     device: every CTA adds them up itself), so that ragged batches, one long sequence and many short ones all keep every SM
//     reading until the end.  What a (sequence, head) cut between warps leaves is joined in the CTA, what one cut between CTAs
//     leaves by the CTA that arrives last, in the order of the positions: one launch, and the same bits whoever is last.
//   * S^T = K q^T on mma.sync.m16n8k16: positions are the sixteen rows, query heads the eight columns (two column blocks for
//     nine to sixteen).  tcgen05 has no shape for eight columns by sixteen rows that would not idle.  O^T = V^T P^T with V^T by
//     transposed ldmatrix.  Of int8 rows a 16-bit element is two codes, neighbours in a row: the contraction index of K and the
//     rows of V^T are permuted accordingly, queries and outputs with them.
//   * Types of the products.  A bf16 cache multiplies in bf16, and the weights enter the second product as the sum of three bf16
//     numbers, eight bits each of the 24 that a weight has, cut off and not rounded, and 2^-30 of the weight on top: no part is negative or zero (unless
//     the weight is below 2^-80), so that an infinity among the values stays that infinity.  An int8 cache multiplies in
//     fp16, where codes are exact and cost least to make: queries are scaled by a power of two per row (exact down to 2^-32 of the row's
//     largest: bf16 has fewer bits), and the weights, 2^14 at most, enter as the sum of two fp16 numbers, 2^-22 relative down to 2^-17 of
//     the largest and 2^-39 of the largest below that.  (One number, 2^-11, shows where values cancel.)  gamma_k
//     scales the scores; the weights of the second product are w / gamma_v, w = exp2(s - m) with m the maximum of s - log2 gamma_v less 14,
//     so that they stay in range.  m is an offset and nothing else (an approximate logarithm will do), and what is summed up is w itself:
//     gammas from 2^-121 to 2^24, rows of the largest numbers and rows of zeros, may lie beside one another.
// Measured (us, GB/s of the cache): sixty-four ragged sequences of up to 4096 positions, eight heads of 128 with four query heads each, bf16
// 112 to 116, 5900; 131072 positions of one sequence, the same heads, int8 62 to 65, 4300; sixteen of up to 2048, sixteen heads 35, 4900;
// sixteen of up to 2048, thirty-two heads of 100, int8 45, 3100; one of 200, sixteen heads 7.6.  Sixteen of up to 4096, eight heads of 256, bf16, with 8,
// 16 and 32 query heads each: 100, 143 and 237.  While the tiles stream they come at the rate of the memory; beside that a call has a head
// of about 4 us (lengths, page ids, first rows: three trips to memory one after another) and a tail of 3 to 5 (warps that end apart, two
// joins, the count between CTAs).  int8 rows also cost instructions, three in ten of them conversions: 62 % of the issue slots.  Eight or
// twelve warps instead of sixteen: heads of 100 47 and 41 where sixteen took 41; addresses carried along, pieces behind head_dim skipped,
// rows packed densely in the ring: no gain.
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <chrono>
#include <mutex>
#include <utility>

#include "pq_kernels.cuh"

namespace pq {

constexpr int kAttnTile = 16;                 // positions of a tile; pages are multiples of it
constexpr int kAttnRingBytes = 204 * 1024;    // of 227 KB a CTA can have, 18 of them static
constexpr int kAttnSmemMost = 209 * 1024;     // what a launch can ask for beside them
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

template <int DP, int NT, bool I8>
struct AttnForm {
  static constexpr int kRow = DP * (I8 ? 1 : 2);                       // bytes of a row in the ring
  static constexpr int kChunks = kRow / 16;                            // ... and its 16-byte pieces
  static constexpr int kTileBytes = kAttnTile * kRow;                  // keys of a tile; values behind them
  static constexpr int kCopies = kTileBytes / 512;                     // copies of a warp for a tile's keys
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kGammaBytes = I8 ? 128 : 0;                     // 16 of the keys, 16 of the values
  // As many warps as registers allow: sixteen where accumulators and queries fit in 128
  static constexpr int kWarps = DP * NT <= 128 && kStageBytes <= 4096 ? 16 : kStageBytes <= 8192 ? 8 : 4;
  static constexpr int kFit = kAttnRingBytes / ((kStageBytes + kGammaBytes) * kWarps);
  static constexpr int kStages = kFit > 6 ? 6 : kFit;
  static constexpr int kGammaAt = kStages * kStageBytes * kWarps;      // the gammas behind all rings
  static constexpr int kSmem = kGammaAt + kStages * kGammaBytes * kWarps;
  static_assert(kStages >= 3, "two stages in flight and one in use");
  static_assert(8 * NT * DP * 4 <= kStages * kStageBytes, "a warp's last partial sums fit in its ring");
};
// Where piece c of row r lies in a tile: the eight rows that ldmatrix reads at once fall into eight different bank groups
template <int ROW>
__device__ __forceinline__ uint32_t attn_place(int r, int c) {
  return r * ROW + ((c ^ (ROW >= 128 ? r & 7 : r >> 1 & 3)) << 4);
}

// 16 bytes; the offsets are part of the instruction, which spares an addition or two at every copy of a tile
template <int DST, int SRC>
__device__ __forceinline__ void attn_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0+%2], [%1+%3], 16;" ::"r"(dst), "l"(src), "n"(DST), "n"(SRC) : "memory");
}
template <bool ALL, int VALUES, int... I>       // the copies of a tile's keys and values that this lane has (32 i < have), or all
__device__ __forceinline__ void attn_copy_tile(std::integer_sequence<int, I...>, uint32_t dst, const uint32_t* place, const void* kp, const void* vp, int have) {
  ([&] { if (ALL || 32 * I < have) attn_copy16<0, 512 * I>(dst + place[I], kp); }(), ...);
  ([&] { if (ALL || 32 * I < have) attn_copy16<VALUES, 512 * I>(dst + place[I], vp); }(), ...);
}
__device__ __forceinline__ void attn_copy4(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
__device__ __forceinline__ void attn_copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void attn_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The sum of a tile to that of the tiles before.  A tensor core cuts off what does not fit where it adds to its accumulator: over a thousand tiles
// that would be 2^-14 of the sum for each part of the weights, always towards zero.  This addition rounds.
__device__ __forceinline__ void attn_add(float (&o)[4], const float (&sum)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] += sum[i];
}
// A word that counts arrivals of one launch: the launch's number above 16 bits, the count below.  Whoever is going to count first makes
// sure that the word is this launch's (a failed exchange means that another CTA of it did), so that the workspace may hold anything before.
__device__ __forceinline__ void count_open(unsigned long long* word, unsigned long long call) {
  const unsigned long long seen = *reinterpret_cast<volatile unsigned long long*>(word);
  if (seen >> 16 != call >> 16) atomicCAS(word, seen, call);
}
// One more: releases what the CTA has written (behind its barrier) and acquires what those before it have.  The last one leaves 0.
__device__ __forceinline__ bool count_last(unsigned long long* word, int of) {
  unsigned long long old;
  asm volatile("atom.acq_rel.gpu.global.add.u64 %0, [%1], 1;" : "=l"(old) : "l"(word) : "memory");
  const bool last = (int)(old & 0xffff) == of - 1;
  if (last) *reinterpret_cast<volatile unsigned long long*>(word) = 0;
  return last;
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p) : "memory"); }
__device__ __forceinline__ float attn_exp2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float attn_log2(float x) { float y; asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// Factors are taken as the square of this: a sum of weights times it twice survives where its square is below fp32's range
__device__ __forceinline__ float attn_half(float d) { return attn_exp2(0.5f * d); }
__device__ __forceinline__ float attn_rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t (&v)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t (&v)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Four int8 codes with their sign bits flipped (0 to 255) -> two pairs of fp16: behind an exponent byte 0x64 they read 1024 + u,
// and 1152 less is the code
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t halves) {
  const uint32_t bias = 0xE480E480u;      // -1152, twice
  const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&halves), *reinterpret_cast<const __half2*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int SEL>      // which two bytes
__device__ __forceinline__ uint32_t codes_pair(uint32_t flipped) { return codes_to_f16(__byte_perm(flipped, 0x64646464u, SEL)); }
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// The leading eight bits of a number, as a number and, of two, as a pair of bf16
__device__ __forceinline__ float bf16_part(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_parts(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
constexpr float kWeightTop = 14.f;        // int8 caches: the largest weight is 2^14, so that small ones keep their bits in fp16

// Division by a number that the host knows, of 0 <= n < 2^31: multiply and shift (Granlund and Montgomery's round-up method)
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  explicit FastDiv(uint32_t by) : d(by), shift(0) {
    while ((1ull << shift) < by) ++shift;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - by)) / by + 1);
  }
  __device__ int operator()(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
  __device__ long long wide(long long n) const { return n >> 31 ? n / d : (long long)operator()((int)n); }
};

struct AttnArgs {
  KvCache c;
  const uint16_t* Q;
  long long q_stride;
  const int* lens;
  uint16_t* O;
  float* lse;
  float scale_log2;          // scale x log2(e): weights are powers of two
  int q_heads, group;        // query heads, and of them per cache head
  int blocks;                // column blocks of 8 NT query heads per cache head
  FastDiv by_blocks, by_per_seq, by_page_tiles, by_chunks;   // blocks, heads x blocks, tiles of a page, 16-byte pieces of a row
  int first_in_smem;         // a warp's first piece fits in shared memory, behind the rings
  // workspace
  float* warp_part;          // [CTAs x warps][8 NT][DP] unnormalised sums of a warp's first piece, if that is not its last
  float* cta_part;           // [2 CTAs][8 NT][DP] the same of a CTA: 2 c + 1 where its piece is the item's beginning, 2 c elsewhere
  float2* cta_ml;            // [2 CTAs][8 NT] what was taken off the scores, and the sum of weights
  unsigned long long* arrived;   // [CTAs] of the item that begins in the CTA: how many of its pieces are there, marked with `call`
  unsigned long long call;   // a number of this launch, above 16 bits: what the workspace held before is recognised by its absence
};

constexpr int kFewPieces = 4;
constexpr int kAttnLens = 1024;      // lengths kept in shared memory

__device__ __forceinline__ int attn_len(const AttnArgs& a, const int* lens, int seq) {
  const int len = a.c.num_seqs <= kAttnLens ? lens[seq] : __ldcg(a.lens + seq);
  return min(len, a.c.max_pages * a.c.page_size);       // longer: reported where the lengths are added up
}

// A walk over a warp's share: its segments are stretches of tiles of one item = (sequence, cache head, column block).
struct AttnWalk {
  long long left;            // tiles of the share behind the current segment
  int seq, hb, t0, t1, len, tiles;
  __device__ bool next(const AttnArgs& a, const int* lens, int per_seq) {
    if (left <= 0) return false;
    if (++hb == per_seq) {
      hb = 0;
      do { len = attn_len(a, lens, ++seq); } while (len <= 0);
      tiles = (len + kAttnTile - 1) / kAttnTile;
    }
    t0 = 0;
    t1 = (int)(left < tiles ? left : tiles);
    left -= t1;
    return true;
  }
};

// Equal shares of all tiles: the first `more` CTAs take one tile more than the others
struct AttnShares {
  bool by_chunk;
  int used, more;
  long long each;
  __device__ long long begin(int cta) const { return cta * each + min(cta, more); }
  __device__ int holder(long long tile) const {               // the CTA whose share it is in
    const long long cut = (each + 1) * more;
    return (int)(tile < cut ? tile / (each + 1) : more + (tile - cut) / each);
  }
};

// One piece of a cut item: what a warp leaves for the CTA's join
struct AttnPiece {
  int item;                  // -1: none
  int seq, hb, whole_from, whole_to;   // whether the item begins, ends here
};

__device__ __forceinline__ void attn_store(const AttnArgs& a, long long qrow, int dim, float v0, float v1, float v2, float v3, float inv) {
  *reinterpret_cast<uint2*>(a.O + qrow * a.c.dim + dim) = make_uint2(pack_bf16x2(v0 * inv, v1 * inv), pack_bf16x2(v2 * inv, v3 * inv));
}
__device__ __forceinline__ float attn_inv(float l) { return l == 0.f ? 0.f : 1.f / l; }      // no weight: zeros
__device__ __forceinline__ float attn_lse(float m, float l) {      // m and the exponent of l may be large and cancel
  int e;
  const float f = frexpf(l, &e);
  return l == 0.f ? -INFINITY : ((m + (float)e) + log2f(f)) * kLn2;
}

template <int DP, int NT, bool I8>
__global__ void __launch_bounds__(AttnForm<DP, NT, I8>::kWarps * 32, 1) k_attn_decode(const __grid_constant__ AttnArgs a) {
  using F = AttnForm<DP, NT, I8>;
  constexpr int kWarps = F::kWarps, kThreads = kWarps * 32, kQ = 8 * NT, kChunkTiles = 4 * kWarps;
  extern __shared__ __align__(1024) uint8_t attn_smem[];      // a name of its own: the swizzle needs this alignment, a shared name takes the first one seen
  uint8_t* const smem = attn_smem;
  __shared__ long long sums[kThreads];          // tiles of the sequences before a thread's own
  __shared__ long long warp_sums[kWarps], warp_chunks[kWarps], cta_share[4];
  __shared__ int lens[kAttnLens];
  __shared__ AttnPiece pieces[2 * kWarps];
  __shared__ float2 piece_ml[2 * kWarps][kQ];   // {taken off the scores, -infinity without weight; sum of weights}
  __shared__ float2 run_ml[2 * kWarps][kQ];     // of the run that begins with a piece
  __shared__ struct { int first, pieces, piece; } open[2];    // items shared with CTAs before, behind: the CTA where it begins, how many hold it; what to join
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int per_seq = a.by_per_seq.d, n = a.c.num_seqs, row_bytes = a.c.pitch * (I8 ? 1 : 2), chunks = row_bytes / 16;
  uint8_t* const ring = smem + warp * (F::kStages * F::kStageBytes);
  // copy i takes this lane's piece 32 i + lane of the tile, whose rows are neighbours in the page
  uint32_t place[F::kCopies];
#pragma unroll
  for (int i = 0; i < F::kCopies; ++i) {
    const int at = 32 * i + lane, r = a.by_chunks(at);
    place[i] = attn_place<F::kRow>(r, at - r * chunks);
  }
  if (chunks < F::kChunks) {                                // pieces behind the rows' end are never copied: zeros once and for all
    for (int s = 0; s < F::kStages; ++s)
      for (int i = lane; i < kAttnTile * F::kChunks; i += 32)
        if (i % F::kChunks >= chunks)
          *reinterpret_cast<uint4*>(ring + s * F::kStageBytes + attn_place<F::kRow>(i / F::kChunks, i % F::kChunks)) = make_uint4(0, 0, 0, 0);
  }
  // lengths, page ids and queries are trips to memory one after another: ask for them to be in L2 (where later writes reach them too)
  {
    const long long line = (long long)(blockIdx.x * kThreads + tid) * 128;
    if (line < (long long)n * 4) prefetch_l2(reinterpret_cast<const uint8_t*>(a.lens) + line);
    if (line < (long long)n * a.c.max_pages * 4) prefetch_l2(reinterpret_cast<const uint8_t*>(a.c.page_table) + line);
    if (line < ((long long)(n - 1) * a.q_stride + (long long)a.q_heads * a.c.dim) * 2) prefetch_l2(reinterpret_cast<const uint8_t*>(a.Q) + line);
  }
  pdl_wait();
  auto first_at = [&](int w) { return reinterpret_cast<float*>(smem + F::kSmem) + w * min(kQ, a.group) * DP; };
  // ---- shares: every CTA adds up the lengths.  Where the items in chunks of kChunkTiles (four tiles a warp) are no more than the CTAs,
  // each chunk is a CTA's share: most items are then whole in a CTA, and a join between CTAs costs more than a few tiles.  Otherwise the
  // CTAs take equal shares of all tiles.
  const int per = (n + kThreads - 1) / kThreads;
  long long mine = 0, mine_chunks = 0;
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s >= n) break;
    const int raw = __ldcg(a.lens + s);
    if (n <= kAttnLens) lens[s] = raw;
    if (raw > a.c.max_pages * a.c.page_size && blockIdx.x == 0) report_index();
    const int tiles = (max(0, min(raw, a.c.max_pages * a.c.page_size)) + kAttnTile - 1) / kAttnTile;
    mine += tiles;
    mine_chunks += (tiles + kChunkTiles - 1) / kChunkTiles;
  }
  long long upto = mine, upto_chunks = mine_chunks;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, d), w = __shfl_up_sync(0xffffffffu, upto_chunks, d);
    if (lane >= d) { upto += v; upto_chunks += w; }
  }
  if (lane == 31) { warp_sums[warp] = upto; warp_chunks[warp] = upto_chunks; }
  if (tid < 2 * kWarps) pieces[tid].item = -1;
  __syncthreads();
  long long before = 0, before_chunks = 0, total = 0, chunks_all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) { before += warp_sums[w]; before_chunks += warp_chunks[w]; }
    total += warp_sums[w];
    chunks_all += warp_chunks[w];
  }
  sums[tid] = before + upto - mine;
  const long long tiles_all = total * per_seq;
  chunks_all *= per_seq;
  const int cta = blockIdx.x;
  AttnShares sh;
  sh.by_chunk = chunks_all <= gridDim.x;
  sh.used = sh.by_chunk ? (int)chunks_all : gridDim.x;
  sh.each = sh.used == 0 ? 0 : tiles_all >> 31 ? tiles_all / sh.used : (long long)((uint32_t)tiles_all / (uint32_t)sh.used);
  sh.more = sh.used ? (int)(tiles_all - sh.each * sh.used) : 0;
  if (sh.by_chunk) {                                          // chunks are few, and so are sequences: the thread that has this CTA's chunk says so
    long long first = before_chunks + upto_chunks - mine_chunks, at = sums[tid];
    if (cta >= first * per_seq && cta < (first + mine_chunks) * per_seq)
      for (int s = tid * per; s < n && s < (tid + 1) * per; ++s) {
        const int tiles = (max(0, attn_len(a, lens, s)) + kAttnTile - 1) / kAttnTile, nc = (tiles + kChunkTiles - 1) / kChunkTiles;
        const int c = cta - (int)(first * per_seq);
        if (c < nc * per_seq) {
          const int hb = c / nc, k = c - hb * nc;
          cta_share[0] = at * per_seq + (long long)hb * tiles + (long long)tiles * k / nc;
          cta_share[1] = at * per_seq + (long long)hb * tiles + (long long)tiles * (k + 1) / nc;
          cta_share[2] = cta - k;                             // the CTA of the item's first chunk, ...
          cta_share[3] = nc;                                  // ... and how many there are
          break;
        }
        first += nc;
        at += tiles;
      }
  }
  __syncthreads();
  long long c0 = 0, c1 = 0;
  if (cta < sh.used) {
    c0 = sh.by_chunk ? cta_share[0] : sh.begin(cta);
    c1 = sh.by_chunk ? cta_share[1] : sh.begin(cta + 1);
  }
  const long long r0 = c0 + (unsigned long long)((c1 - c0) * warp) / kWarps, r1 = c0 + (unsigned long long)((c1 - c0) * (warp + 1)) / kWarps;
  if (r0 < r1) {
    // ---- first segment: the sequence whose tiles hold r0
    const long long x = a.by_per_seq.wide(r0);                         // compared per sequence, not per head
    int lo = 0, hi = kThreads;                                // last thread whose sequences begin at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (sums[mid] <= x) lo = mid; else hi = mid;
    }
    AttnWalk cw;
    long long base = sums[lo];
    cw.seq = lo * per;
    for (;; ++cw.seq) {
      cw.len = attn_len(a, lens, cw.seq);
      cw.tiles = (max(0, cw.len) + kAttnTile - 1) / kAttnTile;
      if (x < base + cw.tiles) break;
      base += cw.tiles;
    }
    const long long in_seq = r0 - base * per_seq;
    cw.hb = in_seq >> 31 ? (int)(in_seq / cw.tiles) : (int)((uint32_t)in_seq / (uint32_t)cw.tiles);
    cw.t0 = (int)(in_seq - (long long)cw.hb * cw.tiles);
    cw.t1 = (int)(cw.tiles - cw.t0 < r1 - r0 ? cw.tiles : cw.t0 + (r1 - r0));
    cw.left = r1 - r0 - (cw.t1 - cw.t0);
    AttnWalk pw = cw;                                         // the loads run ahead of the products, across segments
    int pt = cw.t0, run = 0;                                  // next tile to load, and how many more of its page
    bool more = true;
    long long row0 = 0;                                       // its first row
    const int tiles_per_page = a.by_page_tiles.d;
    const uint32_t ring_at = smem_u32(ring), gamma_at = smem_u32(smem) + F::kGammaAt + warp * (F::kStages * F::kGammaBytes);
    // page ids of the sequence, a window of 32 at a time: lane i holds the one of page window + i
    int window = a.by_page_tiles(pt), ids;
    auto ask = [&]() {
      const int at = window + lane, most = a.by_page_tiles(pw.tiles - 1) + 1;
      ids = at < most ? __ldcg(a.c.page_table + (long long)pw.seq * a.c.max_pages + at) : -1;
    };
    ask();
    auto issue = [&](int stage) {
      if (more) {
        bool known = true;
        if (run == 0) {                                       // another page
          const int slot = a.by_page_tiles(pt), in_page = pt - slot * tiles_per_page;
          if (slot >= window + 32) {
            window = slot;
            ask();
          }
          const int page = __shfl_sync(0xffffffffu, ids, slot - window);
          known = (unsigned)page < (unsigned)a.c.num_pages;
          if (!known && lane == 0) report_index();
          run = known ? min(tiles_per_page - in_page, pw.t1 - pt) : 1;
          row0 = known ? ((long long)page * a.c.heads + a.by_blocks(pw.hb)) * a.c.page_size + in_page * kAttnTile : 0;
        }
        const int rows = known ? pw.len - pt * kAttnTile : 0;
        const uint8_t* const kp = static_cast<const uint8_t*>(a.c.K) + row0 * row_bytes + lane * 16;
        const uint8_t* const vp = static_cast<const uint8_t*>(a.c.V) + row0 * row_bytes + lane * 16;
        const uint32_t dst = ring_at + stage * F::kStageBytes;
        const int have = min(rows, kAttnTile) * chunks - lane;            // this lane's pieces: 32 i < have
        using Copies = std::make_integer_sequence<int, F::kCopies>;
        if (rows >= kAttnTile && chunks == F::kChunks) {
          attn_copy_tile<true, F::kTileBytes>(Copies{}, dst, place, kp, vp, have);
        } else if (rows >= kAttnTile) {
          attn_copy_tile<false, F::kTileBytes>(Copies{}, dst, place, kp, vp, have);
        } else {                                              // the sequence ends inside: rows behind its end are zero, and not read
#pragma unroll
          for (int i = 0; i < F::kCopies; ++i)
            if (32 * i + lane < kAttnTile * chunks) {
              const bool ok = 32 * i < have;
              cp_async16(dst + place[i], ok ? kp + 512 * i : static_cast<const uint8_t*>(a.c.K), ok);
              cp_async16(dst + F::kTileBytes + place[i], ok ? vp + 512 * i : static_cast<const uint8_t*>(a.c.V), ok);
            }
        }
        if constexpr (I8) {
          const int r = lane & 15;
          attn_copy4(gamma_at + stage * F::kGammaBytes + lane * 4, (lane < 16 ? a.c.k_gamma : a.c.v_gamma) + (r < rows ? row0 + r : 0), r < rows);
        }
        row0 += kAttnTile;
        ++pt;
        if (--run == 0) {
          if (pt == pw.t1) {
            const int seq = pw.seq;
            more = pw.next(a, lens, per_seq);
            pt = pw.t0;
            if (more && (pw.seq != seq || window != 0)) {     // from the beginning of another sequence, or of the same one again
              window = 0;
              ask();
            }
          }
        }
      }
      attn_copy_commit();
    };
    uint32_t qf[NT][DP / 16][2];
    auto load_q = [&](const AttnWalk& w) {
      const int head = a.by_blocks(w.hb), q0 = (w.hb - head * a.blocks) * kQ, qn = min(kQ, a.group - q0);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int q = nt * 8 + g;
        const uint16_t* src = a.Q + w.seq * a.q_stride + (long long)(head * a.group + q0 + q) * a.c.dim;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          qf[nt][k][0] = qf[nt][k][1] = 0;
          if constexpr (I8) {                                 // a thread of the product holds four neighbouring codes
            const int dim = k * 16 + t * 4;
            if (q < qn && dim < a.c.dim) {
              const uint2 v = __ldcg(reinterpret_cast<const uint2*>(src + dim));
              qf[nt][k][0] = v.x;
              qf[nt][k][1] = v.y;
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int dim = k * 16 + 8 * h + t * 2;
              if (q < qn && dim < a.c.dim) qf[nt][k][h] = __ldcg(reinterpret_cast<const uint32_t*>(src + dim));
            }
          }
        }
      }
    };
    load_q(cw);                                               // in front of the ring's loads, not behind them
    bool q_there = true;
#pragma unroll
    for (int s = 0; s < F::kStages - 1; ++s) issue(s);
    // counts of the items that this CTA may share: the one that it begins inside of, and one that begins here (while the first loads are on their way)
    if (lane == 0 && (r0 == c0 || r1 == c1) && !(sh.by_chunk && cta_share[3] == 1)) {
      if (r0 == c0 && cw.t0 > 0) {
        const long long x0 = r0 - cw.t0;
        open[0].first = sh.by_chunk ? (int)cta_share[2] : sh.holder(x0);
        open[0].pieces = sh.by_chunk ? (int)cta_share[3] : sh.holder(x0 + cw.tiles - 1) - open[0].first + 1;
        count_open(a.arrived + open[0].first, a.call);
      }
      if (r1 == c1) count_open(a.arrived + cta, a.call);
    }
    int stage = 0, ahead = F::kStages - 1;
    // ldmatrix addresses: of the keys the matrices (rows 0-7, 8-15) of a piece, then of the next one; of the values (transposed) the same
    // by pieces first for bf16, whose m-tiles are two pieces, by rows first for int8, whose m-tile is one
    const int mr = lane & 7, m1 = lane >> 3 & 1, m2 = lane >> 4;
    const uint32_t k_mat = attn_place<F::kRow>(mr + 8 * m1, m2);
    const uint32_t v_mat = F::kTileBytes + (I8 ? attn_place<F::kRow>(mr + 8 * m1, m2) : attn_place<F::kRow>(mr + 8 * m2, m1));

    do {
      // ---- one segment
      const int head = a.by_blocks(cw.hb), q0 = (cw.hb - head * a.blocks) * kQ, qn = min(kQ, a.group - q0);
      if (!q_there) load_q(cw);
      q_there = false;
      float sc[NT][2];                                        // scores in powers of two per unit of the product, by query column
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        sc[nt][0] = sc[nt][1] = a.scale_log2;
        if constexpr (I8) {                                   // to fp16, the largest of the row just below 2^15
          uint32_t top = 0;
#pragma unroll
          for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) top = max(top, max(qf[nt][k][i] << 16 & 0x7fff0000u, qf[nt][k][i] & 0x7fff0000u));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const int up = top >= 0x7f800000u ? 0 : min(126, 127 + 14 - (int)(top >> 23));
          const float f = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
          for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) qf[nt][k][i] = pack_f16x2(bf16lo(qf[nt][k][i]) * f, bf16hi(qf[nt][k][i]) * f);
          const float down = __uint_as_float((uint32_t)(127 - up) << 23) * a.scale_log2;
          sc[nt][0] = __shfl_sync(0xffffffffu, down, 8 * t);
          sc[nt][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
        }
      }
      // m: maximum so far of the scores (int8: less log2 gamma_v), mu: what is taken off them (0 while there is no weight: every score is -infinity)
      float o[NT][DP / 16][4] = {}, m[NT][2], mu[NT][2] = {}, l[NT][2] = {};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = -INFINITY;
      const int seg_len = cw.len;
      for (int tile = cw.t0; tile < cw.t1; ++tile) {
        attn_copy_wait<F::kStages - 2>();
        __syncwarp();                                          // every lane's copies are there, and the tile before has been read
        issue(ahead);                                          // into the place that it has left
        const uint32_t src = ring_at + stage * F::kStageBytes;
        // scores: rows g, g + 8 of the tile, query columns 2 t, 2 t + 1
        float s[NT][4] = {}, s2[NT][4] = {};
#pragma unroll
        for (int j = 0; j < F::kChunks / 2; ++j) {
          uint32_t w[4];
          ldmatrix4((src + k_mat) ^ (j << 5), w);
          if constexpr (I8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t xa = w[2 * h] ^ 0x80808080u, xb = w[2 * h + 1] ^ 0x80808080u;
              const uint32_t a0 = codes_pair<0x4140>(xa), a1 = codes_pair<0x4140>(xb), a2 = codes_pair<0x4342>(xa), a3 = codes_pair<0x4342>(xb);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(h ? s2[nt] : s[nt], a0, a1, a2, a3, qf[nt][2 * j + h][0], qf[nt][2 * j + h][1]);
            }
          } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16(j & 1 ? s2[nt] : s[nt], w[0], w[1], w[2], w[3], qf[nt][j][0], qf[nt][j][1]);
          }
        }
        float rv[2], lg[2];                                     // int8: 1 / gamma_v, about log2 gamma_v
        if constexpr (I8) {
          const float* gm = reinterpret_cast<const float*>(smem + F::kGammaAt + warp * (F::kStages * F::kGammaBytes) + stage * F::kGammaBytes);
          const float rk[2] = {attn_rcp(gm[g]), attn_rcp(gm[g + 8])};
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float gv = gm[16 + 8 * r + g];
            rv[r] = attn_rcp(gv);
            lg[r] = gv == gv ? attn_log2(gv) : 0.f;             // a row that is not a number moves no offset
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = (s[nt][i] + s2[nt][i]) * (rk[i >> 1] * sc[nt][i & 1]);
        } else {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = (s[nt][i] + s2[nt][i]) * sc[nt][i & 1];
        }
        const int valid = seg_len - tile * kAttnTile;         // rows of the tile that the sequence holds
        if (valid < kAttnTile) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (g + 8 * (i >> 1) >= valid) {
              if constexpr (I8) rv[i >> 1] = lg[i >> 1] = 0.f;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) s[nt][i] = -INFINITY;
            }
        }
        bool grew = false;
        float top[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float v = I8 ? fmaxf(s[nt][c] - lg[0], s[nt][c + 2] - lg[1]) : fmaxf(s[nt][c], s[nt][c + 2]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
            top[nt][c] = v;
            grew |= v > m[nt][c];
          }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              if (!(top[nt][c] > m[nt][c])) continue;
              const float h = attn_half(m[nt][c] - top[nt][c]), f = h * h;
              m[nt][c] = top[nt][c];
              mu[nt][c] = I8 ? top[nt][c] - kWeightTop : top[nt][c];
              l[nt][c] = l[nt][c] * h * h;
#pragma unroll
              for (int i = 0; i < DP / 16; ++i) { o[nt][i][c] *= f; o[nt][i][c + 2] *= f; }
            }
        }
        uint32_t ph[NT][2], pl[NT][2], pm[I8 ? 1 : NT][2];      // the parts of the weights, largest first
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] = attn_exp2(s[nt][i] - mu[nt][i & 1]);
            l[nt][i & 1] += p[i];
            if constexpr (I8) p[i] *= rv[i >> 1];
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (I8) {
              const uint32_t hi = pack_f16x2(p[2 * h], p[2 * h + 1]);
              const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              ph[nt][h] = transpose8x8(hi);
              pl[nt][h] = transpose8x8(pack_f16x2(p[2 * h] - back.x, p[2 * h + 1] - back.y));
            } else {
              const float x = p[2 * h], y = p[2 * h + 1];
              const float x1 = fmaf(x, 0x1p-30f, x - bf16_part(x)), x2 = fmaf(x, 0x1p-40f, x1 - bf16_part(x1));
              const float y1 = fmaf(y, 0x1p-30f, y - bf16_part(y)), y2 = fmaf(y, 0x1p-40f, y1 - bf16_part(y1));
              ph[nt][h] = transpose8x8(bf16_parts(x, y));
              pl[nt][h] = transpose8x8(bf16_parts(x1, y1));
              pm[I8 ? 0 : nt][h] = transpose8x8(bf16_parts(x2, y2));
            }
          }
        }
#pragma unroll
        for (int j = 0; j < F::kChunks / 2; ++j) {
          uint32_t w[4];
          ldmatrix4_trans((src + v_mat) ^ (j << 5), w);
          if constexpr (I8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {                      // an m-tile: row g the even dim of the g-th pair of a piece, row g + 8 the odd one
              const uint32_t x0 = w[2 * h] ^ 0x80808080u, x1 = w[2 * h + 1] ^ 0x80808080u;
              const uint32_t a0 = codes_pair<0x4240>(x0), a1 = codes_pair<0x4341>(x0), a2 = codes_pair<0x4240>(x1), a3 = codes_pair<0x4341>(x1);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float sum[4] = {};
                mma_f16(sum, a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
                mma_f16(sum, a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
                attn_add(o[nt][2 * j + h], sum);
              }
            }
          } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float sum[4] = {};
              mma_bf16(sum, w[0], w[1], w[2], w[3], pm[I8 ? 0 : nt][0], pm[I8 ? 0 : nt][1]);
              mma_bf16(sum, w[0], w[1], w[2], w[3], pl[nt][0], pl[nt][1]);
              mma_bf16(sum, w[0], w[1], w[2], w[3], ph[nt][0], ph[nt][1]);
              attn_add(o[nt][j], sum);
            }
          }
        }
        stage = stage + 1 == F::kStages ? 0 : stage + 1;
        ahead = ahead + 1 == F::kStages ? 0 : ahead + 1;
      }
      // ---- the segment's sums: out, or left for the join -- a warp's last piece in its ring, whose copies have all landed and been
      // read, one before it in global memory
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], d);
      const bool whole = cw.t0 == 0 && cw.t1 == cw.tiles, last = cw.left == 0;
      float* const part = last ? reinterpret_cast<float*>(ring) : a.first_in_smem ? first_at(warp) : a.warp_part + (long long)(cta * kWarps + warp) * kQ * DP;
      const int at = 2 * warp + (last ? 1 : 0);
      if (!whole) {
        if (last) { attn_copy_wait<0>(); __syncwarp(); }
        if (lane == 0) {
          pieces[at] = AttnPiece{cw.seq * per_seq + cw.hb, cw.seq, cw.hb, cw.t0 == 0, cw.t1 == cw.tiles};
          if (last && r1 == c1 && cw.t1 < cw.tiles) {          // the CTA's share ends inside: if the item began here, how many CTAs hold it
            open[1].first = cta;
            open[1].pieces = sh.by_chunk ? (int)cta_share[3] : sh.holder(c1 + (cw.tiles - cw.t1) - 1) - cta + 1;
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int q = nt * 8 + 2 * t + c;
          if (q >= qn) continue;
          const float inv = attn_inv(l[nt][c]);
          const long long qrow = (long long)cw.seq * a.q_heads + head * a.group + q0 + q;
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) {
            const int dim = 16 * i + (I8 ? 2 * g : g), dim2 = I8 ? dim + 1 : dim + 8;      // of rows g and g + 8
            if (!whole) {
              part[q * DP + dim] = o[nt][i][c];
              part[q * DP + dim2] = o[nt][i][c + 2];
            } else {
              const uint32_t two = pack_bf16x2(o[nt][i][c] * inv, o[nt][i][c + 2] * inv);
              uint16_t* out = a.O + qrow * a.c.dim;
              if (I8) {
                if (dim < a.c.dim) *reinterpret_cast<uint32_t*>(out + dim) = two;
              } else {
                if (dim < a.c.dim) out[dim] = (uint16_t)two;
                if (dim2 < a.c.dim) out[dim2] = (uint16_t)(two >> 16);
              }
            }
          }
          if (g == 0) {
            if (!whole) piece_ml[at][q] = make_float2(l[nt][c] == 0.f ? -INFINITY : mu[nt][c], l[nt][c]);
            else if (a.lse) a.lse[qrow] = attn_lse(mu[nt][c], l[nt][c]);
          }
        }
    } while (cw.next(a, lens, per_seq));
    attn_copy_wait<0>();
  }
  // ---- sequences without a position: zeros, or, of negative length, left as they were
  for (int s = cta * kWarps + warp; s < n; s += gridDim.x * kWarps) {
    if (attn_len(a, lens, s) != 0) continue;
    for (int i = lane * 4; i < a.q_heads * a.c.dim; i += 128) *reinterpret_cast<uint2*>(a.O + (long long)s * a.q_heads * a.c.dim + i) = make_uint2(0, 0);
    if (a.lse) for (int i = lane; i < a.q_heads; i += 32) a.lse[(long long)s * a.q_heads + i] = -INFINITY;
  }
  if (c0 >= c1) return;
  __syncthreads();
  // ---- join in the CTA.  Pieces of one item follow one another: a run.  Every warp finds the runs for itself, lane e looking at piece e.
  const int item_e = lane < 2 * kWarps ? pieces[lane].item : -1;
  const uint32_t have = __ballot_sync(0xffffffffu, item_e >= 0);
  const uint32_t below = have & ((1u << lane) - 1u);
  const int prev = __shfl_sync(0xffffffffu, item_e, below ? 31 - __clz(below) : 0);
  const uint32_t starts = __ballot_sync(0xffffffffu, item_e >= 0 && (below == 0 || prev != item_e));
  const int runs = __popc(starts), qmost = min(kQ, a.group);
  if (runs == 0) return;
  auto run_start = [&](int run) {                              // its first piece
    uint32_t left = starts;
    for (; run > 0; --run) left &= left - 1;
    return __ffs(left) - 1;
  };
  auto run_mask = [&](int e0) {                                // and all of them
    const uint32_t later = starts & ~((2u << e0) - 1u);
    return have & ~((1u << e0) - 1u) & (later ? (1u << (__ffs(later) - 1)) - 1u : 0xffffffffu);
  };
  // factors of the pieces: a warp for each run and query head, a lane for each piece
  for (int k = warp; k < runs * qmost; k += kWarps) {
    const int q = k % qmost, e0 = run_start(k / qmost);
    const bool in = run_mask(e0) >> lane & 1;
    const float2 ml = in ? piece_ml[lane][q] : make_float2(-INFINITY, 0.f);
    float top = ml.x, l;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float h = attn_half(ml.x - (top == -INFINITY ? 0.f : top)), f = h * h;
    l = ml.y * h * h;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    if (in) piece_ml[lane][q].x = f;
    if (lane == 0) run_ml[e0][q] = make_float2(top, l);
  }
  __syncthreads();
  // a thread for four dims of a query head of a run
  const int run_units = qmost * (DP / 4);
  for (int u = tid; u < runs * run_units; u += kThreads) {
    const int run = u / run_units, q = (u - run * run_units) / (DP / 4), dim = u % (DP / 4) * 4;
    const int e0 = run_start(run);
    const AttnPiece pc = pieces[e0];
    const uint32_t mask = run_mask(e0);
    const int head = a.by_blocks(pc.hb), q0 = (pc.hb - head * a.blocks) * kQ;
    if (q0 + q >= a.group || dim >= a.c.dim) continue;
    float4 acc = make_float4(0, 0, 0, 0);
    auto add = [&](const float4& v, float f) { acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f; };
    auto last_of = [&](int w) { return *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem + w * (F::kStages * F::kStageBytes)) + q * DP + dim); };
    for (uint32_t left = mask & 0x55555555u; left; left &= left - 1) {
      const int e = __ffs(left) - 1;
      add(a.first_in_smem ? *reinterpret_cast<const float4*>(first_at(e >> 1) + q * DP + dim)
                          : __ldcg(reinterpret_cast<const float4*>(a.warp_part + ((long long)(cta * kWarps + (e >> 1)) * kQ + q) * DP + dim)), piece_ml[e][q].x);
    }
    const uint32_t lasts = mask & 0xaaaaaaaau;
    if (lasts) {
      const int w0 = (__ffs(lasts) - 1) >> 1, w1 = (31 - __clz(lasts)) >> 1;
#pragma unroll 4
      for (int w = w0; w <= w1; ++w)
        if (lasts >> (2 * w + 1) & 1) add(last_of(w), piece_ml[2 * w + 1][q].x);
    }
    const bool from = pc.whole_from, to = pieces[31 - __clz(mask)].whole_to;
    const float2 ml = run_ml[e0][q];
    if (from && to) {
      const long long qrow = (long long)pc.seq * a.q_heads + head * a.group + q0 + q;
      attn_store(a, qrow, dim, acc.x, acc.y, acc.z, acc.w, attn_inv(ml.y));
      if (dim == 0 && a.lse) a.lse[qrow] = attn_lse(ml.x, ml.y);
    } else {
      const long long slot = 2 * cta + (from ? 1 : 0);
      __stcg(reinterpret_cast<float4*>(a.cta_part + (slot * kQ + q) * DP + dim), acc);
      if (dim == 0) __stcg(a.cta_ml + slot * kQ + q, ml);
    }
  }
  // ---- join between CTAs: by the last to arrive, for the first run if its item began before this CTA (side 0), for the last one if its
  // item goes on behind it and began here (side 1).  The CTA where the item begins keeps the count.
  const int ea = __ffs(starts) - 1, ez = 31 - __clz(starts);
  const bool open0 = !pieces[ea].whole_from, open1 = pieces[ez].whole_from && !pieces[31 - __clz(have)].whole_to;
  if (!open0 && !open1) return;
  __syncthreads();                                             // this CTA's pieces are written
  if (tid == 0 || tid == 32) {
    const int side = tid >> 5;
    open[side].piece = -1;
    if ((side ? open1 : open0) && count_last(a.arrived + open[side].first, open[side].pieces)) open[side].piece = side ? ez : ea;
  }
  __syncthreads();
  for (int side = 0; side < 2; ++side) {
    if (open[side].piece < 0) continue;
    const int np = open[side].pieces, f0 = open[side].first;
    const AttnPiece pc = pieces[open[side].piece];
    const int head = a.by_blocks(pc.hb), q0 = (pc.hb - head * a.blocks) * kQ, qn = min(kQ, a.group - q0);
    auto slot_of = [&](int i) { return (long long)(2 * (f0 + i) + (i == 0 ? 1 : 0)); };
    auto out = [&](int q, int dim, const float4& acc, float top, float l) {
      const long long qrow = (long long)pc.seq * a.q_heads + head * a.group + q0 + q;
      attn_store(a, qrow, dim, acc.x, acc.y, acc.z, acc.w, attn_inv(l));
      if (dim == 0 && a.lse) a.lse[qrow] = attn_lse(top, l);
    };
    const int units = qn * (DP / 4);
    if (np <= kFewPieces) {                                    // one trip to memory
      for (int u = tid; u < units; u += kThreads) {
        const int q = u / (DP / 4), dim = u % (DP / 4) * 4;
        if (dim >= a.c.dim) continue;
        float2 ml[kFewPieces];
        float4 v[kFewPieces];
#pragma unroll
        for (int i = 0; i < kFewPieces; ++i) {
          ml[i] = make_float2(-INFINITY, 0.f);
          v[i] = make_float4(0, 0, 0, 0);
          if (i < np) {
            ml[i] = __ldcg(&a.cta_ml[slot_of(i) * kQ + q]);
            v[i] = __ldcg(reinterpret_cast<const float4*>(a.cta_part + (slot_of(i) * kQ + q) * DP + dim));
          }
        }
        float top = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < kFewPieces; ++i) top = fmaxf(top, ml[i].x);
        const float off = top == -INFINITY ? 0.f : top;
        float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kFewPieces; ++i) {
          const float h = attn_half(ml[i].x - off), f = h * h;
          l += ml[i].y * h * h;
          acc.x += v[i].x * f; acc.y += v[i].y * f; acc.z += v[i].z * f; acc.w += v[i].w * f;
        }
        out(q, dim, acc, top, l);
      }
      continue;
    }
    // factors into shared memory (the rings are free), then the units, split over the pieces where threads are left
    __syncthreads();
    float* const fac = reinterpret_cast<float*>(smem);         // [np][kQ]
    float* const tops = fac + np * kQ;                         // [kQ] top, [kQ] l
    for (int q = warp; q < qn; q += kWarps) {
      float top = -INFINITY, l = 0.f;
      for (int i = lane; i < np; i += 32) top = fmaxf(top, __ldcg(&a.cta_ml[slot_of(i) * kQ + q]).x);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float off = top == -INFINITY ? 0.f : top;
      for (int i = lane; i < np; i += 32) {
        const float2 ml = __ldcg(&a.cta_ml[slot_of(i) * kQ + q]);
        const float h = attn_half(ml.x - off);
        fac[i * kQ + q] = h * h;
        l += ml.y * h * h;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
      if (lane == 0) { tops[q] = top; tops[kQ + q] = l; }
    }
    __syncthreads();
    int split = 1;                                             // threads that share a unit's pieces: a power of two, in one warp
    while (split < 32 && units * split * 2 <= kThreads && split < np) split *= 2;
    for (int u0 = 0; u0 < units; u0 += kThreads / split) {
      const int u = u0 + tid / split, part = tid % split, q = u / (DP / 4), dim = u % (DP / 4) * 4;
      float4 acc = make_float4(0, 0, 0, 0);
      if (u < units && dim < a.c.dim) {
#pragma unroll 4
        for (int i = part; i < np; i += split) {
          const float4 v = __ldcg(reinterpret_cast<const float4*>(a.cta_part + (slot_of(i) * kQ + q) * DP + dim));
          const float f = fac[i * kQ + q];
          acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
        }
      }
      for (int d = 1; d < split; d <<= 1) {
        acc.x += __shfl_xor_sync(0xffffffffu, acc.x, d); acc.y += __shfl_xor_sync(0xffffffffu, acc.y, d);
        acc.z += __shfl_xor_sync(0xffffffffu, acc.z, d); acc.w += __shfl_xor_sync(0xffffffffu, acc.w, d);
      }
      if (u < units && dim < a.c.dim && part == 0) out(q, dim, acc, tops[q], tops[kQ + q]);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
using AttnKernel = void (*)(AttnArgs);
struct AttnChoice { AttnKernel kernel; int smem, warps; };
template <int DP, int NT>
static AttnChoice attn_choice(bool i8) {
  return i8 ? AttnChoice{k_attn_decode<DP, NT, true>, AttnForm<DP, NT, true>::kSmem, AttnForm<DP, NT, true>::kWarps}
            : AttnChoice{k_attn_decode<DP, NT, false>, AttnForm<DP, NT, false>::kSmem, AttnForm<DP, NT, false>::kWarps};
}
static AttnChoice attn_choice(int dp, int nt, bool i8) {
  if (dp == 64) return nt == 1 ? attn_choice<64, 1>(i8) : attn_choice<64, 2>(i8);
  if (dp == 128) return nt == 1 ? attn_choice<128, 1>(i8) : attn_choice<128, 2>(i8);
  return attn_choice<256, 1>(i8);
}
struct AttnPlan { AttnChoice choice; int dp, nt, blocks; };
static AttnPlan attn_plan(const KvCache& c, int q_heads) {
  AttnPlan p{};
  p.dp = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
  const int group = q_heads / c.heads;
  p.nt = group > 8 && p.dp < 256 ? 2 : 1;         // head_dim above 128: the accumulators of two blocks do not fit
  p.blocks = (group + 8 * p.nt - 1) / (8 * p.nt);
  p.choice = attn_choice(p.dp, p.nt, c.format == PQ_KV_INT8);
  return p;
}
static size_t attn_carve(const AttnPlan& p, void* base, AttnArgs* a) {
  size_t off = 0;
  const size_t ctas = sm_count(), piece = (size_t)8 * p.nt * p.dp;
  auto take = [&](size_t bytes) { uint8_t* q = static_cast<uint8_t*>(base) + off; off += (bytes + 255) / 256 * 256; return q; };
  uint8_t* warp_part = take(ctas * p.choice.warps * piece * 4);
  uint8_t* cta_part = take(2 * ctas * piece * 4);
  uint8_t* ml = take(2 * ctas * 8 * p.nt * 8);
  uint8_t* arrived = take(ctas * 8);
  if (a) {
    a->warp_part = reinterpret_cast<float*>(warp_part); a->cta_part = reinterpret_cast<float*>(cta_part);
    a->cta_ml = reinterpret_cast<float2*>(ml); a->arrived = reinterpret_cast<unsigned long long*>(arrived);
  }
  return off;
}
size_t attn_workspace_bytes(const KvCache& c, int q_heads) { return attn_carve(attn_plan(c, q_heads), nullptr, nullptr); }

// Numbers of launches, so that a count left in a workspace by something else is not taken for one of this launch: from a start that the
// clock and this library's address spread over 48 bits.  A launch in a graph keeps its number; the last to arrive clears the count.
static unsigned long long attn_call_number() {
  static std::atomic<unsigned long long> next{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull ^
                                              reinterpret_cast<uintptr_t>(&attn_call_number)};
  unsigned long long v;
  do { v = next.fetch_add(1, std::memory_order_relaxed) << 16; } while (v == 0);
  return v;
}

// The opt-in limits, once per device
static cudaError_t attn_limits() {
  constexpr int kMaxDevices = 64;
  static std::once_flag done[kMaxDevices];
  static cudaError_t result[kMaxDevices] = {};
  int dev = 0;
  if (const cudaError_t e = cudaGetDevice(&dev)) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::call_once(done[dev], [&] {
    for (int dp = 64; dp <= 256; dp *= 2)
      for (int nt = 1; nt <= 2; ++nt)
        for (int i8 = 0; i8 < 2; ++i8) {
          if (result[dev] != cudaSuccess) return;
          const AttnChoice ch = attn_choice(dp, nt, i8);
          result[dev] = cudaFuncSetAttribute(ch.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmemMost);
        }
  });
  return result[dev];
}

cudaError_t launch_attn_decode(const KvCache& c, int q_heads, const uint16_t* Q, long long q_stride, const int* lens, float scale, uint16_t* O, float* lse,
                               void* ws, cudaStream_t st) {
  if (const cudaError_t e = attn_limits()) return e;
  const AttnPlan p = attn_plan(c, q_heads);
  AttnArgs a{};
  a.c = c; a.Q = Q; a.q_stride = q_stride; a.lens = lens; a.O = O; a.lse = lse;
  a.scale_log2 = scale * kLog2e;
  a.q_heads = q_heads; a.group = q_heads / c.heads; a.blocks = p.blocks;
  a.by_blocks = FastDiv(p.blocks);
  a.by_per_seq = FastDiv(c.heads * p.blocks);
  a.by_page_tiles = FastDiv(c.page_size / kAttnTile);
  a.by_chunks = FastDiv(c.pitch * (c.format == PQ_KV_INT8 ? 1 : 2) / 16);
  const size_t firsts = (size_t)p.choice.warps * std::min(a.group, 8 * p.nt) * p.dp * 4;
  a.first_in_smem = p.choice.smem + firsts <= (size_t)kAttnSmemMost;
  a.call = attn_call_number();
  attn_carve(p, ws, &a);
  LaunchScope ls(KID_ATTN_DECODE, st);
  return launch_pdl(p.choice.kernel, sm_count(), p.choice.warps * 32, p.choice.smem + (a.first_in_smem ? firsts : 0), st, a);
}

}  // namespace pq
