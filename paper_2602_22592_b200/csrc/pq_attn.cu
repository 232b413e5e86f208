// Attention of one new token per sequence over the paged key-value cache:
//     o = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale (q . k_j) - m),   m = max_j scale (q . k_j),   j < length of the sequence.
//
// A pass reads every cached row once and multiplies it with the group x head_dim query values that share its head: one to
// sixteen multiplications per byte, far below what the tensor cores need to be the limit, so that the memory is.  What
// follows from that:
//   * A warp works alone.  It walks tiles of sixteen positions; all loads of a tile are 16-byte asynchronous copies into a ring
//     that is private to each LANE (a lane copies exactly the pieces that it will multiply), so that nothing is shared, no barrier
//     is met and no bank conflicts: the ring (about 200 KB per SM) is the latency cover.
//   * The work is cut into equal shares of tiles per warp over ALL sequences and heads (lengths live on the device: every CTA
//     sums them itself), so that ragged batches, one long sequence and many short ones all keep every SM reading until the
//     end.  A (sequence, head) cut between warps leaves partial sums, which k_attn_join adds.
//   * S^T = K q^T on mma.sync.m16n8k16: positions are the sixteen rows, query heads the eight columns (two column blocks for
//     nine to sixteen).  tcgen05 has no shape for eight columns by sixteen rows that would not idle.  The contraction index may
//     be permuted at will as long as both operands agree: a lane's 16 bytes of a key row are eight neighbouring values, so that
//     cache rows stay in their natural order.  O^T = V^T P^T the same way: a lane holds four positions of the same dims, byte
//     permutes pair neighbouring positions.
//   * P enters the second product as the sum of two bf16 numbers (2^-17 relative): the tensor cores have room, and a single
//     rounding of P would be as large as the output's own.  int8 codes are exact in bf16; gamma_k scales the scores and
//     1 / gamma_v the weights, in fp32.
#include <algorithm>
#include <mutex>

#include "pq_kernels.cuh"

namespace pq {

constexpr int kAttnTile = 16;                 // positions of a tile; pages are multiples of it
constexpr int kAttnRingBytes = 200 * 1024;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

template <int DP, int NT, bool I8>
struct AttnForm {
  static constexpr int kWarps = DP == 256 ? 4 : 8;
  static constexpr int kK = I8 ? DP / 64 : DP / 32;                    // 16-byte pieces of a key row per lane (four lanes a row)
  static constexpr int kV = I8 ? (DP + 127) / 128 : DP / 64;           // pieces of a value row per lane (eight lanes a row)
  static constexpr int kVBytes = I8 && DP == 64 ? 8 : 16;              // ... and their size
  static constexpr int kSlots = 2 * kK + 4 * kV + (I8 ? 1 : 0);        // ring places of 16 bytes x 32 lanes of a stage
  static constexpr int kStageBytes = kSlots * 512;
  static constexpr int kFit = kAttnRingBytes / (kStageBytes * kWarps);
  static constexpr int kStages = kFit > 6 ? 6 : kFit;
  static constexpr int kSmem = kStages * kStageBytes * kWarps;
  static_assert(kStages >= 3, "two stages in flight and one in use");
};

__device__ __forceinline__ void attn_copy8(uint32_t dst, const void* src, bool valid) {      // zeros where not valid: nothing is read
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(valid ? 8 : 0) : "memory");
}
__device__ __forceinline__ void attn_copy4(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
__device__ __forceinline__ void attn_copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void attn_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 attn_lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Four int8 codes -> two pairs of bf16, exactly: behind an exponent byte 0x43 the low seven bits read 128 + low, the sign bit
// alone 128 or 256, and the difference is the code.
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t halves) {
  const uint32_t a = halves & 0xFF7FFF7Fu, b = halves & 0xFF80FF80u;
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return codes_to_bf16(__byte_perm(w, 0x43434343u, 0x4140)); }
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return codes_to_bf16(__byte_perm(w, 0x43434343u, 0x4342)); }

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
  // workspace
  float* part;               // [2 teams][8 NT][DP] unnormalised sums, ...
  float2* part_ml;           // [2 teams][8 NT] ... their maximum (in powers of two) and sum of weights
  int4* head;                // [min(teams, items)] what k_attn_join has to add: {first slot, pieces, item, -} or pieces = 0
  int teams;                 // warps of the launch
  int head_by_item;          // head's index is the item (else the team that holds its beginning)
};

__device__ __forceinline__ int attn_len(const AttnArgs& a, int seq) {
  return min(__ldcg(a.lens + seq), a.c.max_pages * a.c.page_size);       // longer: reported where the lengths are added up
}

// A walk over a team's share: its segments are stretches of tiles of one item = (sequence, cache head, column block).
struct AttnWalk {
  long long left;            // tiles of the share behind the current segment
  int seq, hb, t0, t1, len, tiles;
  __device__ bool next(const AttnArgs& a, int per_seq) {
    if (left <= 0) return false;
    if (++hb == per_seq) {
      hb = 0;
      do { len = attn_len(a, ++seq); } while (len <= 0);
      tiles = (len + kAttnTile - 1) / kAttnTile;
    }
    t0 = 0;
    t1 = (int)(left < tiles ? left : tiles);
    left -= t1;
    return true;
  }
};

template <int DP, int NT, bool I8>
__global__ void __launch_bounds__(AttnForm<DP, NT, I8>::kWarps * 32, 1) k_attn_decode(const __grid_constant__ AttnArgs a) {
  using F = AttnForm<DP, NT, I8>;
  constexpr int kThreads = F::kWarps * 32, kQ = 8 * NT;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long sums[kThreads + 1];      // tiles of the sequences before a thread's own
  __shared__ long long warp_sums[F::kWarps];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int per_seq = a.c.heads * a.blocks, n = a.c.num_seqs;
  // ---- shares: every CTA adds up the lengths
  const int per = (n + kThreads - 1) / kThreads;
  long long mine = 0;
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s >= n) break;
    const int raw = __ldcg(a.lens + s);
    if (raw > a.c.max_pages * a.c.page_size && blockIdx.x == 0) report_index();
    mine += (max(0, attn_len(a, s)) + kAttnTile - 1) / kAttnTile;
  }
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 31) warp_sums[warp] = upto;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < F::kWarps; ++w) {
    if (w < warp) before += warp_sums[w];
    total += warp_sums[w];
  }
  sums[tid] = before + upto - mine;
  __syncthreads();
  const long long tiles_all = total * per_seq;
  const int team = warp * gridDim.x + blockIdx.x;            // few teams with work: one per SM
  const long long used = tiles_all < a.teams ? tiles_all : a.teams;
  const long long r0 = team < used ? team * tiles_all / used : 0, r1 = team < used ? (team + 1) * tiles_all / used : 0;
  bool headed = false;                                        // head[team] written
  if (r0 < r1) {
    // ---- first segment: the sequence whose tiles hold r0
    const long long x = r0 / per_seq;                         // sums[.] <= x: compared per sequence, not per head
    int lo = 0, hi = kThreads;                                // last thread whose sequences begin at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (sums[mid] <= x) lo = mid; else hi = mid;
    }
    AttnWalk cw;
    long long base = sums[lo];
    cw.seq = lo * per;
    for (;; ++cw.seq) {
      cw.len = attn_len(a, cw.seq);
      cw.tiles = (max(0, cw.len) + kAttnTile - 1) / kAttnTile;
      if (x < base + cw.tiles) break;
      base += cw.tiles;
    }
    const long long in_seq = r0 - base * per_seq;
    cw.hb = (int)(in_seq / cw.tiles);
    cw.t0 = (int)(in_seq - (long long)cw.hb * cw.tiles);
    cw.t1 = (int)(cw.tiles - cw.t0 < r1 - r0 ? cw.tiles : cw.t0 + (r1 - r0));
    cw.left = r1 - r0 - (cw.t1 - cw.t0);
    AttnWalk pw = cw;                                         // the loads run ahead of the products, across segments
    int pt = cw.t0;
    bool more = true;
    const int tiles_per_page = a.c.page_size / kAttnTile;
    const uint32_t ring = smem_u32(smem) + warp * (F::kStages * F::kStageBytes) + lane * 16;
    const int row_bytes = a.c.pitch * (I8 ? 1 : 2);
    auto page_of = [&]() { return __ldcg(a.c.page_table + (long long)pw.seq * a.c.max_pages + pt / tiles_per_page); };
    int page = page_of();                                     // of tile pt, asked for a tile ahead
    auto issue = [&](int stage) {
      if (more) {
        const bool known = (unsigned)page < (unsigned)a.c.num_pages;
        if (!known && lane == 0) report_index();
        const int rows = known ? min(kAttnTile, pw.len - pt * kAttnTile) : 0;
        const int head = pw.hb / a.blocks;
        const long long row0 = known ? ((long long)page * a.c.heads + head) * a.c.page_size + (pt % tiles_per_page) * kAttnTile : 0;
        const uint8_t* kp = static_cast<const uint8_t*>(a.c.K) + row0 * row_bytes;
        const uint8_t* vp = static_cast<const uint8_t*>(a.c.V) + row0 * row_bytes;
        uint32_t dst = ring + stage * F::kStageBytes;
#pragma unroll
        for (int j = 0; j < F::kK; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = g + 8 * h, at = j * 64 + t * 16;
            const bool ok = row < rows && at < row_bytes;
            cp_async16(dst, kp + (ok ? row * row_bytes + at : 0), ok);
            dst += 512;
          }
#pragma unroll
        for (int j = 0; j < F::kV; ++j)
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int row = 2 * t + (h & 1) + (h >> 1) * 8, at = j * 8 * F::kVBytes + g * F::kVBytes;
            const bool ok = row < rows && at < row_bytes;
            if constexpr (F::kVBytes == 16) cp_async16(dst, vp + (ok ? row * row_bytes + at : 0), ok);
            else attn_copy8(dst, vp + (ok ? row * row_bytes + at : 0), ok);
            dst += 512;
          }
        if constexpr (I8) {
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int row = g + 8 * (h & 1);
            const bool ok = row < rows;
            attn_copy4(dst + 4 * h, (h < 2 ? a.c.k_gamma : a.c.v_gamma) + (ok ? row0 + row : 0), ok);
          }
        }
        if (++pt == pw.t1) {
          more = pw.next(a, per_seq);
          pt = pw.t0;
        }
        if (more) page = page_of();
      }
      attn_copy_commit();
    };
#pragma unroll
    for (int s = 0; s < F::kStages - 1; ++s) issue(s);
    int stage = 0, ahead = F::kStages - 1;

    do {
      // ---- one segment
      const int head = cw.hb / a.blocks, q0 = (cw.hb - head * a.blocks) * kQ, qn = min(kQ, a.group - q0);
      uint32_t qf[NT][DP / 16][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          const int dim = I8 ? (k / 4) * 64 + t * 16 + (k % 4) * 4 : (k / 2) * 32 + t * 8 + (k % 2) * 4, q = nt * 8 + g;
          uint2 v = make_uint2(0, 0);
          if (q < qn && dim < a.c.dim)
            v = __ldcg(reinterpret_cast<const uint2*>(a.Q + cw.seq * a.q_stride + (long long)(head * a.group + q0 + q) * a.c.dim + dim));
          qf[nt][k][0] = v.x;
          qf[nt][k][1] = v.y;
        }
      float o[NT][DP / 16][4] = {}, m[NT][2], l[NT][2] = {};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = -INFINITY;
      const int seg_len = cw.len;
      for (int tile = cw.t0; tile < cw.t1; ++tile) {
        attn_copy_wait<F::kStages - 2>();
        issue(ahead);                                          // into the place that this tile's predecessor has left
        const uint32_t src = ring + stage * F::kStageBytes;
        // scores: rows g, g + 8 of the tile, query columns 2 t, 2 t + 1
        float s[NT][4] = {}, s2[NT][4] = {};
#pragma unroll
        for (int j = 0; j < F::kK; ++j) {
          const uint4 ka = attn_lds128(src + (2 * j) * 512), kb = attn_lds128(src + (2 * j + 1) * 512);
          const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
          if constexpr (I8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a0 = codes_lo(wa[i]), a1 = codes_lo(wb[i]), a2 = codes_hi(wa[i]), a3 = codes_hi(wb[i]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_bf16(i & 1 ? s2[nt] : s[nt], a0, a1, a2, a3, qf[nt][4 * j + i][0], qf[nt][4 * j + i][1]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_bf16(i & 1 ? s2[nt] : s[nt], wa[2 * i], wb[2 * i], wa[2 * i + 1], wb[2 * i + 1], qf[nt][2 * j + i][0], qf[nt][2 * j + i][1]);
          }
        }
        float fk[2] = {a.scale_log2, a.scale_log2}, fv[2] = {1.f, 1.f};
        const int valid = seg_len - tile * kAttnTile;         // rows of the tile that the sequence holds
        if constexpr (I8) {
          const uint4 gm = attn_lds128(src + (F::kSlots - 1) * 512);
          fk[0] = __fdividef(a.scale_log2, __uint_as_float(gm.x)); fk[1] = __fdividef(a.scale_log2, __uint_as_float(gm.y));
          fv[0] = __fdividef(1.f, __uint_as_float(gm.z)); fv[1] = __fdividef(1.f, __uint_as_float(gm.w));
        }
        bool grew = false;
        float top[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[nt][i] = (s[nt][i] + s2[nt][i]) * fk[i >> 1];
            if (g + 8 * (i >> 1) >= valid) s[nt][i] = -INFINITY;
          }
#pragma unroll
          for (int cidx = 0; cidx < 2; ++cidx) {
            float v = fmaxf(s[nt][cidx], s[nt][cidx + 2]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
            top[nt][cidx] = fmaxf(v, m[nt][cidx]);
            grew |= top[nt][cidx] > m[nt][cidx];
          }
        }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int cidx = 0; cidx < 2; ++cidx) {
              const float f = top[nt][cidx] > m[nt][cidx] ? exp2f(m[nt][cidx] - top[nt][cidx]) : 1.f;
              m[nt][cidx] = top[nt][cidx];
              l[nt][cidx] *= f;
#pragma unroll
              for (int i = 0; i < DP / 16; ++i) { o[nt][i][cidx] *= f; o[nt][i][cidx + 2] *= f; }
            }
        }
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float mm = m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1];      // no weight so far: every score is -infinity
            p[i] = exp2f(s[nt][i] - mm);
            l[nt][i & 1] += p[i];
            if (I8) p[i] = g + 8 * (i >> 1) < valid ? p[i] * fv[i >> 1] : 0.f;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t hi = pack_bf16x2(p[2 * h], p[2 * h + 1]);
            const uint32_t low = pack_bf16x2(p[2 * h] - bf16lo(hi), p[2 * h + 1] - bf16hi(hi));
            ph[nt][h] = transpose8x8(hi);
            pl[nt][h] = transpose8x8(low);
          }
        }
#pragma unroll
        for (int j = 0; j < F::kV; ++j) {
          uint4 r[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) r[h] = attn_lds128(src + (2 * F::kK + 4 * j + h) * 512);
          const uint32_t w0[4] = {r[0].x, r[0].y, r[0].z, r[0].w}, w1[4] = {r[1].x, r[1].y, r[1].z, r[1].w};
          const uint32_t w2[4] = {r[2].x, r[2].y, r[2].z, r[2].w}, w3[4] = {r[3].x, r[3].y, r[3].z, r[3].w};
          auto product = [&](int mt, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma_bf16(o[nt][mt], a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
              mma_bf16(o[nt][mt], a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
            }
          };
          if constexpr (I8) {
#pragma unroll
            for (int i = 0; i < F::kVBytes / 4; ++i) {
              const uint32_t x01 = __byte_perm(w0[i], w1[i], 0x5140), x23 = __byte_perm(w2[i], w3[i], 0x5140);
              const uint32_t y01 = __byte_perm(w0[i], w1[i], 0x7362), y23 = __byte_perm(w2[i], w3[i], 0x7362);
              product(j * 8 + 2 * i, codes_lo(x01), codes_hi(x01), codes_lo(x23), codes_hi(x23));
              product(j * 8 + 2 * i + 1, codes_lo(y01), codes_hi(y01), codes_lo(y23), codes_hi(y23));
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              product(j * 4 + i, __byte_perm(w0[i], w1[i], 0x5410), __byte_perm(w0[i], w1[i], 0x7632), __byte_perm(w2[i], w3[i], 0x5410),
                      __byte_perm(w2[i], w3[i], 0x7632));
          }
        }
        stage = stage + 1 == F::kStages ? 0 : stage + 1;
        ahead = ahead + 1 == F::kStages ? 0 : ahead + 1;
      }
      // ---- the segment's sums
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int cidx = 0; cidx < 2; ++cidx)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[nt][cidx] += __shfl_xor_sync(0xffffffffu, l[nt][cidx], d);
      const bool whole = cw.t0 == 0 && cw.t1 == cw.tiles;
      const int slot = 2 * team + (cw.t0 == 0 ? 1 : 0);
      constexpr int kRun = 2 * F::kVBytes / (I8 ? 2 : 4);      // neighbouring dims of a lane in a piece: 8 (bf16, short int8 rows) or 16
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int cidx = 0; cidx < 2; ++cidx) {
          const int q = nt * 8 + 2 * t + cidx;
          if (q >= qn) continue;
          const float inv = l[nt][cidx] == 0.f ? 0.f : 1.f / l[nt][cidx];
          const long long qrow = (long long)cw.seq * a.q_heads + head * a.group + q0 + q;
#pragma unroll
          for (int j = 0; j < F::kV; ++j)
#pragma unroll
            for (int i = 0; i < kRun / 2; i += 2) {            // four neighbouring dims at a time: head_dim is a multiple of 4
              const int mt = j * (kRun / 2) + i, dim = j * 8 * kRun + g * kRun + 2 * i;
              if (dim >= a.c.dim) continue;
              const float v0 = o[nt][mt][cidx], v1 = o[nt][mt][cidx + 2], v2 = o[nt][mt + 1][cidx], v3 = o[nt][mt + 1][cidx + 2];
              if (whole) *reinterpret_cast<uint2*>(a.O + qrow * a.c.dim + dim) = make_uint2(pack_bf16x2(v0 * inv, v1 * inv), pack_bf16x2(v2 * inv, v3 * inv));
              else *reinterpret_cast<float4*>(a.part + ((long long)slot * kQ + q) * DP + dim) = make_float4(v0, v1, v2, v3);
            }
          if (g == 0) {
            if (!whole) a.part_ml[(long long)slot * kQ + q] = make_float2(m[nt][cidx], l[nt][cidx]);
            else if (a.lse) a.lse[qrow] = l[nt][cidx] == 0.f ? -INFINITY : (m[nt][cidx] + log2f(l[nt][cidx])) * kLn2;
          }
        }
      if (cw.t0 == 0 && lane == 0) {                           // the holder of an item's beginning says what there is to join
        const int item = cw.seq * per_seq + cw.hb;
        int pieces = 0;
        if (!whole) {
          const long long last = r1 - cw.left + (cw.tiles - cw.t1) - 1;     // the item's last tile; its team is the last t with t tiles_all / used <= it
          pieces = (int)(((last + 1) * used - 1) / tiles_all) - team + 1;
        }
        if (a.head_by_item || !whole) a.head[a.head_by_item ? item : team] = make_int4(slot, pieces, item, 0);
        headed |= !whole;
      }
    } while (cw.next(a, per_seq));
  }
  if (!a.head_by_item && lane == 0 && !headed) a.head[team] = make_int4(0, 0, 0, 0);
  // ---- sequences without a position: zeros, or, of negative length, left as they were
  for (int s = team; s < n; s += a.teams) {
    const int len = attn_len(a, s);
    if (len > 0) continue;
    if (len == 0) {
      for (int i = lane * 4; i < a.q_heads * a.c.dim; i += 128) *reinterpret_cast<uint2*>(a.O + (long long)s * a.q_heads * a.c.dim + i) = make_uint2(0, 0);
      if (a.lse) for (int i = lane; i < a.q_heads; i += 32) a.lse[(long long)s * a.q_heads + i] = -INFINITY;
    }
    if (a.head_by_item) for (int i = lane; i < per_seq; i += 32) a.head[s * per_seq + i] = make_int4(0, 0, 0, 0);
  }
}

// ---------------------------------------------------------------------------
// k_attn_join: the pieces of an item that several warps worked on, one block per (entry of head, query head), added in the order
// of their positions.  Slots of the pieces: the first one, then the even slots of the teams behind it.
// ---------------------------------------------------------------------------
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) k_attn_join(const __grid_constant__ AttnArgs a, int width, int cols, int entries) {
  constexpr int kWarps = kJoinThreads / 32;
  __shared__ float tops[kWarps], sums[kWarps], out[kWarps][256];
  pdl_launch_dependents();
  pdl_wait();
  const int q = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, per_seq = a.c.heads * a.blocks;
  for (int entry = blockIdx.x; entry < entries; entry += gridDim.x) {
    const int4 e = __ldcg(a.head + entry);
    const int pieces = e.y, item = e.z;
    if (pieces == 0) continue;
    const int seq = item / per_seq, hb = item - seq * per_seq, head = hb / a.blocks, q0 = (hb - head * a.blocks) * cols;
    if (q0 + q >= a.group) continue;
    auto slot = [&](int i) { return (long long)(i == 0 ? e.x : (e.x & ~1) + 2 * i) * cols + q; };
    // a warp takes every eighth piece, a lane four neighbouring dims and the four 128 behind them
    float m = -INFINITY;
    for (int i = tid; i < pieces; i += kJoinThreads) m = fmaxf(m, __ldcg(&a.part_ml[slot(i)]).x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) tops[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, tops[w]);
    if (m == -INFINITY) m = 0.f;                    // no weight anywhere
    float4 acc[2] = {make_float4(0, 0, 0, 0), make_float4(0, 0, 0, 0)};
    float l = 0.f;
    for (int i = warp; i < pieces; i += kWarps) {
      const float2 ml = __ldcg(&a.part_ml[slot(i)]);
      const float f = exp2f(ml.x - m);
      l += ml.y * f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int dim = lane * 4 + 128 * h;
        if (dim >= a.c.dim) continue;
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part + slot(i) * width + dim));
        acc[h].x += v.x * f; acc[h].y += v.y * f; acc[h].z += v.z * f; acc[h].w += v.w * f;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<float4*>(&out[warp][lane * 4 + 128 * h]) = acc[h];
    if (lane == 0) sums[warp] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) l += sums[w];
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long long qrow = (long long)seq * a.q_heads + head * a.group + q0 + q;
    if (tid < a.c.dim) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += out[w][tid];
      a.O[qrow * a.c.dim + tid] = (uint16_t)(pack_bf16x2(v * inv, 0.f) & 0xffffu);
    }
    if (tid == 0 && a.lse) a.lse[qrow] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct AttnPlan { int dp, nt, warps, teams, blocks; long long items, heads; };
static AttnPlan attn_plan(const KvCache& c, int q_heads) {
  AttnPlan p{};
  p.dp = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
  const int group = q_heads / c.heads;
  p.nt = group > 8 && p.dp < 256 ? 2 : 1;         // head_dim above 128: the accumulators of two blocks do not fit
  p.blocks = (group + 8 * p.nt - 1) / (8 * p.nt);
  p.warps = p.dp == 256 ? 4 : 8;
  p.teams = p.warps * sm_count();
  p.items = (long long)c.num_seqs * c.heads * p.blocks;
  p.heads = std::min<long long>(p.items, p.teams);
  return p;
}
static size_t attn_carve(const AttnPlan& p, void* base, AttnArgs* a) {
  size_t off = 0;
  auto take = [&](size_t bytes) { uint8_t* q = static_cast<uint8_t*>(base) + off; off += (bytes + 255) / 256 * 256; return q; };
  uint8_t* part = take((size_t)2 * p.teams * 8 * p.nt * p.dp * 4);
  uint8_t* ml = take((size_t)2 * p.teams * 8 * p.nt * 8);
  uint8_t* head = take((size_t)p.heads * 16);
  if (a) { a->part = reinterpret_cast<float*>(part); a->part_ml = reinterpret_cast<float2*>(ml); a->head = reinterpret_cast<int4*>(head); }
  return off;
}
size_t attn_workspace_bytes(const KvCache& c, int q_heads) { return attn_carve(attn_plan(c, q_heads), nullptr, nullptr); }

using AttnKernel = void (*)(AttnArgs);
struct AttnChoice { AttnKernel kernel; int smem; };
template <int DP, int NT>
static AttnChoice attn_choice(bool i8) {
  return i8 ? AttnChoice{k_attn_decode<DP, NT, true>, AttnForm<DP, NT, true>::kSmem} : AttnChoice{k_attn_decode<DP, NT, false>, AttnForm<DP, NT, false>::kSmem};
}
static AttnChoice attn_choice(int dp, int nt, bool i8) {
  if (dp == 64) return nt == 1 ? attn_choice<64, 1>(i8) : attn_choice<64, 2>(i8);
  if (dp == 128) return nt == 1 ? attn_choice<128, 1>(i8) : attn_choice<128, 2>(i8);
  return attn_choice<256, 1>(i8);
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
          result[dev] = cudaFuncSetAttribute(ch.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ch.smem);
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
  a.q_heads = q_heads; a.group = q_heads / c.heads; a.blocks = p.blocks; a.teams = p.teams;
  a.head_by_item = p.items <= p.teams;
  attn_carve(p, ws, &a);
  const AttnChoice ch = attn_choice(p.dp, p.nt, c.format == PQ_KV_INT8);
  {
    LaunchScope ls(KID_ATTN_DECODE, st);
    if (const cudaError_t e = launch_pdl(ch.kernel, p.teams / p.warps, p.warps * 32, ch.smem, st, a)) return e;
  }
  LaunchScope ls(KID_ATTN_JOIN, st);
  const int rows = std::min(a.group, 8 * p.nt);
  return launch_pdl(k_attn_join, dim3((unsigned)std::min<long long>(p.heads, std::max(1, 4 * sm_count() / rows)), (unsigned)rows), kJoinThreads, 0, st, a,
                    p.dp, 8 * p.nt, (int)p.heads);
}

}  // namespace pq
