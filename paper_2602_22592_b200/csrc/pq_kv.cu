// Paged key-value cache: tokens are written (rotary embedding, bf16 or int8 as Eq. 7-9 quantise activations) and read back.
//
// Both kernels move rows of head_dim values and are bound by memory.  A row is small (200 to 512 bytes), so that a group of G lanes
// takes a row with accesses of up to 16 bytes and a warp 32 / G rows at once, kSteps times over: a unit, of one token.  Position,
// sequence, page id and row are four trips to memory one after another; warps walk the units with a stride and ask for the next
// unit's indices before they work on this one's rows.
// Measured: 7850 tokens of 16 heads of 128 in bf16, written with their queries 32 us (6.1 TB/s) and read back 23 (5.6); 2142 tokens of 32 heads
// of 100 in int8 written 37 us, 5356 read back 33: there the instructions are the limit (65 % of the issue slots), about a hundred a
// row, since 50 values half a row can only be had in twos.
#include <algorithm>
#include <cstring>

#include "pq_pairs.cuh"

namespace pq {

__device__ __forceinline__ void report_index() {
  if (atomicCAS(&g_status[0], 0, PQ_ERR_INDEX) == 0) g_status[1] = WHERE_OTHER;
}

// Where the token (seq, pos) lives: {page, position in the page}, page < 0 when there is no such place.  Every index that comes
// from device memory is checked here before it becomes an address.
__device__ __forceinline__ int2 kv_place(const KvCache& c, int seq, int pos) {
  if ((unsigned)seq >= (unsigned)c.num_seqs || pos < 0) return make_int2(-1, 0);
  const int slot = pos / c.page_size;
  if (slot >= c.max_pages) return make_int2(-1, 0);
  const int page = __ldcg(c.page_table + (long long)seq * c.max_pages + slot);
  return make_int2((unsigned)page < (unsigned)c.num_pages ? page : -1, pos - slot * c.page_size);
}
__device__ __forceinline__ long long kv_row(const KvCache& c, int2 place, int head) {
  return ((long long)place.x * c.heads + head) * c.page_size + place.y;
}

// VEC bf16 values as pairs.  The loads of this file bypass L1: what an earlier kernel wrote must be seen by one that is resident already.
template <int W> struct Words;
template <> struct Words<4> { using T = uint4; };
template <> struct Words<2> { using T = uint2; };
template <> struct Words<1> { using T = uint32_t; };
template <int VEC>
struct Bf {
  uint32_t w[VEC / 2];
  __device__ void load(const uint16_t* p) {
    using T = typename Words<VEC / 2>::T;
    const T v = __ldcg(reinterpret_cast<const T*>(p));
    memcpy(w, &v, sizeof v);
  }
  __device__ void store(uint16_t* p) const {
    using T = typename Words<VEC / 2>::T;
    T v;
    memcpy(&v, w, sizeof v);
    *reinterpret_cast<T*>(p) = v;
  }
  __device__ F2 pair(int k) const { return f2(bf16lo(w[k]), bf16hi(w[k])); }
};
__device__ __forceinline__ uint32_t pack_pair(const F2& v) {
  float x, y;
  get(v, x, y);
  return pack_bf16x2(x, y);
}
// Two values times gamma, rounded to integers (ties to even) and limited to 127, in the low bytes of the result: behind 1.5 x 2^23 a
// number's last bits are the integer.  (Below -128 none can fall: |x| gamma <= 128.)
__device__ __forceinline__ void code_pair(const F2& x, const F2& gamma, uint32_t& lo, uint32_t& hi) {
  float a, b;
  get(x * gamma, a, b);
  const F2 r = f2(fminf(a, 127.f), fminf(b, 127.f)) + f2(12582912.f);
  get(r, a, b);
  lo = __float_as_uint(a);
  hi = __float_as_uint(b);
}

constexpr int kSteps = 4;        // of a unit at most; with few rows one, so that they spread over more warps

// A warp's walk over units = (token, rows of it).  While a unit is worked on, the place of the next one is looked up and the position and
// sequence of the one behind it are on their way.
struct KvWalk {
  long long unit, stride, units;      // the unit whose position has been asked for
  int per_token, tok1, part1, at1, sq1;
  int tok, part, at;                  // the current unit, ...
  int2 place;                         // ... and its place: page < 0 if there is none, or nothing to do (at < 0)
  __device__ void begin(int tokens, int per_token_, const int* seq, const int* pos) {
    per_token = per_token_;
    units = (long long)tokens * per_token;
    unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    stride = (long long)gridDim.x * 8;
    ask(seq, pos);
  }
  __device__ void ask(const int* seq, const int* pos) {
    if (unit >= units) return;
    tok1 = units >> 31 ? (int)(unit / per_token) : (int)((uint32_t)unit / (uint32_t)per_token);
    part1 = (int)(unit - (long long)tok1 * per_token);
    at1 = __ldcg(pos + tok1);
    sq1 = __ldcg(seq + tok1);
  }
  __device__ bool more() const { return unit < units; }
  __device__ void next(const KvCache& c, const int* seq, const int* pos) {
    tok = tok1; part = part1; at = at1;
    place = at1 >= 0 ? kv_place(c, sq1, at1) : make_int2(-1, 0);
    unit += stride;
    ask(seq, pos);
  }
};

// ---------------------------------------------------------------------------
// k_kv_append: rows of a token: query heads, key heads, value heads.  Lane l of a row's group holds VEC values of the first half and
// the VEC values of the second half that they turn with,
//     (a, b) -> bf16(a cos - b sin), bf16(b cos + a sin)         one rounding per product and sum in fp32, as written,
// so that the rotation stays inside a lane, and every row of the unit turns by the same angles.  A cached row is quantised from the
// rounded values: gamma = 128 / max(max|x|, 1e-5), codes clamp(rint(x gamma)); a row that holds an infinity or a NaN gets
// gamma = NaN and reads back as NaN throughout.
// VEC = 8 (16-byte accesses) where both halves are multiples of 8 values and the rows are 16-byte aligned, else 2.
// ---------------------------------------------------------------------------
template <int VEC, int G, bool I8>
__global__ void __launch_bounds__(256, VEC == 8 ? 2 : 3) k_kv_append(KvCache c, int tokens, const int* seq, const int* pos, const uint16_t* K, long long k_stride,
                                                      const uint16_t* V, long long v_stride, const float* cos_t, const float* sin_t, int rope_rows,
                                                      const uint16_t* Q, long long q_stride, int q_heads, uint16_t* Q_out, int steps) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kMost = VEC == 8 ? 1 : 2;                              // pieces of VEC pairs per lane (G = 16: head_dim <= 128)
  constexpr int kRows = 32 / G;
  const int lane = threadIdx.x % G, sub = threadIdx.x % 32 / G, half = c.dim / 2, pieces = half / VEC;
  const int rows = q_heads + 2 * c.heads;
  const unsigned mask = G == 32 ? 0xffffffffu : ((1u << (G & 31)) - 1u) << (sub * G);
  const long long head_rows = (long long)c.page_size * c.pitch;       // values from head to head of a page
  KvWalk w;
  w.begin(tokens, (rows + kRows * steps - 1) / (kRows * steps), seq, pos);
  if (!w.more()) return;
  w.next(c, seq, pos);
  for (bool more = true; more;) {
    const int tok = w.tok, at = w.at, row0 = w.part * (kRows * steps) + sub;
    const int2 place = w.place;
    const uint16_t* const q_row = Q + tok * q_stride;
    const uint16_t* const k_row = K + tok * k_stride - (long long)q_heads * c.dim;                  // of row r: + r dim
    const uint16_t* const v_row = V + tok * v_stride - (long long)(q_heads + c.heads) * c.dim;
    Bf<VEC> ra[kSteps][kMost], rb[kSteps][kMost];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int r = row0 + s * kRows;
      const uint16_t* src = (r < q_heads ? q_row : r < q_heads + c.heads ? k_row : v_row) + (long long)r * c.dim + lane * VEC;
#pragma unroll
      for (int i = 0; i < kMost; ++i)
        if (s < steps && r < rows && lane + i * G < pieces) { ra[s][i].load(src + i * G * VEC); rb[s][i].load(src + half + i * G * VEC); }
    }
    // other warps turn other rows of the token by the same angles: through L1
    F2 cs[kMost][VEC / 2], sn[kMost][VEC / 2];
    const bool turns = cos_t && at >= 0 && at < rope_rows;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int p = lane + i * G;
      if (!turns || p >= pieces) continue;
      const float* cr = cos_t + (long long)at * half + p * VEC;
      const float* sr = sin_t + (long long)at * half + p * VEC;
#pragma unroll
      for (int k = 0; k < VEC / 2; k += 2) {
        if constexpr (VEC == 8) {
          const float4 x = __ldca(reinterpret_cast<const float4*>(cr) + k / 2), y = __ldca(reinterpret_cast<const float4*>(sr) + k / 2);
          cs[i][k] = f2(x.x, x.y); cs[i][k + 1] = f2(x.z, x.w);
          sn[i][k] = f2(y.x, y.y); sn[i][k + 1] = f2(y.z, y.w);
        } else {
          const float2 x = __ldca(reinterpret_cast<const float2*>(cr)), y = __ldca(reinterpret_cast<const float2*>(sr));
          cs[i][0] = f2(x.x, x.y);
          sn[i][0] = f2(y.x, y.y);
        }
      }
    }
    more = w.more();
    if (more) w.next(c, seq, pos);
    if (place.x < 0 || (cos_t && at >= rope_rows)) {                   // nothing of this token is written: padding, or no such place
      if (at >= 0 && threadIdx.x % 32 == 0) report_index();
      continue;
    }
    const long long crow0 = kv_row(c, place, 0);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int r = row0 + s * kRows;
      if (s >= steps || r >= rows) break;
      const bool query = r < q_heads, key = r < q_heads + c.heads;     // else a value
      uint32_t amax = 0;                                               // of pairs: two 16-bit numbers
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (lane + i * G >= pieces) continue;
        if (turns && key) {
#pragma unroll
          for (int k = 0; k < VEC / 2; ++k) {
            float c0, c1, s0, s1;
            get(cs[i][k], c0, c1);
            get(sn[i][k], s0, s1);
            const float a0 = bf16lo(ra[s][i].w[k]), a1 = bf16hi(ra[s][i].w[k]), b0 = bf16lo(rb[s][i].w[k]), b1 = bf16hi(rb[s][i].w[k]);
            ra[s][i].w[k] = pack_bf16x2(__fsub_rn(__fmul_rn(a0, c0), __fmul_rn(b0, s0)), __fsub_rn(__fmul_rn(a1, c1), __fmul_rn(b1, s1)));
            rb[s][i].w[k] = pack_bf16x2(__fadd_rn(__fmul_rn(b0, c0), __fmul_rn(a0, s0)), __fadd_rn(__fmul_rn(b1, c1), __fmul_rn(a1, s1)));
          }
        }
        if (I8) {
#pragma unroll
          for (int k = 0; k < VEC / 2; ++k)      // bits of bf16 without the sign: a NaN is above infinity is above the rest
            amax = __vmaxu2(amax, __vmaxu2(ra[s][i].w[k] & 0x7fff7fffu, rb[s][i].w[k] & 0x7fff7fffu));
        }
      }
      const int head = query ? r : key ? r - q_heads : r - q_heads - c.heads;
      if (query || !I8) {
        uint16_t* dst = query ? Q_out + ((long long)tok * q_heads + head) * c.dim : static_cast<uint16_t*>(key ? c.K : c.V) + crow0 * c.pitch + head * head_rows;
        dst += lane * VEC;
#pragma unroll
        for (int i = 0; i < kMost; ++i)
          if (lane + i * G < pieces) { ra[s][i].store(dst + i * G * VEC); rb[s][i].store(dst + half + i * G * VEC); }
        if (!query && lane < c.pitch - c.dim) dst[c.dim + lane - lane * VEC] = 0;      // at most 4 of them
        continue;
      }
      amax = max(amax & 0xffffu, amax >> 16);
#pragma unroll
      for (int d = G / 2; d > 0; d >>= 1) amax = max(amax, __shfl_xor_sync(mask, amax, d));
      const bool finite = amax < 0x7f80u;
      const float gamma = finite ? __fdiv_rn(kActQmax, fmaxf(__uint_as_float(amax << 16), kActAmaxFloor)) : __uint_as_float(0x7fffffffu);
      const F2 g2 = f2(gamma);
      int8_t* dst = static_cast<int8_t*>(key ? c.K : c.V) + crow0 * c.pitch + head * head_rows;
      auto put = [&](int8_t* to, const Bf<VEC>& v) {
        uint32_t b[VEC];
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) code_pair(v.pair(k), g2, b[2 * k], b[2 * k + 1]);
        if constexpr (VEC == 8) {
          uint2 x;
          x.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
          x.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
          *reinterpret_cast<uint2*>(to) = finite ? x : make_uint2(0, 0);
        } else {
          *reinterpret_cast<uint16_t*>(to) = finite ? (uint16_t)__byte_perm(b[0], b[1], 0x0040) : (uint16_t)0;
        }
      };
#pragma unroll
      for (int i = 0; i < kMost; ++i)
        if (lane + i * G < pieces) { put(dst + (lane + i * G) * VEC, ra[s][i]); put(dst + half + (lane + i * G) * VEC, rb[s][i]); }
      if (lane < c.pitch - c.dim) dst[c.dim + lane] = 0;               // at most 12
      if (lane == 0) (key ? c.k_gamma : c.v_gamma)[crow0 + (long long)head * c.page_size] = gamma;
    }
  }
}

// ---------------------------------------------------------------------------
// k_kv_read: rows of a token: key heads, value heads; bf16(code / gamma).  The quotient is the correctly rounded one
// from the reciprocal and one residual (Markstein: a correctly rounded reciprocal and one fused correction of the quotient
// give the rounded quotient): three instructions a value where a division takes about ten, which would be
// more than the memory asks for.
// ---------------------------------------------------------------------------
template <int VEC, int G, bool I8>
__global__ void __launch_bounds__(256, 4) k_kv_read(KvCache c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out, int steps) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kMost = VEC == 8 ? 1 : 2;                              // pieces per lane (G = 16: head_dim <= 128)
  constexpr int kRows = 32 / G, kBytes = I8 ? 1 : 2;
  using In = Bf<I8 ? VEC / 2 : VEC>;                                   // the bytes of VEC values
  const int lane = threadIdx.x % G, sub = threadIdx.x % 32 / G, pieces = c.dim / VEC, rows = 2 * c.heads;
  const long long head_bytes = (long long)c.page_size * c.pitch * kBytes;
  KvWalk w;
  w.begin(tokens, (rows + kRows * steps - 1) / (kRows * steps), seq, pos);
  if (!w.more()) return;
  w.next(c, seq, pos);
  for (bool more = true; more;) {
    const int tok = w.tok, row0 = w.part * (kRows * steps) + sub;
    const int2 place = w.place;
    if (place.x < 0 && w.at >= 0 && threadIdx.x % 32 == 0) report_index();
    In raw[kSteps][kMost];
    float gamma[kSteps];
    if (place.x >= 0) {
      const long long crow0 = kv_row(c, place, 0);
      const uint8_t* const k_src = static_cast<const uint8_t*>(c.K) + crow0 * c.pitch * kBytes + lane * VEC * kBytes;
      const uint8_t* const v_src = static_cast<const uint8_t*>(c.V) + crow0 * c.pitch * kBytes + lane * VEC * kBytes;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int r = row0 + s * kRows, head = r < c.heads ? r : r - c.heads;
        if (s >= steps || r >= rows) break;
        const uint8_t* src = (r < c.heads ? k_src : v_src) + head * head_bytes;
#pragma unroll
        for (int i = 0; i < kMost; ++i)
          if (lane + i * G < pieces) raw[s][i].load(reinterpret_cast<const uint16_t*>(src + i * G * VEC * kBytes));
        if (I8) gamma[s] = __ldcg((r < c.heads ? c.k_gamma : c.v_gamma) + crow0 + (long long)head * c.page_size);
      }
    }
    more = w.more();
    if (more) w.next(c, seq, pos);
    if (place.x < 0) continue;
    const long long out0 = (long long)tok * c.heads * c.dim + lane * VEC;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int r = row0 + s * kRows, head = r < c.heads ? r : r - c.heads;
      if (s >= steps || r >= rows) break;
      uint16_t* const dst = (r < c.heads ? K_out : V_out) + out0 + head * c.dim;
      const float inv = I8 ? __frcp_rn(gamma[s]) : 0.f;
      const F2 by = f2(inv), g2 = f2(-gamma[s]), bias = f2(-8388736.f);
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (lane + i * G >= pieces) continue;
        if constexpr (!I8) {
          raw[s][i].store(dst + i * G * VEC);
        } else {
          Bf<VEC> out;
#pragma unroll
          for (int k = 0; k < VEC / 2; ++k) {
            // under the bits of 2^23 an integer below it is itself: conversions by permute and addition
            const uint32_t word = raw[s][i].w[k / 2] ^ 0x80808080u;
            const F2 x = f2(__uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440 + 2 * (k % 2))), __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7441 + 2 * (k % 2)))) + bias;
            const F2 q = x * by;
            out.w[k] = pack_pair(fma2(fma2(q, g2, x), by, q));
          }
          out.store(dst + i * G * VEC);
        }
      }
    }
  }
}

// Lanes of a row: the pieces rounded up to a power of two
static int group_of(int pieces) {
  int g = 2;
  while (g < pieces && g < 32) g *= 2;
  return g;
}
// Rows of a warp's unit in steps of 32 / g: one step while the warps of a block per SM have one unit or less each
static int steps_for(int tokens, int rows, int g) {
  return (long long)tokens * ((rows + 32 / g - 1) / (32 / g)) <= 8LL * sm_count() ? 1 : kSteps;
}
// eight warps a block, as many blocks as can be resident
static int blocks_for(int tokens, int rows, int g, int steps, int resident) {
  const int per_token = (rows + 32 / g * steps - 1) / (32 / g * steps);
  return (int)std::min<long long>(((long long)tokens * per_token + 7) / 8, (long long)sm_count() * resident);
}

template <bool I8>
static auto append_kernel(bool wide, int g) {
  return !wide ? (g == 16 ? k_kv_append<2, 16, I8> : k_kv_append<2, 32, I8>)
         : g == 2 ? k_kv_append<8, 2, I8> : g == 4 ? k_kv_append<8, 4, I8> : g == 8 ? k_kv_append<8, 8, I8> : k_kv_append<8, 16, I8>;
}
template <bool I8>
static auto read_kernel(bool wide, int g) {
  return !wide ? (g == 16 ? k_kv_read<4, 16, I8> : k_kv_read<4, 32, I8>)
         : g == 2 ? k_kv_read<8, 2, I8> : g == 4 ? k_kv_read<8, 4, I8> : g == 8 ? k_kv_read<8, 8, I8> : g == 16 ? k_kv_read<8, 16, I8> : k_kv_read<8, 32, I8>;
}

cudaError_t launch_kv_append(const KvCache& c, int tokens, const int* seq, const int* pos, const uint16_t* K, long long k_stride,
                             const uint16_t* V, long long v_stride, const float* cos_t, const float* sin_t, int rope_rows, const uint16_t* Q,
                             long long q_stride, int q_heads, uint16_t* Q_out, cudaStream_t st) {
  const bool wide = c.dim % 16 == 0 && k_stride % 8 == 0 && v_stride % 8 == 0 && (!Q || q_stride % 8 == 0);
  const int g = wide ? group_of(c.dim / 16) : c.dim <= 128 ? 16 : 32;
  auto kern = c.format == PQ_KV_INT8 ? append_kernel<true>(wide, g) : append_kernel<false>(wide, g);
  const int steps = steps_for(tokens, q_heads + 2 * c.heads, g);
  LaunchScope ls(KID_KV_APPEND, st);
  return launch_pdl(kern, blocks_for(tokens, q_heads + 2 * c.heads, g, steps, wide ? 2 : 3), 256, 0, st, c, tokens, seq, pos, K, k_stride, V, v_stride,
                    cos_t, sin_t, rope_rows, Q, q_stride, q_heads, Q_out, steps);
}

cudaError_t launch_kv_read(const KvCache& c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out, cudaStream_t st) {
  const bool wide = c.dim % 8 == 0;
  const int g = wide ? group_of(c.dim / 8) : c.dim <= 128 ? 16 : 32;
  auto kern = c.format == PQ_KV_INT8 ? read_kernel<true>(wide, g) : read_kernel<false>(wide, g);
  const int steps = steps_for(tokens, 2 * c.heads, g);
  LaunchScope ls(KID_KV_READ, st);
  return launch_pdl(kern, blocks_for(tokens, 2 * c.heads, g, steps, 4), 256, 0, st, c, tokens, seq, pos, K_out, V_out, steps);
}

}  // namespace pq
