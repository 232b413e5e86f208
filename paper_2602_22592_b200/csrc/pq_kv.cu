// Paged key-value cache: tokens are written (rotary embedding, bf16 or int8 as Eq. 7-9 quantise activations) and read back.
//
// Both kernels move rows of head_dim values and are bound by memory.  A row is small (200 to 512 bytes), so that a group of G lanes
// takes a row with accesses of up to 16 bytes and a warp 32 / G rows at once, kSteps times over: a unit, of one token.  Position,
// sequence, page id and row are four trips to memory one after another; warps walk the units with a stride and ask for the next
// unit's indices before they work on this one's rows.
#include <algorithm>

#include "pq_kernels.cuh"

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

// rounded to the nearest integer (ties to even), saturated to -128 .. 127
__device__ __forceinline__ int sat_s8(float x) {
  int v;
  asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(v) : "f"(x));
  return v;
}
// The loads of this file bypass L1: what an earlier kernel wrote must be seen by one that is resident already
template <int VEC>
__device__ __forceinline__ void store_bf16(uint16_t* p, const float (&v)[VEC]) {
  if constexpr (VEC == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  else if constexpr (VEC == 4)
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else
    *reinterpret_cast<uint32_t*>(p) = pack_bf16x2(v[0], v[1]);
}

constexpr int kSteps = 4;        // of a unit

// The raw bits of VEC bf16 values
template <int VEC> struct Raw;
template <> struct Raw<8> { uint4 v; };
template <> struct Raw<4> { uint2 v; };
template <> struct Raw<2> { uint32_t v; };
template <int VEC>
__device__ __forceinline__ void load_raw(const uint16_t* p, Raw<VEC>& r) { r.v = __ldcg(reinterpret_cast<const decltype(r.v)*>(p)); }
__device__ __forceinline__ void raw_floats(const Raw<8>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = bf16lo(w[i]); v[2 * i + 1] = bf16hi(w[i]); }
}
__device__ __forceinline__ void raw_floats(const Raw<2>& r, float (&v)[2]) { v[0] = bf16lo(r.v); v[1] = bf16hi(r.v); }

// A warp's walk over units = (token, rows of it).  Indices of the unit behind the current one are asked for early.
struct KvWalk {
  long long unit, stride, units;
  int per_token, tok, part, at, sq;      // of the next unit
  __device__ void begin(int tokens, int per_token_, const int* seq, const int* pos) {
    per_token = per_token_;
    units = (long long)tokens * per_token;
    unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    stride = (long long)gridDim.x * 8;
    ask(seq, pos);
  }
  __device__ void ask(const int* seq, const int* pos) {
    if (unit >= units) return;
    tok = units >> 31 ? (int)(unit / per_token) : (int)((uint32_t)unit / (uint32_t)per_token);
    part = (int)(unit - (long long)tok * per_token);
    at = __ldcg(pos + tok);
    sq = __ldcg(seq + tok);
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
template <int VEC, int G>
__global__ void __launch_bounds__(256, VEC == 8 ? 2 : 3) k_kv_append(KvCache c, int tokens, const int* seq, const int* pos, const uint16_t* K, long long k_stride,
                                                      const uint16_t* V, long long v_stride, const float* cos_t, const float* sin_t, int rope_rows,
                                                      const uint16_t* Q, long long q_stride, int q_heads, uint16_t* Q_out) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kMost = VEC == 8 ? 1 : 2;                              // pieces of VEC pairs per lane (G = 16: head_dim <= 128)
  constexpr int kRows = 32 / G;
  const int lane = threadIdx.x % G, sub = threadIdx.x % 32 / G, half = c.dim / 2, pieces = half / VEC;
  const int rows = q_heads + 2 * c.heads;
  const unsigned mask = G == 32 ? 0xffffffffu : ((1u << (G & 31)) - 1u) << (sub * G);
  KvWalk w;
  w.begin(tokens, (rows + kRows * kSteps - 1) / (kRows * kSteps), seq, pos);
  while (w.unit < w.units) {
    const int tok = w.tok, at = w.at, sq = w.sq, row0 = w.part * (kRows * kSteps) + sub;
    // the rows do not wait for the indices
    Raw<VEC> ra[kSteps][kMost], rb[kSteps][kMost];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int r = row0 + s * kRows;
      const uint16_t* src = r < q_heads ? Q + tok * q_stride + (long long)r * c.dim
                            : r < q_heads + c.heads ? K + tok * k_stride + (long long)(r - q_heads) * c.dim
                                                    : V + tok * v_stride + (long long)(r - q_heads - c.heads) * c.dim;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const int p = lane + i * G;
        if (r < rows && p < pieces) { load_raw<VEC>(src + p * VEC, ra[s][i]); load_raw<VEC>(src + half + p * VEC, rb[s][i]); }
      }
    }
    w.unit += w.stride;
    w.ask(seq, pos);
    if (at < 0) continue;                           // padding: nothing of this token is written
    const int2 place = kv_place(c, sq, at);
    if (place.x < 0 || (cos_t && at >= rope_rows)) {
      if (threadIdx.x % 32 == 0) report_index();
      continue;
    }
    float cs[kMost][VEC], sn[kMost][VEC];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int p = lane + i * G;
      if (!cos_t || p >= pieces) continue;
      const float* cr = cos_t + (long long)at * half + p * VEC;
      const float* sr = sin_t + (long long)at * half + p * VEC;
      // other warps turn other rows of the token by the same angles: through L1
      if constexpr (VEC == 8) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float4 x = __ldca(reinterpret_cast<const float4*>(cr) + k), y = __ldca(reinterpret_cast<const float4*>(sr) + k);
          cs[i][4 * k] = x.x; cs[i][4 * k + 1] = x.y; cs[i][4 * k + 2] = x.z; cs[i][4 * k + 3] = x.w;
          sn[i][4 * k] = y.x; sn[i][4 * k + 1] = y.y; sn[i][4 * k + 2] = y.z; sn[i][4 * k + 3] = y.w;
        }
      } else {
        const float2 x = __ldca(reinterpret_cast<const float2*>(cr)), y = __ldca(reinterpret_cast<const float2*>(sr));
        cs[i][0] = x.x; cs[i][1] = x.y; sn[i][0] = y.x; sn[i][1] = y.y;
      }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int r = row0 + s * kRows;
      if (r >= rows) break;
      const int kind = r < q_heads ? 0 : r < q_heads + c.heads ? 1 : 2;      // query, key, value
      float a[kMost][VEC], b[kMost][VEC];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (lane + i * G >= pieces) continue;
        raw_floats(ra[s][i], a[i]);
        raw_floats(rb[s][i], b[i]);
        if (cos_t && kind < 2) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float u = __fsub_rn(__fmul_rn(a[i][k], cs[i][k]), __fmul_rn(b[i][k], sn[i][k]));
            const float v = __fadd_rn(__fmul_rn(b[i][k], cs[i][k]), __fmul_rn(a[i][k], sn[i][k]));
            a[i][k] = u;
            b[i][k] = v;
          }
#pragma unroll
          for (int k = 0; k < VEC; k += 2) {
            const uint32_t x = pack_bf16x2(a[i][k], a[i][k + 1]), y = pack_bf16x2(b[i][k], b[i][k + 1]);
            a[i][k] = bf16lo(x); a[i][k + 1] = bf16hi(x);
            b[i][k] = bf16lo(y); b[i][k + 1] = bf16hi(y);
          }
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k)      // as integers: a NaN is above infinity is above the rest
          amax = max(amax, max(__float_as_uint(a[i][k]) & 0x7fffffffu, __float_as_uint(b[i][k]) & 0x7fffffffu));
      }
      const int head = kind == 0 ? r : kind == 1 ? r - q_heads : r - q_heads - c.heads;
      const long long crow = kv_row(c, place, head);
      if (kind == 0 || c.format == PQ_KV_BF16) {
        uint16_t* dst = kind == 0 ? Q_out + ((long long)tok * q_heads + head) * c.dim : static_cast<uint16_t*>(kind == 1 ? c.K : c.V) + crow * c.pitch;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          const int p = lane + i * G;
          if (p < pieces) { store_bf16<VEC>(dst + p * VEC, a[i]); store_bf16<VEC>(dst + half + p * VEC, b[i]); }
        }
        if (kind != 0)
          for (int i = c.dim + lane; i < c.pitch; i += G) dst[i] = 0;
        continue;
      }
#pragma unroll
      for (int d = G / 2; d > 0; d >>= 1) amax = max(amax, __shfl_xor_sync(mask, amax, d));
      const bool finite = amax < 0x7f800000u;
      const float gamma = finite ? __fdiv_rn(kActQmax, fmaxf(__uint_as_float(amax), kActAmaxFloor)) : __uint_as_float(0x7fffffffu);
      int8_t* dst = static_cast<int8_t*>(kind == 1 ? c.K : c.V) + crow * c.pitch;
      auto code = [&](float x) { return finite ? sat_s8(__fmul_rn(x, gamma)) & 0xff : 0; };
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const int p = lane + i * G;
        if (p >= pieces) continue;
        auto put = [&](int8_t* to, const float (&v)[VEC]) {
          if constexpr (VEC == 8) {
            uint2 x;
            x.x = code(v[0]) | code(v[1]) << 8 | code(v[2]) << 16 | code(v[3]) << 24;
            x.y = code(v[4]) | code(v[5]) << 8 | code(v[6]) << 16 | code(v[7]) << 24;
            *reinterpret_cast<uint2*>(to) = x;
          } else {
            *reinterpret_cast<uint16_t*>(to) = (uint16_t)(code(v[0]) | code(v[1]) << 8);
          }
        };
        put(dst + p * VEC, a[i]);
        put(dst + half + p * VEC, b[i]);
      }
      for (int i = c.dim + lane; i < c.pitch; i += G) dst[i] = 0;
      if (lane == 0) (kind == 1 ? c.k_gamma : c.v_gamma)[crow] = gamma;
    }
  }
}

// ---------------------------------------------------------------------------
// k_kv_read: rows of a token: key heads, value heads; bf16(code / gamma).  The quotient is the correctly rounded one
// from the reciprocal and one residual (Markstein: a correctly rounded reciprocal and one fused correction of the quotient
// give the rounded quotient): three instructions a value where a division takes about ten, which would be
// more than the memory asks for.
// ---------------------------------------------------------------------------
template <int VEC, int G>
__global__ void __launch_bounds__(256, 4) k_kv_read(KvCache c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kMost = VEC == 8 ? 1 : 2;                              // pieces per lane (G = 16: head_dim <= 128)
  constexpr int kRows = 32 / G;
  const int lane = threadIdx.x % G, sub = threadIdx.x % 32 / G, pieces = c.dim / VEC, rows = 2 * c.heads;
  KvWalk w;
  w.begin(tokens, (rows + kRows * kSteps - 1) / (kRows * kSteps), seq, pos);
  auto locate = [&](int& tok, int& row0, int& at) -> int2 {            // of the unit that the walk stands at; moves on
    tok = w.tok; at = w.at; row0 = w.part * (kRows * kSteps) + sub;
    const int2 p = at >= 0 ? kv_place(c, w.sq, at) : make_int2(-1, 0);
    w.unit += w.stride;
    w.ask(seq, pos);
    return p;
  };
  if (w.unit >= w.units) return;
  int tok, row0, at;
  int2 place = locate(tok, row0, at);
  for (bool more = true; more;) {
    int tok1 = 0, row1 = 0, at1 = -1;
    int2 place1 = make_int2(-1, 0);
    const bool bf = c.format == PQ_KV_BF16;
    Raw<VEC> raw[kSteps][kMost];                                       // bf16 rows; of int8 rows the first half of the bits
    float gamma[kSteps];
    if (place.x >= 0) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int r = row0 + s * kRows;
        if (r >= rows) break;
        const bool key = r < c.heads;
        const long long crow = kv_row(c, place, key ? r : r - c.heads);
        const uint8_t* src = static_cast<const uint8_t*>(key ? c.K : c.V) + crow * c.pitch * (bf ? 2 : 1);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          const int p = lane + i * G;
          if (p >= pieces) continue;
          if (bf) load_raw<VEC>(reinterpret_cast<const uint16_t*>(src) + p * VEC, raw[s][i]);
          else if constexpr (VEC == 8) { const uint2 u = __ldcg(reinterpret_cast<const uint2*>(src) + p); raw[s][i].v = make_uint4(u.x, u.y, 0, 0); }
          else raw[s][i].v.x = __ldcg(reinterpret_cast<const uint32_t*>(src) + p);
        }
        if (!bf) gamma[s] = __ldcg((key ? c.k_gamma : c.v_gamma) + crow);
      }
    } else if (at >= 0 && threadIdx.x % 32 == 0) {
      report_index();
    }
    more = w.unit < w.units;
    if (more) place1 = locate(tok1, row1, at1);                        // its page id is on the way while this unit's rows are
    if (place.x >= 0) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int r = row0 + s * kRows;
        if (r >= rows) break;
        const bool key = r < c.heads;
        uint16_t* dst = (key ? K_out : V_out) + ((long long)tok * c.heads + (key ? r : r - c.heads)) * c.dim;
        const float inv = bf ? 0.f : __frcp_rn(gamma[s]);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          const int p = lane + i * G;
          if (p >= pieces) continue;
          if (bf) {
            *reinterpret_cast<decltype(raw[s][i].v)*>(dst + p * VEC) = raw[s][i].v;
          } else {
            float v[VEC];
            const uint32_t word[2] = {raw[s][i].v.x, raw[s][i].v.y};
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
              const float x = (float)(int8_t)(word[k / 4] >> (8 * (k % 4)) & 0xff), q = __fmul_rn(x, inv);
              v[k] = __fmaf_rn(__fmaf_rn(-q, gamma[s], x), inv, q);
            }
            store_bf16<VEC>(dst + p * VEC, v);
          }
        }
      }
    }
    place = place1; tok = tok1; row0 = row1; at = at1;
  }
}

// Lanes of a row: the pieces rounded up to a power of two
static int group_of(int pieces) {
  int g = 2;
  while (g < pieces && g < 32) g *= 2;
  return g;
}
// Units of kSteps x (32 / g) rows, eight warps a block, as many blocks as can be resident
static int blocks_for(int tokens, int rows, int g, int resident) {
  const int per_token = (rows + 32 / g * kSteps - 1) / (32 / g * kSteps);
  return (int)std::min<long long>(((long long)tokens * per_token + 7) / 8, (long long)sm_count() * resident);
}

cudaError_t launch_kv_append(const KvCache& c, int tokens, const int* seq, const int* pos, const uint16_t* K, long long k_stride,
                             const uint16_t* V, long long v_stride, const float* cos_t, const float* sin_t, int rope_rows, const uint16_t* Q,
                             long long q_stride, int q_heads, uint16_t* Q_out, cudaStream_t st) {
  const bool wide = c.dim % 16 == 0 && k_stride % 8 == 0 && v_stride % 8 == 0 && (!Q || q_stride % 8 == 0);
  const int g = wide ? group_of(c.dim / 16) : c.dim <= 128 ? 16 : 32;
  auto kern = !wide ? (g == 16 ? k_kv_append<2, 16> : k_kv_append<2, 32>) : g == 2 ? k_kv_append<8, 2> : g == 4 ? k_kv_append<8, 4> : g == 8 ? k_kv_append<8, 8> : k_kv_append<8, 16>;
  LaunchScope ls(KID_KV_APPEND, st);
  return launch_pdl(kern, blocks_for(tokens, q_heads + 2 * c.heads, g, wide ? 2 : 3), 256, 0, st, c, tokens, seq, pos, K, k_stride, V, v_stride,
                    cos_t, sin_t, rope_rows, Q, q_stride, q_heads, Q_out);
}

cudaError_t launch_kv_read(const KvCache& c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out, cudaStream_t st) {
  const bool wide = c.dim % 8 == 0;
  const int g = wide ? group_of(c.dim / 8) : c.dim <= 128 ? 16 : 32;
  auto kern = !wide ? (g == 16 ? k_kv_read<4, 16> : k_kv_read<4, 32>)
              : g == 2 ? k_kv_read<8, 2> : g == 4 ? k_kv_read<8, 4> : g == 8 ? k_kv_read<8, 8> : g == 16 ? k_kv_read<8, 16> : k_kv_read<8, 32>;
  LaunchScope ls(KID_KV_READ, st);
  return launch_pdl(kern, blocks_for(tokens, 2 * c.heads, g, 4), 256, 0, st, c, tokens, seq, pos, K_out, V_out);
}

}  // namespace pq
