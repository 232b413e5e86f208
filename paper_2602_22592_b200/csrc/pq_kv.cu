// Paged key-value cache: tokens are written (rotary embedding, bf16 or int8 as Eq. 7-9 quantise activations) and read back.
//
// Both kernels move rows of head_dim values, one row per group of lanes, and are bound by memory.  A row is small (200 to 512
// bytes), so that groups are as narrow as 16-byte accesses allow and a block holds many of them.
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

// VEC values as 32-bit floats; the loads bypass L1: what an earlier kernel wrote must be seen by one that is resident already
template <int VEC>
__device__ __forceinline__ void load_bf16(const uint16_t* p, float (&v)[VEC]) {
  if constexpr (VEC == 8) {
    const uint4 u = __ldcg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16lo(w[i]); v[2 * i + 1] = bf16hi(w[i]); }
  } else if constexpr (VEC == 4) {
    const uint2 u = __ldcg(reinterpret_cast<const uint2*>(p));
    v[0] = bf16lo(u.x); v[1] = bf16hi(u.x); v[2] = bf16lo(u.y); v[3] = bf16hi(u.y);
  } else {
    const uint32_t u = __ldcg(reinterpret_cast<const uint32_t*>(p));
    v[0] = bf16lo(u); v[1] = bf16hi(u);
  }
}
template <int VEC>
__device__ __forceinline__ void store_bf16(uint16_t* p, const float (&v)[VEC]) {
  if constexpr (VEC == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  else if constexpr (VEC == 4)
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else
    *reinterpret_cast<uint32_t*>(p) = pack_bf16x2(v[0], v[1]);
}

// ---------------------------------------------------------------------------
// k_kv_append: rows in the order token, then query heads, key heads, value heads.  A group of G lanes owns a row; lane l holds
// VEC values of the first half and the VEC values of the second half that they turn with,
//     (a, b) -> bf16(a cos - b sin), bf16(b cos + a sin)         one rounding per product and sum in fp32, as written,
// so that the rotation stays inside a lane and 8192 tokens of 16 heads read every byte once.  A cached row is quantised from the
// rounded values: gamma = 128 / max(max|x|, 1e-5), codes clamp(rint(x gamma)); a row that holds an infinity or a NaN gets
// gamma = NaN and reads back as NaN throughout.
// VEC = 8 (16-byte accesses) where both halves are multiples of 8 values and the rows are 16-byte aligned, else 2.
// ---------------------------------------------------------------------------
template <int VEC, int G>
__global__ void __launch_bounds__(256) k_kv_append(KvCache c, int tokens, const int* seq, const int* pos, const uint16_t* K, long long k_stride,
                                                   const uint16_t* V, long long v_stride, const float* cos_t, const float* sin_t, int rope_rows,
                                                   const uint16_t* Q, long long q_stride, int q_heads, uint16_t* Q_out) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kMost = VEC == 8 ? 1 : 2;          // pieces of VEC pairs per lane: head_dim <= 256
  const int lane = threadIdx.x % G, half = c.dim / 2, pieces = half / VEC;
  const int per_token = q_heads + 2 * c.heads;
  const long long rows = (long long)tokens * per_token;
  const unsigned mask = G == 32 ? 0xffffffffu : ((1u << (G & 31)) - 1u) << ((threadIdx.x % 32) / G * G);
  for (long long row = ((long long)blockIdx.x * 256 + threadIdx.x) / G; row < rows; row += (long long)gridDim.x * (256 / G)) {
    const int tok = (int)(row / per_token), r = (int)(row - (long long)tok * per_token);
    const int at = __ldcg(pos + tok), sq = __ldcg(seq + tok);
    const int kind = r < q_heads ? 0 : r < q_heads + c.heads ? 1 : 2;      // query, key, value
    const int head = kind == 0 ? r : kind == 1 ? r - q_heads : r - q_heads - c.heads;
    const uint16_t* src = kind == 0 ? Q + tok * q_stride : kind == 1 ? K + tok * k_stride : V + tok * v_stride;
    src += (long long)head * c.dim;
    float a[kMost][VEC], b[kMost][VEC];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int p = lane + i * G;
      if (p < pieces) { load_bf16<VEC>(src + p * VEC, a[i]); load_bf16<VEC>(src + half + p * VEC, b[i]); }
    }
    if (at < 0) continue;                           // padding: nothing of this token is written
    const int2 place = kv_place(c, sq, at);
    if (place.x < 0 || (cos_t && at >= rope_rows)) {
      if (lane == 0) report_index();
      continue;
    }
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int p = lane + i * G;
      if (p >= pieces) continue;
      if (cos_t && kind < 2) {
        float cs[VEC], sn[VEC];
        const float* cr = cos_t + (long long)at * half + p * VEC;
        const float* sr = sin_t + (long long)at * half + p * VEC;
        // every head of the token reads the same angles: through L1
        if constexpr (VEC == 8) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float4 x = __ldca(reinterpret_cast<const float4*>(cr) + k), y = __ldca(reinterpret_cast<const float4*>(sr) + k);
            cs[4 * k] = x.x; cs[4 * k + 1] = x.y; cs[4 * k + 2] = x.z; cs[4 * k + 3] = x.w;
            sn[4 * k] = y.x; sn[4 * k + 1] = y.y; sn[4 * k + 2] = y.z; sn[4 * k + 3] = y.w;
          }
        } else {
          const float2 x = __ldca(reinterpret_cast<const float2*>(cr)), y = __ldca(reinterpret_cast<const float2*>(sr));
          cs[0] = x.x; cs[1] = x.y; sn[0] = y.x; sn[1] = y.y;
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float u = __fsub_rn(__fmul_rn(a[i][k], cs[k]), __fmul_rn(b[i][k], sn[k]));
          const float w = __fadd_rn(__fmul_rn(b[i][k], cs[k]), __fmul_rn(a[i][k], sn[k]));
          a[i][k] = __bfloat162float(__float2bfloat16_rn(u));
          b[i][k] = __bfloat162float(__float2bfloat16_rn(w));
        }
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k)      // as integers: a NaN is above infinity is above the rest
        amax = max(amax, max(__float_as_uint(a[i][k]) & 0x7fffffffu, __float_as_uint(b[i][k]) & 0x7fffffffu));
    }
    if (kind == 0) {
      uint16_t* dst = Q_out + ((long long)tok * q_heads + head) * c.dim;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const int p = lane + i * G;
        if (p < pieces) { store_bf16<VEC>(dst + p * VEC, a[i]); store_bf16<VEC>(dst + half + p * VEC, b[i]); }
      }
      continue;
    }
    const long long crow = kv_row(c, place, head);
    if (c.format == PQ_KV_BF16) {
      uint16_t* dst = static_cast<uint16_t*>(kind == 1 ? c.K : c.V) + crow * c.pitch;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const int p = lane + i * G;
        if (p < pieces) { store_bf16<VEC>(dst + p * VEC, a[i]); store_bf16<VEC>(dst + half + p * VEC, b[i]); }
      }
      for (int i = c.dim + lane; i < c.pitch; i += G) dst[i] = 0;
      continue;
    }
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) amax = max(amax, __shfl_xor_sync(mask, amax, d));
    const bool finite = amax < 0x7f800000u;
    const float gamma = finite ? __fdiv_rn(kActQmax, fmaxf(__uint_as_float(amax), kActAmaxFloor)) : __uint_as_float(0x7fffffffu);
    int8_t* dst = static_cast<int8_t*>(kind == 1 ? c.K : c.V) + crow * c.pitch;
    auto code = [&](float x) { return finite ? min(127, max(-128, __float2int_rn(__fmul_rn(x, gamma)))) & 0xff : 0; };
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int p = lane + i * G;
      if (p >= pieces) continue;
      auto put = [&](int8_t* to, const float (&v)[VEC]) {
        if constexpr (VEC == 8) {
          uint2 w;
          w.x = code(v[0]) | code(v[1]) << 8 | code(v[2]) << 16 | code(v[3]) << 24;
          w.y = code(v[4]) | code(v[5]) << 8 | code(v[6]) << 16 | code(v[7]) << 24;
          *reinterpret_cast<uint2*>(to) = w;
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

// ---------------------------------------------------------------------------
// k_kv_read: rows in the order token, then key heads, value heads; bf16(code / gamma).  The quotient is the correctly rounded one
// from the reciprocal and one residual (Markstein: a correctly rounded reciprocal and one fused correction of the quotient
// give the rounded quotient): three instructions a value where a division takes about ten, which would be
// more than the memory asks for.
// ---------------------------------------------------------------------------
template <int VEC, int G>
__global__ void __launch_bounds__(256) k_kv_read(KvCache c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x % G, pieces = c.dim / VEC;
  const long long rows = (long long)tokens * 2 * c.heads;
  for (long long row = ((long long)blockIdx.x * 256 + threadIdx.x) / G; row < rows; row += (long long)gridDim.x * (256 / G)) {
    const int tok = (int)(row / (2 * c.heads)), r = (int)(row - (long long)tok * 2 * c.heads);
    const int at = __ldcg(pos + tok);
    if (at < 0) continue;
    const int2 place = kv_place(c, __ldcg(seq + tok), at);
    if (place.x < 0) {
      if (lane == 0) report_index();
      continue;
    }
    const bool key = r < c.heads;
    const int head = key ? r : r - c.heads;
    const long long crow = kv_row(c, place, head);
    uint16_t* dst = (key ? K_out : V_out) + ((long long)tok * c.heads + head) * c.dim;
    const void* pages = key ? c.K : c.V;
    if (c.format == PQ_KV_BF16) {
      const uint16_t* src = static_cast<const uint16_t*>(pages) + crow * c.pitch;
      for (int p = lane; p < pieces; p += G) {
        if constexpr (VEC == 8) *reinterpret_cast<uint4*>(dst + 8 * p) = __ldcg(reinterpret_cast<const uint4*>(src + 8 * p));
        else *reinterpret_cast<uint2*>(dst + 4 * p) = __ldcg(reinterpret_cast<const uint2*>(src + 4 * p));
      }
      continue;
    }
    const int8_t* src = static_cast<const int8_t*>(pages) + crow * c.pitch;
    const float gamma = __ldcg((key ? c.k_gamma : c.v_gamma) + crow), inv = __frcp_rn(gamma);
    for (int p = lane; p < pieces; p += G) {
      uint32_t w[VEC / 4];
      if constexpr (VEC == 8) { const uint2 u = __ldcg(reinterpret_cast<const uint2*>(src + 8 * p)); w[0] = u.x; w[1] = u.y; }
      else w[0] = __ldcg(reinterpret_cast<const uint32_t*>(src + 4 * p));
      float v[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float x = (float)(int8_t)(w[k / 4] >> (8 * (k % 4)) & 0xff), q = __fmul_rn(x, inv);
        v[k] = __fmaf_rn(__fmaf_rn(-q, gamma, x), inv, q);
      }
      store_bf16<VEC>(dst + VEC * p, v);
    }
  }
}

// Lanes of a row: the pieces rounded up to a power of two
static int group_of(int pieces) {
  int g = 2;
  while (g < pieces && g < 32) g *= 2;
  return g;
}
static int blocks_for(long long rows, int g) {
  const long long b = (rows * g + 255) / 256, most = 1 << 20;      // beyond it the rows are walked with the grid's stride
  return (int)(b < most ? b : most);
}

cudaError_t launch_kv_append(const KvCache& c, int tokens, const int* seq, const int* pos, const uint16_t* K, long long k_stride,
                             const uint16_t* V, long long v_stride, const float* cos_t, const float* sin_t, int rope_rows, const uint16_t* Q,
                             long long q_stride, int q_heads, uint16_t* Q_out, cudaStream_t st) {
  const bool wide = c.dim % 16 == 0 && k_stride % 8 == 0 && v_stride % 8 == 0 && (!Q || q_stride % 8 == 0);
  const int g = wide ? group_of(c.dim / 16) : 32;
  auto kern = !wide ? k_kv_append<2, 32> : g == 2 ? k_kv_append<8, 2> : g == 4 ? k_kv_append<8, 4> : g == 8 ? k_kv_append<8, 8> : k_kv_append<8, 16>;
  LaunchScope ls(KID_KV_APPEND, st);
  return launch_pdl(kern, blocks_for((long long)tokens * (q_heads + 2 * c.heads), g), 256, 0, st, c, tokens, seq, pos, K, k_stride, V, v_stride,
                    cos_t, sin_t, rope_rows, Q, q_stride, q_heads, Q_out);
}

cudaError_t launch_kv_read(const KvCache& c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out, cudaStream_t st) {
  const bool wide = c.dim % 8 == 0;
  const int g = group_of(c.dim / (wide ? 8 : 4));
  auto kern = wide ? (g == 2 ? k_kv_read<8, 2> : g == 4 ? k_kv_read<8, 4> : g == 8 ? k_kv_read<8, 8> : g == 16 ? k_kv_read<8, 16> : k_kv_read<8, 32>)
                   : (g == 2 ? k_kv_read<4, 2> : g == 4 ? k_kv_read<4, 4> : g == 8 ? k_kv_read<4, 8> : g == 16 ? k_kv_read<4, 16> : k_kv_read<4, 32>);
  LaunchScope ls(KID_KV_READ, st);
  return launch_pdl(kern, blocks_for((long long)tokens * 2 * c.heads, g), 256, 0, st, c, tokens, seq, pos, K_out, V_out);
}

}  // namespace pq
