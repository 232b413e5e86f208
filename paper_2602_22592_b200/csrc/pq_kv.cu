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

constexpr int kSteps = 4;        // of a unit at most; with few rows one, so that they spread over more warps

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
    Raw<VEC> ra[kSteps][kMost], rb[kSteps][kMost];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int r = row0 + s * kRows;
      const uint16_t* src = (r < q_heads ? q_row : r < q_heads + c.heads ? k_row : v_row) + (long long)r * c.dim + lane * VEC;
#pragma unroll
      for (int i = 0; i < kMost; ++i)
        if (s < steps && r < rows && lane + i * G < pieces) { load_raw<VEC>(src + i * G * VEC, ra[s][i]); load_raw<VEC>(src + half + i * G * VEC, rb[s][i]); }
    }
    // other warps turn other rows of the token by the same angles: through L1
    float cs[kMost][VEC], sn[kMost][VEC];
    const bool turns = cos_t && at >= 0 && at < rope_rows;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int p = lane + i * G;
      if (!turns || p >= pieces) continue;
      const float* cr = cos_t + (long long)at * half + p * VEC;
      const float* sr = sin_t + (long long)at * half + p * VEC;
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
      float a[kMost][VEC], b[kMost][VEC];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (lane + i * G >= pieces) continue;
        raw_floats(ra[s][i], a[i]);
        raw_floats(rb[s][i], b[i]);
        if (turns && key) {
#pragma unroll
          for (int k = 0; k < VEC; k += 2) {
            float u[2], v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              u[j] = __fsub_rn(__fmul_rn(a[i][k + j], cs[i][k + j]), __fmul_rn(b[i][k + j], sn[i][k + j]));
              v[j] = __fadd_rn(__fmul_rn(b[i][k + j], cs[i][k + j]), __fmul_rn(a[i][k + j], sn[i][k + j]));
            }
            const uint32_t x = pack_bf16x2(u[0], u[1]), y = pack_bf16x2(v[0], v[1]);
            a[i][k] = bf16lo(x); a[i][k + 1] = bf16hi(x);
            b[i][k] = bf16lo(y); b[i][k + 1] = bf16hi(y);
          }
        }
        if (I8) {
#pragma unroll
          for (int k = 0; k < VEC; ++k)      // as integers: a NaN is above infinity is above the rest
            amax = max(amax, max(__float_as_uint(a[i][k]) & 0x7fffffffu, __float_as_uint(b[i][k]) & 0x7fffffffu));
        }
      }
      const int head = query ? r : key ? r - q_heads : r - q_heads - c.heads;
      if (query || !I8) {
        uint16_t* dst = query ? Q_out + ((long long)tok * q_heads + head) * c.dim : static_cast<uint16_t*>(key ? c.K : c.V) + crow0 * c.pitch + head * head_rows;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          const int p = lane + i * G;
          if (p < pieces) { store_bf16<VEC>(dst + p * VEC, a[i]); store_bf16<VEC>(dst + half + p * VEC, b[i]); }
        }
        if (!query && lane < c.pitch - c.dim) dst[c.dim + lane] = 0;      // at most 4 of them
        continue;
      }
#pragma unroll
      for (int d = G / 2; d > 0; d >>= 1) amax = max(amax, __shfl_xor_sync(mask, amax, d));
      const bool finite = amax < 0x7f800000u;
      const float gamma = finite ? __fdiv_rn(kActQmax, fmaxf(__uint_as_float(amax), kActAmaxFloor)) : __uint_as_float(0x7fffffffu);
      int8_t* dst = static_cast<int8_t*>(key ? c.K : c.V) + crow0 * c.pitch + head * head_rows;
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
__global__ void __launch_bounds__(256, I8 ? 5 : 4) k_kv_read(KvCache c, int tokens, const int* seq, const int* pos, uint16_t* K_out, uint16_t* V_out, int steps) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kMost = VEC == 8 ? 1 : 2;                              // pieces per lane (G = 16: head_dim <= 128)
  constexpr int kRows = 32 / G, kBytes = I8 ? 1 : 2;
  using In = Raw<I8 ? VEC / 2 : VEC>;                                  // the bytes of VEC values
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
          if (lane + i * G < pieces) raw[s][i].v = __ldcg(reinterpret_cast<const decltype(raw[s][i].v)*>(src + i * G * VEC * kBytes));
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
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (lane + i * G >= pieces) continue;
        if constexpr (!I8) {
          *reinterpret_cast<decltype(raw[s][i].v)*>(dst + i * G * VEC) = raw[s][i].v;
        } else {
          uint32_t word[VEC / 4];
          if constexpr (VEC == 8) { word[0] = raw[s][i].v.x; word[1] = raw[s][i].v.y; } else word[0] = raw[s][i].v;
          float v[VEC];
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            // under the bits of 2^23 an integer below it is itself: conversions by permute and addition
            const float x = __uint_as_float(__byte_perm(word[k / 4] ^ 0x80808080u, 0x4B000000u, 0x7440 + k % 4)) - 8388736.f, q = __fmul_rn(x, inv);
            v[k] = __fmaf_rn(__fmaf_rn(-q, gamma[s], x), inv, q);
          }
          store_bf16<VEC>(dst + i * G * VEC, v);
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
  return launch_pdl(kern, blocks_for(tokens, 2 * c.heads, g, steps, c.format == PQ_KV_INT8 ? 5 : 4), 256, 0, st, c, tokens, seq, pos, K_out, V_out, steps);
}

}  // namespace pq
