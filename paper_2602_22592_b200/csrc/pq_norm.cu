// The norms before and after a block, with its gate and residual scale, forward and backward:
//     u = rms(y) post | y,     s = res_scale x + gate u,     h = rms(s) pre,     rms(z) = z / sqrt(mean z^2 + eps)
// y is the block's output, x the stream in front of it, s the stream behind it, h the next block's input.  Sums, norms and s itself
// are held in fp32; s and h are rounded once, each from fp32.
//
// Every tensor moves once: rows come through shared memory by asynchronous copies, several ahead, and are finished where they are.
// Measured at 8192 x 2048 with a norm behind the block and a gate per feature: forward 30 us (134 MB, 4.5 TB/s; a copy of as much 20.5), backward
// 50 us (201 MB, 4.0 TB/s).  The forward waits at two meetings of a row's warps; the backward issues in 69 % of its slots: 27 fp32 operations a
// value and as much again to unpack, address and add up.  999 x 3200 without a norm behind the block: 18 us, 5 of them the sums over blocks.
// Above N = 2048 the backward behind a norm needs more than the 128 registers a thread has (two or four pieces, two rows, three running sums): 70 to 490
// bytes of it live in local memory for two pieces, 400 to 940 for four, and it shows: 4096 x 3200 with a gate per feature 87 us, without a norm
// behind the block 32; 1024 x 8640 97 and 28.
#include <algorithm>
#include <mutex>

#include "pq_pairs.cuh"

namespace pq {

constexpr int kNormSmemLimit = 224 * 1024;

__device__ __forceinline__ void unpack8(const uint4& u, F2 (&v)[4]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = f2(bf16lo(w[i]), bf16hi(w[i]));
}
__device__ __forceinline__ uint4 pack8(const F2 (&v)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x, y;
    get(v[i], x, y);
    w[i] = pack_bf16x2(x, y);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 ldcg8(const uint16_t* p, int chunk) { return __ldcg(reinterpret_cast<const uint4*>(p) + chunk); }
__device__ __forceinline__ void ldcg_f8(const float* p, int chunk, F2 (&v)[4]) {
  const float4 a = __ldcg(reinterpret_cast<const float4*>(p) + 2 * chunk), b = __ldcg(reinterpret_cast<const float4*>(p) + 2 * chunk + 1);
  v[0] = f2(a.x, a.y); v[1] = f2(a.z, a.w); v[2] = f2(b.x, b.y); v[3] = f2(b.z, b.w);
}
__device__ __forceinline__ void norm_copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
template <int N>
__device__ __forceinline__ void norm_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void norm_copy_wait(int pending) {
  switch (pending) {
    case 0: norm_copy_wait<0>(); break;
    case 1: norm_copy_wait<1>(); break;
    case 2: norm_copy_wait<2>(); break;
    default: norm_copy_wait<3>(); break;
  }
}

// Rows of up to four tensors on their way through shared memory by asynchronous copies, [stage][tensor][piece][thread]: a thread copies what it
// will read itself, so that nothing has to be waited for but its own copies.  Pieces behind the row's end and absent tensors
// stay zero.  THREADS, the most a block can have, is the stride, so that every place is an offset the compiler knows: with strides and
// rows multiplied out at every access half of these kernels' instructions were integer ones.
template <int K, int CH, int RB, int THREADS>
struct RowRing {
  static constexpr int kPiece = THREADS * 16, kStage = K * CH * kPiece;
  uint8_t* base;             // this thread's column
  const uint16_t* from[K];   // this thread's first piece of the next row to ask for, or null
  long long left, hop;       // rows of this team still to ask for; values from one to the next
  int gap, mine;             // values from piece to piece of a thread; how many pieces it has
  int most, at, into;        // bytes of the stages; where the row at work, the next copies are
  __device__ void begin() {
    for (int s = 0; s < most; s += kStage)
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (!from[k] || i >= mine) *reinterpret_cast<uint4*>(base + s + (k * CH + i) * kPiece) = make_uint4(0, 0, 0, 0);
    at = into = 0;
    for (int s = 0; s < most / kStage - RB; ++s) issue();
  }
  __device__ void issue() {
    if (left > 0) {
      const uint32_t dst = smem_u32(base) + into;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!from[k]) continue;
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (i < mine) norm_copy16(dst + (k * CH + i) * kPiece, from[k] + i * gap);
        from[k] += hop;
      }
      --left;
    }
    into = into + kStage == most ? 0 : into + kStage;
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ int after(int s) const { return s + kStage == most ? 0 : s + kStage; }
  __device__ void next() {                                     // the RB rows to work on are there, those behind them on their way
#pragma unroll
    for (int b = 0; b < RB; ++b) issue();
    norm_copy_wait(most / kStage - RB);
  }
  __device__ uint4 get(int b, int k, int i) const { return *reinterpret_cast<const uint4*>(base + (b == 0 ? at : after(at)) + (k * CH + i) * kPiece); }
  __device__ void done() {
#pragma unroll
    for (int b = 0; b < RB; ++b) at = after(at);
  }
};

// Sums over the `warps` warps of a row's owners (a named barrier of theirs where a block holds several rows): every lane gets
// them.  `slot` alternates between the two halves of `part`, so that one barrier a sum is enough.
struct RowTeam {
  float* part;               // [2][warps][8] floats of this team in shared memory
  int warps, warp, bar, slot;
  template <int K>
  __device__ void sum(float (&v)[K]) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
    if (warps == 1) return;
    float4* p = reinterpret_cast<float4*>(part) + slot * 2 * warps;
    slot ^= 1;
    if ((threadIdx.x & 31) == 0) {
      p[2 * warp] = make_float4(v[0], K > 1 ? v[K > 1 ? 1 : 0] : 0.f, K > 2 ? v[K > 2 ? 2 : 0] : 0.f, K > 3 ? v[K > 3 ? 3 : 0] : 0.f);
      if (K > 4) p[2 * warp + 1] = make_float4(v[K > 4 ? 4 : 0], K > 5 ? v[K > 5 ? 5 : 0] : 0.f, 0.f, 0.f);
    }
    asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(warps * 32) : "memory");
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.f;
    for (int w = 0; w < warps; ++w) {
      const float4 x = p[2 * w], y = K > 4 ? p[2 * w + 1] : make_float4(0, 0, 0, 0);
      const float all[6] = {x.x, x.y, x.z, x.w, y.x, y.y};
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += all[k];
    }
  }
};
__host__ __device__ constexpr int team_floats(int warps) { return 2 * 8 * warps; }

// ---------------------------------------------------------------------------
// k_block_norm: `warps` warps per row, CH pieces of 8 values per thread; teams of warps walk the rows with a stride.  The gains of a
// thread's columns stay in its registers.
// ---------------------------------------------------------------------------
template <int CH> constexpr int kNormThreads = CH == 1 ? 1024 : 512;
template <int CH, bool Y, bool POST>
__global__ void __launch_bounds__(kNormThreads<CH>) k_block_norm(const __grid_constant__ BlockNormArgs a, int warps, int stages) {
  extern __shared__ float smem_f[];
  pdl_launch_dependents();
  constexpr int K = Y ? 2 : 1;
  const int tid = threadIdx.x, lanes = warps * 32, teams = blockDim.x / lanes, team = tid / lanes, l = tid - team * lanes;
  RowTeam rt{smem_f + team * team_floats(warps), warps, l >> 5, 1 + team, 0};
  const int chunks = a.N / 8;
  long long row = (long long)blockIdx.x * teams + team;
  const long long step = (long long)gridDim.x * teams;
  const int mine = l < chunks ? min(CH, (chunks - l + lanes - 1) / lanes) : 0, gap = lanes * 8;
  long long off = row * a.N + l * 8;                           // of this thread's first piece of the row
  const long long hop = step * a.N;
  RowRing<K, CH, 1, kNormThreads<CH>> ring;
  ring.base = reinterpret_cast<uint8_t*>(smem_f + teams * team_floats(warps)) + tid * 16;
  ring.from[0] = a.x + off;
  if (Y) ring.from[K - 1] = a.y + off;
  ring.left = row < a.T ? (a.T - row + step - 1) / step : 0;
  ring.hop = hop; ring.gap = gap; ring.mine = mine; ring.most = stages * ring.kStage;
  pdl_wait();
  ring.begin();
  const float gate1 = a.gate && !a.gate_vector ? __ldcg(a.gate) : 1.f, inv_n = 1.f / a.N;
  uint4 pre[CH], post[POST ? CH : 1];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = l + i * lanes;
    pre[i] = a.h && i < mine ? ldcg8(a.pre, c) : make_uint4(0, 0, 0, 0);
    if (POST) post[POST ? i : 0] = i < mine ? ldcg8(a.post, c) : make_uint4(0, 0, 0, 0);
  }
  for (; row < a.T; row += step, off += hop) {
    ring.next();
    float ry = 1.f;
    if (POST) {
      F2 sq = f2(0.f);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        F2 y[4];
        unpack8(ring.get(0, K - 1, i), y);
#pragma unroll
        for (int k = 0; k < 4; ++k) sq = fma2(y[k], y[k], sq);
      }
      float v[1] = {both(sq)};
      rt.sum(v);
      ry = rsqrtf(v[0] * inv_n + a.eps);
    }
    const F2 by = f2(gate1 * ry), scale = f2(a.res_scale);
    F2 s[CH][4], sq = f2(0.f);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      unpack8(ring.get(0, 0, i), s[i]);
      F2 u[4];
      if (Y) {
        unpack8(ring.get(0, K - 1, i), u);
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = u[k] * by;
        if (POST) {
          F2 w[4];
          unpack8(post[POST ? i : 0], w);
#pragma unroll
          for (int k = 0; k < 4; ++k) u[k] = u[k] * w[k];
        }
        if (a.gate_vector && i < mine) {                       // 32 bytes a piece: read again, from L1
          const float4* at = reinterpret_cast<const float4*>(a.gate + l * 8 + i * gap);
          const float4 g0 = __ldca(at), g1 = __ldca(at + 1);
          u[0] = u[0] * f2(g0.x, g0.y); u[1] = u[1] * f2(g0.z, g0.w); u[2] = u[2] * f2(g1.x, g1.y); u[3] = u[3] * f2(g1.z, g1.w);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s[i][k] = Y ? fma2(scale, s[i][k], u[k]) : scale * s[i][k];
        sq = fma2(s[i][k], s[i][k], sq);
      }
      if (a.x_out && i < mine) *reinterpret_cast<uint4*>(a.x_out + off + i * gap) = pack8(s[i]);
    }
    ring.done();
    if (!a.h) continue;
    float v[1] = {both(sq)};
    rt.sum(v);
    const F2 r = f2(rsqrtf(v[0] * inv_n + a.eps));
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (i >= mine) continue;
      F2 w[4];
      unpack8(pre[i], w);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = s[i][k] * r * w[k];
      *reinterpret_cast<uint4*>(a.h + off + i * gap) = pack8(w);
    }
  }
  norm_copy_wait<0>();
}

// ---------------------------------------------------------------------------
// k_block_norm_backward.  With n = s r, r = 1 / sqrt(mean s^2 + eps) and d = dh pre:
//     g = ds + r (d - n mean(d n)),   dx = res_scale g,   dpre = sum_t dh n,   dgate = sum_t g u (over the features too if it is one number)
//     e = gate g;  dy = e, or behind a norm with m = y ry:  dy = ry (e post - m mean(e post m)),   dpost = sum_t e m
// mean(d n) = r mean(d s): one sum over the row gives both r and it.  Teams of threads walk the rows with a stride; a thread owns
// its columns for the whole launch, so that the sums over tokens stay in its registers; teams of a block meet in shared memory and
// blocks in k_norm_sums, in a fixed order.
// ---------------------------------------------------------------------------
template <int CH, bool POST, int GATE>     // GATE: 0 none, 1 one number, 2 per feature
__global__ void __launch_bounds__(512, 1) k_block_norm_backward(const __grid_constant__ BlockNormArgs a, int warps, int stages, float* part, double* gate_part) {
  extern __shared__ float smem_f[];
  __shared__ double gate_sums[32];
  pdl_launch_dependents();
  constexpr bool kY = POST || GATE > 0;
  constexpr int K = kY ? 4 : 3;
  const int tid = threadIdx.x, lanes = warps * 32, teams = blockDim.x / lanes, team = tid / lanes, l = tid - team * lanes;
  RowTeam rt{smem_f + team * team_floats(warps), warps, l >> 5, 1 + team, 0};
  const int chunks = a.N / 8;
  const long long step = (long long)gridDim.x * teams;
  long long row = (long long)blockIdx.x * teams + team;
  constexpr int RB = CH == 4 ? 1 : 2;                          // rows worked on at once: their sums meet in the same barriers
  const int mine = l < chunks ? min(CH, (chunks - l + lanes - 1) / lanes) : 0, gap = lanes * 8;
  long long off = row * a.N + l * 8;                           // of this thread's first piece of the row
  const long long hop = step * a.N;
  RowRing<K, CH, RB, 512> ring;
  ring.base = reinterpret_cast<uint8_t*>(smem_f + teams * team_floats(warps)) + tid * 16;
  ring.from[0] = a.dh ? a.x + off : nullptr;
  ring.from[1] = a.dh ? a.dh + off : nullptr;
  ring.from[2] = a.dx_out ? a.dx_out + off : nullptr;
  if (kY) ring.from[K - 1] = a.y + off;
  ring.left = row < a.T ? (a.T - row + step - 1) / step : 0;
  ring.hop = hop; ring.gap = gap; ring.mine = mine; ring.most = stages * ring.kStage;
  pdl_wait();
  ring.begin();
  const float gate1 = GATE == 1 ? __ldcg(a.gate) : 1.f, inv_n = 1.f / a.N;
  const F2 zero = f2(0.f);
  F2 spre[CH][4], sgate[GATE == 2 ? CH : 1][4], spost[POST ? CH : 1][4];
  double sgate1 = 0.0;
  // this thread's columns of the gains, zeros behind the row's end
  uint4 pre[CH], post[POST ? CH : 1];
  F2 gate[GATE == 2 ? CH : 1][4];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = l + i * lanes;
    const bool ok = i < mine;
    pre[i] = ok && a.dh ? ldcg8(a.pre, c) : make_uint4(0, 0, 0, 0);
    if (POST) post[POST ? i : 0] = ok ? ldcg8(a.post, c) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      spre[i][k] = zero;
      if (GATE == 2) sgate[GATE == 2 ? i : 0][k] = gate[GATE == 2 ? i : 0][k] = zero;
      if (POST) spost[POST ? i : 0][k] = zero;
    }
    if (GATE == 2 && ok) ldcg_f8(a.gate, c, gate[GATE == 2 ? i : 0]);
  }
  for (; row < a.T; row += RB * step, off += RB * hop) {
    ring.next();
    float sums[3 * RB];                                        // of each row: s^2, dh pre s, y^2
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      F2 sq = zero, dot = zero, ysq = zero;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        F2 s[4], dh[4], w[4];
        unpack8(ring.get(rb, 0, i), s);
        unpack8(ring.get(rb, 1, i), dh);
        unpack8(pre[i], w);
#pragma unroll
        for (int k = 0; k < 4; ++k) { sq = fma2(s[k], s[k], sq); dot = fma2(dh[k] * w[k], s[k], dot); }
        if (POST) {
          F2 y[4];
          unpack8(ring.get(rb, K - 1, i), y);
#pragma unroll
          for (int k = 0; k < 4; ++k) ysq = fma2(y[k], y[k], ysq);
        }
      }
      sums[3 * rb] = both(sq);
      sums[3 * rb + 1] = both(dot);
      sums[3 * rb + 2] = POST ? both(ysq) : 0.f;
    }
    rt.sum(sums);
    F2 e[RB][CH][4], ry2[RB];
    float edot[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      edot[rb] = 0.f;
      if (row + rb * step >= a.T) break;                                  // the ring still holds an older row there
      const float r = rsqrtf(sums[3 * rb] * inv_n + a.eps), ry = POST ? rsqrtf(sums[3 * rb + 2] * inv_n + a.eps) : 1.f;
      const F2 r2 = f2(r), corr = f2(-sums[3 * rb + 1] * inv_n * r * r), scale = f2(a.res_scale), g1 = f2(gate1);
      ry2[rb] = f2(ry);
      F2 edot2 = zero;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        F2 s[4], dh[4], w[4], g[4];
        unpack8(ring.get(rb, 0, i), s);
        unpack8(ring.get(rb, 1, i), dh);
        unpack8(ring.get(rb, 2, i), g);
        unpack8(pre[i], w);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          spre[i][k] = fma2(dh[k], s[k] * r2, spre[i][k]);
          g[k] = fma2(r2, fma2(s[k], corr, dh[k] * w[k]), g[k]);
        }
        if (i < mine) {
          F2 dx[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) dx[k] = scale * g[k];
          *reinterpret_cast<uint4*>(a.dx + off + rb * hop + i * gap) = pack8(dx);
        }
        if (kY) {
          F2 y[4], pw[4], line = zero;
          unpack8(ring.get(rb, K - 1, i), y);
          if (POST) unpack8(post[POST ? i : 0], pw);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const F2 m = POST ? y[k] * ry2[rb] : y[k], u = POST ? m * pw[k] : m;
            if (GATE == 2) sgate[GATE == 2 ? i : 0][k] = fma2(g[k], u, sgate[GATE == 2 ? i : 0][k]);
            if (GATE == 1) line = fma2(g[k], u, line);
            const F2 ge = GATE == 2 ? g[k] * gate[GATE == 2 ? i : 0][k] : GATE == 1 ? g[k] * g1 : g[k];
            if (POST) {
              spost[POST ? i : 0][k] = fma2(ge, m, spost[POST ? i : 0][k]);
              e[rb][i][k] = ge * pw[k];
              edot2 = fma2(e[rb][i][k], m, edot2);
            } else {
              e[rb][i][k] = ge;
            }
          }
          if (GATE == 1) sgate1 += (double)both(line);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) e[rb][i][k] = g[k];
        }
        if (!POST && a.dy && i < mine) *reinterpret_cast<uint4*>(a.dy + off + rb * hop + i * gap) = pack8(e[rb][i]);
      }
      edot[rb] = both(edot2);
    }
    if (POST) {
      rt.sum(edot);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (row + rb * step >= a.T) break;
        float ry, ry_;
        get(ry2[rb], ry, ry_);
        const F2 take = f2(-edot[rb] * inv_n * ry);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          if (i >= mine) continue;
          F2 y[4];
          unpack8(ring.get(rb, K - 1, i), y);
#pragma unroll
          for (int k = 0; k < 4; ++k) e[rb][i][k] = ry2[rb] * fma2(y[k], take, e[rb][i][k]);
          *reinterpret_cast<uint4*>(a.dy + off + rb * hop + i * gap) = pack8(e[rb][i]);
        }
      }
    }
    ring.done();
  }
  norm_copy_wait<0>();
  // ---- the block's sums: teams one after another into shared memory (the rings are free), [dpre, dgate, dpost][N]
  float* acc = smem_f + teams * team_floats(warps);
  const int n = a.N;
  for (int turn = 0; turn < teams; ++turn) {
    __syncthreads();
    if (turn != team) continue;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = l + i * lanes;
      if (c >= chunks) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        auto put = [&](float* p, const F2& v) {
          float x, y;
          get(v, x, y);
          p[0] = x + (turn ? p[0] : 0.f);
          p[1] = y + (turn ? p[1] : 0.f);
        };
        float* p = acc + c * 8 + 2 * k;
        put(p, spre[i][k]);
        if (GATE == 2) put(p + n, sgate[GATE == 2 ? i : 0][k]);
        if (POST) put(p + (GATE == 2 ? 2 : 1) * n, spost[POST ? i : 0][k]);
      }
    }
  }
  if (GATE == 1) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sgate1 += __shfl_xor_sync(0xffffffffu, sgate1, d);
    if ((tid & 31) == 0) gate_sums[tid >> 5] = sgate1;
  }
  __syncthreads();
  constexpr int kSums = 1 + (GATE == 2) + POST;
  for (int i = tid * 4; i < kSums * n; i += blockDim.x * 4)
    *reinterpret_cast<float4*>(part + (long long)blockIdx.x * kSums * n + i) = *reinterpret_cast<const float4*>(acc + i);
  if (GATE == 1 && tid == 0) {
    double v = 0.0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) v += gate_sums[w];
    gate_part[blockIdx.x] = v;
  }
}

// Sums over the blocks, in their order: 32 columns by 32 slices of blocks (eight were 1.2 us slower: a trip to memory more).  One block more than the columns need adds the one
// number of a scalar gate.
__global__ void __launch_bounds__(1024) k_norm_sums(const float* part, int blocks, int n, int sums, float* out0, float* out1, float* out2, const double* gate_part,
                                                   float* dgate1) {
  __shared__ float red[32][33];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, x = tid & 31, y = tid >> 5, width = sums * n;
  const int col = blockIdx.x * 32 + x;
  if (blockIdx.x * 32 >= width) {
    if (tid == 0) {
      double v = 0.0;
      for (int b = 0; b < blocks; ++b) v += __ldcg(gate_part + b);
      *dgate1 = (float)v;
    }
    return;
  }
  float v = 0.f;
  if (col < width) {
    const int b0 = (int)((long long)blocks * y / 32), b1 = (int)((long long)blocks * (y + 1) / 32);
#pragma unroll 8
    for (int b = b0; b < b1; ++b) v += __ldcg(part + (long long)b * width + col);
  }
  red[y][x] = v;
  __syncthreads();
  if (y == 0 && col < width) {
    v = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) v += red[k][x];
    const int which = col / n;
    float* out = which == 0 ? out0 : which == 1 ? out1 : out2;
    if (out) out[col - which * n] = v;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// The opt-in limits, once per device
template <int CH>
static auto norm_kernel(bool y, bool post) { return post ? k_block_norm<CH, true, true> : y ? k_block_norm<CH, true, false> : k_block_norm<CH, false, false>; }
template <int CH>
static auto norm_bwd_kernel(bool post, int gate) {
  return post ? (gate == 0 ? k_block_norm_backward<CH, true, 0> : gate == 1 ? k_block_norm_backward<CH, true, 1> : k_block_norm_backward<CH, true, 2>)
              : (gate == 0 ? k_block_norm_backward<CH, false, 0> : gate == 1 ? k_block_norm_backward<CH, false, 1> : k_block_norm_backward<CH, false, 2>);
}
static cudaError_t norm_limits() {
  constexpr int kMaxDevices = 64;
  static std::once_flag done[kMaxDevices];
  static cudaError_t result[kMaxDevices] = {};
  int dev = 0;
  if (const cudaError_t e = cudaGetDevice(&dev)) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::call_once(done[dev], [&] {
    auto set = [&](auto k) { if (result[dev] == cudaSuccess) result[dev] = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormSmemLimit); };
    for (int post = 0; post < 2; ++post) {
      for (int y = post; y < 2; ++y) { set(norm_kernel<1>(y, post)); set(norm_kernel<4>(y, post)); }
      for (int gate = 0; gate < 3; ++gate) { set(norm_bwd_kernel<1>(post, gate)); set(norm_bwd_kernel<2>(post, gate)); set(norm_bwd_kernel<4>(post, gate)); }
    }
  });
  return result[dev];
}
// as many rows in flight as fit, four at most
static int norm_stages(size_t row_bytes, size_t fixed, int least, int most) {
  return (int)std::max<size_t>(least, std::min<size_t>(most, (kNormSmemLimit - fixed) / row_bytes));
}

cudaError_t launch_block_norm_forward(const BlockNormArgs& a, cudaStream_t st) {
  if (const cudaError_t e = norm_limits()) return e;
  const int chunks = a.N / 8, tensors = a.y ? 2 : 1;
  // few rows: a thread per piece, the row's latency; many: four pieces a thread, fewer warps to meet per row (8192 x 2048 with four pieces and
  // sixteen warps an SM 29.6 us, with two and thirty-two 33.5, with one 35)
  const int ch = chunks <= 1024 && a.T <= sm_count() ? 1 : 4, most = ch == 1 ? 32 : 16;
  const int warps = (chunks + 32 * ch - 1) / (32 * ch);
  const int teams = std::max(1, std::min(most / warps, 15));                                  // named barriers
  const int blocks = (int)std::min<long long>(((long long)a.T + teams - 1) / teams, sm_count());
  const bool few = a.T <= blocks * teams;                                                     // one row a team: nothing behind it
  const size_t fixed = (size_t)teams * team_floats(warps) * sizeof(float), row = (size_t)tensors * ch * 16 * (ch == 1 ? kNormThreads<1> : kNormThreads<4>);
  const int stages = norm_stages(row, fixed, 1, few ? 1 : 4);
  auto kern = ch == 1 ? norm_kernel<1>(a.y != nullptr, a.post != nullptr) : norm_kernel<4>(a.y != nullptr, a.post != nullptr);
  LaunchScope ls(KID_NORM_FWD, st);
  return launch_pdl(kern, blocks, teams * warps * 32, fixed + stages * row, st, a, warps, stages);
}

struct NormBwdPlan { int ch, warps, teams, blocks; };
static NormBwdPlan norm_bwd_plan(int T, int N) {
  NormBwdPlan p{};
  const int chunks = N / 8;
  p.ch = chunks <= 256 ? 1 : chunks <= 1024 ? 2 : 4;           // two rows at work in a block as long as they fit
  p.warps = (chunks + 32 * p.ch - 1) / (32 * p.ch);
  p.teams = std::max(1, std::min(16 / p.warps, 15));           // named barriers
  p.blocks = (int)std::min<long long>(sm_count(), ((long long)T + p.teams - 1) / p.teams);
  return p;
}
size_t block_norm_workspace_bytes(int T, int N) {
  const NormBwdPlan p = norm_bwd_plan(T, N);
  return ((size_t)p.blocks * 3 * N * 4 + 255) / 256 * 256 + (size_t)p.blocks * 8;
}

cudaError_t launch_block_norm_backward(const BlockNormArgs& a, void* ws, cudaStream_t st) {
  const NormBwdPlan p = norm_bwd_plan(a.T, a.N);
  float* part = static_cast<float*>(ws);
  double* gate_part = reinterpret_cast<double*>(static_cast<uint8_t*>(ws) + ((size_t)p.blocks * 3 * a.N * 4 + 255) / 256 * 256);
  const int gate = !a.gate ? 0 : a.gate_vector ? 2 : 1, sums = 1 + (gate == 2) + (a.post != nullptr);
  const bool post = a.post != nullptr;
  auto kern = p.ch == 1 ? norm_bwd_kernel<1>(post, gate) : p.ch == 2 ? norm_bwd_kernel<2>(post, gate) : norm_bwd_kernel<4>(post, gate);
  if (const cudaError_t e = norm_limits()) return e;
  // the sums over tokens take the ring's place in the end
  const size_t row = (size_t)(a.post || a.gate ? 4 : 3) * p.ch * 16 * 512, fixed = (size_t)p.teams * team_floats(p.warps) * sizeof(float);
  const int stages = norm_stages(row, fixed, p.ch == 4 ? 1 : 2, 4);
  const size_t smem = fixed + std::max(stages * row, (size_t)sums * a.N * sizeof(float));
  {
    LaunchScope ls(KID_NORM_BWD, st);
    if (const cudaError_t e = launch_pdl(kern, p.blocks, p.teams * p.warps * 32, smem, st, a, p.warps, stages, part, gate_part)) return e;
  }
  LaunchScope ls(KID_NORM_SUMS, st);
  return launch_pdl(k_norm_sums, (sums * a.N + 31) / 32 + (gate == 1 ? 1 : 0), 1024, 0, st, part, p.blocks, a.N, sums, a.dh ? a.dpre : nullptr,
                    gate == 2 ? a.dgate : a.dpost, a.dpost, gate_part, a.dgate);
}

}  // namespace pq
