// The norms before and after a block, with its gate and residual scale, forward and backward:
//     u = rms(y) post | y,     s = res_scale x + gate u,     h = rms(s) pre,     rms(z) = z / sqrt(mean z^2 + eps)
// y is the block's output, x the stream in front of it, s the stream behind it, h the next block's input.  Sums, norms and s itself
// are held in fp32; s and h are rounded once, each from fp32.
//
// Bound by memory: a row stays in the registers of the warps that own it from its load to its store, so that every tensor moves
// once.
#include <algorithm>

#include "pq_kernels.cuh"

namespace pq {

constexpr int kNormSmemLimit = 224 * 1024;

__device__ __forceinline__ void unpack8(const uint4& u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = bf16lo(w[i]); v[2 * i + 1] = bf16hi(w[i]); }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
// gains and gates, which every row reads again: through L1
__device__ __forceinline__ uint4 ldca8(const uint16_t* p, int chunk) { return __ldca(reinterpret_cast<const uint4*>(p) + chunk); }
__device__ __forceinline__ uint4 ldcg8(const uint16_t* p, int chunk) { return __ldcg(reinterpret_cast<const uint4*>(p) + chunk); }
__device__ __forceinline__ void ldca_f8(const float* p, int chunk, float (&v)[8]) {
  const float4 a = __ldca(reinterpret_cast<const float4*>(p) + 2 * chunk), b = __ldca(reinterpret_cast<const float4*>(p) + 2 * chunk + 1);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// Sums over the `warps` warps of a row's owners (a named barrier of theirs where a block holds several rows): every lane gets
// them.  `slot` alternates between the two halves of `part`, so that one barrier a sum is enough.
struct RowTeam {
  float* part;               // [2][32][4] floats of this team in shared memory
  int warps, warp, bar, slot;
  __device__ void sum(float& a) { float b = 0.f, c = 0.f; sum(a, b, c); }
  __device__ void sum(float& a, float& b, float& c) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, d);
      b += __shfl_xor_sync(0xffffffffu, b, d);
      c += __shfl_xor_sync(0xffffffffu, c, d);
    }
    if (warps == 1) return;
    float4* p = reinterpret_cast<float4*>(part) + slot * 32;
    slot ^= 1;
    if ((threadIdx.x & 31) == 0) p[warp] = make_float4(a, b, c, 0.f);
    asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(warps * 32) : "memory");
    a = b = c = 0.f;
    for (int w = 0; w < warps; ++w) { a += p[w].x; b += p[w].y; c += p[w].z; }
  }
};
constexpr int kTeamFloats = 2 * 32 * 4;

// ---------------------------------------------------------------------------
// k_block_norm: `warps` warps per row, CH pieces of 8 values per lane
// ---------------------------------------------------------------------------
template <int CH>
__global__ void __launch_bounds__(CH == 4 ? 512 : 1024) k_block_norm(const __grid_constant__ BlockNormArgs a, int warps) {
  extern __shared__ float smem_f[];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, lanes = warps * 32, team = tid / lanes, l = tid - team * lanes;
  const long long row = (long long)blockIdx.x * (blockDim.x / lanes) + team;
  if (row >= a.T) return;                       // a whole team: its barrier is its own
  RowTeam rt{smem_f + team * kTeamFloats, warps, l >> 5, 1 + team, 0};
  const int chunks = a.N / 8;
  uint4 xr[CH], yr[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = l + i * lanes;
    xr[i] = yr[i] = make_uint4(0, 0, 0, 0);
    if (c < chunks) {
      xr[i] = ldcg8(a.x + row * a.N, c);
      if (a.y) yr[i] = ldcg8(a.y + row * a.N, c);
    }
  }
  float ry = 1.f;
  if (a.post) {
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float v[8];
      unpack8(yr[i], v);
#pragma unroll
      for (int k = 0; k < 8; ++k) sq += v[k] * v[k];
    }
    rt.sum(sq);
    ry = rsqrtf(sq / a.N + a.eps);
  }
  float s[CH][8], sq = 0.f;
  const float gate1 = a.gate && !a.gate_vector ? __ldcg(a.gate) : 1.f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = l + i * lanes;
    float u[8];
    unpack8(xr[i], s[i]);
    unpack8(yr[i], u);
    if (c < chunks) {
      if (a.post) {
        float w[8];
        unpack8(ldca8(a.post, c), w);
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = u[k] * ry * w[k];
      }
      if (a.gate_vector) {
        float w[8];
        ldca_f8(a.gate, c, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] *= w[k];
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      s[i][k] = a.res_scale * s[i][k] + gate1 * u[k];
      sq += s[i][k] * s[i][k];
    }
    if (a.x_out && c < chunks) reinterpret_cast<uint4*>(a.x_out + row * a.N)[c] = pack8(s[i]);
  }
  if (!a.h) return;
  rt.sum(sq);
  const float r = rsqrtf(sq / a.N + a.eps);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = l + i * lanes;
    if (c >= chunks) continue;
    float w[8];
    unpack8(ldca8(a.pre, c), w);
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = s[i][k] * r * w[k];
    reinterpret_cast<uint4*>(a.h + row * a.N)[c] = pack8(w);
  }
}

// ---------------------------------------------------------------------------
// k_block_norm_backward.  With n = s r, r = 1 / sqrt(mean s^2 + eps) and d = dh pre:
//     g = ds + r (d - n mean(d n)),   dx = res_scale g,   dpre = sum_t dh n,   dgate = sum_t g u (over the features too if it is one number)
//     e = gate g;  dy = e, or behind a norm with m = y ry:  dy = ry (e post - m mean(e post m)),   dpost = sum_t e m
// mean(d n) = r mean(d s): one sum over the row gives both r and it.  Teams of threads walk the rows with a stride; a thread owns
// its columns for the whole launch, so that the sums over tokens stay in its registers; teams of a block meet in shared memory and
// blocks in k_norm_sums, in a fixed order.
// ---------------------------------------------------------------------------
template <int N>
__device__ __forceinline__ void norm_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int CH, bool POST, int GATE>     // GATE: 0 none, 1 one number, 2 per feature
__global__ void __launch_bounds__(512, 1) k_block_norm_backward(const __grid_constant__ BlockNormArgs a, int warps, int stages, float* part, double* gate_part) {
  extern __shared__ float smem_f[];
  __shared__ double gate_sums[32];
  pdl_launch_dependents();
  pdl_wait();
  constexpr bool kY = POST || GATE > 0;
  constexpr int kTensors = kY ? 4 : 3;
  const int tid = threadIdx.x, lanes = warps * 32, teams = blockDim.x / lanes, team = tid / lanes, l = tid - team * lanes;
  RowTeam rt{smem_f + team * kTeamFloats, warps, l >> 5, 1 + team, 0};
  const int chunks = a.N / 8;
  const float gate1 = GATE == 1 ? __ldcg(a.gate) : 1.f, inv_n = 1.f / a.N;
  float spre[CH][8] = {}, sgate[GATE == 2 ? CH : 1][8] = {}, spost[POST ? CH : 1][8] = {};
  double sgate1 = 0.0;
  // this thread's columns of the gains, zeros behind the row's end
  uint4 pre[CH], post[POST ? CH : 1];
  float gate[GATE == 2 ? CH : 1][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = l + i * lanes;
    const bool ok = c < chunks;
    pre[i] = ok && a.dh ? ldcg8(a.pre, c) : make_uint4(0, 0, 0, 0);
    if (POST) post[POST ? i : 0] = ok ? ldcg8(a.post, c) : make_uint4(0, 0, 0, 0);
    if (GATE == 2) {
#pragma unroll
      for (int k = 0; k < 8; ++k) gate[GATE == 2 ? i : 0][k] = 0.f;
      if (ok) ldca_f8(a.gate, c, gate[GATE == 2 ? i : 0]);
    }
  }
  // Rows come through a ring in shared memory by asynchronous copies, [stage][tensor][piece][thread]: a thread copies what it will read itself,
  // so that nothing has to be waited for but its own copies.  Absent tensors and pieces behind the row's end stay zero.
  uint4* const ring = reinterpret_cast<uint4*>(smem_f + teams * kTeamFloats) + (size_t)team * stages * kTensors * CH * lanes + l;
  const uint16_t* const from[4] = {a.dh ? a.x : nullptr, a.dh, a.dx_out, kY ? a.y : nullptr};
  auto place = [&](int stage, int tensor, int i) { return ring + (size_t)((stage * kTensors + tensor) * CH + i) * lanes; };
  for (int s = 0; s < stages; ++s)
#pragma unroll
    for (int k = 0; k < kTensors; ++k)
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (!from[k] || l + i * lanes >= chunks) *place(s, k, i) = make_uint4(0, 0, 0, 0);
  const long long step = (long long)gridDim.x * teams;
  long long row = (long long)blockIdx.x * teams + team, ahead = row;
  auto issue = [&](int stage) {
    if (ahead < a.T) {
#pragma unroll
      for (int k = 0; k < kTensors; ++k)
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (from[k] && l + i * lanes < chunks) cp_async16(smem_u32(place(stage, k, i)), from[k] + ahead * a.N + (l + i * lanes) * 8, true);
    }
    ahead += step;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int s = 0; s < stages - 1; ++s) issue(s);
  int stage = 0, into = stages - 1;
  for (; row < a.T; row += step) {
    issue(into);                                               // where the row before this one was
    switch (stages) {
      case 1: norm_copy_wait<0>(); break;
      case 2: norm_copy_wait<1>(); break;
      case 3: norm_copy_wait<2>(); break;
      default: norm_copy_wait<3>(); break;
    }
    float sq = 0.f, dot = 0.f, ysq = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float s[8], dh[8], w[8];
      unpack8(*place(stage, 0, i), s);
      unpack8(*place(stage, 1, i), dh);
      unpack8(pre[i], w);
#pragma unroll
      for (int k = 0; k < 8; ++k) { sq += s[k] * s[k]; dot += dh[k] * w[k] * s[k]; }
      if (POST) {
        float y[8];
        unpack8(*place(stage, 3, i), y);
#pragma unroll
        for (int k = 0; k < 8; ++k) ysq += y[k] * y[k];
      }
    }
    rt.sum(sq, dot, ysq);
    const float r = rsqrtf(sq * inv_n + a.eps), corr = dot * inv_n * r * r, ry = POST ? rsqrtf(ysq * inv_n + a.eps) : 1.f;
    float e[CH][8], edot = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = l + i * lanes;
      float s[8], dh[8], w[8], g[8];
      unpack8(*place(stage, 0, i), s);
      unpack8(*place(stage, 1, i), dh);
      unpack8(*place(stage, 2, i), g);
      unpack8(pre[i], w);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        spre[i][k] += dh[k] * (s[k] * r);
        g[k] += r * (dh[k] * w[k] - s[k] * corr);
      }
      if (c < chunks) {
        float dx[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) dx[k] = a.res_scale * g[k];
        reinterpret_cast<uint4*>(a.dx + row * a.N)[c] = pack8(dx);
      }
      if (kY) {
        float y[8], pw[8];
        unpack8(*place(stage, kTensors - 1, i), y);
        if (POST) unpack8(post[POST ? i : 0], pw);
        float line = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float m = y[k] * ry, u = POST ? m * pw[k] : m;
          if (GATE == 2) sgate[GATE == 2 ? i : 0][k] += g[k] * u;
          if (GATE == 1) line += g[k] * u;
          const float ge = g[k] * (GATE == 2 ? gate[GATE == 2 ? i : 0][k] : gate1);
          if (POST) {
            spost[POST ? i : 0][k] += ge * m;
            e[i][k] = ge * pw[k];
            edot += e[i][k] * m;
          } else {
            e[i][k] = ge;
          }
        }
        if (GATE == 1) sgate1 += (double)line;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) e[i][k] = g[k];
      }
    }
    if (a.dy) {
      if (POST) { rt.sum(edot); edot *= inv_n; }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = l + i * lanes;
        if (c >= chunks) continue;
        if (POST) {
          float y[8];
          unpack8(*place(stage, kTensors - 1, i), y);
#pragma unroll
          for (int k = 0; k < 8; ++k) e[i][k] = ry * (e[i][k] - y[k] * ry * edot);
        }
        reinterpret_cast<uint4*>(a.dy + row * a.N)[c] = pack8(e[i]);
      }
    }
    stage = stage + 1 == stages ? 0 : stage + 1;
    into = into + 1 == stages ? 0 : into + 1;
  }
  norm_copy_wait<0>();
  // ---- the block's sums: teams one after another into shared memory (the rings are free), [dpre, dgate, dpost][N]
  float* acc = smem_f + teams * kTeamFloats;
  const int n = a.N;
  for (int turn = 0; turn < teams; ++turn) {
    __syncthreads();
    if (turn != team) continue;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = l + i * lanes;
      if (c >= chunks) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float* p = acc + c * 8 + k;
        p[0] = spre[i][k] + (turn ? p[0] : 0.f);
        if (GATE == 2) p[n] = sgate[GATE == 2 ? i : 0][k] + (turn ? p[n] : 0.f);
        if (POST) p[(GATE == 2 ? 2 : 1) * n] = spost[POST ? i : 0][k] + (turn ? p[(GATE == 2 ? 2 : 1) * n] : 0.f);
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

// Sums over the blocks, in their order: 32 columns by 8 slices of blocks.  One block more than the columns need adds the one
// number of a scalar gate.
__global__ void __launch_bounds__(256) k_norm_sums(const float* part, int blocks, int n, int sums, float* out0, float* out1, float* out2, const double* gate_part,
                                                   float* dgate1) {
  __shared__ float red[8][32];
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
    const int b0 = (int)((long long)blocks * y / 8), b1 = (int)((long long)blocks * (y + 1) / 8);
#pragma unroll 8
    for (int b = b0; b < b1; ++b) v += __ldcg(part + (long long)b * width + col);
  }
  red[y][x] = v;
  __syncthreads();
  if (y == 0 && col < width) {
    v = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v += red[k][x];
    const int which = col / n;
    float* out = which == 0 ? out0 : which == 1 ? out1 : out2;
    if (out) out[col - which * n] = v;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
cudaError_t launch_block_norm_forward(const BlockNormArgs& a, cudaStream_t st) {
  const int chunks = a.N / 8;
  // few rows: a lane per piece, the row's latency; many: four pieces a lane
  const int ch = a.T <= 2 * sm_count() ? 1 : 4;
  int warps = 1;
  while (warps < 32 && warps * 32 * ch < chunks) warps *= 2;
  const int use = warps * 32 >= chunks ? 1 : warps * 64 >= chunks ? 2 : 4;
  auto kern = use == 1 ? k_block_norm<1> : use == 2 ? k_block_norm<2> : k_block_norm<4>;
  const int rows = std::max(1, 8 / warps);
  LaunchScope ls(KID_NORM_FWD, st);
  return launch_pdl(kern, (a.T + rows - 1) / rows, rows * warps * 32, rows * kTeamFloats * sizeof(float), st, a, warps);
}

struct NormBwdPlan { int ch, warps, teams, blocks; };
static NormBwdPlan norm_bwd_plan(int T, int N) {
  NormBwdPlan p{};
  const int chunks = N / 8;
  p.ch = chunks <= 512 ? 1 : chunks <= 1024 ? 2 : 4;
  p.warps = (chunks + 32 * p.ch - 1) / (32 * p.ch);
  p.teams = p.ch == 1 ? std::max(1, 16 / p.warps) : 1;
  p.blocks = std::min(sm_count(), (T + p.teams - 1) / p.teams);
  return p;
}
size_t block_norm_workspace_bytes(int T, int N) {
  const NormBwdPlan p = norm_bwd_plan(T, N);
  return ((size_t)p.blocks * 3 * N * 4 + 255) / 256 * 256 + (size_t)p.blocks * 8;
}

template <int CH>
static auto norm_bwd_kernel(bool post, int gate) {
  return post ? (gate == 0 ? k_block_norm_backward<CH, true, 0> : gate == 1 ? k_block_norm_backward<CH, true, 1> : k_block_norm_backward<CH, true, 2>)
              : (gate == 0 ? k_block_norm_backward<CH, false, 0> : gate == 1 ? k_block_norm_backward<CH, false, 1> : k_block_norm_backward<CH, false, 2>);
}
cudaError_t launch_block_norm_backward(const BlockNormArgs& a, void* ws, cudaStream_t st) {
  const NormBwdPlan p = norm_bwd_plan(a.T, a.N);
  float* part = static_cast<float*>(ws);
  double* gate_part = reinterpret_cast<double*>(static_cast<uint8_t*>(ws) + ((size_t)p.blocks * 3 * a.N * 4 + 255) / 256 * 256);
  const int gate = !a.gate ? 0 : a.gate_vector ? 2 : 1, sums = 1 + (gate == 2) + (a.post != nullptr);
  const bool post = a.post != nullptr;
  auto kern = p.ch == 1 ? norm_bwd_kernel<1>(post, gate) : p.ch == 2 ? norm_bwd_kernel<2>(post, gate) : norm_bwd_kernel<4>(post, gate);
  // as many rows in flight as fit, four at most; the sums over tokens take the ring's place in the end
  const size_t row = (size_t)(a.post || a.gate ? 4 : 3) * p.ch * p.warps * 32 * 16 * p.teams, fixed = (size_t)p.teams * kTeamFloats * sizeof(float);
  const int stages = (int)std::max<size_t>(1, std::min<size_t>(4, (kNormSmemLimit - fixed) / row));
  const size_t smem = fixed + std::max(stages * row, (size_t)sums * a.N * sizeof(float));
  if (const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormSmemLimit)) return e;
  {
    LaunchScope ls(KID_NORM_BWD, st);
    if (const cudaError_t e = launch_pdl(kern, p.blocks, p.teams * p.warps * 32, smem, st, a, p.warps, stages, part, gate_part)) return e;
  }
  LaunchScope ls(KID_NORM_SUMS, st);
  return launch_pdl(k_norm_sums, (sums * a.N + 31) / 32 + (gate == 1 ? 1 : 0), 256, 0, st, part, p.blocks, a.N, sums, a.dh ? a.dpre : nullptr,
                    gate == 2 ? a.dgate : a.dpost, a.dpost, gate_part, a.dgate);
}

}  // namespace pq
