// Gradients of the gated residual and norms (block_norm_fwd.cu).  With
// n(v) = (v - mean) rho and, for a vector d, the norm's transposed Jacobian
//   J(v)^T d = rho (d - mean(d) - n mean(d n))      (RMS: without mean(d)):
//   dn = dh (1 + scale) pre_weight      d  = dr + J_pre(r)^T dn
//   dx = a d                            dy = J_post(y)^T (d gate post_weight)
// and the sums over tokens
//   A = sum dh n(r)    C = sum dh    E = sum d n(y)
//   dscale = pre_weight A, dshift = C, dgate = post_weight E   per group,
//   dpre_weight = sum_g (1 + scale) A,  dpost_weight = sum_g gate E.
//
// Bound by memory: dr, dh, r, y are read once, dx, dy written once (18 bytes
// per element with a float32 residual stream).  A thread owns 8 columns for
// all the rows that its CTA takes, so A, C and E stay in its registers and
// every token sum has a fixed order; a row's eight sums go across the CTA in
// four exchanges.
#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

// Sums of N values over all threads of the CTA (at most 32 warps).
template <int N>
__device__ __forceinline__ void cta_sum(float (&v)[N], float* smem, int warps) {
#pragma unroll
  for (int m = 16; m > 0; m >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], m);
  if (warps == 1) return;
  const int warp = threadIdx.x / 32;
  __syncthreads();  // the previous sums have been read
  if (threadIdx.x % 32 == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) smem[i * 32 + warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += smem[i * 32 + w];
}

template <typename TR, typename TY>
__global__ void __launch_bounds__(1024)
norm_bwd_kernel(const __grid_constant__ NormBwdParams p) {
  __shared__ float smem[2 * 32];
  pdl_trigger();
  pdl_wait();
  const int c = threadIdx.x * 8;
  const bool on = c < p.dim;
  const int warps = blockDim.x / 32;
  const float inv_dim = 1.f / (float)p.dim;
  const bool has_y = p.y != nullptr, has_h = p.dh != nullptr;

  float w_pre[8], w_post[8];
  if (on) {
    load8_or(p.pre_weight, c, 1.f, w_pre);
    load8_or(p.post == kNormNone ? nullptr : p.post_weight, c, 1.f, w_post);
  }
  float d_pre[8], d_post[8];  // weight gradients over all groups of the CTA
#pragma unroll
  for (int e = 0; e < 8; ++e) d_pre[e] = d_post[e] = 0.f;

  // The CTA's groups: one slice of one group, or several whole groups.
  const int64_t g0 = p.slices > 1 ? blockIdx.x / p.slices
                                  : (int64_t)blockIdx.x * p.cta_groups;
  const int64_t g1 =
      p.slices > 1 ? g0 + 1 : min(g0 + p.cta_groups, p.all_groups);
  const int slice = p.slices > 1 ? (int)(blockIdx.x % p.slices) : 0;
  for (int64_t g = g0; g < g1; ++g) {
    const int64_t t0 = slice * p.group_tokens / p.slices;
    const int64_t t1 = (slice + 1) * p.group_tokens / p.slices;
    float gate[8], sc[8];
    float sum_a[8], sum_c[8], sum_e[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum_a[e] = sum_c[e] = sum_e[e] = 0.f;
    if (on) {
      load8_or(p.gate, g * p.dim + c, 1.f, gate);
      load8_or(p.scale, g * p.dim + c, 0.f, sc);
    }
    for (int64_t t = t0; t < t1; ++t) {
      const int64_t at = (g * p.group_tokens + t) * p.dim + c;
      float d[8], dh[8], n[8], u[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = dh[e] = n[e] = u[e] = 0.f;
      if (on) {
        if (p.dr != nullptr) {
          Raw8<TR> v;
          v.load(p.dr, at);
          v.widen(d);
        }
        if (has_h) {
          Raw8<TY> v;
          v.load(p.dh, at);
          v.widen(dh);
          Raw8<TR> q;
          q.load(p.r, at);
          q.widen(n);
        }
        if (has_y) {
          Raw8<TY> v;
          v.load(p.y, at);
          v.widen(u);
        }
      }
      const bool post = has_y && p.post != kNormNone;
      // means of r and y
      float s[2] = {0.f, 0.f};
      if ((has_h && p.pre == kNormLayer) || (post && p.post == kNormLayer)) {
        s[0] = p.pre == kNormLayer ? sum8(n) : 0.f;
        s[1] = post && p.post == kNormLayer ? sum8(u) : 0.f;
        cta_sum(s, smem, warps);
        if (on) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            n[e] -= s[0] * inv_dim;
            u[e] -= s[1] * inv_dim;
          }
        }
      }
      float rho = 1.f, rho_y = 1.f;
      if (has_h || post) {
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[0] = fmaf(n[e], n[e], s[0]);
          s[1] = fmaf(u[e], u[e], s[1]);
        }
        cta_sum(s, smem, warps);
        rho = rsqrtf(s[0] * inv_dim + p.eps);
        if (post) rho_y = rsqrtf(s[1] * inv_dim + p.eps);
      }
      if (has_h) {
        float dn[8];
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          n[e] *= rho;
          dn[e] = on ? dh[e] * (1.f + sc[e]) * w_pre[e] : 0.f;
          s[0] += dn[e];
          s[1] = fmaf(dn[e], n[e], s[1]);
          sum_a[e] = fmaf(dh[e], n[e], sum_a[e]);
          sum_c[e] += dh[e];
        }
        cta_sum(s, smem, warps);
        const float m0 = p.pre == kNormLayer ? s[0] * inv_dim : 0.f;
        const float m1 = s[1] * inv_dim;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          d[e] = fmaf(rho, dn[e] - m0 - n[e] * m1, d[e]);
      }
      if (on) {
        float dx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[e] = p.residual_scale * d[e];
        store8(static_cast<TR*>(p.dx), at, dx);
      }
      if (has_y) {
        float du[8];
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= rho_y;
          sum_e[e] = fmaf(d[e], u[e], sum_e[e]);
          du[e] = on ? d[e] * gate[e] * w_post[e] : 0.f;
          s[0] += du[e];
          s[1] = fmaf(du[e], u[e], s[1]);
        }
        if (post) {
          cta_sum(s, smem, warps);
          const float m0 = p.post == kNormLayer ? s[0] * inv_dim : 0.f;
          const float m1 = s[1] * inv_dim;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            du[e] = rho_y * (du[e] - m0 - u[e] * m1);
        }
        if (on) store8(static_cast<TY*>(p.dy), at, du);
      }
    }
    if (on) {
      if (p.slices > 1) {
        float* part = p.partial + (int64_t)blockIdx.x * 3 * p.dim + c;
        store8(part, 0, sum_a);
        store8(part, p.dim, sum_c);
        store8(part, 2 * p.dim, sum_e);
      } else {
        float o[8];
        if (p.dshift != nullptr) store8(p.dshift, g * p.dim + c, sum_c);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = sum_a[e] * w_pre[e];
        if (p.dscale != nullptr) store8(p.dscale, g * p.dim + c, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = has_y ? sum_e[e] * w_post[e] : 0.f;
        if (p.dgate != nullptr) store8(p.dgate, g * p.dim + c, o);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        d_pre[e] = fmaf(1.f + sc[e], sum_a[e], d_pre[e]);
        d_post[e] = fmaf(gate[e], sum_e[e], d_post[e]);
      }
    }
  }
  if (on && p.weight_partial != nullptr) {
    float* part = p.weight_partial + (int64_t)blockIdx.x * 2 * p.dim + c;
    store8(part, 0, d_pre);
    store8(part, p.dim, d_post);
  }
}

// Adds the CTAs' partial sums up, in order.  blockIdx.y < all_groups: one
// group's slices into dscale, dshift and dgate; the last one or two
// blockIdx.y: every CTA's share of a weight gradient.  A CTA takes 32
// columns; its 8 warps take every eighth partial row.
constexpr int kSumThreads = 256;

__global__ void __launch_bounds__(kSumThreads)
norm_bwd_sum_kernel(const __grid_constant__ NormBwdParams p) {
  __shared__ float smem[3][8][33];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int c = blockIdx.x * 32 + lane;
  const bool on = c < p.dim;
  const int64_t group_jobs = p.slices > 1 ? p.all_groups : 0;
  const int64_t job = (int64_t)blockIdx.y + (int64_t)blockIdx.z * 65535;
  if (job >= group_jobs + 2) return;
  float s[3] = {0.f, 0.f, 0.f};
  if (job < group_jobs) {
    if (on)
      for (int i = warp; i < p.slices; i += 8) {
        const float* part =
            p.partial + (job * p.slices + i) * 3 * (int64_t)p.dim + c;
#pragma unroll
        for (int q = 0; q < 3; ++q) s[q] += part[(int64_t)q * p.dim];
      }
  } else {
    float* out = job == group_jobs ? p.dpre_weight : p.dpost_weight;
    if (out == nullptr) return;
    if (on)
      for (int64_t i = warp; i < p.ctas; i += 8)
        s[0] += p.weight_partial[(i * 2 + (job - group_jobs)) * p.dim + c];
  }
#pragma unroll
  for (int q = 0; q < 3; ++q) smem[q][warp][lane] = s[q];
  __syncthreads();
  if (warp != 0 || !on) return;
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    s[q] = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s[q] += smem[q][w][lane];
  }
  if (job < group_jobs) {
    const int64_t o = job * p.dim + c;
    const float w_pre = p.pre_weight ? p.pre_weight[c] : 1.f;
    const float w_post =
        p.post != kNormNone && p.post_weight ? p.post_weight[c] : 1.f;
    if (p.dscale != nullptr) p.dscale[o] = s[0] * w_pre;
    if (p.dshift != nullptr) p.dshift[o] = s[1];
    if (p.dgate != nullptr) p.dgate[o] = s[2] * w_post;
  } else {
    (job == group_jobs ? p.dpre_weight : p.dpost_weight)[c] = s[0];
  }
}

}  // namespace

// How the rows are shared out: groups are cut into slices when there are
// fewer of them than CTAs wanted, else a CTA takes several whole groups.
NormBwdSplit norm_bwd_split(int64_t all_groups, int64_t group_tokens, int sms) {
  NormBwdSplit s;
  const int64_t want = (int64_t)sms * 3;
  s.slices = 1;
  s.cta_groups = 1;
  if (all_groups < want) {
    int64_t n = want / all_groups;
    if (n > group_tokens) n = group_tokens;
    s.slices = (int32_t)n;
    s.ctas = all_groups * n;
  } else {
    s.cta_groups = (all_groups + want - 1) / want;
    s.ctas = (all_groups + s.cta_groups - 1) / s.cta_groups;
  }
  return s;
}

cudaError_t launch_norm_bwd(const NormBwdParams& p, bool res_f32,
                            bool block_f32, cudaStream_t stream) {
  using B = __nv_bfloat16;
  const dim3 grid((unsigned)p.ctas), block((p.dim / 8 + 31) / 32 * 32);
  cudaError_t e;
  if (res_f32)
    e = block_f32
            ? launch_pdl(norm_bwd_kernel<float, float>, grid, block, 0, stream, p)
            : launch_pdl(norm_bwd_kernel<float, B>, grid, block, 0, stream, p);
  else
    e = block_f32
            ? launch_pdl(norm_bwd_kernel<B, float>, grid, block, 0, stream, p)
            : launch_pdl(norm_bwd_kernel<B, B>, grid, block, 0, stream, p);
  if (e != cudaSuccess) return e;
  const bool sums = p.slices > 1 && (p.dscale || p.dshift || p.dgate);
  if (!sums && p.weight_partial == nullptr) return cudaSuccess;
  const int64_t jobs = (p.slices > 1 ? p.all_groups : 0) + 2;
  const dim3 grid2((p.dim + 31) / 32,
                   (unsigned)(jobs < 65535 ? jobs : 65535),
                   (unsigned)((jobs + 65534) / 65535));
  return launch_pdl(norm_bwd_sum_kernel, grid2, dim3(kSumThreads), 0, stream,
                    p);
}

}  // namespace fastvr
