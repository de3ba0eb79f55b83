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
// every token sum has a fixed order; the next row is loaded while a row's eight
// sums go across the CTA in three exchanges.
#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

// The four inputs of a row, a thread's 8 columns of each.
template <typename TR, typename TY>
struct RowIn {
  Raw8<TR> dr, r;
  Raw8<TY> dh, y;
};

template <typename TR, typename TY, int TPR, int kMinCtas>
__global__ void __launch_bounds__(Shape<TPR>::kThreads, kMinCtas)
norm_bwd_kernel(const __grid_constant__ NormBwdParams p) {
  using S = Shape<TPR>;
  constexpr int kRows = S::kRows;
  extern __shared__ __align__(16) float dyn[];  // [2][dim] weight sums
  __shared__ float4 s_stat[S::kWarps];
  __shared__ float2 s_dn[S::kWarps], s_du[S::kWarps];
  __shared__ __align__(16) float s_fold[kRows > 1 ? 3 * 8 * 128 : 4];
  pdl_trigger();
  pdl_wait();
  const Cols k = make_cols<TPR>(p.dim);
  const int c = k.c;
  const bool on = k.on;
  const float inv_dim = k.inv_dim;
  const int slot = kRows > 1 ? threadIdx.x / TPR : 0;
  const bool has_y = p.y != nullptr, has_h = p.dh != nullptr;
  const bool has_dr = p.dr != nullptr;
  const bool post = has_y && p.post != kNormNone;
  const bool mean_r = has_h && p.pre == kNormLayer;
  const bool mean_y = post && p.post == kNormLayer;
  const bool weights = p.weight_partial != nullptr;
  if (weights && slot == 0 && on) {
    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    store8(dyn, c, zero);
    store8(dyn, p.dim + c, zero);
  }

  // The CTA's groups: one slice of one group, or several whole groups.
  const int64_t g0 = p.slices > 1 ? blockIdx.x / p.slices
                                  : (int64_t)blockIdx.x * p.cta_groups;
  const int64_t g1 =
      p.slices > 1 ? g0 + 1 : min(g0 + p.cta_groups, p.all_groups);
  const int slice = p.slices > 1 ? (int)(blockIdx.x % p.slices) : 0;
  const int64_t t0 = slice * p.group_tokens / p.slices;
  const int64_t t1 = (slice + 1) * p.group_tokens / p.slices;

  RowIn<TR, TY> in;
  auto fetch = [&](int64_t g, int64_t t) {
    if (!on || t >= t1) return;
    const int64_t at = (g * p.group_tokens + t) * p.dim + c;
    if (has_dr) in.dr.load(p.dr, at);
    if (has_h) {
      in.dh.load(p.dh, at);
      in.r.load(p.r, at);
    }
    if (has_y) in.y.load(p.y, at);
  };
  fetch(g0, t0 + slot);
  for (int64_t g = g0; g < g1; ++g) {
    float gp[8], sw[8];  // gate post_weight, (1 + scale) pre_weight
    float sum_a[8], sum_c[8], sum_e[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      sum_a[e] = sum_c[e] = sum_e[e] = gp[e] = sw[e] = 0.f;
    if (on) {
      float x[8];
      load8_or(p.gate, g * p.dim + c, 1.f, gp);
      load8_or(p.post == kNormNone ? nullptr : p.post_weight, c, 1.f, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) gp[e] *= x[e];
      load8_or(p.scale, g * p.dim + c, 0.f, sw);
      load8_or(p.pre_weight, c, 1.f, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sw[e] = (1.f + sw[e]) * x[e];
    }
    // Every thread makes every pass (barriers and shuffles inside); a slot
    // past the last row works on zeros.
    for (int64_t tb = t0; tb < t1; tb += kRows) {
      const int64_t t = tb + slot;
      const bool row_on = on && t < t1;
      float d[8], dh[8], n[8], u[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = dh[e] = n[e] = u[e] = 0.f;
      if (row_on) {
        if (has_dr) in.dr.widen(d);
        if (has_h) {
          in.dh.widen(dh);
          in.r.widen(n);
        }
        if (has_y) in.y.widen(u);
      }
      // the next row is on its way while this one is worked on
      if (tb + kRows < t1)
        fetch(g, t + kRows);
      else if (g + 1 < g1)
        fetch(g + 1, t0 + slot);

      float rho = 1.f, rho_y = 1.f;
      if (has_h || post) {
        const Stats st = row_stats<TPR>(n, u, mean_r, mean_y, k, s_stat);
        rho = rsqrtf(st.sq_a * inv_dim + p.eps);
        if (post) rho_y = rsqrtf(st.sq_b * inv_dim + p.eps);
        if (row_on) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            n[e] = (n[e] - st.mu_a) * rho;
            u[e] = (u[e] - st.mu_b) * rho_y;
          }
        }
      }
      if (has_h) {
        float dn[8], s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dn[e] = dh[e] * sw[e];
          s0 += dn[e];
          s1 = fmaf(dn[e], n[e], s1);
          sum_a[e] = fmaf(dh[e], n[e], sum_a[e]);
          sum_c[e] += dh[e];
        }
        row_sums<TPR>(s0, s1, k, s_dn);
        const float m0 = p.pre == kNormLayer ? s0 * inv_dim : 0.f;
        const float m1 = s1 * inv_dim;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          d[e] = fmaf(rho, dn[e] - m0 - n[e] * m1, d[e]);
      }
      const int64_t at = (g * p.group_tokens + t) * p.dim + c;
      if (row_on) {
        float dx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[e] = p.residual_scale * d[e];
        store8(static_cast<TR*>(p.dx), at, dx);
      }
      if (has_y) {
        float du[8], s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum_e[e] = fmaf(d[e], u[e], sum_e[e]);
          du[e] = d[e] * gp[e];
          s0 += du[e];
          s1 = fmaf(du[e], u[e], s1);
        }
        if (post) {
          row_sums<TPR>(s0, s1, k, s_du);
          const float m0 = p.post == kNormLayer ? s0 * inv_dim : 0.f;
          const float m1 = s1 * inv_dim;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            du[e] = rho_y * (du[e] - m0 - u[e] * m1);
        }
        if (row_on) store8(static_cast<TY*>(p.dy), at, du);
      }
    }

    // The group's sums: over the rows side by side, then to memory.
    if constexpr (kRows > 1) {
      __syncthreads();  // the previous group's sums have been read
      store8(s_fold, threadIdx.x * 8, sum_a);
      store8(s_fold, 1024 + threadIdx.x * 8, sum_c);
      store8(s_fold, 2048 + threadIdx.x * 8, sum_e);
      __syncthreads();
      if (slot == 0) {
#pragma unroll
        for (int r = 1; r < kRows; ++r) {
          float x[8];
          load8_or(s_fold, r * TPR * 8 + c, 0.f, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum_a[e] += x[e];
          load8_or(s_fold, 1024 + r * TPR * 8 + c, 0.f, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum_c[e] += x[e];
          load8_or(s_fold, 2048 + r * TPR * 8 + c, 0.f, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum_e[e] += x[e];
        }
      }
    }
    if (on && slot == 0) {
      float x[8], w[8];
      if (p.slices > 1) {
        float* part = p.partial + (int64_t)blockIdx.x * 3 * p.dim + c;
        store8(part, 0, sum_a);
        store8(part, p.dim, sum_c);
        store8(part, 2 * p.dim, sum_e);
      } else {
        if (p.dshift != nullptr) store8(p.dshift, g * p.dim + c, sum_c);
        load8_or(p.pre_weight, c, 1.f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sum_a[e] * w[e];
        if (p.dscale != nullptr) store8(p.dscale, g * p.dim + c, x);
        load8_or(p.post == kNormNone ? nullptr : p.post_weight, c, 1.f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sum_e[e] * w[e];
        if (p.dgate != nullptr) store8(p.dgate, g * p.dim + c, x);
      }
      if (weights) {
        load8_or(p.scale, g * p.dim + c, 0.f, w);
        load8_or(dyn, c, 0.f, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(1.f + w[e], sum_a[e], x[e]);
        store8(dyn, c, x);
        load8_or(p.gate, g * p.dim + c, 1.f, w);
        load8_or(dyn, p.dim + c, 0.f, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(w[e], sum_e[e], x[e]);
        store8(dyn, p.dim + c, x);
      }
    }
  }
  if (weights && on && slot == 0) {
    float* part = p.weight_partial + (int64_t)blockIdx.x * 2 * p.dim + c;
    float x[8];
    load8_or(dyn, c, 0.f, x);
    store8(part, 0, x);
    load8_or(dyn, p.dim + c, 0.f, x);
    store8(part, p.dim, x);
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

// CTAs per SM: the registers of a thread (8 columns of
// every input, the sums) want about 112 of them, up to 2048 columns.
int ctas_per_sm(int dim) {
  const int n = row_threads(dim);
  return n <= 32 ? 4 : n <= 64 ? 8 : n <= 128 ? 4 : n <= 192 ? 3
                                   : n <= 256 ? 2 : 1;
}

template <typename TR, typename TY>
cudaError_t launch_t(const NormBwdParams& p, cudaStream_t stream) {
  const dim3 grid((unsigned)p.ctas);
  const size_t smem =
      p.weight_partial != nullptr ? (size_t)2 * p.dim * sizeof(float) : 0;
  const int n = row_threads(p.dim);
  const dim3 block(n <= 32 ? 128 : n);
  if (n == 8)
    return launch_pdl(norm_bwd_kernel<TR, TY, 8, 4>, grid, block, smem, stream, p);
  if (n == 16)
    return launch_pdl(norm_bwd_kernel<TR, TY, 16, 4>, grid, block, smem, stream, p);
  if (n == 32)
    return launch_pdl(norm_bwd_kernel<TR, TY, 32, 4>, grid, block, smem, stream, p);
  if (n <= 64)
    return launch_pdl(norm_bwd_kernel<TR, TY, 64, 8>, grid, block, smem, stream, p);
  if (n <= 128)
    return launch_pdl(norm_bwd_kernel<TR, TY, 128, 4>, grid, block, smem, stream, p);
  if (n <= 192)
    return launch_pdl(norm_bwd_kernel<TR, TY, 192, 3>, grid, block, smem, stream, p);
  if (n <= 256)
    return launch_pdl(norm_bwd_kernel<TR, TY, 256, 2>, grid, block, smem, stream, p);
  if (n <= 512)
    return launch_pdl(norm_bwd_kernel<TR, TY, 512, 1>, grid, block, smem, stream, p);
  // 64 KB of weight sums at dim 8192
  auto kernel = norm_bwd_kernel<TR, TY, 1024, 1>;
  const cudaError_t e = cudaFuncSetAttribute(
      kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * 8192 * 4);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, grid, block, smem, stream, p);
}

}  // namespace

// How the rows are shared out: groups are cut into slices when there are
// fewer of them than CTAs wanted, else a CTA takes several whole groups.
NormBwdSplit norm_bwd_split(int64_t all_groups, int64_t group_tokens, int dim,
                            int sms) {
  NormBwdSplit s;
  const int64_t want = (int64_t)sms * ctas_per_sm(dim);
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
  const cudaError_t e =
      res_f32 ? (block_f32 ? launch_t<float, float>(p, stream)
                           : launch_t<float, B>(p, stream))
              : (block_f32 ? launch_t<B, float>(p, stream)
                           : launch_t<B, B>(p, stream));
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
