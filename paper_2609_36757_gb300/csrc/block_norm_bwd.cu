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
// per element with a float32 residual stream).  A thread owns the same columns
// of all the rows that its CTA takes, so A, C and E are its own and every token
// sum has a fixed order; the next row is loaded while a row's eight sums go
// across the CTA in three exchanges, whose latency is what is left: 73.7 us
// (4.6 TB/s) for 12288 rows of 1536 with a float32 residual.
#include "block_norm.cuh"

namespace fastvr {
namespace {

using namespace norm;

// The four inputs of a row, 8 columns of each.
template <typename TR, typename TY>
struct RowIn {
  Raw8<TR> dr, r;
  Raw8<TY> dh, y;
};

// The end of a group in a CTA: sums over its tokens of 8 columns into a partial
// result or the group's gradients, and their share of the weight gradients into
// dyn [2][dim].
__device__ __forceinline__ void end_group(const NormBwdParams& p, int64_t g,
                                          int c, const F8& sum_a,
                                          const F8& sum_c, const F8& sum_e,
                                          float* dyn) {
  const int64_t gc = g * p.dim + c;
  if (p.slices > 1) {
    float* part = p.partial + (int64_t)blockIdx.x * 3 * p.dim + c;
    store8(part, 0, sum_a);
    store8(part, p.dim, sum_c);
    store8(part, 2 * p.dim, sum_e);
  } else {
    if (p.dshift != nullptr) store8(p.dshift, gc, sum_c);
    if (p.dscale != nullptr)
      store8(p.dscale, gc, mul(sum_a, load8_or(p.pre_weight, c, 1.f)));
    if (p.dgate != nullptr)
      store8(p.dgate, gc,
             mul(sum_e,
                 load8_or(p.post == kNormNone ? nullptr : p.post_weight, c,
                          1.f)));
  }
  if (p.weight_partial != nullptr) {
    store8(dyn, c,
           fma(add(load8_or(p.scale, gc, 0.f), splat(1.f)), sum_a,
               load8_or(dyn, c, 0.f)));
    store8(dyn, p.dim + c,
           fma(load8_or(p.gate, gc, 1.f), sum_e,
               load8_or(dyn, p.dim + c, 0.f)));
  }
}

template <typename TR, typename TY, int TPR, int NV, bool kAhead, bool kRegs,
          int kMinCtas>
__global__ void __launch_bounds__(Shape<TPR>::kThreads, kMinCtas)
norm_bwd_kernel(const __grid_constant__ NormBwdParams p) {
  using S = Shape<TPR>;
  constexpr int kRows = S::kRows;
  // mine: gate post_weight (j), (1 + scale) pre_weight (NV + j), and the sums
  // over tokens A, C, E ((2, 3, 4) NV + j); then [2][dim] weight sums
  extern __shared__ float4 dyn4[];
  Kept<kRegs, 5 * NV> mine;
  mine.m = Private{dyn4};
  static_assert(!kRegs || S::kRows == 1, "rows side by side are added there");
  float* dyn = reinterpret_cast<float*>(
      dyn4 + (kRegs ? 0 : 10 * NV * S::kThreads));
  __shared__ float4 s_stat[S::kWarps];
  __shared__ float2 s_dn[S::kWarps], s_du[S::kWarps];
  __shared__ float s_n[S::kWarps];
  pdl_trigger();
  const Cols<TPR, NV> k(p.dim, s_n);
  const float inv_dim = k.inv_dim;
  const int slot = kRows > 1 ? threadIdx.x / TPR : 0;
  const bool has_y = p.y != nullptr, has_h = p.dh != nullptr;
  const bool has_dr = p.dr != nullptr;
  const bool post = has_y && p.post != kNormNone;
  const bool mean_r = has_h && p.pre == kNormLayer;
  const bool mean_y = post && p.post == kNormLayer;
  const bool weights = p.weight_partial != nullptr;
  if (weights && slot == 0)
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (k.on(j)) {
        store8(dyn, k.at(j), splat(0.f));
        store8(dyn, p.dim + k.at(j), splat(0.f));
      }
  pdl_wait();

  // The CTA's groups: one slice of one group, or several whole groups.
  const int64_t g0 = p.slices > 1 ? blockIdx.x / p.slices
                                  : (int64_t)blockIdx.x * p.cta_groups;
  const int64_t g1 =
      p.slices > 1 ? g0 + 1 : min(g0 + p.cta_groups, p.all_groups);
  const int slice = p.slices > 1 ? (int)(blockIdx.x % p.slices) : 0;
  const int64_t t0 = slice * p.group_tokens / p.slices;
  const int64_t t1 = (slice + 1) * p.group_tokens / p.slices;

  RowIn<TR, TY> in[NV];
  auto fetch = [&](int64_t g, int64_t t) {
    if (t >= t1) return;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (k.on(j)) {
        const int64_t at = (g * p.group_tokens + t) * p.dim + k.at(j);
        if (has_dr) in[j].dr.load(p.dr, at);
        if (has_h) {
          in[j].dh.load(p.dh, at);
          in[j].r.load(p.r, at);
        }
        if (has_y) in[j].y.load(p.y, at);
      }
  };
  if (kAhead) fetch(g0, t0 + slot);
  for (int64_t g = g0; g < g1; ++g) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      F8 gp = splat(0.f), sw = gp;
#pragma unroll
      for (int q = 2; q < 5; ++q) mine.set(q * NV + j, gp);
      if (k.on(j)) {
        const int64_t at = g * p.dim + k.at(j);
        gp = mul(load8_or(p.gate, at, 1.f),
                 load8_or(p.post == kNormNone ? nullptr : p.post_weight,
                          k.at(j), 1.f));
        sw = mul(add(load8_or(p.scale, at, 0.f), splat(1.f)),
                 load8_or(p.pre_weight, k.at(j), 1.f));
      }
      mine.set(j, gp);
      mine.set(NV + j, sw);
    }
    // Every thread makes every pass (barriers and shuffles inside); a slot
    // past the last row works on zeros.
    for (int64_t tb = t0; tb < t1; tb += kRows) {
      const int64_t t = tb + slot;
      if (!kAhead) fetch(g, t);
      F8 d[NV], dh[NV], n[NV], u[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bool on = t < t1 && k.on(j);
        d[j] = on && has_dr ? in[j].dr.widen() : splat(0.f);
        dh[j] = on && has_h ? in[j].dh.widen() : splat(0.f);
        n[j] = on && has_h ? in[j].r.widen() : splat(0.f);
        u[j] = on && has_y ? in[j].y.widen() : splat(0.f);
      }
      // the next row is on its way while this one is worked on
      if (kAhead && tb + kRows < t1)
        fetch(g, t + kRows);
      else if (kAhead && g + 1 < g1)
        fetch(g + 1, t0 + slot);

      float rho = 1.f, rho_y = 1.f;
      if (has_h || post) {
        const Stats st = row_stats<TPR, NV>(n, u, mean_r, mean_y, k, s_stat);
        rho = rsqrtf(st.sq_a * inv_dim + p.eps);
        if (post) rho_y = rsqrtf(st.sq_b * inv_dim + p.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (t < t1 && k.on(j)) {
            n[j] = fma(n[j], rho, -st.mu_a * rho);
            u[j] = fma(u[j], rho_y, -st.mu_b * rho_y);
          }
      }
      if (has_h) {
        F8 s0 = splat(0.f), s1 = s0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          mine.set(2 * NV + j, fma(dh[j], n[j], mine.get(2 * NV + j)));
          mine.set(3 * NV + j, add(dh[j], mine.get(3 * NV + j)));
          dh[j] = mul(dh[j], mine.get(NV + j));
          s0 = add(s0, dh[j]);
          s1 = fma(dh[j], n[j], s1);
        }
        float m0 = sum(s0), m1 = sum(s1);
        row_sums<TPR>(m0, m1, s_dn);
        m0 = p.pre == kNormLayer ? -m0 * inv_dim : 0.f;
        m1 *= -inv_dim;
#pragma unroll
        for (int j = 0; j < NV; ++j)
          d[j] = fma(fma(n[j], m1, add(dh[j], splat(m0))), rho, d[j]);
      }
      const int64_t at = (g * p.group_tokens + t) * p.dim;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (t < t1 && k.on(j))
          store8(static_cast<TR*>(p.dx), at + k.at(j),
                 mul(d[j], p.residual_scale));
      if (has_y) {
        F8 s0 = splat(0.f), s1 = s0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          mine.set(4 * NV + j, fma(d[j], u[j], mine.get(4 * NV + j)));
          d[j] = mul(d[j], mine.get(j));
          s0 = add(s0, d[j]);
          s1 = fma(d[j], u[j], s1);
        }
        if (post) {
          float m0 = sum(s0), m1 = sum(s1);
          row_sums<TPR>(m0, m1, s_du);
          m0 = p.post == kNormLayer ? -m0 * inv_dim : 0.f;
          m1 *= -inv_dim;
#pragma unroll
          for (int j = 0; j < NV; ++j)
            d[j] = mul(fma(u[j], m1, add(d[j], splat(m0))), rho_y);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (t < t1 && k.on(j))
            store8(static_cast<TY*>(p.dy), at + k.at(j), d[j]);
      }
    }

    // The group's sums: over the rows side by side, then to memory.
    if (kRows > 1) __syncthreads();
    if (slot == 0)
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (k.on(j)) {
          F8 sums[3];
#pragma unroll
          for (int q = 0; q < 3; ++q) {
            sums[q] = mine.get((2 + q) * NV + j);
#pragma unroll
            for (int r = 1; r < kRows; ++r)
              sums[q] = add(sums[q], Private{dyn4 + r * TPR}.get(
                                         (2 + q) * NV + j));
          }
          end_group(p, g, k.at(j), sums[0], sums[1], sums[2], dyn);
        }
    if (kRows > 1) __syncthreads();  // before the next group's zeros
  }
  if (weights && slot == 0) {
    float* part = p.weight_partial + (int64_t)blockIdx.x * 2 * p.dim;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (k.on(j)) {
        store8(part, k.at(j), load8_or(dyn, k.at(j), 0.f));
        store8(part, p.dim + k.at(j), load8_or(dyn, p.dim + k.at(j), 0.f));
      }
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

// CTAs per SM of the kernel that dim selects, see launch_t.
int ctas_per_sm(int dim) {
  return dim <= 256 ? 4 : dim <= 512 ? 5 : dim <= 1024 ? 3 : dim <= 2048 ? 2 : 1;
}

template <typename TR, typename TY, int TPR, int NV, bool kAhead, bool kRegs,
          int kMinCtas>
cudaError_t launch_v(const NormBwdParams& p, cudaStream_t stream) {
  const size_t smem =
      (kRegs ? 0 : (size_t)10 * NV * Shape<TPR>::kThreads * sizeof(float4)) +
      (p.weight_partial != nullptr ? (size_t)2 * p.dim * sizeof(float) : 0);
  auto kernel = norm_bwd_kernel<TR, TY, TPR, NV, kAhead, kRegs, kMinCtas>;
  if (smem > 32768) {  // up to 224 KB at dim 8192
    const cudaError_t e = cudaFuncSetAttribute(
        kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kernel, dim3((unsigned)p.ctas),
                    dim3(Shape<TPR>::kThreads), smem, stream, p);
}

// Threads and vectors of a row, whether its sums stay in registers, and CTAs
// per SM: what was fastest of those that do not spill (12288 rows of 1536 with
// a float32 residual: 96 threads of 16 columns 73.7 us, 192 of 8 76.1, the
// same with the sums in shared memory 82; one more CTA per SM at the price of
// spills 115 and more).  With groups of a few rows, whose ends then count, 192
// threads of 8 columns: 84.8 us for 8160 groups of one row, against 120.9.
template <typename TR, typename TY>
cudaError_t launch_t(const NormBwdParams& p, cudaStream_t stream) {
  if (p.dim <= 64) return launch_v<TR, TY, 8, 1, true, false, 4>(p, stream);
  if (p.dim <= 128) return launch_v<TR, TY, 16, 1, true, false, 4>(p, stream);
  if (p.dim <= 256) return launch_v<TR, TY, 32, 1, true, false, 4>(p, stream);
  if (p.dim <= 512) return launch_v<TR, TY, 64, 1, true, true, 5>(p, stream);
  if (p.dim <= 1024) return launch_v<TR, TY, 128, 1, true, true, 3>(p, stream);
  if (p.dim <= 1536 && p.group_tokens < 16)
    return launch_v<TR, TY, 192, 1, true, true, 2>(p, stream);
  if (p.dim <= 1536) return launch_v<TR, TY, 96, 2, true, true, 2>(p, stream);
  if (p.dim <= 2048) return launch_v<TR, TY, 256, 1, true, false, 2>(p, stream);
  if (p.dim <= 4096) return launch_v<TR, TY, 256, 2, true, false, 1>(p, stream);
  if (p.dim <= 5120) return launch_v<TR, TY, 320, 2, true, false, 1>(p, stream);
  return launch_v<TR, TY, 1024, 1, false, false, 1>(p, stream);
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
