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
// d is not needed for the sums that J_post takes over it: with s(.) a sum over
// the row and w = gate post_weight n(y),
//   s(d w) = s(dr w) + rho (s(dn w) + m0 s(w) + m1 s(n(r) w)),
//   m0 = -mean(dn), m1 = -mean(dn n(r)),
// so a row needs one exchange between its warps: of up to twelve sums and two
// means, each taken about the warp's own mean and moved when they are put
// together.
//
// Bound by memory: dr, dh, r, y are read once, dx, dy written once (18 bytes
// per element with a float32 residual stream).  A thread owns the same columns
// of all the rows that its CTA takes, so A, C and E are its own and every token
// sum has a fixed order.  The slices of a group take its rows in turn, so that
// neighbours in memory are asked for together.  72.0 us (4.7 TB/s) for 12288
// rows of 1536 with a float32 residual, layer norm and RMS post norm; three
// exchanges, one after the other, took 73.7, and 88.6 instead of 80.9 for 3600
// rows of 5120.  With a bfloat16 residual, a third of the bytes less, it gains
// 2 to 12 % up to 2048 columns and loses at 1536 and 5120 (93.6 and 93.5 us
// against 74.5 and 81.5 in the same run; the cause is not known).  These and
// the times below are of calls replayed from a graph, a few per cent below a
// call's own.
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

// What a row's gradients need of all its columns, with r and y less their means
// where the norm takes them off, dn = dh (1 + scale) pre_weight, gp = gate
// post_weight and w = gp y: sums of r r, y y, dn r, dn, dr w, dn w, r w, w, and
// for a post norm with a mean of dr gp, dn gp, r gp, gp.
struct RowSums {
  float mu_r, mu_y, rr, yy, dn_r, dn, dr_w, dn_w, r_w, w, dr_g, dn_g, r_g, g;
};

// Means over the row's columns in this warp.
template <int TPR, int NV>
__device__ __forceinline__ void warp_means(const F8 (&r)[NV], const F8 (&y)[NV],
                                           const Cols<TPR, NV>& k, float& mu_r,
                                           float& mu_y) {
  F8 a = r[0], b = y[0];
#pragma unroll
  for (int i = 1; i < NV; ++i) {
    a = add(a, r[i]);
    b = add(b, y[i]);
  }
  mu_r = sum(a);
  mu_y = sum(b);
  both_sums<Shape<TPR>::kLanes>(mu_r, mu_y);
  mu_r *= k.inv_warp;
  mu_y *= k.inv_warp;
}

// The sums over the row from a thread's parts (v: rr to w, v4: dr_g to g), that
// were taken about its warp's means.  One exchange: the warps' parts are moved
// to the row's means when they are put together.  `part`: not written again
// before the next exchange.
template <int TPR, int NV>
__device__ __forceinline__ RowSums row_part_sums(float (&v)[8], float (&v4)[4],
                                                 float mu_r, float mu_y,
                                                 bool mean_r, bool mean_y,
                                                 const Cols<TPR, NV>& k,
                                                 float4 (*part)[4]) {
  using S = Shape<TPR>;
  constexpr int L = S::kLanes;
  const int lane = threadIdx.x % 32;
  RowSums s = {};
  const float mine = keep_sum<L>(v);
  const float mine4 = mean_y ? keep_sum<L>(v4) : 0.f;
  if constexpr (!S::kMany) {
    const int first = lane & ~(L - 1);
    auto of = [&](float x, int lanes, int i) {
      return __shfl_sync(0xffffffffu, x, first + i * lanes);
    };
    s.mu_r = mu_r;
    s.mu_y = mu_y;
    s.rr = of(mine, L / 8, 0);
    s.yy = of(mine, L / 8, 1);
    s.dn_r = of(mine, L / 8, 2);
    s.dn = of(mine, L / 8, 3);
    s.dr_w = of(mine, L / 8, 4);
    s.dn_w = of(mine, L / 8, 5);
    s.r_w = of(mine, L / 8, 6);
    s.w = of(mine, L / 8, 7);
    if (mean_y) {
      s.dr_g = of(mine4, L / 4, 0);
      s.dn_g = of(mine4, L / 4, 1);
      s.r_g = of(mine4, L / 4, 2);
      s.g = of(mine4, L / 4, 3);
    }
  } else {
    float4* to = part[threadIdx.x / 32];
    if (lane == 0) to[0] = make_float4(mu_r, mu_y, 0.f, 0.f);
    if (lane % 4 == 0) reinterpret_cast<float*>(to + 1)[lane / 4] = mine;
    if (mean_y && lane % 8 == 0)
      reinterpret_cast<float*>(to + 3)[lane / 8] = mine4;
    __syncthreads();
    if (mean_r || mean_y) {
#pragma unroll(S::kUnroll)
      for (int i = 0; i < S::kWarps; ++i) {
        s.mu_r = fmaf(part[i][0].x, k.counts[i], s.mu_r);
        s.mu_y = fmaf(part[i][0].y, k.counts[i], s.mu_y);
      }
      s.mu_r *= k.inv_dim;
      s.mu_y *= k.inv_dim;
    }
#pragma unroll(S::kUnroll)
    for (int i = 0; i < S::kWarps; ++i) {
      const float4 a = part[i][1], b = part[i][2];
      s.rr += a.x;
      s.yy += a.y;
      s.dn_r += a.z;
      s.dn += a.w;
      s.dr_w += b.x;
      s.dn_w += b.y;
      s.r_w += b.z;
      s.w += b.w;
      if (mean_r) {
        const float by = part[i][0].x - s.mu_r;
        s.rr = fmaf(by * by, k.counts[i], s.rr);
        s.dn_r = fmaf(by, a.w, s.dn_r);
        s.r_w = fmaf(by, b.w, s.r_w);
      }
      if (mean_y) {
        const float4 c = part[i][3];
        const float by = part[i][0].y - s.mu_y;
        const float by_r = mean_r ? part[i][0].x - s.mu_r : 0.f;
        const float r_g = fmaf(by_r, c.w, c.z);
        s.yy = fmaf(by * by, k.counts[i], s.yy);
        s.dr_w = fmaf(by, c.x, s.dr_w);
        s.dn_w = fmaf(by, c.y, s.dn_w);
        s.r_w = fmaf(by, r_g, s.r_w);
        s.w = fmaf(by, c.w, s.w);
        s.dr_g += c.x;
        s.dn_g += c.y;
        s.r_g += r_g;
        s.g += c.w;
      }
    }
  }
  return s;
}

template <typename TR, typename TY, int TPR, int NV, bool kAhead, int kRegs,
          int kMinCtas>
__global__ void __launch_bounds__(Shape<TPR>::kThreads, kMinCtas)
norm_bwd_kernel(const __grid_constant__ NormBwdParams p) {
  using S = Shape<TPR>;
  constexpr int kRows = S::kRows;
  // mine: gate post_weight (j), (1 + scale) pre_weight (NV + j), and the sums
  // over tokens A, C, E ((2, 3, 4) NV + j); then [2][dim] weight sums
  extern __shared__ float4 dyn4[];
  Kept<kRegs * NV, 5 * NV> mine;
  mine.m = Private{dyn4};
  static_assert(kRegs <= 2 || S::kRows == 1,
                "rows side by side are added there");
  static_assert(kAhead || S::kRows == 1, "");
  float* dyn =
      reinterpret_cast<float*>(dyn4 + 2 * (5 - kRegs) * NV * S::kThreads);
  __shared__ float4 s_part[2][S::kWarps][4];
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
  const int64_t t0 = (int64_t)slice * kRows, step = (int64_t)p.slices * kRows;
  const int64_t t1 = p.group_tokens;

  RowIn<TR, TY> in[NV];
  // (fg, ft): the pass to load next
  int64_t fg = g0, ft = t0;
  auto fetch = [&] {
    const int64_t t = ft + slot;
    if (fg < g1 && t < t1)
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (k.on(j)) {
          const int64_t at = (fg * p.group_tokens + t) * p.dim + k.at(j);
          if (has_dr) in[j].dr.load(p.dr, at);
          if (has_h) {
            in[j].dh.load(p.dh, at);
            in[j].r.load(p.r, at);
          }
          if (has_y) in[j].y.load(p.y, at);
        }
    // without registers to load the next row ahead, at least to L2
    if (!kAhead && threadIdx.x == 0 && fg < g1 && ft + step < t1) {
      const int64_t at = (fg * p.group_tokens + ft + step) * p.dim;
      if (has_dr)
        prefetch_l2(static_cast<const TR*>(p.dr) + at, p.dim * sizeof(TR));
      if (has_h) {
        prefetch_l2(static_cast<const TR*>(p.r) + at, p.dim * sizeof(TR));
        prefetch_l2(static_cast<const TY*>(p.dh) + at, p.dim * sizeof(TY));
      }
      if (has_y)
        prefetch_l2(static_cast<const TY*>(p.y) + at, p.dim * sizeof(TY));
    }
    ft += step;
    if (ft >= t1) {
      ft = t0;
      ++fg;
    }
  };
  if (kAhead) fetch();
  int turn = 0;
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
    for (int64_t tb = t0; tb < t1; tb += step) {
      const int64_t t = tb + slot;
      if (!kAhead) fetch();
      const bool on = t < t1;
      F8 d[NV], dh[NV], n[NV], u[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bool here = on && k.on(j);
        d[j] = here && has_dr ? in[j].dr.widen() : splat(0.f);
        dh[j] = here && has_h ? in[j].dh.widen() : splat(0.f);
        n[j] = here && has_h ? in[j].r.widen() : splat(0.f);
        u[j] = here && has_y ? in[j].y.widen() : splat(0.f);
      }
      // the next row is on its way while this one is worked on
      if (kAhead) fetch();

      RowSums s = {};
      if (has_h || post) {
        float mu_r = 0.f, mu_y = 0.f;  // of this warp's columns
        if (mean_r || mean_y) warp_means<TPR, NV>(n, u, k, mu_r, mu_y);
        if (!mean_r) mu_r = 0.f;
        if (!mean_y) mu_y = 0.f;
        F2 q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = f2(0.f);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (on && k.on(j)) {
            const F8 r = add(n[j], splat(-mu_r)), y = add(u[j], splat(-mu_y));
            const F8 dn = mul(dh[j], mine.get(NV + j));
            const F8 w = mul(y, mine.get(j));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              q[0] = fma(r.v[e], r.v[e], q[0]);
              q[1] = fma(y.v[e], y.v[e], q[1]);
              q[2] = fma(dn.v[e], r.v[e], q[2]);
              q[3] = add(dn.v[e], q[3]);
              q[4] = fma(d[j].v[e], w.v[e], q[4]);
              q[5] = fma(dn.v[e], w.v[e], q[5]);
              q[6] = fma(r.v[e], w.v[e], q[6]);
              q[7] = add(w.v[e], q[7]);
            }
          }
        float v[8], v4[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sum(q[i]);
        if (mean_y) {
#pragma unroll
          for (int i = 0; i < 4; ++i) q[i] = f2(0.f);
#pragma unroll
          for (int j = 0; j < NV; ++j)
            if (on && k.on(j)) {
              const F8 gp = mine.get(j), r = add(n[j], splat(-mu_r));
              const F8 dn = mul(dh[j], mine.get(NV + j));
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                q[0] = fma(d[j].v[e], gp.v[e], q[0]);
                q[1] = fma(dn.v[e], gp.v[e], q[1]);
                q[2] = fma(r.v[e], gp.v[e], q[2]);
                q[3] = add(gp.v[e], q[3]);
              }
            }
#pragma unroll
          for (int i = 0; i < 4; ++i) v4[i] = sum(q[i]);
        }
        s = row_part_sums<TPR, NV>(v, v4, mu_r, mu_y, mean_r, mean_y, k,
                                   s_part[turn]);
        turn ^= 1;
      }
      // d = dr + rho (dn + m0 + m1 n(r)), dy = rho_y (d gp + m2 + m3 n(y))
      const float rho = rsqrtf(s.rr * inv_dim + p.eps);
      const float rho_y = post ? rsqrtf(s.yy * inv_dim + p.eps) : 1.f;
      const float m0 = mean_r ? -s.dn * inv_dim : 0.f;
      const float m1 = -s.dn_r * rho * inv_dim;
      const float m2 =
          mean_y ? -(s.dr_g + rho * (s.dn_g + m0 * s.g + m1 * rho * s.r_g)) *
                       inv_dim
                 : 0.f;
      const float m3 =
          -(s.dr_w + rho * (s.dn_w + m0 * s.w + m1 * rho * s.r_w)) * rho_y *
          inv_dim;
      const int64_t at = (g * p.group_tokens + t) * p.dim;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (has_h) {
          const F8 unit = fma(n[j], rho, -s.mu_r * rho);
          mine.set(2 * NV + j, fma(dh[j], unit, mine.get(2 * NV + j)));
          mine.set(3 * NV + j, add(dh[j], mine.get(3 * NV + j)));
          d[j] = fma(fma(unit, m1, fma(dh[j], mine.get(NV + j), splat(m0))),
                     rho, d[j]);
        }
        if (on && k.on(j))
          store8(static_cast<TR*>(p.dx), at + k.at(j),
                 mul(d[j], p.residual_scale));
        if (!has_y) continue;
        if (post) u[j] = fma(u[j], rho_y, -s.mu_y * rho_y);
        mine.set(4 * NV + j, fma(d[j], u[j], mine.get(4 * NV + j)));
        d[j] = mul(d[j], mine.get(j));
        if (post) d[j] = mul(fma(u[j], m3, add(d[j], splat(m2))), rho_y);
        if (on && k.on(j))
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
                                         (2 + q - kRegs) * NV + j));
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
    // without a post norm its weight is not used: a gradient of zeros
    if (on && (job == group_jobs || p.post != kNormNone))
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

// CTAs per SM of the kernel that is selected, see launch_t.
int ctas_per_sm(int dim, int64_t group_tokens) {
  if (dim > 1024 && dim <= 1536 && group_tokens < kFewTokens) return 3;
  return dim <= 256    ? 4
         : dim <= 512  ? 6
         : dim <= 768  ? 4
         : dim <= 1024 ? 3
         : dim <= 2048 ? 2
                       : 1;
}

template <typename TR, typename TY, int TPR, int NV, bool kAhead, int kRegs,
          int kMinCtas>
cudaError_t launch_v(const NormBwdParams& p, cudaStream_t stream) {
  const size_t smem =
      (size_t)2 * (5 - kRegs) * NV * Shape<TPR>::kThreads * sizeof(float4) +
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

// Threads and vectors of a row, whether the next row is loaded ahead, how many
// of a thread's five vectors stay in registers, CTAs per SM: what was fastest
// of those that spill nothing, or next to nothing in float32 throughout (12288
// rows of 1536 with a float32 residual: 96 threads of 16 columns 72.0 us, the
// same with all five in shared memory and four CTAs 73.5, 192 of 8 and three
// CTAs 81.8; rows ahead in shared memory 92 and more; 9000 rows of 2048: 61.7
// us, 128 threads of 16 columns 68.8, bfloat16 and RMS norms).  With groups of
// a few rows, whose ends then count, 192 threads of 8 columns: 78.5 us for 8160
// groups of one row, against 98 (bfloat16, layer norm alone).  Rows above 5120
// leave no registers to load ahead and spill some (3000 rows of 8192, bfloat16,
// RMS norms: 105.8 us; without asking for the next row in L2 128.7).  Asked for
// in L2 as well, narrower rows gain nothing.
template <typename TR, typename TY>
cudaError_t launch_t(const NormBwdParams& p, cudaStream_t stream) {
  if (p.dim <= 64) return launch_v<TR, TY, 8, 1, true, 0, 4>(p, stream);
  if (p.dim <= 128) return launch_v<TR, TY, 16, 1, true, 0, 4>(p, stream);
  if (p.dim <= 256) return launch_v<TR, TY, 32, 1, true, 0, 4>(p, stream);
  if (p.dim <= 512) return launch_v<TR, TY, 64, 1, true, 5, 6>(p, stream);
  if (p.dim <= 768) return launch_v<TR, TY, 96, 1, true, 5, 4>(p, stream);
  if (p.dim <= 1024) return launch_v<TR, TY, 128, 1, true, 5, 3>(p, stream);
  if (p.dim <= 1536 && p.group_tokens < kFewTokens)
    return launch_v<TR, TY, 192, 1, true, 0, 3>(p, stream);
  if (p.dim <= 1536) return launch_v<TR, TY, 96, 2, true, 5, 2>(p, stream);
  if (p.dim <= 2048) return launch_v<TR, TY, 256, 1, true, 3, 2>(p, stream);
  if (p.dim <= 4096) return launch_v<TR, TY, 256, 2, true, 0, 1>(p, stream);
  if (p.dim <= 5120) return launch_v<TR, TY, 320, 2, true, 0, 1>(p, stream);
  return launch_v<TR, TY, 512, 2, false, 0, 1>(p, stream);
}

}  // namespace

// How the rows are shared out: groups are cut into slices when there are
// fewer of them than CTAs wanted, else a CTA takes several whole groups.
NormBwdSplit norm_bwd_split(int64_t all_groups, int64_t group_tokens, int dim,
                            int sms) {
  NormBwdSplit s;
  const int64_t want = (int64_t)sms * ctas_per_sm(dim, group_tokens);
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
