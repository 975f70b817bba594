// Plain kernels of attention with shaped scores over packed sequences, fp32 arithmetic, any storage dtype and alignment:
//   s_ij = scale q_i.k_j,  capped c tanh(s / c),  minus slope_h |i - j|;   o_i = sum_j softmax_j(s_ij) v_j
//   dS_ij = P_ij (dO_i.v_j - delta_i) (1 - t_ij^2) scale,  dq_i = sum_j dS_ij k_j,  dk_j = sum_i dS_ij q_i,  dv_j = sum_i P_ij dO_i
// with t = tanh(s / c) (0 without a cap) and delta_i = dO_i.o_i.  One workgroup per (row, head); only pairs that count are read,
// so nothing behind a mask reaches a result, an infinity or NaN included.
#include "score.h"

namespace stg {
namespace {

constexpr int NT = 256;               // keys (queries) of one step: one per thread

__device__ __forceinline__ float wg_reduce(float v, bool is_max, float* red) {
  for (int o = 32; o > 0; o >>= 1) {
    const float t = __shfl_xor(v, o, 64);
    v = is_max ? fmaxf(v, t) : v + t;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = red[0];
  for (int i = 1; i < NT / 64; ++i) r = is_max ? fmaxf(r, red[i]) : r + red[i];
  return r;
}

template <typename T>
__global__ __launch_bounds__(NT) void score_fwd_ref_kernel(ScoreArgs a) {
  __shared__ float p[NT], qs[128], red[NT / 64];
  const int i = blockIdx.x, j = blockIdx.y, g = j / (a.h / a.hkv), t = threadIdx.x;
  SeqSpan sp;
  if (!seq_of_row(a, i, sp)) return;
  const int end = keys_end(a, sp, i);
  const float slope = a.slope ? a.slope[j] : 0.f;
  if (t < a.hd) qs[t] = to_f32(((const T*)a.q)[(int64_t)i * a.ldq + j * a.hd + t]);
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int u0 = sp.lo; u0 < end; u0 += NT) {
    const int u = u0 + t, n = min(NT, end - u0);
    __syncthreads();
    float sc = -INFINITY;
    if (t < n) {
      const T* kr = (const T*)a.k + (int64_t)u * a.ldk + g * a.hd;
      float dot = 0.f, dcap;
      for (int x = 0; x < a.hd; ++x) dot = fmaf(qs[x], to_f32(kr[x]), dot);
      sc = shaped(dot, a, slope, i - u, dcap);
    }
    const float mn = fmaxf(m, wg_reduce(sc, true, red));
    const float sub = mn == -INFINITY ? 0.f : mn, e = t < n ? expf(sc - sub) : 0.f, alpha = expf(m - sub);
    p[t] = e;
    l = l * alpha + wg_reduce(e, false, red);      // (the barriers in it publish p)
    m = mn;
    if (t < a.hd) {
      o *= alpha;
      for (int x = 0; x < n; ++x) o = fmaf(p[x], to_f32(((const T*)a.v)[(int64_t)(u0 + x) * a.ldv + g * a.hd + t]), o);
    }
  }
  if (t < a.hd) ((T*)a.o)[(int64_t)i * a.ldo + j * a.hd + t] = from_f32<T>(o / l);
  if (t == 0 && a.lse) a.lse[(int64_t)j * a.rows + i] = m + logf(l);
}

template <typename T>
__global__ __launch_bounds__(NT) void score_dq_ref_kernel(ScoreArgs a) {
  __shared__ float ds[NT], qs[128], dos[128], red[NT / 64];
  const int i = blockIdx.x, j = blockIdx.y, g = j / (a.h / a.hkv), t = threadIdx.x;
  SeqSpan sp;
  if (!seq_of_row(a, i, sp)) return;
  const int end = keys_end(a, sp, i);
  const float slope = a.slope ? a.slope[j] : 0.f, lse = a.lse[(int64_t)j * a.rows + i];
  float part = 0.f;
  if (t < a.hd) {
    qs[t] = to_f32(((const T*)a.q)[(int64_t)i * a.ldq + j * a.hd + t]);
    dos[t] = to_f32(((const T*)a.dout)[(int64_t)i * a.lddo + j * a.hd + t]);
    part = dos[t] * to_f32(((const T*)a.o)[(int64_t)i * a.ldo + j * a.hd + t]);
  }
  const float delta = wg_reduce(part, false, red);
  if (t == 0) a.delta[(int64_t)j * a.rows + i] = delta;
  float acc = 0.f;
  for (int u0 = sp.lo; u0 < end; u0 += NT) {
    const int u = u0 + t, n = min(NT, end - u0);
    __syncthreads();
    if (t < n) {
      const T* kr = (const T*)a.k + (int64_t)u * a.ldk + g * a.hd;
      const T* vr = (const T*)a.v + (int64_t)u * a.ldv + g * a.hd;
      float dot = 0.f, dp = 0.f, dcap;
      for (int x = 0; x < a.hd; ++x) { dot = fmaf(qs[x], to_f32(kr[x]), dot); dp = fmaf(dos[x], to_f32(vr[x]), dp); }
      const float sc = shaped(dot, a, slope, i - u, dcap);
      ds[t] = expf(sc - lse) * (dp - delta) * dcap;
    }
    __syncthreads();
    if (t < a.hd)
      for (int x = 0; x < n; ++x) acc = fmaf(ds[x], to_f32(((const T*)a.k)[(int64_t)(u0 + x) * a.ldk + g * a.hd + t]), acc);
  }
  if (t < a.hd) ((T*)a.dq)[(int64_t)i * a.lddq + j * a.hd + t] = from_f32<T>(acc * a.scale);
}

// one workgroup per (key, KV head): the query heads of the group and their queries in a fixed order
template <typename T>
__global__ __launch_bounds__(NT) void score_dkv_ref_kernel(ScoreArgs a) {
  __shared__ float ps[NT], dss[NT], ks[128], vs[128];
  const int u = blockIdx.x, g = blockIdx.y, t = threadIdx.x, grp = a.h / a.hkv;
  SeqSpan sp;
  if (!seq_of_row(a, u, sp)) return;
  if (t < a.hd) {
    ks[t] = to_f32(((const T*)a.k)[(int64_t)u * a.ldk + g * a.hd + t]);
    vs[t] = to_f32(((const T*)a.v)[(int64_t)u * a.ldv + g * a.hd + t]);
  }
  const int begin = queries_begin(a, sp, u);
  float dk = 0.f, dv = 0.f;
  for (int j = g * grp; j < (g + 1) * grp; ++j) {
    const float slope = a.slope ? a.slope[j] : 0.f;
    for (int i0 = begin; i0 < sp.hi; i0 += NT) {
      const int i = i0 + t, n = min(NT, sp.hi - i0);
      __syncthreads();
      if (t < n) {
        const T* qr = (const T*)a.q + (int64_t)i * a.ldq + j * a.hd;
        const T* dor = (const T*)a.dout + (int64_t)i * a.lddo + j * a.hd;
        float dot = 0.f, dp = 0.f, dcap;
        for (int x = 0; x < a.hd; ++x) { dot = fmaf(to_f32(qr[x]), ks[x], dot); dp = fmaf(to_f32(dor[x]), vs[x], dp); }
        const int64_t row = (int64_t)j * a.rows + i;
        const float sc = shaped(dot, a, slope, i - u, dcap), p = expf(sc - a.lse[row]);
        ps[t] = p;
        dss[t] = p * (dp - a.delta[row]) * dcap;
      }
      __syncthreads();
      if (t < a.hd)
        for (int x = 0; x < n; ++x) {
          dv = fmaf(ps[x], to_f32(((const T*)a.dout)[(int64_t)(i0 + x) * a.lddo + j * a.hd + t]), dv);
          dk = fmaf(dss[x], to_f32(((const T*)a.q)[(int64_t)(i0 + x) * a.ldq + j * a.hd + t]), dk);
        }
    }
  }
  if (t < a.hd) {
    ((T*)a.dk)[(int64_t)u * a.lddk + g * a.hd + t] = from_f32<T>(dk * a.scale);
    ((T*)a.dv)[(int64_t)u * a.lddv + g * a.hd + t] = from_f32<T>(dv);
  }
}

template <typename T>
hipError_t bwd_t(const ScoreArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((score_dq_ref_kernel<T>), dim3(a.rows, a.h), dim3(NT), 0, s, a);
  hipLaunchKernelGGL((score_dkv_ref_kernel<T>), dim3(a.rows, a.hkv), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t score_fwd_ref(DType dt, const ScoreArgs& a, hipStream_t s) {
  if (dt == DT_F32) hipLaunchKernelGGL((score_fwd_ref_kernel<float>), dim3(a.rows, a.h), dim3(NT), 0, s, a);
  else hipLaunchKernelGGL((score_fwd_ref_kernel<bf16>), dim3(a.rows, a.h), dim3(NT), 0, s, a);
  return hipGetLastError();
}
hipError_t score_bwd_ref(DType dt, const ScoreArgs& a, hipStream_t s) { return dt == DT_F32 ? bwd_t<float>(a, s) : bwd_t<bf16>(a, s); }

}  // namespace stg
