// Log probabilities of the rows' tokens, entropy, alternatives and the logits' gradient: plain kernels, one mathematical step behind the other.
// A workgroup takes a row: its largest logit m, then S = sum e^(s(x - m)) and T = sum e^(s(x - m)) s(m - x), whose terms have one sign, so that
// the entropy ln S + T / S loses nothing; then the alternatives one by one, each the first of what comes behind the one before it.
#include "common.h"

namespace stg {
namespace {

constexpr int NT = 256;

template <typename Op> __device__ float over_all(float v, Op op) {
  __shared__ float red[NT];
  __syncthreads();
  red[threadIdx.x] = v;
  for (int w = NT / 2; w > 0; w >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < w) red[threadIdx.x] = op(red[threadIdx.x], red[threadIdx.x + w]);
  }
  __syncthreads();
  return red[0];
}

// whether (v, c) comes before (w, d): the larger logit, of equal ones the lower column
__device__ __forceinline__ bool before(float v, int c, float w, int d) { return v > w || (v == w && c < d); }

template <typename T>
__global__ __launch_bounds__(NT) void logprob_ref_kernel(LogprobArgs a) {
  __shared__ float bv[NT];
  __shared__ int bc[NT];
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x;
  const T* x = (const T*)a.x + row * a.ldx;
  float top = -INFINITY;
  for (int j = t; j < a.vocab; j += NT) top = fmaxf(top, to_f32(x[j]));      // a NaN is passed over here and spoils the sum
  const float m = over_all(top, [](float p, float q) { return fmaxf(p, q); });
  const float at = m == -INFINITY ? 0.f : m;
  float s = 0.f, h = 0.f;
  for (int j = t; j < a.vocab; j += NT) {
    const float z = a.scale * (to_f32(x[j]) - at), e = expf(z);
    s += e;
    if (!(e == 0.f)) h -= e * z;
  }
  s = over_all(s, [](float p, float q) { return p + q; });
  h = over_all(h, [](float p, float q) { return p + q; });
  const bool bad = !(s < INFINITY);
  const float ln = bad ? NAN : logf(s);
  auto logp = [&](float v) { return v == -INFINITY && !bad ? -INFINITY : a.scale * (v - at) - ln; };
  if (t == 0) {
    const int id = a.target ? a.target[row] : -1;
    if (a.logp) a.logp[row] = id >= 0 && id < a.vocab ? logp(to_f32(x[id])) : 0.f;
    if (a.stats) { a.stats[2 * row] = m; a.stats[2 * row + 1] = ln; }
    if (a.entropy) a.entropy[row] = s == 0.f ? 0.f : ln + h / s;
  }
  float lv = INFINITY;
  int lc = -1;
  for (int r = 0; r < a.top; ++r) {
    float v = -INFINITY;
    int c = INT32_MAX;
    if (!bad)
      for (int j = t; j < a.vocab; j += NT) {
        const float w = to_f32(x[j]);
        if (before(lv, lc, w, j) && before(w, j, v, c)) { v = w; c = j; }
      }
    bv[t] = v; bc[t] = c;
    for (int w = NT / 2; w > 0; w >>= 1) {
      __syncthreads();
      if (t < w && before(bv[t + w], bc[t + w], bv[t], bc[t])) { bv[t] = bv[t + w]; bc[t] = bc[t + w]; }
    }
    __syncthreads();
    lv = bv[0]; lc = bc[0];
    __syncthreads();
    if (t == 0) {
      a.top_id[row * a.top + r] = bad ? -1 : lc;
      a.top_logp[row * a.top + r] = bad ? NAN : logp(lv);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(NT) void logprob_grad_ref_kernel(LogprobArgs a) {
  const int64_t row = blockIdx.x;
  const T* x = (const T*)a.x + row * a.ldx;
  T* dx = (T*)a.dx + row * a.lddx;
  const int id = a.target ? a.target[row] : -1;
  const float w = a.dlogp && id >= 0 && id < a.vocab ? a.dlogp[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f, dl = a.dlse ? a.dlse[row] : 0.f;
  const float m = a.stats[2 * row], ln = a.stats[2 * row + 1], h = a.dentropy ? a.entropy[row] : 0.f;
  const bool none = (w == 0.f && dh == 0.f && dl == 0.f) || empty_row(m, ln);
  for (int j = threadIdx.x; j < a.vocab; j += NT) {
    float g = 0.f;
    if (!none) {
      const float lp = a.scale * (to_f32(x[j]) - m) - ln, p = expf(lp);
      g = p == 0.f ? 0.f : p * (dl - w - dh * (lp + h));
      if (j == id) g += w;
    }
    dx[j] = from_f32<T>(a.scale * g);
  }
}

}  // namespace

hipError_t logprob_ref(DType dt, const LogprobArgs& a, hipStream_t s) {
  if (dt == DT_F32) hipLaunchKernelGGL((logprob_ref_kernel<float>), dim3(a.rows), dim3(NT), 0, s, a);
  else hipLaunchKernelGGL((logprob_ref_kernel<bf16>), dim3(a.rows), dim3(NT), 0, s, a);
  return hipGetLastError();
}
hipError_t logprob_grad_ref(DType dt, const LogprobArgs& a, hipStream_t s) {
  if (dt == DT_F32) hipLaunchKernelGGL((logprob_grad_ref_kernel<float>), dim3(a.rows), dim3(NT), 0, s, a);
  else hipLaunchKernelGGL((logprob_grad_ref_kernel<bf16>), dim3(a.rows), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace stg
