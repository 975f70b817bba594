// What happens to a stage's gradients between iterations: their common norm, the clip to a largest one, and the AdamW step.
//   sumsq = sum g^2,  c = min(1, max_norm / sqrt(sumsq)),  out = c g
//   m = b1 m + (1 - b1) c g,  v = b2 v + (1 - b2) (c g)^2,  w -= lr (wd w + (m / c1) / (sqrt(v / c2) + eps)),  c_i = 1 - b_i^step
// Every element is moved once per kernel and a few operations are done on it: what bounds all of it is bytes.
//
// A list of tensors is cut into chunks of one size, and a launch takes the chunks of as many tensors as travel with its arguments: nothing is copied to the
// device beforehand, so that a captured launch holds all that it needs.  Clip and step have a workgroup to each chunk, and loads and stores that ask the
// caches to keep nothing: 202 million fp32 gradients, norm and clip 378 us (ordinary accesses 423, and in 2048 workgroups that walk 468), the AdamW step with bf16 weights 1037 to
// 1055 us (1283 in workgroups that walk).
#include "common.h"

#include <type_traits>

namespace stg {
namespace {

constexpr int NT = 256;
constexpr int MOST_WGS = 1 << 22;    // of a launch; lists of more chunks than that are walked
// tensors of K arrays each to a launch: what 4 KB of arguments hold
template <int K> constexpr int most_tensors() { return 3900 / (24 + 8 * K); }

template <typename T> constexpr int vec() { return 16 / (int)sizeof(T); }

// `first`: chunks before the tensor.  `head`: elements of it before the first that lies on a boundary of a group in every
// array, or -1 where there is none in common, which makes the accesses single elements.  (All of a tensor in one entry of 8-byte fields: from an array
// of bytes beside the arrays of pointers, indexed by the same number t, the compiler made scalar loads at base + t with an offset of 7 t, and scalar loads drop the low two
// bits of each.)
template <int K> struct Entry {
  int64_t first, size, head;
  const void* p[K];
};
template <int K> struct Lists {
  int64_t n, chunks;
  Entry<K> e[most_tensors<K>()];
};
// One chunk: elements [lo, body) one by one, groups from body on, and what is left of them one by one up to hi
struct Chunk { int t; int64_t lo, body, hi; bool groups; };
template <int K, int CHUNK> __device__ __forceinline__ Chunk chunk_of(const Lists<K>& l, int64_t c) {
  int t = 0;
  for (int step = 64; step > 0; step >>= 1)
    if (t + step < l.n && l.e[t + step].first <= c) t += step;
  const int64_t i = c - l.e[t].first, size = l.e[t].size, head = l.e[t].head > 0 ? l.e[t].head : 0;
  Chunk r;
  r.t = t;
  r.body = min(head + i * CHUNK, size);
  r.lo = i ? r.body : 0;
  r.hi = min(head + (i + 1) * CHUNK, size);
  r.groups = l.e[t].head >= 0;
  return r;
}

// ONCE: a list beyond what the last-level cache holds, of which nothing will be found there
template <typename T, bool ONCE> struct Group {
  union { u32x4 raw; T v[vec<T>()]; } u;
  __device__ __forceinline__ void load(const T* p) { u.raw = fetch<ONCE, u32x4>(p); }
  __device__ __forceinline__ void store(T* p) const { put<ONCE>(p, u.raw); }
};

template <int N> __device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[N / 64];
  for (int w = 32; w > 0; w >>= 1) v += __shfl_xor(v, w, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < N / 64; ++w) v += red[w];
  return v;
}

constexpr int SUM_U = 8;
// Squares are formed and added in 64 bits: no gradient is too large or too small for them, and the vector units take fp64 as fast as memory brings it.
// part[workgroup] += its chunks' sum, or = where no launch before has left one (`left` of them have).
template <typename T, bool ONCE>
__global__ __launch_bounds__(NT) void sumsq_kernel(Lists<1> l, double* part, int left) {
  constexpr int V = vec<T>(), CHUNK = NT * V * SUM_U;
  double acc[4] = {};
  for (int64_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const Chunk k = chunk_of<1, CHUNK>(l, c);
    const T* g = (const T*)l.e[k.t].p[0];
    auto one = [&](int64_t i) { const double v = (double)to_f32(g[i]); acc[0] = fma(v, v, acc[0]); };
    auto group = [&](const Group<T, ONCE>& q) {
#pragma unroll
      for (int e = 0; e < V; ++e) { const double v = (double)to_f32(q.u.v[e]); acc[e & 3] = fma(v, v, acc[e & 3]); }
    };
    if (k.hi - k.body == CHUNK) {
      Group<T, ONCE> q[SUM_U];
#pragma unroll
      for (int u = 0; u < SUM_U; ++u) q[u].load(g + k.body + (int64_t)(u * NT + threadIdx.x) * V);
#pragma unroll
      for (int u = 0; u < SUM_U; ++u) group(q[u]);
    } else {
      const int64_t n = (k.hi - k.body) / V;
      for (int64_t i = threadIdx.x; i < n; i += NT) {
        Group<T, ONCE> q;
        q.load(g + k.body + i * V);
        group(q);
      }
      for (int64_t i = k.body + n * V + threadIdx.x; i < k.hi; i += NT) one(i);
    }
    for (int64_t i = k.lo + threadIdx.x; i < k.body; i += NT) one(i);
  }
  const double s = block_sum<NT>((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (threadIdx.x == 0) part[blockIdx.x] = ((int)blockIdx.x < left ? part[blockIdx.x] : 0.0) + s;
}

constexpr int NTT = 1024;
__global__ __launch_bounds__(NTT) void sumsq_total_kernel(const double* part, int parts, int add, double* sumsq) {
  static_assert(GRAD_PARTS == 2 * NTT, "two of them to a thread");
  const int i = threadIdx.x;
  const double a = i < parts ? part[i] : 0.0, b = i + NTT < parts ? part[i + NTT] : 0.0, s = block_sum<NTT>(a + b);
  if (i == 0) sumsq[0] = add ? sumsq[0] + s : s;
}

// The factor that brings a norm down to max_norm; 1 where the norm is not finite.  Norms that are more than 2^100 times max_norm have their factor in two, the first of
// which fp32 holds in all of its bits: the second is a power of two, and for all others 1, by which nothing changes.
struct Factor {
  float f, then;
  __device__ __forceinline__ float operator()(float g) const { return g * f * then; }
};
__device__ __forceinline__ Factor clip_factor(double sumsq, float max_norm) {
  const double norm = sqrt(sumsq), r = norm > (double)max_norm && norm < INFINITY ? (double)max_norm / norm : 1.0;
  const bool low = r < 0x1p-100;
  return {(float)(low ? r * 0x1p64 : r), low ? 0x1p-64f : 1.f};
}

constexpr int CLIP_U = 4;
template <typename T, bool ONCE>
__global__ __launch_bounds__(NT) void clip_kernel(Lists<2> l, const double* sumsq, float max_norm, float* norm) {
  constexpr int V = vec<T>(), CHUNK = NT * V * CLIP_U;
  const Factor f = clip_factor(*sumsq, max_norm);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)sqrt(*sumsq);
  for (int64_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const Chunk k = chunk_of<2, CHUNK>(l, c);
    const T* g = (const T*)l.e[k.t].p[0];
    T* o = (T*)l.e[k.t].p[1];
    if (f.f == 1.f && g == o) continue;              // nothing to change
    auto one = [&](int64_t i) { o[i] = from_f32<T>(f(to_f32(g[i]))); };
    auto group = [&](Group<T, ONCE>& q) {
#pragma unroll
      for (int e = 0; e < V; ++e) q.u.v[e] = from_f32<T>(f(to_f32(q.u.v[e])));
    };
    if (k.groups && k.hi - k.body == CHUNK) {
      Group<T, ONCE> q[CLIP_U];
#pragma unroll
      for (int u = 0; u < CLIP_U; ++u) q[u].load(g + k.body + (int64_t)(u * NT + threadIdx.x) * V);
#pragma unroll
      for (int u = 0; u < CLIP_U; ++u) {
        group(q[u]);
        q[u].store(o + k.body + (int64_t)(u * NT + threadIdx.x) * V);
      }
    } else {
      const int64_t n = k.groups ? (k.hi - k.body) / V : 0;
      for (int64_t i = threadIdx.x; i < n; i += NT) {
        Group<T, ONCE> q;
        q.load(g + k.body + i * V);
        group(q);
        q.store(o + k.body + i * V);
      }
      for (int64_t i = k.body + n * V + threadIdx.x; i < k.hi; i += NT) one(i);
    }
    for (int64_t i = k.lo + threadIdx.x; i < k.body; i += NT) one(i);
  }
}

// four elements side by side, on a boundary of four
template <typename T, bool ONCE> struct Four {
  union { u32x4 w; u32x2 h; T v[4]; } u;
  __device__ __forceinline__ void load(const T* p) {
    if (sizeof(T) == 4) u.w = fetch<ONCE, u32x4>(p);
    else u.h = fetch<ONCE, u32x2>(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    if (sizeof(T) == 4) put<ONCE>(p, u.w);
    else put<ONCE>(p, u.h);
  }
};

constexpr int ADAM_V = 4, ADAM_CHUNK = NT * ADAM_V;
enum { A_W, A_MASTER, A_M, A_V, A_G };
// The fp32 weights are `master`; with bf16 weights w receives their rounding.
template <typename TW, typename TG, bool ONCE>
__global__ __launch_bounds__(NT) void adamw_kernel(Lists<5> l, AdamWArgs a) {
  constexpr bool LP = sizeof(TW) == 2;
  __shared__ float sh[2];
  Factor f = {1.f, 1.f};
  if (a.sumsq) {
    if (!(*a.sumsq < INFINITY)) return;
    f = clip_factor(*a.sumsq, a.max_norm);
  }
  float lr = a.lr, i1 = a.inv1, i2 = a.inv2;
  if (a.lr_now) lr = *a.lr_now;
  if (a.step_now) {
    if (threadIdx.x == 0) {
      const double step = (double)max(*a.step_now, 1);
      sh[0] = (float)(-1.0 / expm1(step * a.lnbeta1));
      sh[1] = (float)(-1.0 / expm1(step * a.lnbeta2));
    }
    __syncthreads();
    i1 = sh[0];
    i2 = sh[1];
  }
  auto update = [&](float g, float& w, float& m, float& v) {
    g = f(g);
    m = fmaf(a.beta1, m, a.rest1 * g);
    v = fmaf(a.beta2, v, a.rest2 * g * g);
    w = fmaf(-lr, fmaf(a.decay, w, m * i1 / (sqrtf(v * i2) + a.eps)), w);
  };
  for (int64_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const Chunk k = chunk_of<5, ADAM_CHUNK>(l, c);
    TW* w = (TW*)l.e[k.t].p[A_W];
    float *x = (float*)l.e[k.t].p[A_MASTER], *m = (float*)l.e[k.t].p[A_M], *v = (float*)l.e[k.t].p[A_V];
    const TG* g = (const TG*)l.e[k.t].p[A_G];
    auto one = [&](int64_t i) {
      float xi = x[i], mi = m[i], vi = v[i];
      update(to_f32(g[i]), xi, mi, vi);
      x[i] = xi; m[i] = mi; v[i] = vi;
      if (LP) w[i] = from_f32<TW>(xi);
    };
    const int64_t n = k.groups ? (k.hi - k.body) / ADAM_V : 0, at = k.body + (int64_t)threadIdx.x * ADAM_V;
    if (threadIdx.x < n) {
      Four<float, ONCE> xi, mi, vi;
      Four<TG, ONCE> gi;
      Four<TW, ONCE> wi;
      xi.load(x + at); mi.load(m + at); vi.load(v + at); gi.load(g + at);
  #pragma unroll
      for (int e = 0; e < ADAM_V; ++e) {
        update(to_f32(gi.u.v[e]), xi.u.v[e], mi.u.v[e], vi.u.v[e]);
        wi.u.v[e] = from_f32<TW>(xi.u.v[e]);
      }
      xi.store(x + at); mi.store(m + at); vi.store(v + at);
      if (LP) wi.store(w + at);
    }
    for (int64_t i = k.body + n * ADAM_V + threadIdx.x; i < k.hi; i += NT) one(i);
    for (int64_t i = k.lo + threadIdx.x; i < k.body; i += NT) one(i);
  }
}

// Calls launch(lists, workgroups), one to a chunk, for as many tensors at a time as a launch takes; with `always` once at least.  es: element sizes of the K arrays; the pointers are
// arr[k][i]; an array may be missing (null), which counts as aligned.
template <int K, int CHUNK, int V, typename F>
hipError_t over_lists(const TensorList& t, const void* const* const (&arr)[K], const int (&es)[K], bool always, F launch) {
  int i = 0;
  do {
    Lists<K> l;
    l.n = l.chunks = 0;
    for (; i < t.n && l.n < most_tensors<K>(); ++i) {
      if (t.size[i] == 0) continue;
      Entry<K>& k = l.e[l.n++];
      int64_t head = -2;
      for (int q = 0; q < K; ++q) {
        k.p[q] = arr[q] ? arr[q][i] : nullptr;
        if (!arr[q]) continue;
        const int64_t h = (V - (uintptr_t)arr[q][i] / es[q] % V) % V;
        head = head == -2 || head == h ? h : -1;
      }
      k.first = l.chunks;
      k.size = t.size[i];
      k.head = head < k.size ? head : k.size;
      const int64_t body = k.size - (k.head > 0 ? k.head : 0);
      l.chunks += body > CHUNK ? (body + CHUNK - 1) / CHUNK : 1;
    }
    if (l.n || always) {
      const hipError_t e = launch(l, (int)(l.chunks < 1 ? 1 : l.chunks < MOST_WGS ? l.chunks : MOST_WGS));
      if (e != hipSuccess) return e;
    }
    always = false;
  } while (i < t.n);
  return hipSuccess;
}

// Whether a list's accesses ask the caches to keep nothing: from 256 MB on, what the last-level cache holds.  (4.2 million parameters, 59 MB: AdamW 12.9 us with ordinary
// accesses, 14.0 without keeping; 202 million, 6.1 GB: 1129 against 1099; norm and clip of 151 million bf16 gradients 308 against 269.)
bool once(const TensorList& l, int bytes) {
  int64_t n = 0;
  for (int i = 0; i < l.n; ++i) n += l.size[i];
  return n * bytes > (int64_t)256 << 20;
}
template <typename F> hipError_t by_size(bool large, F f) { return large ? f(std::true_type{}) : f(std::false_type{}); }

template <typename T>
hipError_t sumsq_launch(const TensorList& l, const void* const* grad, int add, double* sumsq, double* part, hipStream_t s) {
  int left = 0;
  const bool large = once(l, sizeof(T));
  const hipError_t e = over_lists<1, NT * vec<T>() * SUM_U, vec<T>()>(l, {grad}, {(int)sizeof(T)}, false, [&](const Lists<1>& t, int chunks) {
    const int wgs = chunks < GRAD_PARTS ? chunks : GRAD_PARTS;
    const hipError_t r = by_size(large, [&](auto o) {
      hipLaunchKernelGGL((sumsq_kernel<T, o()>), dim3(wgs), dim3(NT), 0, s, t, part, left);
      return hipGetLastError();
    });
    left = left > wgs ? left : wgs;
    return r;
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(sumsq_total_kernel, dim3(1), dim3(NTT), 0, s, part, left, add, sumsq);
  return hipGetLastError();
}

template <typename T>
hipError_t clip_launch(const TensorList& l, const void* const* grad, void* const* out, const double* sumsq, float max_norm, float* norm, hipStream_t s) {
  const bool large = once(l, 2 * sizeof(T));
  return over_lists<2, NT * vec<T>() * CLIP_U, vec<T>()>(l, {grad, (const void* const*)out}, {(int)sizeof(T), (int)sizeof(T)}, norm != nullptr, [&](const Lists<2>& t, int wgs) {
    const hipError_t r = by_size(large, [&](auto o) {
      hipLaunchKernelGGL((clip_kernel<T, o()>), dim3(wgs), dim3(NT), 0, s, t, sumsq, max_norm, norm);
      return hipGetLastError();
    });
    norm = nullptr;
    return r;
  });
}

template <typename TW, typename TG>
hipError_t adamw_launch(const AdamWArgs& a, const TensorList& l, void* const* w, float* const* master, float* const* m, float* const* v,
                        const void* const* grad, hipStream_t s) {
  const void* const* fp32 = sizeof(TW) == 2 ? (const void* const*)master : (const void* const*)w;
  const void* const* lp = sizeof(TW) == 2 ? (const void* const*)w : nullptr;
  const bool large = once(l, 24 + sizeof(TG));
  return over_lists<5, ADAM_CHUNK, ADAM_V>(l, {lp, fp32, (const void* const*)m, (const void* const*)v, grad}, {2, 4, 4, 4, (int)sizeof(TG)}, false,
                                                     [&](const Lists<5>& t, int wgs) {
    return by_size(large, [&](auto o) {
      hipLaunchKernelGGL((adamw_kernel<TW, TG, o()>), dim3(wgs), dim3(NT), 0, s, t, a);
      return hipGetLastError();
    });
  });
}

}  // namespace

hipError_t grad_sumsq(DType dt, TensorList l, const void* const* grad, int add, double* sumsq, double* part, hipStream_t s) {
  return dt == DT_F32 ? sumsq_launch<float>(l, grad, add, sumsq, part, s) : sumsq_launch<bf16>(l, grad, add, sumsq, part, s);
}
hipError_t grad_clip(DType dt, TensorList l, const void* const* grad, void* const* out, const double* sumsq, float max_norm, float* norm, hipStream_t s) {
  return dt == DT_F32 ? clip_launch<float>(l, grad, out, sumsq, max_norm, norm, s) : clip_launch<bf16>(l, grad, out, sumsq, max_norm, norm, s);
}
hipError_t adamw(DType dt, DType gdt, const AdamWArgs& a, TensorList l, void* const* w, float* const* master, float* const* m, float* const* v,
                 const void* const* grad, hipStream_t s) {
  if (dt == DT_F32)
    return gdt == DT_F32 ? adamw_launch<float, float>(a, l, w, master, m, v, grad, s) : adamw_launch<float, bf16>(a, l, w, master, m, v, grad, s);
  return gdt == DT_F32 ? adamw_launch<bf16, float>(a, l, w, master, m, v, grad, s) : adamw_launch<bf16, bf16>(a, l, w, master, m, v, grad, s);
}

}  // namespace stg
