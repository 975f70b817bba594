// Rotary positions on several axes (time, height, width), alone or behind the RMS norm of every query and key head, and the way back.
//   norm:      rstd = (mean x^2 + eps)^-1/2 over the hd columns of a head, n = x rstd, y = R(n gamma)
//   rotation:  pair p of a head turns by the row's position on the pair's axis times the pair's frequency,
//              (a, b) -> (a cos - b sin, a sin + b cos); R^T is the rotation by the negative angle
//   backward:  g = R^T dy, dgamma += sum g n, dx = rstd (g gamma - n mean(g gamma n))
// All of it moves every element once and computes a few operations on it: what bounds it is bytes.
//
// A lane holds HALF pairs of a head in registers, so a head is HD / V lanes wide and a wavefront works on 64 V / HD heads of a row
// side by side; the norm's sums run across a head's lanes in registers.  The angle is formed in double precision and in turns
// (a position may be a million, and single precision would leave nothing of its angle), brought into [-1/2, 1/2] and only then
// rounded; a lane's pairs are the same in every head, so sine and cosine are computed once for all heads that it visits of a row.
#include "common.h"

#include <type_traits>

namespace stg {
namespace {

constexpr int WAVES = 4, NT = WAVES * 64;
// Workgroups of the backward, each of which leaves one row of partial sums, and their wavefronts: 16 to a compute unit in all.  (40 heads of
// 128 x 4096 rows, forward and backward: 512 of 8 wavefronts 49.8 us, 256 of 16 49.9, 1024 of 4 52.5, 512 of 4 54.3; the sum over the rows is the difference.)
constexpr int PARTS = 512, WB = 8, NTB = WB * 64;

template <typename T> constexpr int vec() { return 16 / (int)sizeof(T); }

// The pairs c * V/2 .. + V/2 of a head whose first element is at p: adjacent columns (one 16-byte piece) or columns hd / 2 apart
// (two of 8 bytes).
template <typename T, int HD, bool HALVES>
struct Pairs {
  static constexpr int N = vec<T>() / 2;
  union { uint4 raw; uint2 half[2]; T v[2 * N]; } u;
  __device__ __forceinline__ void load(const T* p, int c) {
    if (HALVES) {
      u.half[0] = *reinterpret_cast<const uint2*>(p + c * N);
      u.half[1] = *reinterpret_cast<const uint2*>(p + HD / 2 + c * N);
    } else u.raw = *reinterpret_cast<const uint4*>(p + c * 2 * N);
  }
  __device__ __forceinline__ void store(T* p, int c) const {
    if (HALVES) {
      *reinterpret_cast<uint2*>(p + c * N) = u.half[0];
      *reinterpret_cast<uint2*>(p + HD / 2 + c * N) = u.half[1];
    } else *reinterpret_cast<uint4*>(p + c * 2 * N) = u.raw;
  }
  __device__ __forceinline__ void get(float (&a)[N], float (&b)[N]) const {
#pragma unroll
    for (int q = 0; q < N; ++q) { a[q] = to_f32(u.v[HALVES ? q : 2 * q]); b[q] = to_f32(u.v[HALVES ? N + q : 2 * q + 1]); }
  }
  __device__ __forceinline__ void set(const float (&a)[N], const float (&b)[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) { u.v[HALVES ? q : 2 * q] = from_f32<T>(a[q]); u.v[HALVES ? N + q : 2 * q + 1] = from_f32<T>(b[q]); }
  }
};

// sum over the LPH lanes of a head: within rows of 16 lanes by moves between lanes inside the vector instruction
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LPH> __device__ __forceinline__ float head_sum(float v) {
  v += dpp<0xB1>(v);                   // the neighbour
  v += dpp<0x4E>(v);                   // the other two of four
  v += dpp<0x141>(v);                  // mirrored in eight: the other four
  if (LPH >= 16) v += dpp<0x140>(v);   // mirrored in sixteen
  if (LPH >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}

// cosines and sines of a lane's pairs at a row
template <typename T, int N>
__device__ __forceinline__ void row_turns(const RotateArgs& r, const double (&turn)[N], const int (&axis)[N], int row, int inverse, float (&cs)[N], float (&sn)[N]) {
  int pos[N];
#pragma unroll
  for (int q = 0; q < N; ++q) pos[q] = r.pos[(int64_t)axis[q] * r.pos_stride + row];
#pragma unroll
  for (int q = 0; q < N; ++q) {
    double t = turn[q] * (double)pos[q];
    t -= rint(t);
    const float f = (float)t;
    if (sizeof(T) == 2) {              // the instructions, which take turns: their error of 2^-20 is far below half a step of bf16
      sn[q] = __builtin_amdgcn_sinf(f);
      cs[q] = __builtin_amdgcn_cosf(f);
    } else sincospif(2.f * f, &sn[q], &cs[q]);
    if (inverse) sn[q] = -sn[q];
  }
}
template <int N>
__device__ __forceinline__ void lane_turns(const RotateArgs& r, int c, double (&turn)[N], int (&axis)[N]) {
#pragma unroll
  for (int q = 0; q < N; ++q) { turn[q] = r.turn[c * N + q]; axis[q] = r.axis[c * N + q]; }
}

// Forward, or (without the norm) the rotation alone.  A wavefront's share is U steps of 64 / LPH heads of one row, all of whose
// loads are in flight together.
template <typename T, int HD, bool HALVES, bool NORM, int U>
__global__ __launch_bounds__(NT) void head_rotate_kernel(HeadNormArgs n, RotateArgs r, int chunks) {
  using P = Pairs<T, HD, HALVES>;
  constexpr int N = P::N, LPH = HD / vec<T>(), HPW = 64 / LPH;
  const int lane = threadIdx.x & 63, c = lane % LPH, heads = n.h + n.hkv;
  const int64_t unit = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
  const int row = (int)(unit / chunks), h0 = (int)(unit % chunks) * U * HPW + lane / LPH;
  if (row >= n.rows) return;
  const T* x = (const T*)n.x + (int64_t)row * n.ldx;
  T* y = (T*)n.y + (int64_t)row * n.ldy;
  P v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    v[u].load(x + (int64_t)min(h0 + u * HPW, heads - 1) * HD, c);
  float cs[N], sn[N];
  if (r.pos) {
    double turn[N];
    int axis[N];
    lane_turns(r, c, turn, axis);
    row_turns<T>(r, turn, axis, row, n.inverse, cs, sn);
  }
  float gq[2][N], gk[2][N];
  if (NORM) {
    P g;
    g.load((const T*)n.gq, c);
    g.get(gq[0], gq[1]);
    g.load((const T*)n.gk, c);
    g.get(gk[0], gk[1]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int head = h0 + u * HPW;
    float a[N], b[N];
    v[u].get(a, b);
    if (NORM) {
      float ss = 0.f;
#pragma unroll
      for (int q = 0; q < N; ++q) ss = fmaf(a[q], a[q], fmaf(b[q], b[q], ss));
      const float rstd = rsqrtf(head_sum<LPH>(ss) * (1.f / HD) + n.eps);
      const bool is_q = head < n.h;
#pragma unroll
      for (int q = 0; q < N; ++q) { a[q] *= rstd * (is_q ? gq[0][q] : gk[0][q]); b[q] *= rstd * (is_q ? gq[1][q] : gk[1][q]); }
      if (n.rstd && c == 0 && head < heads) n.rstd[(int64_t)row * heads + head] = rstd;
    }
    if (r.pos) {
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const float ra = a[q] * cs[q] - b[q] * sn[q], rb = a[q] * sn[q] + b[q] * cs[q];
        a[q] = ra; b[q] = rb;
      }
    }
    v[u].set(a, b);
    if (head < heads) v[u].store(y + (int64_t)head * HD, c);
  }
}

// Backward: the same shares, walked by PARTS workgroups that keep the weights' gradients in registers and leave one row of
// partial sums each; another launch adds those in a fixed order.
constexpr int UB = 2;
template <typename T, int HD, bool HALVES>
__global__ __launch_bounds__(NTB) void head_norm_bwd_kernel(HeadNormArgs n, RotateArgs r, int chunks) {
  using P = Pairs<T, HD, HALVES>;
  constexpr int N = P::N, LPH = HD / vec<T>(), HPW = 64 / LPH;
  __shared__ float red[WB * HPW][2][HD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane % LPH, heads = n.h + n.hkv;
  float gq[2][N], gk[2][N], dgq[2][N], dgk[2][N], cs[N], sn[N];
  {
    P g;
    g.load((const T*)n.gq, c);
    g.get(gq[0], gq[1]);
    g.load((const T*)n.gk, c);
    g.get(gk[0], gk[1]);
  }
  double turn[N];
  int axis[N];
  if (r.pos) lane_turns(r, c, turn, axis);
#pragma unroll
  for (int q = 0; q < N; ++q) dgq[0][q] = dgq[1][q] = dgk[0][q] = dgk[1][q] = 0.f;
  const int64_t units = (int64_t)n.rows * chunks;
  for (int64_t unit = (int64_t)blockIdx.x * WB + wave; unit < units; unit += (int64_t)gridDim.x * WB) {
    const int row = (int)(unit / chunks), h0 = (int)(unit % chunks) * UB * HPW + lane / LPH;
    P xv[UB], dv[UB];
    float rstd[UB];
#pragma unroll
    for (int u = 0; u < UB; ++u) {
      const int head = min(h0 + u * HPW, heads - 1);
      xv[u].load((const T*)n.x + (int64_t)row * n.ldx + (int64_t)head * HD, c);
      dv[u].load((const T*)n.dy + (int64_t)row * n.lddy + (int64_t)head * HD, c);
      rstd[u] = n.rstd[(int64_t)row * heads + head];
    }
    if (r.pos) row_turns<T>(r, turn, axis, row, 1, cs, sn);
#pragma unroll
    for (int u = 0; u < UB; ++u) {
      const int head = h0 + u * HPW;
      const bool live = head < heads, is_q = head < n.h;
      float a[N], b[N], ga[N], gb[N], dot = 0.f;
      xv[u].get(a, b);
      dv[u].get(ga, gb);
#pragma unroll
      for (int q = 0; q < N; ++q) {
        a[q] *= rstd[u]; b[q] *= rstd[u];
        if (r.pos) {
          const float ra = ga[q] * cs[q] - gb[q] * sn[q], rb = ga[q] * sn[q] + gb[q] * cs[q];
          ga[q] = ra; gb[q] = rb;
        }
        const float wa = ga[q] * a[q], wb = gb[q] * b[q];
        if (live && is_q) { dgq[0][q] += wa; dgq[1][q] += wb; }
        if (live && !is_q) { dgk[0][q] += wa; dgk[1][q] += wb; }
        ga[q] *= is_q ? gq[0][q] : gk[0][q];
        gb[q] *= is_q ? gq[1][q] : gk[1][q];
        dot = fmaf(ga[q], a[q], fmaf(gb[q], b[q], dot));
      }
      const float mean = head_sum<LPH>(dot) * (1.f / HD);
#pragma unroll
      for (int q = 0; q < N; ++q) { a[q] = rstd[u] * (ga[q] - a[q] * mean); b[q] = rstd[u] * (gb[q] - b[q] * mean); }
      dv[u].set(a, b);
      if (live) dv[u].store((T*)n.y + (int64_t)row * n.ldy + (int64_t)head * HD, c);
    }
  }
  const int slot = wave * HPW + lane / LPH;
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int p = c * N + q, col = HALVES ? e * (HD / 2) + p : 2 * p + e;
      red[slot][0][col] = dgq[e][q];
      red[slot][1][col] = dgk[e][q];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * HD; i += NTB) {
    float s = 0.f;
    for (int k = 0; k < WB * HPW; ++k) s += (&red[k][0][0])[i];
    n.partial[(int64_t)blockIdx.x * 2 * HD + i] = s;
  }
}

// Steps of a share: what costs a row the least, a share counted as one step more than it has (positions, sine and cosine, weights), but none
// that leaves fewer than 16 wavefronts to a compute unit.  (18 heads of 128 x 8192 rows in one share of 5 steps 16.8 us, in two of 4 20.2.)
int steps_of_share(int steps, int rows) {
  auto cost = [&](int u) { return (steps + u - 1) / u * (u + 1); };
  int best = 1;
  for (const int u : {2, 3, 4, 5, 8})
    if ((int64_t)rows * ((steps + u - 1) / u) >= 4096 && cost(u) <= cost(best)) best = u;
  return best;
}

template <typename T, int HD, bool HALVES, bool NORM>
hipError_t rotate_launch(const HeadNormArgs& n, const RotateArgs& r, hipStream_t s) {
  constexpr int HPW = 64 * vec<T>() / HD;
  const int steps = (n.h + n.hkv + HPW - 1) / HPW;
  auto launch = [&](auto u) {
    constexpr int U = decltype(u)::value;
    const int chunks = (steps + U - 1) / U;
    const int64_t units = (int64_t)n.rows * chunks;
    hipLaunchKernelGGL((head_rotate_kernel<T, HD, HALVES, NORM, U>), dim3((unsigned)((units + WAVES - 1) / WAVES)), dim3(NT), 0, s, n, r, chunks);
    return hipGetLastError();
  };
  using std::integral_constant;
  switch (steps_of_share(steps, n.rows)) {
    case 1: return launch(integral_constant<int, 1>{});
    case 2: return launch(integral_constant<int, 2>{});
    case 3: return launch(integral_constant<int, 3>{});
    case 5: return launch(integral_constant<int, 5>{});
    case 8: return launch(integral_constant<int, 8>{});
    default: return launch(integral_constant<int, 4>{});
  }
}
template <typename T, int HD, bool HALVES>
hipError_t bwd_launch(const HeadNormArgs& n, const RotateArgs& r, hipStream_t s) {
  constexpr int HPW = 64 * vec<T>() / HD;
  const int chunks = (n.h + n.hkv + UB * HPW - 1) / (UB * HPW);
  const int64_t units = (int64_t)n.rows * chunks, want = (units + WB - 1) / WB;
  const int parts = (int)(want < PARTS ? want : PARTS);
  hipLaunchKernelGGL((head_norm_bwd_kernel<T, HD, HALVES>), dim3(parts), dim3(NTB), 0, s, n, r, chunks);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ColSumList l{};
  l.j[l.n++] = ColSum{n.partial, 2 * HD, HD, parts, n.dgq, COL_SUM_PARTS};
  l.j[l.n++] = ColSum{n.partial + HD, 2 * HD, HD, parts, n.dgk, COL_SUM_PARTS};
  return col_sums_add(l, s);
}

// calls f with the constants of one of the eight forms
template <typename F>
hipError_t by_form(DType dt, int hd, int halves, F f) {
  using std::integral_constant;
  auto at = [&](auto t, auto d) { return halves ? f(t, d, std::true_type{}) : f(t, d, std::false_type{}); };
  auto of = [&](auto t) { return hd == 128 ? at(t, integral_constant<int, 128>{}) : at(t, integral_constant<int, 64>{}); };
  return dt == DT_F32 ? of(float{}) : of(bf16{});
}

}  // namespace

size_t head_norm_partial_bytes(int hd) { return (size_t)PARTS * 2 * hd * sizeof(float); }

hipError_t rope_axes(DType dt, const HeadNormArgs& n, const RotateArgs& r, hipStream_t s) {
  return by_form(dt, n.hd, r.halves, [&](auto t, auto d, auto hv) { return rotate_launch<decltype(t), d(), hv(), false>(n, r, s); });
}
hipError_t qk_norm_rope_fwd(DType dt, const HeadNormArgs& n, const RotateArgs& r, hipStream_t s) {
  return by_form(dt, n.hd, r.halves, [&](auto t, auto d, auto hv) { return rotate_launch<decltype(t), d(), hv(), true>(n, r, s); });
}
hipError_t qk_norm_rope_bwd(DType dt, const HeadNormArgs& n, const RotateArgs& r, hipStream_t s) {
  return by_form(dt, n.hd, r.halves, [&](auto t, auto d, auto hv) { return bwd_launch<decltype(t), d(), hv()>(n, r, s); });
}

}  // namespace stg
