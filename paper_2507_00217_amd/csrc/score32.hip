// fp32 attention of shaped scores over packed sequences on the fp32 matrix cores: the blocks, the split over wavefronts and the one-launch
// backward of fp32_mfma.hip's attention, with the scores of score_attn.hip.  One workgroup per 16 queries (forward, dQ) or 16 keys
// (dK/dV) of a head; its wavefronts take every 8th block of 16 keys (queries) and are merged through LDS in wavefront order.  Blocks are cut
// per sequence (its slots: first row / 16 + its number), so the only block with pairs that do not count is a query block's last one.
// What bounds it at the lengths fp32 models are checked at is the latency of a wavefront's few blocks and of the merge, not the matrix rate.
#include "fp32_attn.h"
#include "score.h"

#include <type_traits>

namespace stg {
namespace {

struct Block { int lo, len, prefix, r0; };     // rows of the sequence, its prefix, first row of the block in it; len = 0: nothing to do
__device__ __forceinline__ Block find_block(const ScoreArgs& a, int slot, int lane) {
  int i, t;
  if (!a.seq_start) {
    const int per = (a.rows / a.n_seq + 15) / 16;
    i = slot / per; t = slot % per;
  } else {
    i = 0;
    for (int n = a.n_seq; n > 1;) {
      const int step = (n + 63) >> 6, at = lane * step;
      const bool before = at < n && min(max(a.seq_start[i + min(at, n - 1)], 0), a.rows) / 16 + i + at <= slot;
      const int k = max((int)__popcll(__ballot(before)) - 1, 0) * step;
      i += k;
      n = min(step, n - k);
    }
    i = __builtin_amdgcn_readfirstlane(i);
    t = slot - (min(max(a.seq_start[i], 0), a.rows) / 16 + i);
  }
  const SeqSpan s = seq_span(a, i);
  Block b;
  b.lo = __builtin_amdgcn_readfirstlane(s.lo);
  b.prefix = __builtin_amdgcn_readfirstlane(s.prefix);
  b.r0 = __builtin_amdgcn_readfirstlane(t) * 16;
  b.len = b.r0 >= 0 && b.r0 < __builtin_amdgcn_readfirstlane(s.hi - s.lo) ? __builtin_amdgcn_readfirstlane(s.hi - s.lo) : 0;
  return b;
}

template <int HD>
__global__ __launch_bounds__(AW * 64) void score32_fwd_kernel(ScoreArgs a, int slots) {
  constexpr int NT = HD / 16;
  __shared__ f32x4 red[AW * NT * 64];
  __shared__ float red_m[AW][16], red_l[AW][16];
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.h, kvh = head / (a.h / a.hkv);
  const Block b = find_block(a, slots - 1 - (int)(blockIdx.x / a.h), lane);          // late queries, the longer rows, first
  if (b.len == 0) return;
  const float* kp = (const float*)a.k + (int64_t)b.lo * a.ldk + kvh * HD;
  const float* vp = (const float*)a.v + (int64_t)b.lo * a.ldv + kvh * HD;
  const int q0 = b.r0, q = q0 + c, last = b.len - 1, vis = a.causal ? b.prefix : b.len;
  const int seen = min(max(a.causal ? q : 0, vis - 1), last);                        // the last key of the lane's query
  const float slope = a.slope ? a.slope[head] : 0.f;
  f32x4 qf[NT];
  ld_rows<HD>(qf, (const float*)a.q + (int64_t)(b.lo + min(q, last)) * a.ldq + head * HD, g);
  const int nblk = (max(min(q0 + 16, b.len), vis) + 15) / 16;
  f32x4 o[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  f32x4 kf[NT];
  ld_rows<HD>(kf, kp + (int64_t)min(w * 16 + c, last) * a.ldk, g);
  bool odd = false;                                      // the last block waits for the end if its rows are not finite
  f32x4 sc;
  for (int kb = w; kb < nblk; kb += AW) {
    float vf[4][NT];
    ld_cols<HD>(vf, vp, a.ldv, kb * 16, last, c, g);
    sc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) sc = mfma4(kf[t][j], qf[t][j], sc);
    ld_rows<HD>(kf, kp + (int64_t)min((kb + AW) * 16 + c, last) * a.ldk, g);         // next block, in flight during the rest
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int key = kb * 16 + 4 * g + e;
      float d;
      sc[e] = key <= seen ? shaped(sc[e], a, slope, q - key, d) : -INFINITY;
      mx = fmaxf(mx, sc[e]);
    }
    const float mn = fmaxf(m, max_g(mx));
    const float sub = mn == -INFINITY ? 0.f : mn;
    const float alpha = expf(m - sub);
    float ps = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) { sc[e] = expf(sc[e] - sub); ps += sc[e]; }
    m = mn;
    l = l * alpha + ps;
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i] *= alpha;
    if (kb == nblk - 1 && (odd = odd_rows(vf))) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < NT; ++i) vf[j][i] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < NT; ++i) o[i] = mfma4(vf[j][i], sc[j], o[i]);
  }
  if (odd) {
    float vf[4][NT];
    bool ok[4];
    ld_cols<HD>(vf, vp, a.ldv, (nblk - 1) * 16, last, c, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) ok[e] = (nblk - 1) * 16 + 4 * g + e <= seen;
    mul_seen(o, vf, sc, ok, c, g);
  }
  l = sum_g(l);
  if (g == 0) { red_m[w][c] = m; red_l[w][c] = l; }
#pragma unroll
  for (int p = 0; p < NT; ++p) red[(w * NT + p) * 64 + lane] = piece<HD>(o, p);
  __syncthreads();
  float mt = red_m[0][c];
#pragma unroll
  for (int k = 1; k < AW; ++k) mt = fmaxf(mt, red_m[k][c]);
  float f[AW], lt = 0.f;
#pragma unroll
  for (int k = 0; k < AW; ++k) { f[k] = red_m[k][c] == -INFINITY ? 0.f : expf(red_m[k][c] - mt); lt += red_l[k][c] * f[k]; }
  const float inv = 1.f / lt;
  if (q >= b.len) return;
#pragma unroll
  for (int t = 0; t < (NT + AW - 1) / AW; ++t) {
    const int p = w + t * AW;
    if (p >= NT) break;
    f32x4 v = red[p * 64 + lane] * f[0];
#pragma unroll
    for (int k = 1; k < AW; ++k) v += red[(k * NT + p) * 64 + lane] * f[k];
    *reinterpret_cast<f32x4*>((float*)a.o + (int64_t)(b.lo + q) * a.ldo + head * HD + piece_col<HD>(p, g)) = v * inv;
  }
  if (w == 0 && g == 0 && a.lse) a.lse[(int64_t)head * a.rows + b.lo + q] = mt == -INFINITY ? NAN : mt + logf(lt);
}

template <int HD>
__device__ __forceinline__ void score32_dq(const ScoreArgs& a, const Block& b, int head, f32x4* red) {
  constexpr int NT = HD / 16;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = head / (a.h / a.hkv);
  const float* kp = (const float*)a.k + (int64_t)b.lo * a.ldk + kvh * HD;
  const float* vp = (const float*)a.v + (int64_t)b.lo * a.ldv + kvh * HD;
  const int q0 = b.r0, q = q0 + c, last = b.len - 1, qc = b.lo + min(q, last), vis = a.causal ? b.prefix : b.len;
  const int seen = min(max(a.causal ? q : 0, vis - 1), last);
  const float slope = a.slope ? a.slope[head] : 0.f;
  f32x4 qf[NT], dof[NT];
  ld_rows<HD>(qf, (const float*)a.q + (int64_t)qc * a.ldq + head * HD, g);
  ld_rows<HD>(dof, (const float*)a.dout + (int64_t)qc * a.lddo + head * HD, g);
  float delta = 0.f;
  {
    f32x4 of[NT];
    ld_rows<HD>(of, (const float*)a.o + (int64_t)qc * a.ldo + head * HD, g);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) delta += of[t][e] * dof[t][e];
    delta = sum_g(delta);
  }
  const float lse = a.lse[(int64_t)head * a.rows + qc];
  const int nblk = (max(min(q0 + 16, b.len), vis) + 15) / 16;
  f32x4 dq[NT];
  float odd = 0.f;                                       // becomes NaN with the scores of a key row that holds an infinity or NaN
  auto walk = [&](auto seen_c) __attribute__((always_inline)) {
    constexpr bool again = decltype(seen_c)::value;
#pragma unroll
    for (int i = 0; i < NT; ++i) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kb = w; kb < nblk; kb += AW) {
      const int64_t kr = min(kb * 16 + c, last);
      f32x4 kf[NT], vf[NT];
      float kc[4][NT];
      ld_rows<HD>(kf, kp + kr * a.ldk, g);
      ld_rows<HD>(vf, vp + kr * a.ldv, g);
      ld_cols<HD>(kc, kp, a.ldk, kb * 16, last, c, g);
      f32x4 sc = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) { sc = mfma4(kf[t][j], qf[t][j], sc); dp = mfma4(vf[t][j], dof[t][j], dp); }
      bool ok[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = kb * 16 + 4 * g + e;
        float d;
        ok[e] = key <= seen;
        if (!again) odd = __builtin_fmaf(sc[e], 0.f, odd);
        const float s = shaped(sc[e], a, slope, q - key, d);
        sc[e] = ok[e] ? expf(s - lse) * (dp[e] - delta) * d : 0.f;
      }
      if (again) mul_seen(dq, kc, sc, ok, c, g);
      else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < NT; ++i) dq[i] = mfma4(kc[j][i], sc[j], dq[i]);
      }
    }
  };
  walk(std::false_type{});
  if (__any(odd != 0.f)) walk(std::true_type{});
#pragma unroll
  for (int p = 0; p < NT; ++p) red[(w * NT + p) * 64 + lane] = piece<HD>(dq, p);
  __syncthreads();
  if (q >= b.len) return;
#pragma unroll
  for (int t = 0; t < (NT + AW - 1) / AW; ++t) {
    const int p = w + t * AW;
    if (p >= NT) break;
    f32x4 v = red[p * 64 + lane];
#pragma unroll
    for (int k = 1; k < AW; ++k) v += red[(k * NT + p) * 64 + lane];
    *reinterpret_cast<f32x4*>((float*)a.dq + (int64_t)(b.lo + q) * a.lddq + head * HD + piece_col<HD>(p, g)) = v * a.scale;
  }
}

// dK and dV of 16 keys: the wavefronts take the (query head of the group, block of 16 queries) pairs in turn; K and V fragments wait in LDS
template <int HD>
__device__ __forceinline__ void score32_dkv(const ScoreArgs& a, const Block& b, int kvh, f32x4* red, f32x4* kv) {
  constexpr int NT = HD / 16;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = a.h / a.hkv, k0 = b.r0, key = k0 + c, last = b.len - 1;
  if (w < 2) {
    f32x4 f[NT];
    const int64_t row = b.lo + min(key, last);
    ld_rows<HD>(f, w ? (const float*)a.v + row * a.ldv + kvh * HD : (const float*)a.k + row * a.ldk + kvh * HD, g);
#pragma unroll
    for (int t = 0; t < NT; ++t) kv[(w * NT + t) * 64 + lane] = f[t];
  }
  __syncthreads();
  f32x4 dk[NT], dv[NT];
  const int qb0 = a.causal && k0 >= b.prefix ? k0 / 16 : 0, nqb = (b.len + 15) / 16 - qb0;
  const int from = a.causal && key >= b.prefix ? key : 0;             // the first query that sees the lane's key
  float odd = 0.f;                                       // becomes NaN with the scores or delta of a row of Q or dO that holds an infinity or NaN
  auto walk = [&](auto seen_c) __attribute__((always_inline)) {
    constexpr bool again = decltype(seen_c)::value;
#pragma unroll
    for (int i = 0; i < NT; ++i) dk[i] = dv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int it = w; it < grp * nqb; it += AW) {
      const int head = kvh * grp + it / nqb, q0 = (qb0 + it % nqb) * 16;
      const float* qh = (const float*)a.q + (int64_t)b.lo * a.ldq + head * HD;
      const float* doh = (const float*)a.dout + (int64_t)b.lo * a.lddo + head * HD;
      const float slope = a.slope ? a.slope[head] : 0.f;
      const int64_t qr = min(q0 + c, last);
      f32x4 qf[NT], dof[NT];
      float qc[4][NT], doc[4][NT];
      ld_rows<HD>(qf, qh + qr * a.ldq, g);
      ld_rows<HD>(dof, doh + qr * a.lddo, g);
      ld_cols<HD>(doc, doh, a.lddo, q0, last, c, g);
      if (!again) ld_cols<HD>(qc, qh, a.ldq, q0, last, c, g);
      const float* lse = a.lse + (int64_t)head * a.rows + b.lo;
      float ls[4], dl[4], dc = 0.f;
      {
        f32x4 of[NT];
        ld_rows<HD>(of, (const float*)a.o + (b.lo + qr) * a.ldo + head * HD, g);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) dc += of[t][e] * dof[t][e];
        dc = sum_g(dc);                                    // delta of query q0 + c
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) { ls[e] = lse[min(q0 + 4 * g + e, last)]; dl[e] = __shfl(dc, 4 * g + e, 64); }
      f32x4 sc = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const f32x4 kf = kv[t * 64 + lane], vf = kv[(NT + t) * 64 + lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) { sc = mfma4(qf[t][j], kf[j], sc); dp = mfma4(dof[t][j], vf[j], dp); }
      }
      bool ok[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int q = q0 + 4 * g + e;
        float d;
        ok[e] = q < b.len && q >= from;
        if (!again) odd = __builtin_fmaf(sc[e], 0.f, odd);
        const float s = shaped(sc[e], a, slope, q - key, d);
        const float p = ok[e] ? expf(s - ls[e]) : 0.f;
        sc[e] = p;
        dp[e] = ok[e] ? p * (dp[e] - dl[e]) * d : 0.f;
      }
      if (again) {
        mul_seen(dv, doc, sc, ok, c, g);
        ld_cols<HD>(qc, qh, a.ldq, q0, last, c, g);          // (both at once do not fit the registers)
        mul_seen(dk, qc, dp, ok, c, g);
      } else {
        odd = __builtin_fmaf(dc, 0.f, odd);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            dv[i] = mfma4(doc[j][i], sc[j], dv[i]);
            dk[i] = mfma4(qc[j][i], dp[j], dk[i]);
          }
      }
    }
  };
  walk(std::false_type{});
  if (__any(odd != 0.f)) walk(std::true_type{});
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which) __syncthreads();
#pragma unroll
    for (int p = 0; p < NT; ++p) red[(w * NT + p) * 64 + lane] = which ? piece<HD>(dv, p) : piece<HD>(dk, p);
    __syncthreads();
    const int64_t row = b.lo + key;
    float* out = which ? (float*)a.dv + row * a.lddv + kvh * HD : (float*)a.dk + row * a.lddk + kvh * HD;
#pragma unroll
    for (int t = 0; t < (NT + AW - 1) / AW; ++t) {
      const int p = w + t * AW;
      if (p >= NT || key >= b.len) break;
      f32x4 v = red[p * 64 + lane];
#pragma unroll
      for (int k = 1; k < AW; ++k) v += red[(k * NT + p) * 64 + lane];
      *reinterpret_cast<f32x4*>(out + piece_col<HD>(p, g)) = which ? v : v * a.scale;
    }
  }
}

template <int HD>
__global__ __launch_bounds__(AW * 64) void score32_bwd_kernel(ScoreArgs a, int slots) {
  __shared__ f32x4 red[AW * (HD / 16) * 64], kv[2 * (HD / 16) * 64];
  const int n_kv = slots * a.hkv, lane = threadIdx.x & 63;
  int id = blockIdx.x;
  if (id < n_kv) {                                       // low keys first: they see the most queries
    const Block b = find_block(a, id / a.hkv, lane);
    if (b.len) score32_dkv<HD>(a, b, id % a.hkv, red, kv);
  } else {
    id -= n_kv;
    const Block b = find_block(a, slots - 1 - id / a.h, lane);
    if (b.len) score32_dq<HD>(a, b, id % a.h, red);
  }
}

int64_t slots32(const ScoreArgs& a) { return a.seq_start ? a.rows / 16 + a.n_seq : (int64_t)a.n_seq * ((a.rows / a.n_seq + 15) / 16); }

}  // namespace

bool score32_supported(const ScoreArgs& a) {
  auto ok = [](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 4 == 0; };
  if (!ok(a.q, a.ldq) || !ok(a.k, a.ldk) || !ok(a.v, a.ldv) || !ok(a.o, a.ldo)) return false;
  if (a.dout && (!ok(a.dout, a.lddo) || !ok(a.dq, a.lddq) || !ok(a.dk, a.lddk) || !ok(a.dv, a.lddv))) return false;
  return slots32(a) * (a.h + a.hkv) < (1 << 23);         // threads of a grid
}
hipError_t score32_fwd(const ScoreArgs& a, hipStream_t s) {
  const int n = (int)slots32(a);
  if (a.hd == 64) hipLaunchKernelGGL((score32_fwd_kernel<64>), dim3(n * a.h), dim3(AW * 64), 0, s, a, n);
  else hipLaunchKernelGGL((score32_fwd_kernel<128>), dim3(n * a.h), dim3(AW * 64), 0, s, a, n);
  return hipGetLastError();
}
hipError_t score32_bwd(const ScoreArgs& a, hipStream_t s) {
  const int n = (int)slots32(a);
  if (a.hd == 64) hipLaunchKernelGGL((score32_bwd_kernel<64>), dim3(n * (a.h + a.hkv)), dim3(AW * 64), 0, s, a, n);
  else hipLaunchKernelGGL((score32_bwd_kernel<128>), dim3(n * (a.h + a.hkv)), dim3(AW * 64), 0, s, a, n);
  return hipGetLastError();
}

}  // namespace stg
