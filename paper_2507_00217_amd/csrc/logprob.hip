// Log probabilities of the rows' tokens, entropy, likeliest alternatives and the logits' gradient, every logit read once.
//   m = max x,  e_j = 2^(c (x_j - m)) with c = scale log2 e,  S = sum e_j,  T = sum e_j c (m - x_j) (terms of one sign)
//   ln p_j = scale (x_j - m) - ln S,  H = ln S + ln 2 T / S
//   dx_j = scale [p_j (dlse - dlogp - dH (ln p_j + H)) + dlogp [j = token]]
// An element costs a few operations and an exponential: what bounds it is bytes.
//
// Values alone are a walk over the row: every thread keeps a maximum and sums of its own, which are brought to the row's maximum at the end, so that loads are never waited for
// by more than their own thread, and little is held in registers.  Rows that are too few to fill the chip are cut into parts, and a second launch joins what the parts found.
//
// With the gradient in the same call a row lies in the registers of one workgroup: up to 128 Ki columns of bf16 in 64 registers of each of 1024 threads, half of a compute
// unit's registers.  The logits are read once; half of the workgroup's next row comes to LDS during the sums, the rest into the registers whose gradient has been stored.
//
// Alternatives: the k-th largest of the maxima of 256 (64) groups of columns is a lower bound of the k-th largest logit, found bit by bit with ballots.  The walk has left the maximum
// of every two pieces in LDS; the few that reach the bound are read again, their elements that reach it go to a list in LDS, and each one's rank is the number of
// list entries before it.  A list overflows where many columns equal the bound, which has a way of its own (2048 rows x 128000 of one value with 20 alternatives 120 us,
// of nine tokens and one value below them 128; spread logits 100), or where many columns of few groups are beyond it: those rows are gone through once for each alternative.
#include "common.h"

#include <type_traits>

namespace stg {
namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float FAR = -1e4f;           // an exponent below which 2^x is zero many times over, and x still a number
constexpr float EDGE = 1e6f;          // magnitude of c m up to which its rounding, 2^-24 of it, is far from a whole exponent
constexpr int CAND = 512;
constexpr int MAX_PARTS = 64;
typedef unsigned long long u64;

template <typename T> constexpr int vec() { return 16 / (int)sizeof(T); }

__device__ __forceinline__ float max3(float a, float b, float c) {     // fmaxf would first quiet each operand
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <typename T> struct Piece;
template <> struct Piece<bf16> {
  u32x4 w;
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const unsigned d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __builtin_bit_cast(float, d[i] << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, d[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void none() { w = u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
};
template <> struct Piece<float> {
  u32x4 w;
  __device__ __forceinline__ void get(float (&f)[4]) const {
    const unsigned d[4] = {w.x, w.y, w.z, w.w};    // (a bit_cast of w.y itself gives w.x)
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_bit_cast(float, d[i]);
  }
  __device__ __forceinline__ void none() { w = u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }
};
// From here on the pieces are taken for others: what was unpacked of them is not kept for a later pass, which would be twice the registers.
template <typename P> __device__ __forceinline__ void forget(P& p) { asm volatile("" : "+v"(p.w)); }
template <typename T> union Out {
  u32x4 w;
  T v[vec<T>()];
};

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <typename Op> __device__ __forceinline__ float over_wave(float v, Op op) {
  v = op(v, dpp<0xB1>(v));                        // the neighbour
  v = op(v, dpp<0x4E>(v));                        // the other two of four
  v = op(v, dpp<0x141>(v));                       // mirrored in eight
  v = op(v, dpp<0x140>(v));                       // mirrored in sixteen
  v = op(v, __shfl_xor(v, 16, 64));
  return op(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float wave_max(float v) { return over_wave(v, max_of); }
__device__ __forceinline__ float wave_sum(float v) { return over_wave(v, [](float a, float b) { return a + b; }); }

// an order of fp32 numbers as one of unsigned ones; zeros of both signs are one
__device__ __forceinline__ unsigned ordered(float f) {
  const unsigned u = __builtin_bit_cast(unsigned, f + 0.f);
  return u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float disordered(unsigned u) { return __builtin_bit_cast(float, u ^ ((int)u < 0 ? 0x80000000u : 0xffffffffu)); }
// the larger logit first, of equal ones the lower column; 0 comes behind all
__device__ __forceinline__ u64 key_of(float f, int col) { return (u64)ordered(f) << 32 | (unsigned)~col; }
__device__ __forceinline__ int col_of(u64 key) { return (int)~(unsigned)key; }
__device__ __forceinline__ float value_of(u64 key) { return disordered((unsigned)(key >> 32)); }

__device__ __forceinline__ float log_prob(float x, float m, float scale, float ln) {
  return x == -INFINITY && ln == ln ? -INFINITY : scale * (x - m) - ln;
}

// What a row's gradient is made of: dx = p (a - b (ln p + h)) + at the token w, all times scale already
struct Weights {
  float a, b, h, w;
  int token;
  bool none;
};
__device__ __forceinline__ Weights weights_of(const LogprobArgs& a, int64_t row, bool with_h) {
  Weights r;
  r.token = a.target ? a.target[row] : -1;
  const bool has = r.token >= 0 && r.token < a.vocab;
  const float w = a.dlogp && has ? a.dlogp[row] : 0.f, dh = with_h && a.dentropy ? a.dentropy[row] : 0.f, dl = a.dlse ? a.dlse[row] : 0.f;
  if (!has) r.token = -1;
  r.a = a.scale * (dl - w);
  r.b = a.scale * dh;
  r.w = a.scale * w;
  r.h = 0.f;
  r.none = w == 0.f && dh == 0.f && dl == 0.f;
  return r;
}
template <bool H> __device__ __forceinline__ float grad_of(float x, float m, float c, float log2s, const Weights& w) {
  const float u = fmaf(x - m, c, -log2s), p = __builtin_amdgcn_exp2f(u);
  return H ? p * fmaf(-w.b, fmaf(fmaxf(u, FAR), LN2, w.h), w.a) : p * w.a;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <bool H> __device__ __forceinline__ void piece_out(const float (&f)[8], float m, float c, float log2s, const Weights& w, Out<bf16>& o) {
  unsigned d[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 g = {grad_of<H>(f[2 * i], m, c, log2s, w), grad_of<H>(f[2 * i + 1], m, c, log2s, w)};
    d[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(g, bf16x2));
  }
  o.w = u32x4{d[0], d[1], d[2], d[3]};
}
template <bool H> __device__ __forceinline__ void piece_out(const float (&f)[4], float m, float c, float log2s, const Weights& w, Out<float>& o) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o.v[i] = grad_of<H>(f[i], m, c, log2s, w);
}
template <typename T, bool H> __device__ __forceinline__ void piece_grad(const Piece<T>& p, float m, float c, float log2s, const Weights& w, Out<T>& o) {
  float f[vec<T>()];
  p.get(f);
  piece_out<H>(f, m, c, log2s, w, o);
}
template <bool ONCE, typename T> __device__ __forceinline__ void put_apart(T* to, const Out<T>& o, bool together) {
  if (together) put<ONCE>(to, o.w);
  else
#pragma unroll
    for (int e = 0; e < vec<T>(); ++e) to[e] = o.v[e];
}
// n more entries of a list: the first one's place.  (The address is hidden from the compiler, which would make a loop over the lanes of additions to one address.)
__device__ __forceinline__ int list_take(int* length, int n) {
  unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) int*)length;
  asm volatile("" : "+v"(at));
  return __hip_atomic_fetch_add((__attribute__((address_space(3))) int*)(uintptr_t)at, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
// entries of a list before `key`; the list is filled up with zeros to a multiple of eight
__device__ __forceinline__ int rank_of(u64 key, const u64* list, int n) {
  int rank = 0;
  for (int j = 0; j < n; j += 8)
#pragma unroll
    for (int e = 0; e < 8; ++e) rank += list[j + e] > key;
  return rank;
}

// How a row's columns lie: `lead` before the first 16-byte boundary, `full` pieces, and the rest
template <typename T> struct Span {
  int n, lead, full, tail;
  __device__ __forceinline__ Span(const T* x, int cols) : n(cols) {
    constexpr int V = vec<T>();
    lead = min(n, (int)((V - (unsigned)((uintptr_t)x / sizeof(T)) % V) % V));
    full = (n - lead) / V;
    tail = lead + full * V;
  }
  // the column that thread t takes by itself, or -1
  __device__ __forceinline__ int edge(int t) const { return t < lead ? t : t - lead < n - tail ? tail + t - lead : -1; }
};

template <typename T> __device__ __forceinline__ float piece_max(const Piece<T>& p) {
  constexpr int V = vec<T>();
  float f[V];
  p.get(f);
  float m = max3(f[0], f[1], f[2]);
#pragma unroll
  for (int e = 3; e < V; e += 2) m = max3(m, f[e], e + 1 < V ? f[e + 1] : f[e]);
  return m;
}
// what exponents are taken from: the maximum, or zero where there is nothing but -inf
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// One row, or part `blockIdx.x % parts` of one, whose findings go to rec (m, S, T) and keys.  WALK pieces of every thread are loaded while the WALK before them are worked on.
// (Four pieces in the place of two: 2000 rows x 50000 46.8 us against 42.5.  Workgroups that go on to a next row, whose first pieces they load before the sums are joined, take
// registers that leave six wavefronts to a SIMD in the place of eight: 4000 x 32000 with 20 alternatives 75 us against 58.)
constexpr int WALK = 2;
template <typename T, int NT, bool TOP, bool H, bool ONCE>
__global__ __launch_bounds__(NT, 8) void logprob_kernel(LogprobArgs a, int parts, int cols, float4* rec, u64* keys) {
  constexpr int V = vec<T>(), WAVES = NT / 64, BARS = NT < 256 ? NT : 256;      // BARS: groups of threads whose maxima are compared
  constexpr int KEPT = NT == 64 ? WALK : 1;         // maxima that are kept of a thread's WALK pieces
  extern __shared__ float group_max[];             // TOP: [groups * KEPT][NT]
  __shared__ float gmax[BARS], red[2][WAVES];
  __shared__ u64 cand[TOP ? CAND : 1], best[TOP ? WAVES : 1];
  __shared__ int ncand;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t unit = blockIdx.x, row = parts > 1 ? unit / parts : unit;
  const int c0 = parts > 1 ? (int)(unit % parts) * cols : 0;
  const T* x = (const T*)a.x + row * a.ldx + c0;
  const Span<T> sp(x, min(cols, a.vocab - c0));
  const int groups = (sp.full + NT * WALK - 1) / (NT * WALK);
  auto load = [&](Piece<T> (&v)[WALK], int g) {
#pragma unroll
    for (int u = 0; u < WALK; ++u) {
      const int i = (g * WALK + u) * NT + t;
      if ((g + 1) * WALK * NT <= sp.full) v[u].w = fetch<ONCE, u32x4>(x + sp.lead + i * V);
      else {
        v[u].none();
        if (i < sp.full) v[u].w = fetch<ONCE, u32x4>(x + sp.lead + i * V);
      }
    }
  };
  Piece<T> now[WALK];
  load(now, 0);
  const int token = a.target ? a.target[row] : -1;
  const int ecol = sp.edge(t);
  const float xe = ecol >= 0 ? to_f32(x[ecol]) : -INFINITY;
  if (TOP) {
    for (int i = t; i < CAND; i += NT) cand[i] = 0;
    if (t == 0) ncand = 0;
  }

  // Sums of 2^(c x - base), base the rounding of c times the maximum so far: one fma an element, and no matter what base was rounded to.  A maximum so low that c times
  // it is beyond -EDGE counts as that; rows whose own is beyond either way are walked again below.
  const float c = a.scale * LOG2E, low = -EDGE / c;
  auto base_at = [&](float m) {
    float b = fmaxf(m, low) * c;
    asm("" : "+v"(b));                             // rounded here: the compiler would subtract the product itself from another base
    return b;
  };
  float tm = -INFINITY, base = base_at(tm), s = 0.f, h = 0.f;
  auto term = [&](float f) {
    const float z = fmaf(f, c, -base), e = __builtin_amdgcn_exp2f(z);
    s += e;
    if (H) h = fmaf(e, -fmaxf(z, FAR), h);
  };
  auto move = [&](float m) {                       // to a maximum of m
    const float to = base_at(m), z = fmaxf(base - to, FAR), f = __builtin_amdgcn_exp2f(z);
    if (H) h = fmaf(s, -z, h) * f;
    s *= f;
    tm = m;
    base = to;
  };
  for (int g = 0; g < groups; ++g) {
    Piece<T> next[WALK];
    if (g + 1 < groups) load(next, g + 1);
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < WALK; ++u) {
      const float q = piece_max(now[u]);
      m = u ? max_of(m, q) : q;
      if (TOP && KEPT > 1) group_max[(g * WALK + u) * NT + t] = q;
    }
    if (TOP && KEPT == 1) group_max[g * NT + t] = m;
    move(max_of(tm, m));
#pragma unroll
    for (int u = 0; u < WALK; ++u) {
      float f[V];
      now[u].get(f);
#pragma unroll
      for (int e = 0; e < V; ++e) term(f[e]);
      now[u] = next[u];
    }
  }
  const bool has_token = token >= 0 && token < a.vocab;
  const float xt = has_token && t == 0 && parts == 1 ? to_f32(x[token]) : 0.f;
  move(max_of(tm, xe));
  term(xe);
  const float gm = NT > BARS ? max_of(tm, dpp<0xB1>(tm)) : tm;
  if (t % (NT / BARS) == 0) gmax[t / (NT / BARS)] = gm;
  __syncthreads();
  float group[BARS / 64];
#pragma unroll
  for (int i = 0; i < BARS / 64; ++i) group[i] = gmax[i * 64 + lane];
  float m = group[0];
#pragma unroll
  for (int i = 1; i < BARS / 64; ++i) m = max_of(m, group[i]);
  m = wave_max(m);
  const float at = base_of(m);
  move(m);
  // what base is more than c m, so that ln S is that of 2^(c (x - m))
  float more = fmaf(-m, c, base);
  if (!(fabsf(m * c) < EDGE) && m != -INFINITY) {
    s = h = more = 0.f;
    auto far_term = [&](float f) {
      const float z = (f - m) * c, e = __builtin_amdgcn_exp2f(z);
      s += e;
      if (H) h = fmaf(e, -fmaxf(z, FAR), h);
    };
    for (int i = t; i < sp.full; i += NT) {
      Piece<T> p;
      float f[V];
      p.w = fetch<ONCE, u32x4>(x + sp.lead + i * V);
      p.get(f);
#pragma unroll
      for (int e = 0; e < V; ++e) far_term(f[e]);
    }
    if (ecol >= 0) far_term(xe);
  }

  float bar = 0.f;
  auto offer = [&](float f, int col) {
    const int slot = list_take(&ncand, 1);
    if (slot < CAND) cand[slot] = key_of(f, c0 + col);
  };
  // the elements that reach the bar, or are beyond it
  auto collect = [&](auto wanted) {
    for (int g = 0; g < groups * KEPT; ++g) {
      if (!wanted(group_max[g * NT + t])) continue;
      if (*(volatile int*)&ncand > CAND) break;        // it will not be used
      Piece<T> p[WALK / KEPT];
#pragma unroll
      for (int u = 0; u < WALK / KEPT; ++u) {
        const int i = (g * (WALK / KEPT) + u) * NT + t;
        p[u].none();
        if (i < sp.full) p[u].w = fetch<ONCE, u32x4>(x + sp.lead + i * V);
      }
#pragma unroll
      for (int u = 0; u < WALK / KEPT; ++u) {
        const int i = (g * (WALK / KEPT) + u) * NT + t;
        if (!(i < sp.full && wanted(piece_max(p[u])))) continue;
        float f[V];
        p[u].get(f);
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (wanted(f[e])) offer(f[e], sp.lead + i * V + e);
      }
    }
    if (ecol >= 0 && wanted(xe)) offer(xe, ecol);
  };
  if (TOP) {
    // The k-th largest of the groups' maxima, which bf16 has in its leading 16 bits.  One wavefront: of its 64 lanes, or, for more alternatives than half of them, of
    // four groups to a lane: pairs of pieces, pieces, halves or quarters of one (4096 rows x 4000 with 64 alternatives 23 us; by lanes, which leave some 4.7 x 64 elements to the
    // bound and one time in fifty more than the list takes, 230).
    const bool many = NT > 64 || a.top > 32;
    unsigned reach = 0, mine[4];
    if (NT == 64) {
      mine[0] = ordered(group[0]);
      if (many && sp.full <= 128) {
        Piece<T> p[WALK];
        load(p, 0);
        float q[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float f[V];
          p[u].get(f);
#pragma unroll
          for (int i = 0; i < 4; ++i) q[u][i] = max_of(f[i * V / 4], f[i * V / 4 + V / 4 - 1]);
        }
        const bool two = sp.full > 64;
        mine[0] = ordered(max3(xe, q[0][0], two ? q[0][1] : q[0][0]));
        mine[1] = ordered(two ? max_of(q[0][2], q[0][3]) : q[0][1]);
        mine[2] = ordered(two ? max_of(q[1][0], q[1][1]) : q[0][2]);
        mine[3] = ordered(two ? max_of(q[1][2], q[1][3]) : q[0][3]);
      } else if (many) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int step = sp.full <= 256 ? 1 : 2;
          float f = i ? -INFINITY : xe;
          if (i * step < groups * KEPT) f = max3(f, group_max[i * step * NT + t], group_max[(i * step + step - 1) * NT + t]);
          mine[i] = ordered(f);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < BARS / 64; ++i) mine[i] = ordered(group[i]);
    }
#pragma unroll
    for (int b = 31; b >= (sizeof(T) == 2 ? 16 : 0); --b) {
      const unsigned next = reach | 1u << b;
      int n = __builtin_popcountll(__ballot(mine[0] >= next));
      if (many)
#pragma unroll
        for (int i = 1; i < 4; ++i) n += __builtin_popcountll(__ballot(mine[i] >= next));
      if (n >= a.top) reach = next;
    }
    // in the order's numbers the lower half of a negative bf16 is ones: with zeros the bound would be a number that bf16 does not have, below those that tie
    if (sizeof(T) == 2 && !(reach >> 31)) reach |= 0xffffu;
    bar = reach <= 0x007fffffu ? -INFINITY : disordered(reach);
    collect([&](float f) { return f >= bar; });
  }

  s = wave_sum(s);
  if (H) h = wave_sum(h);
  if (lane == 0) { red[0][wave] = s; red[1][wave] = h; }
  __syncthreads();
  s = wave_sum(lane < WAVES ? red[0][lane] : 0.f);
  if (H) h = wave_sum(lane < WAVES ? red[1][lane] : 0.f);

  const bool bad = !(s < INFINITY);
  // sum 2^z with z = c (x - m) - more, and the entropy's mean of -z: -more of it is more of the logarithm
  const float ln = bad ? NAN : s == 0.f ? -INFINITY : logf(s) + LN2 * more;
  if (t == 0) {
    if (parts > 1) rec[unit] = make_float4(m, s, h, s == 0.f ? 0.f : more);
    else {
      if (a.logp) a.logp[row] = has_token ? log_prob(xt, at, a.scale, ln) : 0.f;
      if (a.stats) { a.stats[2 * row] = m; a.stats[2 * row + 1] = ln; }
      if (H && a.entropy) a.entropy[row] = s == 0.f ? 0.f : logf(s) + LN2 * h / s;
    }
  }
  if (!TOP) return;
  auto put = [&](int rank, u64 key) {
    if (parts > 1) keys[unit * a.top + rank] = key;
    else {
      a.top_id[row * a.top + rank] = bad ? -1 : col_of(key);
      a.top_logp[row * a.top + rank] = bad ? NAN : log_prob(value_of(key), at, a.scale, ln);
    }
  };
  auto put_list = [&](int n) {
    for (int i = t; i < n; i += NT) {
      const u64 key = cand[i];
      const int rank = rank_of(key, cand, n);
      if (rank < a.top) put(rank, key);
    }
  };
  int n = ncand;
  if (bad) {
    for (int i = t; i < a.top; i += NT) put(i, 0);
    return;
  }
  if (n <= CAND) {
    put_list(n);
    for (int i = n + t; i < a.top; i += NT) put(i, 0);      // a part with fewer columns
    return;
  }
  // More than the list takes: as a rule columns that are equal to the bar (a constant row, or the -inf of one with fewer tokens left than alternatives).  The list then takes
  // those beyond it, and one wavefront finds the first of the equal ones.
  __syncthreads();
  for (int i = t; i < CAND; i += NT) cand[i] = 0;
  if (t == 0) ncand = 0;
  __syncthreads();
  collect([&](float f) { return f > bar; });
  __syncthreads();
  n = ncand;
  if (n <= CAND) {
    put_list(n);
    if (wave == 0)
      for (int col = lane, rank = n; rank < a.top && col - lane < sp.n; col += 64) {
        const bool equal = col < sp.n && to_f32(x[col]) == bar;
        const u64 mask = __ballot(equal);
        const int at_rank = rank + __builtin_popcountll(mask & ((1ull << lane) - 1));
        if (equal && at_rank < a.top) put(at_rank, key_of(bar, c0 + col));
        rank += __builtin_popcountll(mask);
      }
    return;
  }
  // Still more: one by one.
  u64 last = ~0ull, mine = 0;
  for (int r = 0; r < a.top; ++r) {
    if (mine == 0 || mine == last) {               // the thread's largest behind the last one taken
      mine = 0;
      auto look = [&](float f, int col) {
        const u64 key = key_of(f, c0 + col);
        if (key < last && key > mine) mine = key;
      };
      for (int i = t; i < sp.full; i += NT) {
        Piece<T> p;
        float f[V];
        p.w = fetch<ONCE, u32x4>(x + sp.lead + i * V);
        p.get(f);
#pragma unroll
        for (int e = 0; e < V; ++e) look(f[e], sp.lead + i * V + e);
      }
      if (ecol >= 0) look(xe, ecol);
    }
    u64 b = mine;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) { const u64 o = __shfl_xor(b, d, 64); b = o > b ? o : b; }
    if (lane == 0) best[wave] = b;
    __syncthreads();
    b = best[0];
    for (int i = 1; i < WAVES; ++i) b = best[i] > b ? best[i] : b;
    __syncthreads();
    if (t == 0) put(r, b);
    last = b;
  }
}

// 16 bytes of every lane to LDS, lane l's to lds_addr + 16 l; what lies beyond the buffer's bytes comes as zeros.  Inline assembly because the compiler would wait for such a load
// before any access to LDS; it is awaited by hand.
typedef int rsrc_words __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ rsrc_words raw_rsrc(const void* base, unsigned bytes) {
  const uint64_t a = (uint64_t)base;
  return rsrc_words{(int)(unsigned)a, (int)(unsigned)((a >> 32) & 0xffffu), (int)bytes, 0x00020000};
}
__device__ __forceinline__ void load_to_lds(rsrc_words rsrc, unsigned lds_addr, unsigned offset) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(offset), "s"(rsrc) : "memory");
}

// Values and gradient of whole rows, blockIdx.x and every gridDim.x-th behind it.  H: with the entropy.  The next row's last NL pieces are on their way to LDS while this one's
// exponentials are summed, the others while its gradient is stored.  (4096 rows x 128000: 410 us with half of the pieces by LDS, 429 with a quarter; 446 with none, when memory
// rests during the sums, since all compute units come to them together; 420 with every second piece instead of the last ones.)
constexpr int waves_of(int nv) { return nv > 8 ? 4 : nv > 4 ? 6 : 8; }      // wavefronts to a SIMD whose registers hold nv pieces each
template <typename T, int NT, int NV, int NL, bool H, bool ONCE>
__global__ __launch_bounds__(NT, waves_of(NV)) void logprob_both_kernel(LogprobArgs a) {
  constexpr int V = vec<T>(), WAVES = NT / 64;
  __shared__ float red[3][WAVES];
  __shared__ u32x4 ahead[NL > 0 ? NL : 1][NL > 0 ? NT : 1];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const float c = a.scale * LOG2E;
  auto load = [&](Piece<T>& p, const T* x, const Span<T>& sp, int k) {
    if ((k + 1) * NT <= sp.full) p.w = fetch<ONCE, u32x4>(x + sp.lead + (k * NT + t) * V);
    else {
      p.none();
      if (k * NT + t < sp.full) p.w = fetch<ONCE, u32x4>(x + sp.lead + (k * NT + t) * V);
    }
  };
  Piece<T> v[NV];
  int64_t row = blockIdx.x;
  const T* x = (const T*)a.x + row * a.ldx;
  Span<T> sp(x, a.vocab);
  int ecol = sp.edge(t);
  float xe = ecol >= 0 ? to_f32(x[ecol]) : -INFINITY;
  Weights w = weights_of(a, row, H);
  float xt = w.token >= 0 ? to_f32(x[w.token]) : 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) load(v[k], x, sp, k);
  for (;;) {
    float m = xe;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (k * NT < sp.full) m = max_of(m, piece_max(v[k]));
    // the token's has arrived before any thread puts a gradient in its place, and no load that the compiler counts is behind those to LDS
    asm volatile("" : "+v"(xt), "+v"(m));
    const int64_t after = row + gridDim.x;
    const bool more = after < a.rows;
    const T* xn = more ? (const T*)a.x + after * a.ldx : x;
    const Span<T> spn(xn, more ? a.vocab : 0);
    if (NL > 0 && more) {
      const rsrc_words rsrc = raw_rsrc(xn + spn.lead, (unsigned)spn.full * 16u);
#pragma unroll
      for (int l = 0; l < NL; ++l) load_to_lds(rsrc, (unsigned)(size_t)((lds_char*)&ahead[l][0] + wave * 1024), (unsigned)((NV - NL + l) * NT + t) * 16u);
    }
    m = wave_max(m);
    if (lane == 0) red[2][wave] = m;
    __syncthreads();
    m = wave_max(lane < WAVES ? red[2][lane] : -INFINITY);
    const float at = base_of(m);

    float s = 0.f, h = 0.f;
    auto term = [&](float f) {
      const float z = (f - at) * c, e = __builtin_amdgcn_exp2f(z);
      s += e;
      if (H) h = fmaf(e, -fmaxf(z, FAR), h);
    };
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (k * NT >= sp.full) continue;
      float f[V];
      forget(v[k]);
      v[k].get(f);
#pragma unroll
      for (int e = 0; e < V; ++e) term(f[e]);
    }
    term(xe);
    s = wave_sum(s);
    if (H) h = wave_sum(h);
    if (lane == 0) { red[0][wave] = s; red[1][wave] = h; }
    __syncthreads();
    s = wave_sum(lane < WAVES ? red[0][lane] : 0.f);
    if (H) h = wave_sum(lane < WAVES ? red[1][lane] : 0.f);

    const bool bad = !(s < INFINITY);
    const float ln = bad ? NAN : logf(s), entropy = s == 0.f ? 0.f : ln + LN2 * h / s;
    if (t == 0) {
      if (a.logp) a.logp[row] = w.token >= 0 ? log_prob(xt, at, a.scale, ln) : 0.f;
      if (a.stats) { a.stats[2 * row] = m; a.stats[2 * row + 1] = ln; }
      if (H && a.entropy) a.entropy[row] = entropy;
    }

    T* dx = (T*)a.dx + row * a.lddx;
    if (H) w.h = entropy;
    const bool none = w.none || empty_row(m, ln), together = (((uintptr_t)dx ^ (uintptr_t)x) & 15) == 0;
    const float log2s = ln * LOG2E;
    if (NL > 0) {
      __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): the pieces in LDS have landed
      asm volatile("" ::: "memory");               // and none is read before: the wait by itself names no memory
    }
    const int ecoln = spn.edge(t);
    const float xen = ecoln >= 0 ? to_f32(xn[ecoln]) : -INFINITY;
    const Weights wn = weights_of(a, more ? after : row, H);
    const float xtn = more && wn.token >= 0 ? to_f32(xn[wn.token]) : 0.f;
    auto next = [&](int k) {
      if (k < NV - NL) load(v[k], xn, spn, k);
      else {
        v[k].none();
        if (k * NT + t < spn.full) v[k].w = ahead[k - (NV - NL)][t];
      }
    };
    if (together && !none) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (k * NT + t < sp.full) {
          Out<T> o;
          forget(v[k]);
          piece_grad<T, H>(v[k], at, c, log2s, w, o);
          put<ONCE>(dx + sp.lead + (k * NT + t) * V, o.w);
        }
        next(k);
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (k * NT + t < sp.full) {
          Out<T> o;
          forget(v[k]);
          piece_grad<T, H>(v[k], at, c, log2s, w, o);
          if (none) o.w = u32x4{0, 0, 0, 0};
          put_apart<ONCE>(dx + sp.lead + (k * NT + t) * V, o, together);
        }
        next(k);
      }
    }
    if (ecol >= 0) dx[ecol] = from_f32<T>(none ? 0.f : grad_of<H>(xe, at, c, log2s, w));
    // the token's, by the thread that has stored it above, so that this store comes behind that one
    const int piece = w.token - sp.lead;
    const bool inside = piece >= 0 && w.token < sp.tail;
    if (w.token >= 0 && !none && (inside ? piece / V % NT == t : ecol == w.token)) dx[w.token] = from_f32<T>(grad_of<H>(xt, at, c, log2s, w) + w.w);
    if (!more) break;
    row = after;
    x = xn;
    sp = spn;
    ecol = ecoln;
    xe = xen;
    w = wn;
    xt = xtn;
  }
}

// Joins the parts of a row.
constexpr int NTJ = 256;
template <typename T>
__global__ __launch_bounds__(NTJ) void logprob_join_kernel(LogprobArgs a, int parts, const float4* rec, const u64* keys) {
  __shared__ u64 cand[MAX_PARTS * LOGPROB_MAX_TOP + 8];
  __shared__ int ncand;
  const int t = threadIdx.x, lane = t & 63;
  const int64_t row = blockIdx.x;
  const float4 r = lane < parts ? rec[row * parts + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const float m = wave_max(r.x), at = m == -INFINITY ? 0.f : m, c = a.scale * LOG2E;
  // a part whose maximum is -inf has S = T = 0 (or NaN, which stays one)
  const float z = fmaxf(fmaf(r.x - at, c, r.w), FAR), f = __builtin_amdgcn_exp2f(z);
  const float s = wave_sum(r.y * f), h = wave_sum(fmaf(r.y, -z, r.z) * f);
  const bool bad = !(s < INFINITY);
  const float ln = bad ? NAN : logf(s);
  if (t == 0) {
    const int token = a.target ? a.target[row] : -1;
    if (a.logp) a.logp[row] = token >= 0 && token < a.vocab ? log_prob(to_f32(((const T*)a.x)[row * a.ldx + token]), at, a.scale, ln) : 0.f;
    if (a.stats) { a.stats[2 * row] = m; a.stats[2 * row + 1] = ln; }
    if (a.entropy) a.entropy[row] = s == 0.f ? 0.f : ln + LN2 * h / s;
    ncand = 0;
  }
  if (a.top == 0) return;
  keys += row * parts * a.top;
  // With j = ceil(top / parts) and r = ceil(top / j): r parts have j keys each that reach the r-th largest of the parts' j-th keys, so nothing below it is among the first.
  const int j = (a.top + parts - 1) / parts, r_th = (a.top + j - 1) / j;
  const u64 jth = lane < parts ? keys[lane * a.top + j - 1] : 0;
  u64 bar = 0;
  auto narrow = [&](int from, int to) {
    for (int b = from; b >= to; --b)
      if (__builtin_popcountll(__ballot(jth >= (bar | 1ull << b))) >= r_th) bar |= 1ull << b;
  };
  narrow(63, 32);
  if (__builtin_popcountll(__ballot(jth >= bar)) > r_th) narrow(31, 0);   // ties: the columns decide (8 constant rows of 128000 43 -> 27 us)
  __syncthreads();
  for (int i = t; i < parts * a.top; i += NTJ) {
    const u64 k = keys[i];
    if (k >= bar && k != 0) cand[list_take(&ncand, 1)] = k;
  }
  __syncthreads();
  const int n = ncand;
  if (t < 8) cand[n + t] = 0;
  __syncthreads();
  for (int i = t; i < (bad ? a.top : n); i += NTJ) {
    const u64 key = bad ? 0 : cand[i];
    const int rank = bad ? i : rank_of(key, cand, n);
    if (rank < a.top) {
      a.top_id[row * a.top + rank] = bad ? -1 : col_of(key);
      a.top_logp[row * a.top + rank] = bad ? NAN : log_prob(value_of(key), at, a.scale, ln);
    }
  }
}

// The gradient from a row's statistics: GV pieces of a row to each thread.
constexpr int NTG = 256, GV = 4;
template <typename T, bool H, bool ONCE>
__global__ __launch_bounds__(NTG) void logprob_grad_kernel(LogprobArgs a, int chunks) {
  constexpr int V = vec<T>();
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x / chunks;
  const int chunk = blockIdx.x % chunks;
  const T* x = (const T*)a.x + row * a.ldx;
  T* dx = (T*)a.dx + row * a.lddx;
  const Span<T> sp(x, a.vocab);
  Weights w = weights_of(a, row, H);
  const float m = a.stats[2 * row], ln = a.stats[2 * row + 1], log2s = ln * LOG2E, c = a.scale * LOG2E;
  if (H) w.h = a.entropy[row];
  const bool none = w.none || empty_row(m, ln), together = (((uintptr_t)dx ^ (uintptr_t)x) & 15) == 0;
  const int first = chunk * NTG * GV + t;
  Piece<T> v[GV];
  const int ecol = chunk == chunks - 1 ? sp.edge(t) : -1;
  const int piece = w.token - sp.lead;
  const bool inside = piece >= 0 && w.token < sp.tail;
  // the token's is stored behind the others, by the same thread
  const bool owner = w.token >= 0 && !none && (inside ? piece / V / (NTG * GV) == chunk && piece / V % NTG == t : ecol == w.token);
  float xe = 0.f, xt = 0.f;
  if (!none) {
#pragma unroll
    for (int k = 0; k < GV; ++k)
      if (first + k * NTG < sp.full) v[k].w = fetch<false, u32x4>(x + sp.lead + (int64_t)(first + k * NTG) * V);
    if (ecol >= 0) xe = to_f32(x[ecol]);
    if (owner) xt = to_f32(x[w.token]);
  }
#pragma unroll
  for (int k = 0; k < GV; ++k) {
    if (first + k * NTG >= sp.full) continue;
    Out<T> o;
    if (none) o.w = u32x4{0, 0, 0, 0};
    else piece_grad<T, H>(v[k], m, c, log2s, w, o);
    put_apart<ONCE>(dx + sp.lead + (int64_t)(first + k * NTG) * V, o, together);
  }
  if (ecol >= 0) dx[ecol] = from_f32<T>(none ? 0.f : grad_of<H>(xe, m, c, log2s, w));
  if (owner) dx[w.token] = from_f32<T>(grad_of<H>(xt, m, c, log2s, w) + w.w);
}

// Parts of a row: where the rows do not fill the chip up to a workgroup per compute unit, none below 512 pieces; and so many that a part's group maxima take at most 32 KiB.
template <typename T> int parts_of(const LogprobArgs& a, int forced) {
  const int most = 8192 * WALK * vec<T>(), need = a.top > 0 ? (a.vocab + most - 1) / most : 1;
  const int fill = a.rows < 256 ? 256 / a.rows : 1, room = a.vocab / (512 * vec<T>());
  int p = fill < room ? fill : room;
  p = p > need ? p : need;
  if (forced) p = p > 3 ? p : a.vocab < 3 ? a.vocab : 3;
  return p < 1 ? 1 : p > MAX_PARTS ? MAX_PARTS : p;
}
size_t part_bytes(const LogprobArgs& a, int parts) { return parts > 1 ? (size_t)a.rows * parts * (sizeof(float4) + a.top * sizeof(u64)) : 0; }

using std::integral_constant;
// Whether accesses ask the caches to keep nothing.  Values: logits of more than the last-level cache's 256 MB, which leave nothing in it for a backward (2048 rows x 128000 with
// alternatives 100 us against 109, 4096 x 64000 in two calls 277 against 287; but 1023 x 50333 in two calls, 103 MB that the backward finds there, 63 against 56).  Values and
// gradient: both of more than that together (4096 x 32000 92 us against 108).  The gradient by itself: its stores, from the 32 MB on that the L2s hold (1023 x 50333 in two
// calls 56 us against 64, 4000 x 32000 127 against 156; 400 x 50333, 40 MB, 27.2 either way).
template <typename T> bool more_than(const LogprobArgs& a, int64_t mb) { return (int64_t)a.rows * a.vocab * (int64_t)sizeof(T) > mb << 20; }
template <typename F> hipError_t by_size(bool large, F f) { return large ? f(std::true_type{}) : f(std::false_type{}); }

template <typename T, bool TOP, bool H>
hipError_t values_launch(const LogprobArgs& a, int parts, void* scratch, hipStream_t s) {
  // columns of a part: whole pieces, so that the last parts may have none left
  const int V = vec<T>(), cols = parts > 1 ? ((a.vocab + parts - 1) / parts + V - 1) / V * V : a.vocab;
  const int used = (a.vocab + cols - 1) / cols, pieces = (cols + V - 1) / V;
  float4* rec = (float4*)scratch;
  u64* keys = (u64*)(rec + (int64_t)a.rows * used);
  auto launch = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    const int groups = (pieces + NT * WALK - 1) / (NT * WALK);
    return by_size(more_than<T>(a, 256), [&](auto o) {
      hipLaunchKernelGGL((logprob_kernel<T, NT, TOP, H, o()>), dim3((unsigned)((int64_t)a.rows * used)), dim3(NT), TOP ? groups * (NT == 64 ? WALK : 1) * NT * sizeof(float) : 0, s, a, used, cols, rec,
                         keys);
      return hipGetLastError();
    });
  };
  // One wavefront a row up to 512 pieces (8192 rows x 2000 10.4 us; in 256 threads 18.9), without alternatives up to 1024 where there are rows enough (8192 x 5000 18.9 us, in 256
  // threads 23.6; with alternatives 8192 x 8000 49 against 41).  256 threads up to 4096 (5882 x 17000 43.7 us, in 512 50.0), but 512 from 2048 on where the rows do not
  // fill the chip with them (64 x 128000 in four parts each 14.7 against 18.4).
  const int64_t units = (int64_t)a.rows * used;
  const hipError_t e = pieces <= 512 || (!TOP && pieces <= 1024 && units >= 4096)  ? launch(integral_constant<int, 64>{})
                       : pieces <= 2048 || (pieces <= 4096 && units >= 1024)       ? launch(integral_constant<int, 256>{})
                                                                                   : launch(integral_constant<int, 512>{});
  if (e != hipSuccess || used == 1) return e;
  hipLaunchKernelGGL((logprob_join_kernel<T>), dim3(a.rows), dim3(NTJ), 0, s, a, used, rec, keys);
  return hipGetLastError();
}

// Rows in registers: at most this many pieces
constexpr int MOST_PIECES = 1024 * 16;
constexpr int FEW = 256;               // pieces up to which few rows are spread over 256 threads each
template <typename T, bool H> hipError_t both_launch(const LogprobArgs& a, hipStream_t s) {
  const auto launch = [&](auto nt, auto nv) {
    constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value, NL = NV >= 8 ? NV / 2 : 0;
    const int wgs = cu_count() * (waves_of(NV) * 256 / NT);
    const auto go = [&](auto o) {
      hipLaunchKernelGGL((logprob_both_kernel<T, NT, NV, NL, H, o()>), dim3(a.rows < wgs ? a.rows : wgs), dim3(NT), 0, s, a);
      return hipGetLastError();
    };
    if constexpr (NT == FEW && NV == 1) return go(std::false_type{});        // 2 MB at most
    else return by_size(more_than<T>(a, 128), go);
  };
  const int pieces = (a.vocab + vec<T>() - 1) / vec<T>();
  // One wavefront a row as far as it goes without giving up registers (8192 rows x 2000 16.3 us, in 256 threads 22), but for few rows
  // (512 x 2000 5.3 us, in 256 threads 4.6); two workgroups of 512 to a compute unit rather than one of
  // 1024 (2000 x 50000 88.5 us against 98.5), as long as 64 registers of each thread hold the row.
  return pieces <= 64     ? launch(integral_constant<int, 64>{}, integral_constant<int, 1>{})
         : pieces <= 256 && a.rows <= 512 ? launch(integral_constant<int, 256>{}, integral_constant<int, 1>{})
         : pieces <= 256  ? launch(integral_constant<int, 64>{}, integral_constant<int, 4>{})
         : pieces <= 512  ? launch(integral_constant<int, 64>{}, integral_constant<int, 8>{})
         : pieces <= 1024 ? launch(integral_constant<int, 256>{}, integral_constant<int, 4>{})
         : pieces <= 2048 ? launch(integral_constant<int, 256>{}, integral_constant<int, 8>{})
         : pieces <= 4096 ? launch(integral_constant<int, 512>{}, integral_constant<int, 8>{})
         : pieces <= 8192 ? launch(integral_constant<int, 512>{}, integral_constant<int, 16>{})
                          : launch(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

template <typename T> hipError_t grad_launch(LogprobArgs a, hipStream_t s) {
  const int per = NTG * GV * vec<T>(), chunks = (a.vocab + per - 1) / per, most = (1 << 23) / chunks;
  const bool large = more_than<T>(a, 32);
  // up to 2^23 workgroups a launch: logits of more than 137 GB take more than one
  for (int left = a.rows; left > 0; left -= most) {
    a.rows = left < most ? left : most;
    const hipError_t e = by_size(large, [&](auto o) {
      const dim3 grid(a.rows * chunks);
      if (a.dentropy) hipLaunchKernelGGL((logprob_grad_kernel<T, true, o()>), grid, dim3(NTG), 0, s, a, chunks);
      else hipLaunchKernelGGL((logprob_grad_kernel<T, false, o()>), grid, dim3(NTG), 0, s, a, chunks);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    a.x = (const T*)a.x + most * a.ldx;
    a.dx = (T*)a.dx + most * a.lddx;
    a.stats += 2 * (int64_t)most;
    a.target = a.target ? a.target + most : nullptr;
    a.entropy = a.entropy ? a.entropy + most : nullptr;
    a.dlogp = a.dlogp ? a.dlogp + most : nullptr;
    a.dentropy = a.dentropy ? a.dentropy + most : nullptr;
    a.dlse = a.dlse ? a.dlse + most : nullptr;
  }
  return hipSuccess;
}

template <typename T> hipError_t values(const LogprobArgs& a, bool forced, void* scratch, hipStream_t s) {
  const int parts = parts_of<T>(a, forced);
  if (a.top > 0) return a.entropy ? values_launch<T, true, true>(a, parts, scratch, s) : values_launch<T, true, false>(a, parts, scratch, s);
  return a.entropy ? values_launch<T, false, true>(a, parts, scratch, s) : values_launch<T, false, false>(a, parts, scratch, s);
}
template <typename T> hipError_t both(const LogprobArgs& a, bool forced, void* scratch, hipStream_t s) {
  if (a.top == 0 && parts_of<T>(a, forced) == 1 && a.vocab <= MOST_PIECES * vec<T>())
    return a.entropy ? both_launch<T, true>(a, s) : both_launch<T, false>(a, s);
  const hipError_t e = values<T>(a, forced, scratch, s);
  return e == hipSuccess ? grad_launch<T>(a, s) : e;
}

}  // namespace

size_t logprob_scratch_bytes(DType dt, const LogprobArgs& a) {
  size_t most = 0;
  for (const int forced : {0, 1}) {
    const size_t n = part_bytes(a, dt == DT_F32 ? parts_of<float>(a, forced) : parts_of<bf16>(a, forced));
    most = n > most ? n : most;
  }
  return most;
}
hipError_t logprob(DType dt, const LogprobArgs& a, bool split, void* scratch, hipStream_t s) {
  return dt == DT_F32 ? values<float>(a, split, scratch, s) : values<bf16>(a, split, scratch, s);
}
hipError_t logprob_grad(DType dt, const LogprobArgs& a, hipStream_t s) { return dt == DT_F32 ? grad_launch<float>(a, s) : grad_launch<bf16>(a, s); }
hipError_t logprob_both(DType dt, const LogprobArgs& a, bool split, void* scratch, hipStream_t s) {
  return dt == DT_F32 ? both<float>(a, split, scratch, s) : both<bf16>(a, split, scratch, s);
}

}  // namespace stg
