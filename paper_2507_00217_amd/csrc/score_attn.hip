// Attention of shaped scores over packed sequences for gfx950 in bf16 with fp32 softmax: the tiles, fragments and the split of the
// backward into dQ and dK/dV of attn_mfma.hip, with
//   s_ij = scale q_i.k_j,  capped c tanh(s / c),  minus slope_h |i - j|,
// a causal mask that a sequence's prefix opens, operands in buffers of their own, and sequences of any lengths one behind the other.
//
// Packing: tiles are cut per sequence, so no tile holds rows of two (their descriptors end with the sequence, rows past it read as
// zeros) and a mask is the bound of one interval.  A packed sequence i whose first row is b takes the slots b / BQ + i .. of the grid,
// BQ rows each: that is never less than it needs, so rows / BQ + n_seq slots are enough for any lengths, a workgroup finds its
// sequence by a search over the offsets (64 at a time), and no list of tiles has to be made beforehand.
//
// Exponents are in units of log 2 throughout.  The distance bias is slope times each pair's own distance, an exact whole number in fp32, so that it is off by
// one rounding of itself and a query's own key has none, however steep the slope (taken against a block's first row, as a scalar per lane plus a
// multiple of the row inside the block, one addition a score less, slopes of 1e4 left several percent in P, and it was no faster: forward and backward
// of 8 heads of 128 x 16384 rows 551 + 1724 us, now 554 + 1711).
#include "attn_tile.h"
#include "score.h"

#include <cfloat>
#include <type_traits>

namespace stg {
namespace {

// What a launch hands over beside ScoreArgs: constants of the score in units of log 2, and the shape of the grid.
struct ScoreCall {
  ScoreArgs a;
  float sl2;                     // scale * log2 e
  float raw;                     // 1 / scale: a bias in units of the plain product
  // cap: of the product x itself, s = c2 tanh(x scale / cap), c2 = cap log2 e
  float c2, ic2, kx;             // kx = 2 log2 e scale / cap
  float small, middling;         // |x| up to which the polynomials hold: s = x (sl2 + x^2 (p[0] + x^2 ...))
  float p3[2], p5[4];
  int wide;                      // the cap is far above the scale (and these two below any |x|)
  int tiles;                     // tiles of a sequence (equal sequences)
  int fold, nsplit;
  float* part;                   // [nsplit][rows][2 * hkv * hd] fp32
};

// ---- where a workgroup works ------------------------------------------------------------------------------------------------
struct Work { int lo, len, prefix, t; };       // rows of its sequence, its prefix, its tile; len = 0: nothing to do

// Sums over the lanes up to this one, by moves between lanes inside the instruction: rows of 16, then their ends into the rows behind.
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan_add(int v) {
  v = dpp_add<0x111, 0xf>(v);
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);
  return dpp_add<0x143, 0xc>(v);
}

// The workgroup of rank `rank`: equal sequences and up to 64 packed ones get theirs heaviest tiles first (QUERIES: the more keys, the
// heavier; else tiles of keys: the more queries).  Heaviness is counted in tiles.  Of a packed sequence of nt tiles, tiles of queries
// weigh their number, but those within the prefix as much as its last; tiles of keys nt - 1 minus their number, but those of the prefix
// nt - 1; without a causal mask all weigh the same.  The level that the rank falls into is searched for with the count of
// tiles of at least a weight, one sequence to a lane.
template <int BQ, bool QUERIES>
__device__ __forceinline__ Work find_work(const ScoreCall& c, int rank, int lane) {
  const ScoreArgs& a = c.a;
  Work w;
  if (a.seq_start && a.n_seq <= 64) {
    const SeqSpan s = seq_span(a, min(lane, a.n_seq - 1));
    const int len = lane < a.n_seq ? s.hi - s.lo : 0, nt = (len + BQ - 1) / BQ;
    // tiles 0 .. flat - 1 weigh `top`; QUERIES: tile t >= flat weighs t (more), else nt - 1 - t (less)
    const int inside = (s.prefix + BQ - 1) / BQ;
    const int flat = a.causal ? max(min(inside, nt), min(nt, 1)) : nt, top = QUERIES ? flat - 1 : nt - 1;
    auto heavier = [&](int x) { return QUERIES ? (x <= top ? nt : max(nt - x, 0)) : (x <= top ? flat + max(nt - flat - x, 0) : 0); };   // tiles of weight >= x
    auto total = [&](int x) { return __builtin_amdgcn_readlane(scan_add(heavier(x)), 63); };
    if (rank >= total(0)) { w.lo = w.len = w.prefix = w.t = 0; return w; }
    int lo = 0, hi = 1 + a.rows / BQ;                  // total(lo) > rank >= total(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (total(mid) > rank) lo = mid;
      else hi = mid;
    }
    const int k = rank - total(lo + 1), n = heavier(lo) - heavier(lo + 1), upto = scan_add(n);
    const int i = __builtin_ctzll(__ballot(upto > k));
    w.lo = __builtin_amdgcn_readlane(s.lo, i);
    w.len = __builtin_amdgcn_readlane(len, i);
    w.prefix = __builtin_amdgcn_readlane(s.prefix, i);
    const int nth = k - __builtin_amdgcn_readlane(upto - n, i);
    w.t = lo == __builtin_amdgcn_readlane(top, i) ? nth : QUERIES ? lo : __builtin_amdgcn_readlane(nt, i) - 1 - lo;
    return w;
  }
  int i, t;
  if (!a.seq_start) {
    i = rank % a.n_seq;
    t = QUERIES ? tile_of_rank(rank / a.n_seq, c.tiles, c.fold) : key_tile_of_rank(rank / a.n_seq, c.tiles, c.fold);
  } else {                                             // more sequences: the slots, last rows first for queries
    const int u = QUERIES ? a.rows / BQ + a.n_seq - 1 - rank : rank;
    i = 0;
    for (int n = a.n_seq; n > 1;) {                    // sequences i .. i + n - 1 are left; 64 of them are looked at
      const int step = (n + 63) >> 6, at = lane * step;
      const bool before = at < n && min(max(a.seq_start[i + min(at, n - 1)], 0), a.rows) / BQ + i + at <= u;
      const int k = max((int)__popcll(__ballot(before)) - 1, 0) * step;
      i += k;
      n = min(step, n - k);
    }
    i = __builtin_amdgcn_readfirstlane(i);
    t = u - (min(max(a.seq_start[i], 0), a.rows) / BQ + i);
  }
  const SeqSpan s = seq_span(a, i);
  w.lo = __builtin_amdgcn_readfirstlane(s.lo);
  w.t = __builtin_amdgcn_readfirstlane(t);
  const int len = __builtin_amdgcn_readfirstlane(s.hi - s.lo);
  w.prefix = __builtin_amdgcn_readfirstlane(s.prefix);
  w.len = w.t >= 0 && w.t * BQ < len ? len : 0;
  return w;
}

// ---- tiles ------------------------------------------------------------------------------------------------------------------
// Rows row0 .. row0 + ROWS - 1 of one head of a sequence -> LDS.  Load j of a thread covers rows j * SWEEP + its own inside a sweep; the
// swizzle repeats every 16 rows, so one offset per matrix is enough.  The descriptor starts at the tile's first row and ends with the
// sequence's last, so offsets stay small however long the buffer is.
template <int HD, int NTHR, int ROWS>
struct Loader {
  using G = Geo<HD>;
  static constexpr int SWEEP = NTHR / G::PPR, NLD = ROWS / SWEEP;
  static_assert(SWEEP % 16 == 0 && ROWS % SWEEP == 0, "swizzle period");
  const bf16* base;
  int64_t ld;
  unsigned off0, hop;
  __device__ __forceinline__ void init(const bf16* p, int64_t stride, int wave, int lane) {
    const int sl = wave * 64 + lane, r = sl / G::PPR, c = (sl % G::PPR) ^ G::swz(r);
    base = p; ld = stride;
    off0 = (unsigned)((r * ld + c * 8) * 2);
    hop = (unsigned)(SWEEP * ld * 2);
  }
  __device__ __forceinline__ void fetch(lds_char* tile, int row0, int len, int wave) const {
    const int rem = min(len - row0, ROWS);
    const rsrc_words rs = raw_rsrc(base + (int64_t)row0 * ld, rem > 0 ? (unsigned)(((rem - 1) * ld + HD) * 2) : 0u);
#pragma unroll
    for (int j = 0; j < NLD; ++j) load_to_lds_b128(rs, (unsigned)(size_t)(tile + (j * (NTHR / 64) + wave) * 1024), off0 + j * hop);
  }
};

// ---- scores -----------------------------------------------------------------------------------------------------------------
// 16 products x -> capped scores in units of log 2.  Scores that are not pressed against the cap, |y| <= 0.25 or 0.6 with y = x scale / cap, take
// tanh(y) = y (1 + y^2 (a1 + ...)) with two or four coefficients (fitted by least squares; tanh is off by 8e-8 and 3e-8 at most, a score of
// 12 under a cap of 50 by 4e-6), a block with any larger one 1 - 2 / (exp(2 y) + 1), whose two transcendental instructions each
// cost as much as four others.  That form is off by 2^-22 of the cap, which beside one high score the low ones of the block have too: up to
// WIDE_CAP nothing against the rounding of P to bf16 (8e-5 of P, a 46th of half a step).  The coefficients are those of x itself, one product less,
// and run out of fp32's range where the cap is far above the scale.  For such caps (`wide`) every score goes by itself, cap_one (a cap
// of 1000, 32 heads of 128 on 8 x 4096, forward and backward: 170 + 551 -> 238 + 752 us).
constexpr double TANH2[2] = {-0.33322914994946595, 0.12846042911412406};
constexpr double TANH4[4] = {-0.33332247985930596, 0.13308098290393836, -0.05199433652233533, 0.015319205699263892};
constexpr float WIDE_CAP = 512.f;      // in units of log 2
__device__ __forceinline__ float cap_one(float x, const ScoreCall& c) {
  const float y = x * (c.kx * (0.5f * LN2)), z = y * y;
  const float low = x * c.sl2 * fmaf(z, fmaf(z, fmaf(z, fmaf(z, (float)TANH4[3], (float)TANH4[2]), (float)TANH4[1]), (float)TANH4[0]), 1.f);
  return fabsf(y) <= 0.6f ? low : fmaf(__builtin_amdgcn_rcpf(fast_exp2(x * c.kx) + 1.f), -2.f * c.c2, c.c2);
}
__device__ __forceinline__ void cap_block(f32x16& x, const ScoreCall& c) {
  float mx = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) mx = fmaxf(mx, fabsf(x[e]));
  if (!__any(mx > c.small)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = x[e] * x[e];
      x[e] *= fmaf(y, fmaf(y, c.p3[1], c.p3[0]), c.sl2);
    }
  } else if (!__any(mx > c.middling)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = x[e] * x[e];
      x[e] *= fmaf(y, fmaf(y, fmaf(y, fmaf(y, c.p5[3], c.p5[2]), c.p5[1]), c.p5[0]), c.sl2);
    }
  } else if (!c.wide) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = fmaf(__builtin_amdgcn_rcpf(fast_exp2(x[e] * c.kx) + 1.f), -2.f * c.c2, c.c2);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      asm volatile("" : "+v"(x));        // (the block stays in its registers: left to itself this branch gets a second set)
      x[e] = cap_one(x[e], c);
    }
    asm volatile("" : "+v"(x));
  }
}

// ---- infinities and NaN behind the mask ----------------------------------------------------------------------------------------
// The products of a tile take all of its rows, those that a query does not see with weight zero, which is right as long as they are finite:
// zero times an infinity or NaN is NaN.  The loops carry no branch for it.  Rows that come out not finite, though their own statistics are not
// NaN, are computed again: 32 of them at a time by their wavefront alone, in blocks of 32 x 32 with operands straight from memory.  Only in blocks
// that the mask cuts does a product go row by row and leave out the pairs that do not count, so a walk costs a few times what the tiles cost, at any
// length.  (16384 rows, 8 heads of 128 on 2, causal, biased, forward + backward: 551 + 1724 us; with an infinity in the first value 3400 + 1990, a NaN in
// the first query 580 + 8300, where one workgroup's walk is what all wait for, NaN everywhere 470 + 1760.)

// the rows (of 32) of a wavefront's accumulators, one to a lane and its partner 32 further on, that hold an infinity or NaN
template <int N> __device__ __forceinline__ unsigned odd_rows(const f32x16 (&acc)[N], bool live) {
  float t = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) t = fmaf(acc[n][e], 0.f, t);            // 0, or NaN
  const uint64_t odd = __ballot(live && t != 0.f);
  return __builtin_amdgcn_readfirstlane((unsigned)(odd | odd >> 32));       // (said to be uniform, it leaves the loops' registers alone)
}
// The arguments once more, from where the launch put them (a kernel's ScoreCall is its first argument): what is computed again is found
// again too, from them, the rank and the lane's number; kept to the end it would take registers that the loops lack.
__device__ __forceinline__ ScoreCall call_again() {
  typedef const __attribute__((address_space(4))) uint64_t* words;
  words p = (words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  static_assert(sizeof(ScoreCall) % 8 == 0, "whole words");
  union { ScoreCall c; uint64_t w[sizeof(ScoreCall) / 8]; } u;
#pragma unroll
  for (unsigned i = 0; i < sizeof(ScoreCall) / 8; ++i) u.w[i] = p[i];
  return u.c;
}
// (inside the walks' loops, where the compiler would keep in registers what follows from the lane's number)
__device__ __forceinline__ int lane_again() { 
  int all = -1;
  asm volatile("" : "+s"(all));
  return __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0));
}

// A product's score in units of log 2, and the cap's derivative there
template <bool CAP> __device__ __forceinline__ float walk_score(float x, const ScoreCall& c, float& dcap) {
  const float s = CAP ? cap_one(x, c) : x * c.sl2, t = CAP ? s * c.ic2 : 0.f;
  dcap = fmaf(-t, t, 1.f);
  return s;
}
// A matrix' rows of one sequence, columns of one head
struct Rows { const bf16* p; int64_t ld; };
// products over head_dim of rows x0 .. x0 + 31 of x (an accumulator's rows) with rows y0 .. y0 + 31 of y (its lanes); rows from n on are zeros
template <int HD> __device__ __forceinline__ f32x16 walk_product(Rows x, int x0, Rows y, int y0, int n, int lane) {
  f32x16 s;
  zero(s);
#pragma unroll HD == 128 ? 8 : 2
  for (int kk = 0; kk < HD / 16; ++kk) s = MFMA(frag_rows_global(x.p, x.ld, x0, n, kk * 16, lane), frag_rows_global(y.p, y.ld, y0, n, kk * 16, lane), s);
  return s;
}
// A walk's own rows are one to a lane, and each sees an interval of the others.
struct Seen {
  int from, to;                                        // within the sequence
  __device__ __forceinline__ bool has(int x) const { return x >= from && x < to; }
  // whether some own row does not see all rows of the sequence in the block from x0 on
  __device__ __forceinline__ bool cuts(int x0, int own, int n) const { return __any(own < n && (from > x0 || to < min(x0 + 32, n))); }
};
// acc += x^T . w for the block of rows x0 .. of x: on the matrix cores, w rounded once, or (cut) row by row, each for the lanes that see it
template <int HD> __device__ __forceinline__ void walk_add(f32x16 (&acc)[HD / 32], const f32x16& w, Seen see, bool cut, Rows x, int x0, int n, int lane) {
  const int hf = lane >> 5;
  auto stay = [&] {                                    // the sums stay in their registers: left to themselves the two ways get a set each
#pragma unroll
    for (int hb = 0; hb < HD / 32; ++hb) asm volatile("" : "+v"(acc[hb]));
  };
  stay();
  if (!cut) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 wf;
#pragma unroll
      for (int e = 0; e < 8; ++e) wf[e] = (bf16)w[h * 8 + e];
#pragma unroll
      for (int hb = 0; hb < HD / 32; ++hb) {
        bf16x8 f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int row = x0 + acc_row(h * 8 + e, hf);
          const bf16 v = x.p[(int64_t)min(row, n - 1) * x.ld + hb * 32 + (lane & 31)];
          f[e] = row < n ? v : (bf16)0.f;
        }
        acc[hb] = MFMA(f, wf, acc[hb]);
      }
      SCHED_FENCE;                                     // few registers, so that the loops keep theirs
    }
    stay();
    return;
  }
#pragma unroll 1
  for (int r = 0; r < min(32, n - x0); ++r) {
    const int e = (r >> 3) * 4 + (r & 3), from = (lane & 31) + ((r >> 2) & 1) * 32;      // who holds that row's weight
    const float f = __shfl(w[e], from);
    const bool counts = see.has(x0 + r);
    const bf16* xr = x.p + (int64_t)(x0 + r) * x.ld + hf * 4;
#pragma unroll
    for (int hb = 0; hb < HD / 32; ++hb)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const bf16x4 v = *reinterpret_cast<const bf16x4*>(xr + hb * 32 + q4 * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[hb][q4 * 4 + i] = counts ? fmaf(f, (float)v[i], acc[hb][q4 * 4 + i]) : acc[hb][q4 * 4 + i];
        SCHED_FENCE;
      }
    stay();
  }
}
template <int HD> __device__ __forceinline__ void store_rows(const f32x16 (&acc)[HD / 32], float f, bf16* out, int hf) {
#pragma unroll
  for (int hb = 0; hb < HD / 32; ++hb)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(acc[hb][q4 * 4 + e] * f);
      *reinterpret_cast<bf16x4*>(out + hb * 32 + q4 * 8 + hf * 4) = v;
    }
}
// forward: queries, block qb of 32 of the tile of BQ that `rank` is, head j
template <int HD, int BQ, bool CAP> __device__ __forceinline__ void again_fwd(int j, int rank, int qb, unsigned rows) {
  const ScoreCall c = call_again();
  const ScoreArgs& a = c.a;
  const int lane = lane_again(), hf = lane >> 5, g = j / (a.h / a.hkv);
  const Work w = find_work<BQ, true>(c, rank, lane);
  const int q0 = w.t * BQ + qb * 32, q = q0 + (lane & 31), vis = a.causal ? w.prefix : w.len, end = max(min(q0 + 32, w.len), vis);
  const Rows Q{(const bf16*)a.q + (int64_t)w.lo * a.ldq + j * HD, a.ldq}, K{(const bf16*)a.k + (int64_t)w.lo * a.ldk + g * HD, a.ldk},
      V{(const bf16*)a.v + (int64_t)w.lo * a.ldv + g * HD, a.ldv};
  const float slope2 = a.slope ? a.slope[j] * LOG2E : 0.f;
  f32x16 acc[HD / 32];
#pragma unroll
  for (int hb = 0; hb < HD / 32; ++hb) zero(acc[hb]);
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < end; k0 += 32) {
    const int lane = lane_again(), hf = lane >> 5, q = q0 + (lane & 31);
    f32x16 s = walk_product<HD>(K, k0, Q, q0, w.len, lane);
    const Seen see{0, min(max(a.causal ? q + 1 : 0, vis), w.len)};
    float mx = -INFINITY, d;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = fmaf(-slope2, fabsf((float)(k0 + acc_row(e, hf) - q)), walk_score<CAP>(s[e], c, d));
      s[e] = see.has(k0 + acc_row(e, hf)) ? s[e] : -INFINITY;
      mx = fmaxf(mx, s[e]);
    }
    const float mn = fmaxf(m, half_max(mx, hf)), sub = mn == -INFINITY ? 0.f : mn, alpha = fast_exp2(m - sub);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) { s[e] = fast_exp2(s[e] - sub); sum += s[e]; }
    l = l * alpha + half_sum(sum, hf);
    m = mn;
#pragma unroll
    for (int hb = 0; hb < HD / 32; ++hb)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[hb][e] *= alpha;
    walk_add<HD>(acc, s, see, see.cuts(k0, q, w.len), V, k0, w.len, lane);
  }
  if (!(rows >> (lane & 31) & 1)) return;
  store_rows<HD>(acc, 1.f / l, (bf16*)a.o + (int64_t)(w.lo + q) * a.ldo + j * HD, hf);
  if (hf == 0 && a.lse) a.lse[(int64_t)j * a.rows + w.lo + q] = (m + log2f(l)) * LN2;
}
template <int HD, int BQ, bool CAP> __device__ __forceinline__ void again_dq(int j, int rank, int qb, unsigned rows) {
  const ScoreCall c = call_again();
  const ScoreArgs& a = c.a;
  const int lane = lane_again(), hf = lane >> 5, g = j / (a.h / a.hkv);
  const Work w = find_work<BQ, true>(c, rank, lane);
  const int q0 = w.t * BQ + qb * 32, q = q0 + (lane & 31), vis = a.causal ? w.prefix : w.len, end = max(min(q0 + 32, w.len), vis);
  const Rows Q{(const bf16*)a.q + (int64_t)w.lo * a.ldq + j * HD, a.ldq}, K{(const bf16*)a.k + (int64_t)w.lo * a.ldk + g * HD, a.ldk},
      V{(const bf16*)a.v + (int64_t)w.lo * a.ldv + g * HD, a.ldv}, D{(const bf16*)a.dout + (int64_t)w.lo * a.lddo + j * HD, a.lddo};
  const float slope2 = a.slope ? a.slope[j] * LOG2E : 0.f;
  const int64_t at = (int64_t)j * a.rows + w.lo + min(q, w.len - 1);
  const float lse2 = a.lse[at] * LOG2E, delta = a.delta[at];
  f32x16 acc[HD / 32];
#pragma unroll
  for (int hb = 0; hb < HD / 32; ++hb) zero(acc[hb]);
#pragma unroll 1
  for (int k0 = 0; k0 < end; k0 += 32) {
    const int lane = lane_again(), hf = lane >> 5, q = q0 + (lane & 31);
    f32x16 s = walk_product<HD>(K, k0, Q, q0, w.len, lane);
    const f32x16 dp = walk_product<HD>(V, k0, D, q0, w.len, lane);
    const Seen see{0, min(max(a.causal ? q + 1 : 0, vis), w.len)};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float d;
      const float x = walk_score<CAP>(s[e], c, d), p = fast_exp2(fmaf(-slope2, fabsf((float)(k0 + acc_row(e, hf) - q)), x - lse2));
      s[e] = see.has(k0 + acc_row(e, hf)) ? p * ((dp[e] - delta) * d) : 0.f;
    }
    walk_add<HD>(acc, s, see, see.cuts(k0, q, w.len), K, k0, w.len, lane);
  }
  if (rows >> (lane & 31) & 1) store_rows<HD>(acc, a.scale, (bf16*)a.dq + (int64_t)(w.lo + q) * a.lddq + j * HD, hf);
}
// Which keys of block kw of 32 are seen by a query whose lse (dK: or delta) is NaN: so is every column of theirs, whatever is behind the mask.
template <int TQ, bool OWN_DELTA> __device__ __forceinline__ unsigned settled_keys(int bx, int rank, int kw, bool dk) {
  const ScoreCall c = call_again();
  const ScoreArgs& a = c.a;
  const int lane = lane_again(), g = bx / c.nsplit, sp = bx % c.nsplit, grp = a.h / a.hkv / c.nsplit, j0 = g * (a.h / a.hkv) + sp * grp;
  const Work w = find_work<TQ, false>(c, rank, lane);
  const int k0 = w.t * TQ + kw * 32, key = k0 + (lane & 31);
  int last = -1;
#pragma unroll 1
  for (int j = j0; j < j0 + grp; ++j)
#pragma unroll 1
    for (int i = lane; i < w.len; i += 64) {
      const int64_t at = (int64_t)j * a.rows + w.lo + i;
      const float x = dk && !OWN_DELTA ? a.lse[at] != a.lse[at] ? a.lse[at] : a.delta[at] : a.lse[at];
      if (x != x) last = max(last, i);
    }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) last = max(last, __shfl_xor(last, x));
  const uint64_t is = __ballot(key < w.len && (a.causal && key >= w.prefix ? key : 0) <= last);
  return __builtin_amdgcn_readfirstlane((unsigned)(is | is >> 32));
}
// dV (dk = false) or dK: block kw of 32 keys of the tile of TQ that `rank` is, of the KV head and split bx
template <int HD, int TQ, bool CAP, bool OWN_DELTA> __device__ __forceinline__ void again_dkv(int bx, int rank, int kw, bool dk, unsigned rows) {
  const ScoreCall c = call_again();
  const ScoreArgs& a = c.a;
  const int lane = lane_again(), hf = lane >> 5, g = bx / c.nsplit, sp = bx % c.nsplit, grp = a.h / a.hkv / c.nsplit, j0 = g * (a.h / a.hkv) + sp * grp;
  const Work w = find_work<TQ, false>(c, rank, lane);
  const int k0 = w.t * TQ + kw * 32, key = k0 + (lane & 31), dkv = a.hkv * HD;
  const int first = a.causal && k0 >= w.prefix ? k0 : 0;             // the first query that sees a key of the block
  const Rows K{(const bf16*)a.k + (int64_t)w.lo * a.ldk + g * HD, a.ldk}, V{(const bf16*)a.v + (int64_t)w.lo * a.ldv + g * HD, a.ldv};
  f32x16 acc[HD / 32];
#pragma unroll
  for (int hb = 0; hb < HD / 32; ++hb) zero(acc[hb]);
#pragma unroll 1
  for (int j = j0; j < j0 + grp; ++j) {
    const float slope2 = a.slope ? a.slope[j] * LOG2E : 0.f;
    const Rows Q{(const bf16*)a.q + (int64_t)w.lo * a.ldq + j * HD, a.ldq}, D{(const bf16*)a.dout + (int64_t)w.lo * a.lddo + j * HD, a.lddo};
#pragma unroll 1
    for (int i0 = first; i0 < w.len; i0 += 32) {
      const int lane = lane_again(), hf = lane >> 5, key = k0 + (lane & 31);
      const int i = min(i0 + (lane & 31), w.len - 1);                // the query whose statistics the lane fetches
      const int64_t at = (int64_t)j * a.rows + w.lo + i;
      const float lse2 = a.lse[at] * LOG2E;
      float delta = 0.f;
      if (dk && OWN_DELTA) {
        const bf16* o = (const bf16*)a.o + (int64_t)(w.lo + i) * a.ldo + j * HD + hf * (HD / 2);
        const bf16* d = D.p + i * D.ld + hf * (HD / 2);
#pragma unroll 1
        for (int x = 0; x < HD / 2; x += 8) {
          const bf16x8 u = *reinterpret_cast<const bf16x8*>(o + x), v = *reinterpret_cast<const bf16x8*>(d + x);
#pragma unroll
          for (int e = 0; e < 8; ++e) delta = fmaf((float)u[e], (float)v[e], delta);
        }
        delta = half_sum(delta, hf);
      } else if (dk) delta = a.delta[at];
      f32x16 s = walk_product<HD>(Q, i0, K, k0, w.len, lane), dp;
      if (dk) dp = walk_product<HD>(D, i0, V, k0, w.len, lane);
      const Seen see{a.causal && key >= w.prefix ? key : 0, w.len};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float d;
        const float x = walk_score<CAP>(s[e], c, d), le = __shfl(lse2, acc_row(e, hf)), de = __shfl(delta, acc_row(e, hf));
        const float p = fast_exp2(fmaf(-slope2, fabsf((float)(i0 + acc_row(e, hf) - key)), x - le));
        s[e] = !see.has(i0 + acc_row(e, hf)) ? 0.f : dk ? p * d * (dp[e] - de) : p;
        if (e % 4 == 3) SCHED_FENCE;
      }
      walk_add<HD>(acc, s, see, see.cuts(i0, key, w.len), dk ? Q : D, i0, w.len, lane);
    }
  }
  if (!(rows >> (lane & 31) & 1)) return;
  const float osc = dk ? a.scale : 1.f;
  if (c.nsplit == 1) store_rows<HD>(acc, osc, dk ? (bf16*)a.dk + (int64_t)(w.lo + key) * a.lddk + g * HD : (bf16*)a.dv + (int64_t)(w.lo + key) * a.lddv + g * HD, hf);
  else {
    float* out = c.part + ((int64_t)sp * a.rows + w.lo + key) * (2 * dkv) + g * HD + (dk ? 0 : dkv);
#pragma unroll
    for (int hb = 0; hb < HD / 32; ++hb)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[hb][q4 * 4 + e] * osc;
        *reinterpret_cast<f32x4*>(out + hb * 32 + q4 * 8 + hf * 4) = v;
      }
  }
}

// ---- forward ----------------------------------------------------------------------------------------------------------------
struct Row { int q, last; };           // a lane's query and the last key that it sees, both inside the sequence

template <int HD, int BUF, int NC, bool CAP>
__device__ __forceinline__ void fwd_tile(lds_char* lds, const FragOff<HD>& fo, const ScoreCall& c, const bf16x8 (&qf)[HD / 16], f32x16 (&o)[HD / 32],
                                         float& m, float& l, int kv0, Row row, int hf, float slope2, bool online, bool need_mask) {
  using G = Geo<HD>;
  constexpr int KT = BUF, VT = BUF + G::TILEB, AHEAD = 3, NPV = G::NHB * 2 * NC, VA = 4;
  bf16x8 kf[AHEAD + 1][NC];
#pragma unroll
  for (int kk = 0; kk < AHEAD; ++kk)
#pragma unroll
    for (int n = 0; n < NC; ++n) kf[kk][n] = frag_rows<HD>(lds, fo, KT, n * 32, kk);
  f32x16 s[NC];
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) {
    if (kk + AHEAD < G::NKK) {
#pragma unroll
      for (int n = 0; n < NC; ++n) kf[(kk + AHEAD) % (AHEAD + 1)][n] = frag_rows<HD>(lds, fo, KT, n * 32, kk + AHEAD);
    }
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      if (kk == 0) s[n] = mfma0(kf[0][n], qf[0]);
      else s[n] = MFMA(kf[kk % (AHEAD + 1)][n], qf[kk], s[n]);
    }
    SCHED_FENCE;
  }
  bf16x8 vf[VA];
#pragma unroll
  for (int i = 0; i < VA; ++i) vf[i] = frag_cols_tr<HD>(lds, fo, VT, (i / G::NHB) * 16, i % G::NHB);
  SCHED_FENCE;
  if (CAP) {
#pragma unroll
    for (int n = 0; n < NC; ++n) cap_block(s[n], c);
  }
  const bool bias = c.a.slope != nullptr;
  const float sl = CAP ? 1.f : c.sl2;
  if (bias) {
    const float sb = CAP ? slope2 : slope2 * c.raw * LN2;                // in the units of s
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const float first = (float)(kv0 + n * 32 + hf * 4 - row.q);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[n][e] = fmaf(-sb, fabsf(first + (float)acc_row(e, 0)), s[n][e]);
    }
  }
  if (need_mask) {
    const int bound = row.last - kv0 - hf * 4;
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (n * 32 + acc_row(e, 0) > bound) s[n][e] = -INFINITY;
  }
  if (!CAP || online) {
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[n][e]);
    const float mn = fmaxf(m, half_max(top, hf) * sl);
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[n][e] = fast_exp2(fmaf(s[n][e], sl, -mn));
    if (__any(mn != m)) {                        // the running max moved for some query of the wavefront
      const float alpha = fast_exp2(m - mn);
      l *= alpha;
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[hb][e] *= alpha;
    }
    m = mn;
  } else {
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[n][e] = fast_exp2(s[n][e]);
  }
  // P is rounded to bf16 for its product, since the matrix cores take both operands in one type (so are P and dS in the backward, once each; every such
  // rounding adds to a result's error about what its own does); the row's sum is of what it was before
  bf16x8 pf[NC][2];
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) { sum[e & 3] += s[n][e]; pf[n][e >> 3][e & 7] = (bf16)s[n][e]; }
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  SCHED_FENCE;
#pragma unroll
  for (int i = 0; i < NPV; ++i) {
    const bf16x8 v = vf[i % VA];
    if (i + VA < NPV) {
      const int n = i + VA;
      vf[i % VA] = frag_cols_tr<HD>(lds, fo, VT, (n / G::NHB) * 16, n % G::NHB);
    }
    o[i % G::NHB] = MFMA(v, pf[(i / G::NHB) >> 1][(i / G::NHB) & 1], o[i % G::NHB]);
    SCHED_FENCE;
  }
}

// Workgroup shapes as in attn_mfma.hip: KS wavefronts share 32 queries, each taking its part of a step's keys.
template <int NT, int KS> constexpr int block_q() { return (NT / 64) * 32 / KS; }
constexpr int WIDE = 512, NARROW = 256;

template <int HD, int NT, int KS, bool CAP>
__global__ __launch_bounds__(NT, KS == 4 && HD == 64 ? 4 : 2) void score_fwd_kernel(ScoreCall c) {
  using G = Geo<HD>;
  constexpr int SUB = KS == 4 ? 2 : 1, TS = TK * SUB;
  constexpr int KT = 0, VT = G::TILEB, BUFB = SUB * 2 * G::TILEB;
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  lds_char* lds = (lds_char*)smem_raw;
  const ScoreArgs& a = c.a;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int BQ = block_q<NT, KS>(), KW = KS == 1 ? 64 : 32;
  const int qb = wave / KS, kh = wave % KS;
  const int j = blockIdx.x % a.h, g = j / (a.h / a.hkv);
  const Work w = find_work<BQ, true>(c, blockIdx.x / a.h, lane);
  if (w.len == 0) return;
  const int q0b = w.t * BQ, q0w = q0b + qb * 32, vis = a.causal ? w.prefix : w.len;       // the first `vis` keys are seen by all
  const Row row{q0w + (lane & 31), min(max(a.causal ? q0w + (lane & 31) : 0, vis - 1), w.len - 1)};
  const float slope2 = a.slope ? a.slope[j] * LOG2E : 0.f;
  const int end = max(min(q0b + BQ, w.len), vis), end_w = max(min(q0w + 32, w.len), vis);   // keys that the workgroup, the wavefront sees
  const int nstep = (end + TS - 1) / TS;
  Loader<HD, NT, TK> K, V;
  K.init((const bf16*)a.k + (int64_t)w.lo * a.ldk + g * HD, a.ldk, wave, lane);
  V.init((const bf16*)a.v + (int64_t)w.lo * a.ldv + g * HD, a.ldv, wave, lane);
  auto fetch = [&](int buf, int row0) {
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      K.fetch(lds + buf + u * 2 * G::TILEB + KT, row0 + u * TK, w.len, wave);
      V.fetch(lds + buf + u * 2 * G::TILEB + VT, row0 + u * TK, w.len, wave);
    }
  };
  fetch(0, 0);
  if (nstep > 1) fetch(BUFB, TS);

  const bf16* qp = (const bf16*)a.q + (int64_t)w.lo * a.ldq + j * HD;
  bf16x8 qf[G::NKK];
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) qf[kk] = frag_rows_global(qp, a.ldq, q0w, w.len, kk * 16, lane);
  f32x16 o[G::NHB];
#pragma unroll
  for (int hb = 0; hb < G::NHB; ++hb) zero(o[hb]);
  // Capped scores lie within c2 of zero and a bias only lowers them: up to c2 = 80 exp2 of them and its sums stay well inside fp32, so
  // the running maximum (and the rescaling that comes with it) is not needed.
  const bool online = !CAP || c.c2 > 80.f || slope2 < 0.f;
  float m = online ? -FLT_MAX : 0.f, l = 0.f;            // (finite: wavefronts and rows that see nothing of a tile take differences of it)
  FragOff<HD> fo;
  fo.init(lane, lds);
  if (KS > 1) fo.hop((kh >> 1) * 2 * G::TILEB + (kh & 1) * 32 * G::ROWB);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();

  auto step = [&](int t, auto buf) {
    constexpr int BUF = decltype(buf)::value;
    const int kv0 = t * TS, kvw = kv0 + kh * 32;
    if (kvw < end_w && q0w < w.len) {
      const bool need_mask = (a.causal && kvw + KW > max(q0w + 1, vis)) || kvw + KW > w.len;
      fwd_tile<HD, BUF, KW / 32, CAP>(lds, fo, c, qf, o, m, l, kvw, row, hf, slope2, online, need_mask);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (t + 2 < nstep) fetch(BUF, kv0 + 2 * TS);
  };
  for (int t = 0; t < nstep; t += 2) {
    step(t, std::integral_constant<int, 0>{});
    if (t + 1 < nstep) step(t + 1, std::integral_constant<int, BUFB>{});
  }

  l = half_sum(l, hf);
  if constexpr (KS > 1) {
    constexpr int OB = G::NHB * 4 * 1024, NQB = BQ / 32;
    static_assert((KS - 1) * NQB * (OB + 512) <= 2 * BUFB, "the merge area fits the tile buffers");
    auto area = [&](int part) { return lds + ((part - 1) * NQB + qb) * (OB + 512); };
    if (kh > 0) {
      lds_char* mo = area(kh) + lane * 16;
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *(__attribute__((address_space(3))) f32x4*)(mo + (hb * 4 + q4) * 1024) =
              f32x4{o[hb][q4 * 4], o[hb][q4 * 4 + 1], o[hb][q4 * 4 + 2], o[hb][q4 * 4 + 3]};
      *(__attribute__((address_space(3))) f32x2*)(area(kh) + OB + lane * 8) = f32x2{m, l};
    }
    __syncthreads();
    if (kh > 0) return;
#pragma unroll
    for (int part = 1; part < KS; ++part) {
      lds_char* mo = area(part) + lane * 16;
      const f32x2 other = *(__attribute__((address_space(3))) const f32x2*)(area(part) + OB + lane * 8);
      const float mn = fmaxf(m, other.x);
      const float a0 = fast_exp2(m - mn), a1 = fast_exp2(other.x - mn);
      l = l * a0 + other.y * a1;
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 v = *(__attribute__((address_space(3))) const f32x4*)(mo + (hb * 4 + q4) * 1024);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[hb][q4 * 4 + e] = o[hb][q4 * 4 + e] * a0 + v[e] * a1;
        }
      m = mn;
    }
  }
  // Exponents are taken from the rounded maximum m, which is off by up to 2^-24 of itself: beyond 1e9 that alone may overflow the sums, or leave nothing of
  // them, and the row is computed again.  Below, a sum that is NaN is the row's own: every column of it is, whatever is behind the mask.
  if (fabsf(m) > 1e9f && m != -FLT_MAX) { l = 1.f; o[0][0] = INFINITY; }
  const unsigned odd = odd_rows(o, row.q < w.len && l == l);
  if (row.q < w.len && !(odd >> (lane & 31) & 1)) {
    const float inv = 1.f / l;
    bf16* orow = (bf16*)a.o + (int64_t)(w.lo + row.q) * a.ldo + j * HD;
#pragma unroll
    for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[hb][q4 * 4 + e] * inv);
        *reinterpret_cast<bf16x4*>(orow + hb * 32 + q4 * 8 + hf * 4) = v;
      }
    if (hf == 0 && a.lse) a.lse[(int64_t)j * a.rows + w.lo + row.q] = (m + log2f(l)) * LN2;
  }
  if (__builtin_expect(odd != 0, 0)) again_fwd<HD, BQ, CAP>(j, blockIdx.x / a.h, qb, odd);
}

// ---- backward ---------------------------------------------------------------------------------------------------------------
// 16 scores of a lane's query with keys from k0 on (capped: in units of log 2, else products) -> P = exp(s - lse), zero where masked
template <bool CAP>
__device__ __forceinline__ void probs_block(f32x16& s, const ScoreCall& c, int k0, Row row, int hf, float slope2, float lse2, bool need_mask) {
  const float first = (float)(k0 + hf * 4 - row.q), sl = CAP ? 1.f : c.sl2;
  if (c.a.slope) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fmaf(-slope2, fabsf(first + (float)acc_row(e, 0)), fmaf(s[e], sl, -lse2));
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fast_exp2(s[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fast_exp2(fmaf(s[e], sl, -lse2));
  }
  if (need_mask) {
    const int bound = row.last - k0 - hf * 4;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (acc_row(e, 0) > bound) s[e] = 0.f;
  }
}

// delta = rowsum(dO * O) is what dS = P (dP - delta) subtracts, and where a row's weight sits on few keys it is nearly all of dP: the rounding of
// O to bf16 is then no longer small against what is left (dQ and dK of sequences of 8 rows, scores of 3 in the mean, off by 5.8e-3 of their norm,
// of 4096 rows by 3.0e-3, where the roundings of dS and of the results alone are 2.35e-3).  So a block of 32 queries that sees no more than the
// DELTA_KEYS keys that are in LDS before the loop starts gets delta as the sum of P dP, which costs it their two products once more.
constexpr int DELTA_KEYS = 2 * TK;
template <int HD, int BUF, bool CAP>
__device__ __forceinline__ float delta_block(lds_char* lds, const FragOff<HD>& fo, const ScoreCall& c, const bf16x8 (&qf)[HD / 16], const bf16x8 (&dof)[HD / 16],
                                             int n, int k0, Row row, int hf, float slope2, float lse2, bool need_mask) {
  using G = Geo<HD>;
  constexpr int KT = BUF, VT = BUF + G::TILEB, AHEAD = 3;
  bf16x8 kf[AHEAD + 1][2];
  f32x16 s, dp;
#pragma unroll
  for (int kk = 0; kk < AHEAD; ++kk) { kf[kk][0] = frag_rows<HD>(lds, fo, KT, n * 32, kk); kf[kk][1] = frag_rows<HD>(lds, fo, VT, n * 32, kk); }
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) {
    if (kk + AHEAD < G::NKK) {
      kf[(kk + AHEAD) % (AHEAD + 1)][0] = frag_rows<HD>(lds, fo, KT, n * 32, kk + AHEAD);
      kf[(kk + AHEAD) % (AHEAD + 1)][1] = frag_rows<HD>(lds, fo, VT, n * 32, kk + AHEAD);
    }
    if (kk == 0) { s = mfma0(kf[0][0], qf[0]); dp = mfma0(kf[0][1], dof[0]); }
    else {
      s = MFMA(kf[kk % (AHEAD + 1)][0], qf[kk], s);
      dp = MFMA(kf[kk % (AHEAD + 1)][1], dof[kk], dp);
    }
    SCHED_FENCE;
  }
  if (CAP) cap_block(s, c);
  probs_block<CAP>(s, c, k0, row, hf, slope2, lse2, need_mask);
  const int bound = need_mask ? row.last - k0 - hf * 4 : 32;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) sum += acc_row(e, 0) > bound ? 0.f : s[e] * dp[e];      // (a masked dP may be anything)
  return sum;
}

// ---- dQ ---------------------------------------------------------------------------------------------------------------------
template <int HD, int BUF, bool CAP>
__device__ __forceinline__ void dq_block(lds_char* lds, const FragOff<HD>& fo, const ScoreCall& c, const bf16x8 (&qf)[HD / 16], const bf16x8 (&dof)[HD / 16],
                                         f32x16 (&dq)[HD / 32], int n, int kv0, Row row, int hf, float slope2, float lse2, float dl, const f32x16& ndl,
                                         bool need_mask) {
  using G = Geo<HD>;
  constexpr int KT = BUF, VT = BUF + G::TILEB, AHEAD = 3, NDQ = G::NHB * 2, VA = 4;
  bf16x8 kf[AHEAD + 1][2];
  f32x16 s, dp;
#pragma unroll
  for (int kk = 0; kk < AHEAD; ++kk) { kf[kk][0] = frag_rows<HD>(lds, fo, KT, n * 32, kk); kf[kk][1] = frag_rows<HD>(lds, fo, VT, n * 32, kk); }
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) {
    if (kk + AHEAD < G::NKK) {
      kf[(kk + AHEAD) % (AHEAD + 1)][0] = frag_rows<HD>(lds, fo, KT, n * 32, kk + AHEAD);
      kf[(kk + AHEAD) % (AHEAD + 1)][1] = frag_rows<HD>(lds, fo, VT, n * 32, kk + AHEAD);
    }
    if (kk == 0) { s = mfma0(kf[0][0], qf[0]); dp = CAP ? mfma0(kf[0][1], dof[0]) : MFMA(kf[0][1], dof[0], ndl); }
    else {
      s = MFMA(kf[kk % (AHEAD + 1)][0], qf[kk], s);
      dp = MFMA(kf[kk % (AHEAD + 1)][1], dof[kk], dp);
    }
    SCHED_FENCE;
  }
  bf16x8 tf[VA];
#pragma unroll
  for (int i = 0; i < VA; ++i) tf[i] = frag_cols_tr<HD>(lds, fo, KT, n * 32 + (i / G::NHB) * 16, i % G::NHB);
  SCHED_FENCE;
  if (CAP) {
    cap_block(s, c);
#pragma unroll
    for (int e = 0; e < 16; ++e) {               // dP - delta times the cap's derivative 1 - t^2
      const float t = s[e] * c.ic2;
      dp[e] = (dp[e] - dl) * fmaf(-t, t, 1.f);
    }
  }
  probs_block<CAP>(s, c, kv0 + n * 32, row, hf, slope2, lse2, need_mask);
  bf16x8 dsf[2];
#pragma unroll
  for (int e = 0; e < 16; ++e) dsf[e >> 3][e & 7] = (bf16)(s[e] * dp[e]);
  SCHED_FENCE;
#pragma unroll
  for (int i = 0; i < NDQ; ++i) {
    const bf16x8 v = tf[i % VA];
    if (i + VA < NDQ) {
      const int x = i + VA;
      tf[i % VA] = frag_cols_tr<HD>(lds, fo, KT, n * 32 + (x / G::NHB) * 16, x % G::NHB);
    }
    dq[i % G::NHB] = MFMA(v, dsf[i / G::NHB], dq[i % G::NHB]);
    SCHED_FENCE;
  }
}

template <int HD, int NT, int KS, bool CAP>
__device__ __forceinline__ void dq_workgroup(const ScoreCall& c, lds_char* lds, int j, int rank) {
  using G = Geo<HD>;
  constexpr int SUB = KS == 4 ? 2 : 1, TS = TK * SUB;
  constexpr int KT = 0, VT = G::TILEB, BUFB = SUB * 2 * G::TILEB;
  const ScoreArgs& a = c.a;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int BQ = block_q<NT, KS>();
  const int qb = wave / KS, kh = wave % KS, g = j / (a.h / a.hkv);
  const Work w = find_work<BQ, true>(c, rank, lane);
  if (w.len == 0) return;
  const int q0b = w.t * BQ, q0w = q0b + qb * 32, vis = a.causal ? w.prefix : w.len;
  const Row row{q0w + (lane & 31), min(max(a.causal ? q0w + (lane & 31) : 0, vis - 1), w.len - 1)};
  const float slope2 = a.slope ? a.slope[j] * LOG2E : 0.f;
  const int end = max(min(q0b + BQ, w.len), vis), end_w = max(min(q0w + 32, w.len), vis);
  const int nstep = (end + TS - 1) / TS;
  Loader<HD, NT, TK> K, V;
  K.init((const bf16*)a.k + (int64_t)w.lo * a.ldk + g * HD, a.ldk, wave, lane);
  V.init((const bf16*)a.v + (int64_t)w.lo * a.ldv + g * HD, a.ldv, wave, lane);
  auto fetch = [&](int buf, int row0) {
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      K.fetch(lds + buf + u * 2 * G::TILEB + KT, row0 + u * TK, w.len, wave);
      V.fetch(lds + buf + u * 2 * G::TILEB + VT, row0 + u * TK, w.len, wave);
    }
  };
  fetch(0, 0);
  if (nstep > 1) fetch(BUFB, TS);

  const bf16* qp = (const bf16*)a.q + (int64_t)w.lo * a.ldq + j * HD;
  const bf16* dop = (const bf16*)a.dout + (int64_t)w.lo * a.lddo + j * HD;
  const bf16* op = (const bf16*)a.o + (int64_t)w.lo * a.ldo + j * HD;
  bf16x8 qf[G::NKK], dof[G::NKK];
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) {
    qf[kk] = frag_rows_global(qp, a.ldq, q0w, w.len, kk * 16, lane);
    dof[kk] = frag_rows_global(dop, a.lddo, q0w, w.len, kk * 16, lane);
  }
  // delta of the lane's query, rowsum(dO * O) from the dO fragments in registers
  const int64_t at = (int64_t)j * a.rows + w.lo + row.q;
  const float lse2 = row.q < w.len ? a.lse[at] * LOG2E : 1e30f;          // rows past the end: P = 0
  float part = 0.f;
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) {
    const bf16x8 of = frag_rows_global(op, a.ldo, q0w, w.len, kk * 16, lane);
#pragma unroll
    for (int e = 0; e < 8; ++e) part = fmaf((float)dof[kk][e], (float)of[e], part);
  }
  FragOff<HD> fo;
  fo.init(lane, lds);
  if (KS > 1) fo.hop((kh >> 1) * 2 * G::TILEB + (kh & 1) * 32 * G::ROWB);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (end_w <= DELTA_KEYS && q0w < w.len) {            // or the sum of P dP (the keys of a wavefront with KS > 1: its parts of the steps)
    part = 0.f;
    Row row1 = row;                                    // copies that the compiler takes for others: what both places derive from them it would
    int hf1 = hf;                                      // keep in registers through the loop
    float slope1 = slope2, lse1 = lse2;
    asm volatile("" : "+v"(row1.q), "+v"(row1.last), "+v"(hf1), "+v"(slope1), "+v"(lse1));
    auto add = [&](int t, auto buf) {
      constexpr int BUF = decltype(buf)::value;
#pragma unroll
      for (int n = 0; n < (KS > 1 ? 1 : 2); ++n) {
        const int k0 = t * TS + kh * 32 + n * 32;
        if (k0 >= end_w) break;
        const bool need_mask = (a.causal && k0 + 32 > max(q0w + 1, vis)) || k0 + 32 > w.len;
        part += delta_block<HD, BUF, CAP>(lds, fo, c, qf, dof, n, k0, row1, hf1, slope1, lse1, need_mask);
      }
    };
    add(0, std::integral_constant<int, 0>{});
    if (KS < 4) add(1, std::integral_constant<int, BUFB>{});
  } else if (kh > 0) part = 0.f;
  float dl = half_sum(part, hf);
  if constexpr (KS > 1) {                              // the other key parts' shares, in order
    __attribute__((address_space(3))) float* shares = (__attribute__((address_space(3))) float*)(lds + 2 * BUFB) + (lane & 31);
    if (hf == 0) shares[wave * 32] = dl;
    __syncthreads();
    dl = shares[qb * KS * 32];
#pragma unroll
    for (int p = 1; p < KS; ++p) dl += shares[(qb * KS + p) * 32];
  }
  if (row.q < w.len && hf == 0 && kh == 0) a.delta[at] = dl;         // for the dK/dV pass
  f32x16 dq[G::NHB], ndl;
#pragma unroll
  for (int hb = 0; hb < G::NHB; ++hb) zero(dq[hb]);
#pragma unroll
  for (int e = 0; e < 16; ++e) ndl[e] = -dl;           // what the dP products start at; capped, delta is subtracted behind them, for want of registers

  auto step = [&](int t, auto buf) {
    constexpr int BUF = decltype(buf)::value;
    const int kv0 = t * TS, kvw = kv0 + kh * 32;
    if (kvw < end_w && q0w < w.len) {
#pragma unroll
      for (int n = 0; n < (KS > 1 ? 1 : 2); ++n) {
        const int k0 = kvw + n * 32;
        if (n > 0 && k0 >= end_w) continue;            // no query of the wavefront sees this block
        const bool need_mask = (a.causal && k0 + 32 > max(q0w + 1, vis)) || k0 + 32 > w.len;
        dq_block<HD, BUF, CAP>(lds, fo, c, qf, dof, dq, n, kvw, row, hf, slope2, lse2, dl, ndl, need_mask);
      }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (t + 2 < nstep) fetch(BUF, kv0 + 2 * TS);
  };
  for (int t = 0; t < nstep; t += 2) {
    step(t, std::integral_constant<int, 0>{});
    if (t + 1 < nstep) step(t + 1, std::integral_constant<int, BUFB>{});
  }

  if constexpr (KS > 1) {      // add the other key parts' dQ to the first's, in order, through LDS
    constexpr int OB = G::NHB * 4 * 1024, NQB = BQ / 32;
    static_assert((KS - 1) * NQB * OB <= 2 * BUFB, "the merge area fits the tile buffers");
    if (kh > 0) {
      lds_char* mo = lds + ((kh - 1) * NQB + qb) * OB + lane * 16;
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *(__attribute__((address_space(3))) f32x4*)(mo + (hb * 4 + q4) * 1024) =
              f32x4{dq[hb][q4 * 4], dq[hb][q4 * 4 + 1], dq[hb][q4 * 4 + 2], dq[hb][q4 * 4 + 3]};
    }
    __syncthreads();
    if (kh > 0) return;
#pragma unroll
    for (int p = 1; p < KS; ++p) {
      lds_char* mo = lds + ((p - 1) * NQB + qb) * OB + lane * 16;
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 v = *(__attribute__((address_space(3))) const f32x4*)(mo + (hb * 4 + q4) * 1024);
#pragma unroll
          for (int e = 0; e < 4; ++e) dq[hb][q4 * 4 + e] += v[e];
        }
    }
  }
  const unsigned odd = odd_rows(dq, row.q < w.len && lse2 == lse2 && dl == dl);      // (one of them is NaN: so is every column of the row)
  if (row.q < w.len && !(odd >> (lane & 31) & 1)) {
    bf16* out = (bf16*)a.dq + (int64_t)(w.lo + row.q) * a.lddq + j * HD;
#pragma unroll
    for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16)(dq[hb][q4 * 4 + e] * a.scale);
        *reinterpret_cast<bf16x4*>(out + hb * 32 + q4 * 8 + hf * 4) = v;
      }
  }
  if (__builtin_expect(odd != 0, 0)) again_dq<HD, BQ, CAP>(j, rank, qb, odd);
}
template <int HD, int NT, int KS, bool CAP>
__global__ __launch_bounds__(NT, 2) void score_dq_kernel(ScoreCall c) {
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  dq_workgroup<HD, NT, KS, CAP>(c, (lds_char*)smem_raw, blockIdx.x % c.a.h, blockIdx.x / c.a.h);
}

// ---- dK/dV ------------------------------------------------------------------------------------------------------------------
// One workgroup = TQ keys of one (sequence, KV head): per 32 keys two wavefronts on a SIMD, one for dV, which makes P, one for dK, which
// takes it (times the cap's derivative) from a 4 KiB slot in LDS; QS = 2: two such pairs, on every second 32 queries each.
constexpr int KEYS = 128, KEYS_SMALL = 64;

template <int HD, int TQ, int QS, bool CAP, bool OWN_DELTA>
__device__ __forceinline__ void dkv_workgroup(const ScoreCall& c, lds_char* lds, int bx, int rank) {
  using G = Geo<HD>;
  constexpr int NTHR = TQ * 4 * QS, NB = TQ / 32 / QS, NKW = TQ / 32, TILEB = TQ * G::ROWB;
  constexpr int QT = 0, OT = TILEB, LT = 2 * TILEB, DT = LT + TQ * 4, BUFB = DT + TQ * 4;
  const ScoreArgs& a = c.a;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int role = wave / (NKW * QS), kw = wave % NKW, qs = QS == 2 ? (wave / NKW) % 2 : 0;
  const int g = __builtin_amdgcn_readfirstlane(bx / c.nsplit), sp = bx - g * c.nsplit;
  const int dkv = a.hkv * HD, per_kv = __builtin_amdgcn_readfirstlane(a.h / a.hkv), grp = __builtin_amdgcn_readfirstlane(per_kv / c.nsplit), j0 = g * per_kv + sp * grp;
  const Work w = find_work<TQ, false>(c, rank, lane);
  if (w.len == 0) return;
  const int kt = w.t, nkt = (w.len + TQ - 1) / TQ;
  const bf16* qbase = (const bf16*)a.q + (int64_t)w.lo * a.ldq;
  const bf16* dobase = (const bf16*)a.dout + (int64_t)w.lo * a.lddo;
  const bf16* kp = (const bf16*)a.k + (int64_t)w.lo * a.ldk + g * HD;
  const bf16* vp = (const bf16*)a.v + (int64_t)w.lo * a.ldv + g * HD;
  const int k0b = kt * TQ, k0w = k0b + kw * 32;
  const int key = k0w + (lane & 31);
  const bool bias = a.slope != nullptr;

  const int t_first = a.causal && k0b >= w.prefix ? kt : 0;     // a key of the prefix is seen by every query
  const int per_head = nkt - t_first;
  const int niter = per_head * grp;
  Loader<HD, NTHR, TQ> Q, D;
  Q.init(qbase, a.ldq, wave, lane);
  D.init(dobase, a.lddo, wave, lane);
  constexpr int NLD = Loader<HD, NTHR, TQ>::NLD, SWEEP = Loader<HD, NTHR, TQ>::SWEEP;
  float stat_l = 0.f, stat_d = 0.f;
  bf16x8 of[OWN_DELTA ? NLD : 1];
  auto fetch = [&](int it, lds_char* buf) {
    const int j = j0 + it / per_head, q0 = (t_first + it % per_head) * TQ;
    Q.base = qbase + j * HD;
    D.base = dobase + j * HD;
    Q.fetch(buf + QT, q0, w.len, wave);
    D.fetch(buf + OT, q0, w.len, wave);
    if (wave < TQ / 64) {                // one query per lane; those past the end get P = 0
      const int qi = q0 + wave * 64 + lane;
      const int64_t at = (int64_t)j * a.rows + w.lo + qi;
      stat_l = qi < w.len ? -LOG2E * a.lse[at] : -1e30f;
      if (!OWN_DELTA) stat_d = qi < w.len ? a.delta[at] : 0.f;
    }
    if constexpr (OWN_DELTA) {           // the pieces of O that go with the pieces of dO this thread has just asked for
      const bf16* oh = (const bf16*)a.o + (int64_t)w.lo * a.ldo + j * HD;
      const int sl = wave * 64 + lane, cc = (sl % G::PPR) ^ G::swz(sl / G::PPR);
#pragma unroll
      for (int n = 0; n < NLD; ++n) of[n] = *reinterpret_cast<const bf16x8*>(oh + (int64_t)min(q0 + n * SWEEP + sl / G::PPR, w.len - 1) * a.ldo + cc * 8);
    }
  };
  // the statistics of the tile fetched last: -lse in units of log 2, and -delta
  auto put_stats = [&](lds_char* buf, int q_of) {
    if (wave < TQ / 64) {
      *(__attribute__((address_space(3))) float*)(buf + LT + (wave * 64 + lane) * 4) = stat_l;
      if (!OWN_DELTA) *(__attribute__((address_space(3))) float*)(buf + DT + (wave * 64 + lane) * 4) = -stat_d;
    }
    if constexpr (OWN_DELTA) {
      __builtin_amdgcn_s_waitcnt(0);     // own loads only, so no barrier: thread and piece correspond as in the fetch, PPR lanes hold a row
      float part[NLD];
#pragma unroll
      for (int n = 0; n < NLD; ++n) {
        const bf16x8 dv = *(__attribute__((address_space(3))) const bf16x8*)(buf + OT + (n * (NTHR / 64) + wave) * 1024 + lane * 16);
        part[n] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) part[n] = fmaf((float)dv[e], (float)of[n][e], part[n]);
      }
#pragma unroll
      for (int x = 1; x < G::PPR; x <<= 1)
#pragma unroll
        for (int n = 0; n < NLD; ++n) part[n] += __shfl_xor(part[n], x);
      if (lane % G::PPR == 0) {
#pragma unroll
        for (int n = 0; n < NLD; ++n) {
          const int r = n * SWEEP + (wave * 64 + lane) / G::PPR;
          *(__attribute__((address_space(3))) float*)(buf + DT + r * 4) = q_of + r < w.len ? -part[n] : 0.f;
        }
      }
    }
  };
  fetch(0, lds);
  put_stats(lds, t_first * TQ);
  if (niter > 1) fetch(1, lds + BUFB);

  FragOff<HD> fo;
  fo.init(lane, lds);
  if (QS == 2) fo.hop(qs * 32 * G::ROWB);
  lds_char* cur = lds;
  lds_char* ldp = lds + LT + hf * 16 + qs * 128;
  int hopb = BUFB;
  typedef __attribute__((address_space(3))) const f32x4* lds_f4;
  // the pair's slot and its counts: produced = blocks written, consumed = blocks read; the waits are bounded
  lds_char* pslot = lds + 2 * BUFB + (qs * NKW + kw) * 4096 + lane * 16;
  volatile __attribute__((address_space(3))) int* produced = (volatile __attribute__((address_space(3))) int*)(lds + 2 * BUFB + QS * NKW * 4096) + qs * NKW + kw;
  volatile __attribute__((address_space(3))) int* consumed = produced + QS * NKW;
  if (tid < 2 * QS * NKW) ((volatile __attribute__((address_space(3))) int*)(lds + 2 * BUFB + QS * NKW * 4096))[tid] = 0;
  auto wait_for = [&](volatile __attribute__((address_space(3))) int* count, int value) {
    for (int guard = 0; *count != value && guard < (1 << 20); ++guard) __builtin_amdgcn_s_sleep(1);
    asm volatile("" ::: "memory");
  };
  int nblk = 0;
  auto turn = [&](int it) {
    if (it + 1 < niter) put_stats(cur + hopb, (t_first + (it + 1) % per_head) * TQ);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (it + 2 < niter) fetch(it + 2, cur);
    fo.hop(hopb);
    cur += hopb;
    ldp += hopb;
    hopb = -hopb;
  };

  bf16x8 kf[G::NKK];
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) kf[kk] = frag_rows_global(role ? vp : kp, role ? a.ldv : a.ldk, k0w, w.len, kk * 16, lane);
  f32x16 acc[G::NHB];                                  // dV^T or dK^T of the wavefront's 32 keys
#pragma unroll
  for (int hb = 0; hb < G::NHB; ++hb) zero(acc[hb]);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();

  if (role == 0) {
    for (int it = 0; it < niter; ++it) {
      const int tq = t_first + it % per_head, q0 = tq * TQ;
      const bool diag = a.causal && tq <= kt;          // some query of the tile is ahead of some key: masked unless the key is in the prefix
      const int lim0 = key < w.prefix ? -(1 << 30) : key - q0 - hf * 4 - qs * 32;
      const float slope2 = bias ? a.slope[j0 + it / per_head] * LOG2E : 0.f;
#pragma unroll
      for (int qc = 0; qc < NB; ++qc) {
        f32x4 l4[4];
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) l4[e4] = *reinterpret_cast<lds_f4>(ldp + (qc * QS * 32 + e4 * 8) * 4);
        f32x16 s;
        dkv_rows_product<HD, QT>(lds, fo, qc * QS * 32, kf, s);
        bf16x8 tf[4];
        dkv_tr_read<HD, OT>(lds, fo, qc * QS * 32, tf);
        SCHED_FENCE;
        float wc[CAP ? 16 : 1];
        if (CAP) {
          cap_block(s, c);
#pragma unroll
          for (int e = 0; e < 16; ++e) { const float t = s[e] * c.ic2; wc[e] = fmaf(-t, t, 1.f); }
        }
        if (bias) {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = CAP ? s[e] + l4[e >> 2][e & 3] : fmaf(s[e], c.sl2, l4[e >> 2][e & 3]);
          const float first = (float)(q0 + (qc * QS + qs) * 32 + hf * 4 - key);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = fmaf(-slope2, fabsf(first + (float)acc_row(e, 0)), s[e]);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = fast_exp2(s[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = fast_exp2(CAP ? s[e] + l4[e >> 2][e & 3] : fmaf(s[e], c.sl2, l4[e >> 2][e & 3]));
        }
        if (diag) {
          asm volatile("" ::: "memory");               // keep this a (wave-uniform) branch: it is rarely taken
          const int lim = lim0 - qc * QS * 32;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = acc_row(e, 0) < lim ? 0.f : s[e];
        }
        wait_for(consumed, nblk);                      // the slot is free
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = CAP ? s[e4 * 4 + e] * wc[CAP ? e4 * 4 + e : 0] : s[e4 * 4 + e];
          *(__attribute__((address_space(3))) f32x4*)(pslot + e4 * 1024) = v;
        }
        asm volatile("" ::: "memory");                 // the LDS executes a wavefront's instructions in order: the count
        *produced = ++nblk;                            // is written after the block
        asm volatile("" ::: "memory");
        bf16x8 pf[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) pf[e >> 3][e & 7] = (bf16)s[e];
        SCHED_FENCE;
        dkv_tr_product<HD, OT>(lds, fo, qc * QS * 32, tf, pf, acc);          // dV^T += dO^T . P
      }
      turn(it);
    }
  } else {
    for (int it = 0; it < niter; ++it) {
#pragma unroll
      for (int qc = 0; qc < NB; ++qc) {
        f32x16 dp;                                      // starts at -delta of the block's queries
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const f32x4 d4 = *reinterpret_cast<lds_f4>(ldp + (DT - LT) + (qc * QS * 32 + e4 * 8) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) dp[e4 * 4 + e] = d4[e];
        }
        dkv_rows_product<HD, OT, true>(lds, fo, qc * QS * 32, kf, dp);               // dP - delta
        bf16x8 tf[4];
        dkv_tr_read<HD, QT>(lds, fo, qc * QS * 32, tf);
        SCHED_FENCE;
        wait_for(produced, nblk + 1);
        f32x4 pv[4];
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) pv[e4] = *(__attribute__((address_space(3))) const f32x4*)(pslot + e4 * 1024);
        asm volatile("" ::: "memory");
        *consumed = ++nblk;
        asm volatile("" ::: "memory");
        bf16x8 df[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) df[e >> 3][e & 7] = (bf16)(pv[e >> 2][e & 3] * dp[e]);
        SCHED_FENCE;
        dkv_tr_product<HD, QT>(lds, fo, qc * QS * 32, tf, df, acc);          // dK^T += Q^T . dS
      }
      turn(it);
    }
  }

  if constexpr (QS == 2) {       // add the second pair's sums to the first's, through LDS
    static_assert(2 * NKW * G::NHB * 4 * 1024 <= 2 * BUFB, "the merge area fits the tile buffers");
    lds_char* mo = lds + (role * NKW + kw) * (G::NHB * 4 * 1024) + lane * 16;
    if (qs == 1) {
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *(__attribute__((address_space(3))) f32x4*)(mo + (hb * 4 + q4) * 1024) =
              f32x4{acc[hb][q4 * 4], acc[hb][q4 * 4 + 1], acc[hb][q4 * 4 + 2], acc[hb][q4 * 4 + 3]};
    }
    __syncthreads();
    if (qs == 1) return;
#pragma unroll
    for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 v = *(__attribute__((address_space(3))) const f32x4*)(mo + (hb * 4 + q4) * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[hb][q4 * 4 + e] += v[e];
      }
  }

  unsigned odd = odd_rows(acc, key < w.len);
  if (__builtin_expect(odd != 0, 0)) odd &= ~settled_keys<TQ, OWN_DELTA>(bx, rank, kw, role != 0);
  if (key < w.len && !(odd >> (lane & 31) & 1)) {             // role 0 holds dV, role 1 dK (still to be scaled)
    const float osc = role ? a.scale : 1.f;
    if (c.nsplit == 1) {
      bf16* out = role ? (bf16*)a.dk + (int64_t)(w.lo + key) * a.lddk + g * HD : (bf16*)a.dv + (int64_t)(w.lo + key) * a.lddv + g * HD;
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (bf16)(acc[hb][q4 * 4 + e] * osc);
          *reinterpret_cast<bf16x4*>(out + hb * 32 + q4 * 8 + hf * 4) = v;
        }
    } else {                     // this split's share, fp32; score_dkv_reduce_kernel adds them up in a fixed order
      float* out = c.part + ((int64_t)sp * a.rows + w.lo + key) * (2 * dkv) + g * HD + (role ? 0 : dkv);
#pragma unroll
      for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[hb][q4 * 4 + e] * osc;
          *reinterpret_cast<f32x4*>(out + hb * 32 + q4 * 8 + hf * 4) = v;
        }
    }
  }
  if (__builtin_expect(odd != 0, 0)) again_dkv<HD, TQ, CAP, OWN_DELTA>(bx, rank, kw, role != 0, odd);
}
template <int HD, int TQ, int QS, bool CAP>
__global__ __launch_bounds__(TQ * 4 * QS, 2) void score_dkv_kernel(ScoreCall c) {
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const int nx = c.a.hkv * c.nsplit, rank = __builtin_amdgcn_readfirstlane(blockIdx.x / nx);
  dkv_workgroup<HD, TQ, QS, CAP, false>(c, (lds_char*)smem_raw, blockIdx.x - rank * nx, rank);
}

// dQ and dK/dV of a small problem in one launch, which neither fills by itself; the dK/dV workgroups, the longer ones, come first
template <int HD, int KS, int QS, bool CAP>
__global__ __launch_bounds__(256 * QS, 2) void score_bwd_kernel(ScoreCall c, int n_dkv) {
  static_assert(KS == 2 * QS, "one workgroup size");
  extern __shared__ __attribute__((aligned(1024))) char smem_raw[];
  const int id = blockIdx.x, nx = c.a.hkv * c.nsplit;
  if (id < n_dkv) dkv_workgroup<HD, KEYS_SMALL, QS, CAP, true>(c, (lds_char*)smem_raw, id % nx, id / nx);
  else dq_workgroup<HD, 256 * QS, KS, CAP>(c, (lds_char*)smem_raw, (id - n_dkv) % c.a.h, (id - n_dkv) / c.a.h);
}

// dK | dV = sum over splits, in split order, rounded once; rows of no sequence are left alone
__global__ __launch_bounds__(256) void score_dkv_reduce_kernel(ScoreCall c) {
  const ScoreArgs& a = c.a;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int dkv = a.hkv * a.hd, per_row = 2 * dkv / 4;
  if (i >= (int64_t)a.rows * per_row) return;
  const int row = (int)(i / per_row), col = (int)(i % per_row) * 4;
  SeqSpan s;
  if (!seq_of_row(a, row, s)) return;
  f32x4 acc = *reinterpret_cast<const f32x4*>(c.part + (int64_t)row * (2 * dkv) + col);
  for (int sp = 1; sp < c.nsplit; ++sp) acc += *reinterpret_cast<const f32x4*>(c.part + ((int64_t)sp * a.rows + row) * (2 * dkv) + col);
  bf16x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (bf16)acc[e];
  bf16* out = col < dkv ? (bf16*)a.dk + (int64_t)row * a.lddk + col : (bf16*)a.dv + (int64_t)row * a.lddv + col - dkv;
  *reinterpret_cast<bf16x4*>(out) = o;
}

// ---- host -------------------------------------------------------------------------------------------------------------------
template <int HD, int KS> constexpr size_t fwd_lds() { return (size_t)(KS == 4 ? 8 : 4) * Geo<HD>::TILEB; }
template <int HD, int NT, int KS> constexpr size_t dq_lds() { return fwd_lds<HD, KS>() + (KS > 1 ? NT / 64 * 128 : 0); }      // + shares of delta
template <int HD, int TQ, int QS> constexpr size_t dkv_lds() { return (size_t)2 * (2 * TQ * Geo<HD>::ROWB + 2 * TQ * 4) + QS * (TQ / 32) * 4096 + 64; }

template <typename K>
hipError_t allow_lds(K kern, size_t bytes) {
  return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

constexpr int64_t RESIDENT = 2 * 256;  // workgroups of 4 wavefronts that a chip of 256 CUs holds (a constant: the scratch's size depends on it)

// grid slots of bq rows each (times heads: workgroups), and what of them there is to do at least
int64_t slots(const ScoreArgs& a, int bq) {
  return a.seq_start ? a.rows / bq + a.n_seq : (int64_t)a.n_seq * ((a.rows / a.n_seq + bq - 1) / bq);
}

// What the rules below are: measured on sequences of 30 to 16384 rows, 4 to 40 heads (us; "packed" = lengths drawn, n of them).
int mean_len(const ScoreArgs& a) { return a.rows / a.n_seq; }

enum Shape { SHAPE_WIDE = 1, SHAPE_NARROW = 2, SHAPE_SPLIT = 3, SHAPE_SPLIT4 = 4 };
// Forward and dQ: 8 wavefronts x 32 queries, 4 x 32, or 64 queries whose keys 2 or 4 wavefronts share.
// WIDE reads every K/V tile once for twice the queries, but its last tiles are twice as much masked and its last round of the chip (one workgroup to a
// CU) leaves twice as much idle: for equal sequences where that round is nearly full, or there are so many rows that it weighs little (WIDE / NARROW,
// forward and dQ's difference, head_dim 128: up to two rounds, 40 heads x 2800 97 / 99, -6, 32 x 4096 145 / 154, -9, 20 x 6000 197 / 205, -11, 16 x 8192 269 / 291,
// -27; a little more than two, 40 x 3400 144 / 139, +7, 40 x 3800 171 / 163, +5, 32 x 4500 183 / 180, +3; three and more, 32 x 2 x 3000 170 / 164, +1, 32 x 2 x 4096
// 285 / 282, -3, 16 x 2 x 6500 354 / 346, -20, 16 x 2 x 8192 523 / 530, -36; without a causal mask 40 x 2560 156 / 162, -9, 36 x 3500 221 / 231, -22, but 40 x 3800
// 339 / 305, +34, 32 x 4500 392 / 352, +42).  Not for packed ones (16 x 13 in 8192 71 / 62), nor in the
// forward of head_dim 64, where NARROW has more wavefronts to a CU (32 x 4096 118 / 90).
// SPLIT below about a round and a half of NARROW (SPLIT / NARROW, head_dim 128: 16 x 3000 58 / 64, 40 x 1500 47 / 40), SPLIT4 for few workgroups
// with long chains (SPLIT4 / SPLIT: 4 x 5000 60 / 72, 16 x 2048 45 / 36; head_dim 64, whose workgroups sit two to a CU, 16 x 2048 21.5 / 24.7).
Shape q_shape(const ScoreArgs& a, int width, bool forward) {
  if (width >= 1 && width <= 4) return (Shape)width;
  const int64_t wide = slots(a, 256) * a.h;
  if (!a.seq_start && !(forward && a.hd == 64) && wide >= 400 && ((wide <= 512 && mean_len(a) >= 2500) || mean_len(a) >= 6000)) return SHAPE_WIDE;
  if (slots(a, 128) * a.h >= (forward && a.hd == 64 ? 512 : 450)) return SHAPE_NARROW;
  return forward && slots(a, 64) * a.h <= (a.hd == 64 ? 512 : 384) && mean_len(a) >= 1000 ? SHAPE_SPLIT4 : SHAPE_SPLIT;
}
// dK/dV: into how many workgroups the query heads of a KV head go: until there are two rounds of them (128 keys: one workgroup to a CU; 64 keys:
// two), or every query head has its own.  (Split for one round, 16 heads on 2 x 13 packed in 8192 239, for two 194; their sums cost 13 of it.)
int dkv_splits(const ScoreArgs& a, int tq) {
  const int grp = a.h / a.hkv;
  const int64_t wgs = slots(a, tq) * a.hkv, want = tq == 128 ? 512 : 1024;
  int ns = 1;
  while (ns < grp && wgs * ns < want) {
    int nx = ns + 1;
    while (grp % nx) ++nx;
    ns = nx;
  }
  return ns;
}
// dK/dV: 128 keys to a workgroup, 64, or 64 with two pairs of wavefronts to 32 keys.
// 64 keys for short sequences and enough workgroups (128 keys / 64, 16 heads x 100 packed in 8192 101 / 70, 16 x 4 x 1024 55 / 59; head_dim 64
// 75 / 41, 36 / 33, 32 x 4 x 2048 237 / 207, 12 x 9000 355 / 391); two pairs for few workgroups (128 keys / two pairs, 4 x 5000 134 / 101, 8 x 1024 34 / 25, 12 x 3 x
// 777 36 / 36; head_dim 64 97 / 80, 25 / 19, 24 / 19, 8 x 5 packed in 6000 79 / 66, 12 x 3 packed in 4096 54 / 52).
enum KeyShape { KEYS_128 = 1, KEYS_64 = 3, KEYS_64_TWO = 4 };
KeyShape k_shape(const ScoreArgs& a, int width) {
  if (width >= 1 && width <= 4) return width <= 2 ? KEYS_128 : (KeyShape)width;
  const int64_t n64 = slots(a, 64) * a.hkv * dkv_splits(a, 64), n128 = slots(a, 128) * a.hkv * dkv_splits(a, 128);
  if (mean_len(a) > 320 && n64 <= (a.hd == 64 ? 850 : 320)) return KEYS_64_TWO;
  if (mean_len(a) <= (a.hd == 64 ? 2048 : 512) && n64 >= 960) return KEYS_64;
  return n128 < 450 ? KEYS_64 : KEYS_128;
}

ScoreCall score_call(const ScoreArgs& a) {
  ScoreCall c{};
  c.a = a;
  c.sl2 = a.scale * LOG2E;
  c.raw = 1.f / a.scale;
  c.nsplit = 1;
  if (a.cap > 0.f) {
    const double r = (double)a.scale / a.cap, c2 = (double)a.cap * 1.4426950408889634;
    c.c2 = (float)c2;
    c.ic2 = (float)(1.0 / c2);
    c.kx = (float)(2.0 * 1.4426950408889634 * r);
    c.small = (float)(0.25 / r);
    c.middling = (float)(0.6 / r);
    double f = c2 * r * r * r;
    for (int i = 0; i < 4; ++i, f *= r * r) {
      if (i < 2) c.p3[i] = (float)(TANH2[i] * f);
      c.p5[i] = (float)(TANH4[i] * f);
    }
    c.wide = c.c2 > WIDE_CAP || fabsf(c.p5[3]) < FLT_MIN;
    if (c.wide) c.small = c.middling = -1.f;
  }
  return c;
}

template <int HD, int NT, int KS, bool CAP>
hipError_t fwd_launch(ScoreCall c, hipStream_t s) {
  constexpr size_t lds_bytes = fwd_lds<HD, KS>();
  static const hipError_t ready = allow_lds(score_fwd_kernel<HD, NT, KS, CAP>, lds_bytes);
  if (ready != hipSuccess) return ready;
  const int64_t n = slots(c.a, block_q<NT, KS>()), grid = n * c.a.h;
  c.tiles = c.a.seq_start ? 0 : (int)(n / c.a.n_seq);
  c.fold = (NT == NARROW || KS == 4 || HD == 64) && c.a.causal && grid <= RESIDENT;
  hipLaunchKernelGGL((score_fwd_kernel<HD, NT, KS, CAP>), dim3((unsigned)grid), dim3(NT), lds_bytes, s, c);
  return hipGetLastError();
}
template <int HD, bool CAP>
hipError_t fwd_t(const ScoreCall& c, int width, hipStream_t s) {
  switch (q_shape(c.a, width, true)) {
    case SHAPE_WIDE:
      if constexpr (HD == 128) return fwd_launch<HD, WIDE, 1, CAP>(c, s);
      // fall through
    case SHAPE_NARROW: return fwd_launch<HD, NARROW, 1, CAP>(c, s);
    case SHAPE_SPLIT: return fwd_launch<HD, NARROW, 2, CAP>(c, s);
    default: return fwd_launch<HD, WIDE, 4, CAP>(c, s);
  }
}

template <int HD, int NT, int KS, bool CAP>
hipError_t dq_launch(ScoreCall c, hipStream_t s) {
  constexpr size_t lds_bytes = dq_lds<HD, NT, KS>();
  static const hipError_t ready = allow_lds(score_dq_kernel<HD, NT, KS, CAP>, lds_bytes);
  if (ready != hipSuccess) return ready;
  const int64_t n = slots(c.a, block_q<NT, KS>()), grid = n * c.a.h;
  c.tiles = c.a.seq_start ? 0 : (int)(n / c.a.n_seq);
  c.fold = NT == NARROW && c.a.causal && grid <= RESIDENT;
  hipLaunchKernelGGL((score_dq_kernel<HD, NT, KS, CAP>), dim3((unsigned)grid), dim3(NT), lds_bytes, s, c);
  return hipGetLastError();
}
hipError_t reduce_launch(const ScoreCall& c, hipStream_t s) {
  const int64_t pieces = (int64_t)c.a.rows * (2 * c.a.hkv * c.a.hd / 4);
  hipLaunchKernelGGL(score_dkv_reduce_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, s, c);
  return hipGetLastError();
}
template <int HD, int TQ, int QS, bool CAP>
hipError_t dkv_launch(ScoreCall c, hipStream_t s) {
  constexpr size_t lds_bytes = dkv_lds<HD, TQ, QS>();
  static const hipError_t ready = allow_lds(score_dkv_kernel<HD, TQ, QS, CAP>, lds_bytes);
  if (ready != hipSuccess) return ready;
  c.nsplit = dkv_splits(c.a, TQ);
  const int64_t n = slots(c.a, TQ), grid = n * c.a.hkv * c.nsplit;
  c.tiles = c.a.seq_start ? 0 : (int)(n / c.a.n_seq);
  c.fold = TQ == KEYS_SMALL && c.a.causal && grid <= RESIDENT;
  hipLaunchKernelGGL((score_dkv_kernel<HD, TQ, QS, CAP>), dim3((unsigned)grid), dim3(TQ * 4 * QS), lds_bytes, s, c);
  return c.nsplit > 1 ? reduce_launch(c, s) : hipGetLastError();
}
template <int HD, int KS, int QS, bool CAP>
hipError_t bwd_fused_launch(ScoreCall c, hipStream_t s) {
  constexpr size_t dq_bytes = dq_lds<HD, 256 * QS, KS>(), dkv_bytes = dkv_lds<HD, KEYS_SMALL, QS>(), lds_bytes = dq_bytes > dkv_bytes ? dq_bytes : dkv_bytes;
  static const hipError_t ready = allow_lds(score_bwd_kernel<HD, KS, QS, CAP>, lds_bytes);
  if (ready != hipSuccess) return ready;
  c.nsplit = dkv_splits(c.a, KEYS_SMALL);
  const int64_t n = slots(c.a, 64), n_dkv = n * c.a.hkv * c.nsplit, grid = n_dkv + n * c.a.h;
  c.tiles = c.a.seq_start ? 0 : (int)(n / c.a.n_seq);
  hipLaunchKernelGGL((score_bwd_kernel<HD, KS, QS, CAP>), dim3((unsigned)grid), dim3(256 * QS), lds_bytes, s, c, (int)n_dkv);
  return c.nsplit > 1 ? reduce_launch(c, s) : hipGetLastError();
}
template <int HD, bool CAP>
hipError_t bwd_t(const ScoreCall& c, int width, hipStream_t s) {
  const ScoreArgs& a = c.a;
  const int64_t n64 = slots(a, 64), total = n64 * a.h + n64 * a.hkv * dkv_splits(a, 64);
  const int len = mean_len(a);
  // Both passes in one launch while their workgroups (64 queries, 64 keys) number little more than what is resident; with two pairs of
  // wavefronts up to one to a CU, or with long causal chains somewhat more (one launch / two: head_dim 128 8 x 1024 33 / 46, 4 x 5000 157 / 175, 16 x
  // 2048 115 / 102), with one pair (head_dim 64: three to a CU) for shorter sequences (workgroups: 880, 40 x 700 27 / 31; 936, 12 x 3 x 777 33.5 / 33.9; 1024, 32 x
  // 1000 36 / 38; 1248, 16 x 3 x 777 39 / 42; 1408, 32 x 1400 60 / 59; 1000, 20 x 1600 55 / 53; 4 x 5000 140 / 128).
  // Not for sequences of up to DELTA_KEYS rows: the dK/dV half cannot wait for the dQ half's delta and takes its own from the rounded O.  Nor for packed
  // ones, whose lengths only the device knows: any of them may be that short, whatever their mean.  (That costs small packed batches time: one launch / two,
  // head_dim 128 8 x 3 packed in 600 18 / 26, 4 x 4 in 2048 31 / 41, 4 x 3 in 4000 79 / 79; head_dim 64 8 x 3 in 600 13 / 19, 12 x 3 in 2331 45 / 50.)
  const bool longer = !a.seq_start && len > DELTA_KEYS;
  const bool two_pairs = longer && (2 * total <= RESIDENT || (a.causal && ((total <= RESIDENT && len > 320) || (total <= 700 && len > 1500))));
  if (width == 6 || (width == 0 && two_pairs)) return bwd_fused_launch<HD, 4, 2, CAP>(c, s);
  const bool one_pair = longer && (HD == 128 ? a.causal && len <= 320 && total <= RESIDENT : len <= 1500 && total <= 1280);
  if (width == 5 || (width == 0 && one_pair)) return bwd_fused_launch<HD, 2, 1, CAP>(c, s);
  hipError_t e;      // dQ first: it also leaves delta in the scratch for the dK/dV pass
  switch (q_shape(a, width, false)) {
    case SHAPE_WIDE: e = dq_launch<HD, WIDE, 1, CAP>(c, s); break;
    case SHAPE_NARROW: e = dq_launch<HD, NARROW, 1, CAP>(c, s); break;
    default: e = dq_launch<HD, NARROW, 2, CAP>(c, s); break;
  }
  if (e != hipSuccess) return e;
  switch (k_shape(a, width)) {
    case KEYS_128: return dkv_launch<HD, KEYS, 1, CAP>(c, s);
    case KEYS_64: return dkv_launch<HD, KEYS_SMALL, 1, CAP>(c, s);
    default: return dkv_launch<HD, KEYS_SMALL, 2, CAP>(c, s);
  }
}

bool rows_ok(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1 << 23); }

}  // namespace

// the backward's fp32 shares of dK | dV, behind delta in the scratch; sized for either tile of the dK/dV kernel
size_t score_part_bytes(const ScoreArgs& a) {
  const int n128 = dkv_splits(a, KEYS), n64 = dkv_splits(a, KEYS_SMALL), ns = n128 > n64 ? n128 : n64;
  return ns > 1 ? (size_t)ns * a.rows * 2 * a.hkv * a.hd * sizeof(float) : 0;
}

// (strides below 2^23: a tile of 128 rows has to lie within the 2 GiB that a load's offset reaches)
bool score_mfma_supported(const ScoreArgs& a) {
  if (!rows_ok(a.q, a.ldq) || !rows_ok(a.k, a.ldk) || !rows_ok(a.v, a.ldv) || !rows_ok(a.o, a.ldo)) return false;
  if (a.dout && (!rows_ok(a.dout, a.lddo) || !rows_ok(a.dq, a.lddq) || !rows_ok(a.dk, a.lddk) || !rows_ok(a.dv, a.lddv))) return false;
  return slots(a, 64) * 2 * a.h * 512 < ((int64_t)1 << 32);         // threads of a grid
}
hipError_t score_fwd_mfma(const ScoreArgs& a, int width, hipStream_t s) {
  const ScoreCall c = score_call(a);
  if (a.cap > 0.f) return a.hd == 128 ? fwd_t<128, true>(c, width, s) : fwd_t<64, true>(c, width, s);
  return a.hd == 128 ? fwd_t<128, false>(c, width, s) : fwd_t<64, false>(c, width, s);
}
hipError_t score_bwd_mfma(const ScoreArgs& a, float* part, int width, hipStream_t s) {
  ScoreCall c = score_call(a);
  c.part = part;
  if (a.cap > 0.f) return a.hd == 128 ? bwd_t<128, true>(c, width, s) : bwd_t<64, true>(c, width, s);
  return a.hd == 128 ? bwd_t<128, false>(c, width, s) : bwd_t<64, false>(c, width, s);
}

}  // namespace stg
