// What the bf16 attention kernels share: tiles that go global -> LDS directly, MFMA operand fragments read from them as rows or
// (transposed) as columns, and the moves between the two lanes that hold a row of a 32 x 32 block.
#pragma once
#include "common.h"

namespace stg {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

namespace {

constexpr int TK = 64;            // rows of one LDS tile (keys in forward / dQ, queries in dK/dV)
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

typedef __attribute__((address_space(3))) char lds_char;
typedef int rsrc_words __attribute__((ext_vector_type(4)));

// LDS tile: TK rows of HD bf16, unpadded, filled by buffer loads that write LDS directly (lane l of a wavefront
// lands at the wavefront's LDS address + 16*l, out-of-range lanes store zeros).  The 16-byte piece c (8 columns)
// of row r sits in slot r*PPR + (c ^ swz(r)); the swizzle makes both ways of reading the tile conflict-free:
//   rows as MFMA operand rows (16 consecutive rows, same piece): 16 different 16-byte bank groups
//   transpose reads (4 consecutive rows, 64 contiguous bytes each): 4 different 64-byte bank groups
template <int HD> struct Geo {
  static constexpr int PPR = HD / 8;             // 16-byte pieces per row
  static constexpr int ROWB = HD * 2;            // bytes per row
  static constexpr int TILEB = TK * ROWB;        // bytes per tile
  static constexpr int NKK = HD / 16;            // k-steps of a product reducing over head_dim
  static constexpr int NHB = HD / 32;            // 32-wide head_dim blocks of an output
  __device__ static __forceinline__ int swz(int r) {
    return HD == 128 ? (((r & 3) << 2) | ((r >> 2) & 3)) : ((((r >> 1) & 1) << 2) | ((r >> 2) & 3));
  }
};

__device__ __forceinline__ rsrc_words raw_rsrc(const void* base, unsigned bytes) {
  const uint64_t a = (uint64_t)base;
  return rsrc_words{(int)(unsigned)a, (int)(unsigned)((a >> 32) & 0xffffu), (int)bytes, 0x00020000};
}
// Inline assembly on purpose: with the builtin the compiler cannot tell these LDS writes from the fragment reads
// of the other buffer and drains the vector-memory counter before every LDS read.  Completion is awaited by hand
// (vmcnt(0) before the barrier that publishes a tile).  m0 = the wavefront's LDS destination.
__device__ __forceinline__ void load_to_lds_b128(rsrc_words rsrc, unsigned lds_addr, unsigned voffset) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(lds_addr), "v"(voffset), "s"(rsrc) : "memory");
}

// Per-thread byte offsets (relative to row 0 of the tile's first row, column 0 of the head) of the pieces it
// fetches: load j of wavefront w fills slots (j*NW + w)*64 .. +63.
template <int HD, int NTHR, int ROWS = TK>
__device__ __forceinline__ void tile_offsets(unsigned (&off)[ROWS * (HD / 8) / NTHR], int64_t ld, int wave, int lane) {
  using G = Geo<HD>;
#pragma unroll
  for (int j = 0; j < ROWS * G::PPR / NTHR; ++j) {
    const int s = (j * (NTHR / 64) + wave) * 64 + lane;
    const int r = s / G::PPR, c = (s % G::PPR) ^ G::swz(r);
    off[j] = (unsigned)(((int64_t)r * ld + c * 8) * 2);
  }
}
// rows [row0, row0+TK) of the matrix behind `rsrc` -> LDS tile; the descriptor ends with the last real row, so rows
// past it are out of range and store zeros.  `wave` must be wave-uniform.
template <int HD, int NTHR, int ROWS = TK>
__device__ __forceinline__ void tile_g2s(lds_char* tile, rsrc_words rsrc, const unsigned (&off)[ROWS * (HD / 8) / NTHR],
                                         int64_t ld, int row0, int wave) {
  const unsigned step = (unsigned)((int64_t)row0 * ld * 2);
#pragma unroll
  for (int j = 0; j < ROWS * (HD / 8) / NTHR; ++j)
    load_to_lds_b128(rsrc, (unsigned)(size_t)(tile + (j * (NTHR / 64) + wave) * 1024), off[j] + step);
}
// descriptor of one head's [nrows, HD] slice of a row-major matrix with row stride ld (elements)
__device__ __forceinline__ rsrc_words head_rsrc(const bf16* p, int64_t ld, int nrows, int hd) {
  return raw_rsrc(p, (unsigned)(((int64_t)(nrows - 1) * ld + hd) * 2));
}

// ---- MFMA operand fragments ---------------------------------------------------
// Per-lane byte offsets inside a tile.
//   rows-type operand (rows = tile rows, reduction over head_dim: lane l -> tile row rb + l%32, columns
//   16*ks + (l/32)*8 ..+7):  ro[ks], plus rb * ROWB for the row block
//   transposed operand (rows = head_dim columns hb*32 + l%32, reduction over 16 tile rows r0..r0+15; the 8 reduction
//   slots of lane-half hf = l/32 are tile rows r0 + 4*hf + {0,1,2,3} and r0 + 8 + 4*hf + {0,1,2,3}: the order in
//   which a lane holds a 32x32 accumulator block's rows, so a register-resident P / dS block pairs with it
//   directly):  co[hb][0 or 1] for the two 4-row groups, plus r0 * ROWB (r0 a multiple of 16)
template <int HD>
struct FragOff {
  unsigned ro[HD / 16];
  unsigned co[HD / 32][2];
  // `lds`: the workgroup's LDS base; the offsets are absolute LDS addresses, so a read's address is one register
  // plus an immediate
  __device__ __forceinline__ void init(int lane, lds_char* lds) {
    using G = Geo<HD>;
    const unsigned base = (unsigned)(size_t)lds;
    const int r = lane & 31, hf = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < G::NKK; ++ks) ro[ks] = base + (unsigned)(r * G::ROWB + (((2 * ks + hf) ^ G::swz(r)) << 4));
    const int g = lane >> 4, li = lane & 15;
#pragma unroll
    for (int hb = 0; hb < G::NHB; ++hb)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int row = (g >> 1) * 4 + (li >> 2) + 8 * u;
        const int piece = hb * 4 + (g & 1) * 2 + ((li & 3) >> 1);
        co[hb][u] = base + (unsigned)(row * G::ROWB + ((piece ^ G::swz(row)) << 4) + (li & 1) * 8);
      }
  }
  __device__ __forceinline__ void hop(int bytes) {
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) ro[ks] += bytes;
#pragma unroll
    for (int hb = 0; hb < HD / 32; ++hb) { co[hb][0] += bytes; co[hb][1] += bytes; }
  }
};
template <int HD>
__device__ __forceinline__ bf16x8 frag_rows(lds_char* lds, const FragOff<HD>& f, int tile_off, int rb, int ks) {
  return *(__attribute__((address_space(3))) const bf16x8*)(size_t)(f.ro[ks] + (unsigned)(tile_off + rb * Geo<HD>::ROWB));
}
template <int HD>
__device__ __forceinline__ bf16x8 frag_cols_tr(lds_char* lds, const FragOff<HD>& f, int tile_off, int r0, int hb) {
  typedef s16x4 __attribute__((address_space(3))) * lds_p;
  union { struct { s16x4 a, b; } s; bf16x8 v; } u;
  u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(size_t)(f.co[hb][0] + (unsigned)(tile_off + r0 * Geo<HD>::ROWB)));
  u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(size_t)(f.co[hb][1] + (unsigned)(tile_off + r0 * Geo<HD>::ROWB)));
  return u.v;
}
// rows-type operand straight from global memory (kept in registers for the whole kernel); rows >= nrows read as zero
__device__ __forceinline__ bf16x8 frag_rows_global(const bf16* base, int64_t ld, int row0, int nrows, int kk, int lane) {
  const int row = row0 + (lane & 31);
  bf16x8 z;
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = (bf16)0.f;
  if (row < nrows) z = *reinterpret_cast<const bf16x8*>(base + (int64_t)row * ld + kk + (lane >> 5) * 8);
  return z;
}

__device__ __forceinline__ bf16x8 pack8(const float* v) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16)v[e];
  return r;
}
// The value held by the lane 32 further on (or back): v_permlane32_swap exchanges the upper half of one register with
// the lower half of another, one vector instruction instead of a round trip through the LDS crossbar.  Given v twice, the
// first result holds the partner's value in lanes 32-63 and the second in lanes 0-31.  (The second copy is made opaque
// and the two results are only ever selected between, never combined with each other: the compiler folded a sum of the
// two results into twice the first.)
__device__ __forceinline__ float xhalf(float v, int hf) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  unsigned w = u;
  asm volatile("" : "+v"(w));
  const auto r = __builtin_amdgcn_permlane32_swap(u, w, false, false);
  return __builtin_bit_cast(float, hf ? r[0] : r[1]);
}
__device__ __forceinline__ float half_max(float v, int hf) { return fmaxf(v, xhalf(v, hf)); }
__device__ __forceinline__ float half_sum(float v, int hf) { return v + xhalf(v, hf); }
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// acc + sum of the 8 elements of v (v_dot2c_f32_bf16 against (1, 1): exact products, fp32 accumulation)
__device__ __forceinline__ float dot_ones(bf16x8 v, float acc) {
  bf16x2 one;
  one[0] = (bf16)1.f; one[1] = (bf16)1.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16x2 pr;
    pr[0] = v[2 * i]; pr[1] = v[2 * i + 1];
    acc = __builtin_amdgcn_fdot2_f32_bf16(pr, one, acc, false);
  }
  return acc;
}
__device__ __forceinline__ void zero(f32x16& a) {
#pragma unroll
  for (int e = 0; e < 16; ++e) a[e] = 0.f;
}
#define MFMA(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16((a), (b), (c), 0, 0, 0)
// first product of an accumulation chain: C = 0 as an inline constant, so no registers are cleared beforehand
__device__ __forceinline__ f32x16 mfma0(bf16x8 a, bf16x8 b) {
  const f32x16 z = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, z, 0, 0, 0);
}

// row index inside a 32-row accumulator block held in register e by a lane of half hf
__device__ __forceinline__ int acc_row(int e, int hf) { return (e >> 2) * 8 + hf * 4 + (e & 3); }

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32; -inf -> 0

#define SCHED_FENCE __builtin_amdgcn_sched_barrier(0)

// Which query tile (forward, dQ: the later, the more keys it sees) the workgroup of dispatch rank `rank` takes.
// Plain order is heaviest first.  `fold`: the heavier half first, heaviest first, then the lighter half, lightest
// first -- for grids that are resident all at once with two workgroups per CU, so that a CU's second workgroup is as
// light as its first is heavy (ranks r and r + nh add up to the same work) instead of the chip waiting for the CUs that
// drew two heavy ones.
__device__ __forceinline__ int tile_of_rank(int rank, int n, int fold) {
  const int nh = (n + 1) >> 1;
  return (!fold || rank < nh) ? n - 1 - rank : rank - nh;
}

// early key tiles see the most queries: plain order is kt = rank; folded (see tile_of_rank) the heavy half first, then
// the light half, lightest first
__device__ __forceinline__ int key_tile_of_rank(int rank, int n, int fold) { return n - 1 - tile_of_rank(rank, n, fold); }

// acc = (ADD: acc +) sum over head_dim of rows(tile `TILE`, rows rb..rb+31) x bfr (the wavefront's K or V fragments); fragment
// reads run three k-steps ahead
template <int HD, int TILE, bool ADD = false>
__device__ __forceinline__ void dkv_rows_product(lds_char* lds, const FragOff<HD>& fo, int rb, const bf16x8 (&bfr)[HD / 16], f32x16& acc) {
  using G = Geo<HD>;
  constexpr int AHEAD = 3;
  bf16x8 f[AHEAD + 1];
#pragma unroll
  for (int kk = 0; kk < AHEAD; ++kk) f[kk] = frag_rows<HD>(lds, fo, TILE, rb, kk);
#pragma unroll
  for (int kk = 0; kk < G::NKK; ++kk) {
    if (kk + AHEAD < G::NKK) f[(kk + AHEAD) % (AHEAD + 1)] = frag_rows<HD>(lds, fo, TILE, rb, kk + AHEAD);
    if (kk == 0 && !ADD) acc = mfma0(f[0], bfr[0]);
    else acc = MFMA(f[kk % (AHEAD + 1)], bfr[kk], acc);
    SCHED_FENCE;
  }
}
// out[hb]^T += (tile `TILE`, rows rb..rb+31)^T . w, w = the 32 x 32 block of P or dS held as two bf16 fragments;
// the first transposed fragments must already be in tf[] (read before the vector arithmetic that made w)
template <int HD, int TILE>
__device__ __forceinline__ void dkv_tr_read(lds_char* lds, const FragOff<HD>& fo, int rb, bf16x8 (&tf)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) tf[i] = frag_cols_tr<HD>(lds, fo, TILE, rb + (i / Geo<HD>::NHB) * 16, i % Geo<HD>::NHB);
}
template <int HD, int TILE>
__device__ __forceinline__ void dkv_tr_product(lds_char* lds, const FragOff<HD>& fo, int rb, bf16x8 (&tf)[4], const bf16x8 (&w)[2],
                                               f32x16 (&out)[HD / 32]) {
  using G = Geo<HD>;
  constexpr int N = G::NHB * 2, VA = 4;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bf16x8 v = tf[i % VA];
    if (i + VA < N) {
      const int n = i + VA;
      tf[i % VA] = frag_cols_tr<HD>(lds, fo, TILE, rb + (n / G::NHB) * 16, n % G::NHB);
    }
    out[i % G::NHB] = MFMA(v, w[i / G::NHB], out[i % G::NHB]);
    SCHED_FENCE;
  }
}

}  // namespace
}  // namespace stg
