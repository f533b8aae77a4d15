// What the kernels of the experts' products share (expert_product.hip, block_product.hip): operands, tiles in LDS and their loads, scales, stores, and the kernels
// that serve both, with the scales of 8-bit operands as a template parameter.
#pragma once
#include <type_traits>

#include "row_ops.hpp"

namespace lasnet {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef unsigned uint2_t __attribute__((ext_vector_type(2)));
typedef uint2_t uint2_any __attribute__((aligned(1)));

struct ProductArgs {
  RowsArg I, J, out;               // .pitch: bytes from one row in memory to the next
  long long i_expert, out_expert;  // bytes from one expert's matrix to the next (I: forward, dx; out: dW)
  const int32_t* offsets;
  const uint8_t* scale;            // of J's rows
  const float* wscale;             // [E][ni]
  long long rows;                  // all rows
  int E, ni, nj, nk;               // output columns; output rows (dW); reduction (forward, dx)
  int tiles_i, tiles_j;            // dW: tiles of an expert's matrix
  int part_rows, parts;            // dW in parts: rows of a part, and how many parts there may be
  bool relu;
  const uint8_t* xblocks;          // scales of blocks of 128 (see SCALES): [rows][kb] bytes
  const void* wblocks;             // [E][(ni + 127) / 128][kb] bytes or floats
  int kb;                          // blocks of the reduction
  bool past;                       // whether the output is written past the caches (see writes_past)
};

// Which scales 8-bit operands have (SCALES).  ROWS: one for each row of J and of I, applied where the sums are stored.  Blocks of 128 of the reduction, those of I shared by 128 of
// its rows: POWERS: both powers of two, bytes 127 + e, which the matrix core applies to the products for nothing; FLOATS: J's powers of two, likewise, and I's in
// 32 bits, m 2^e with m from 1 to 2: the matrix core applies 2^e, too (it adds the two exponents: neither scale by itself takes a sum out of fp32's range), and with m the sum of a block,
// 128 products from 0, is added to the whole: an fma for each element and step, run while the matrix core multiplies.
enum { ROWS = 0, POWERS = 1, FLOATS = 2 };
// The byte and m of a scale in 32 bits.  (Below the normal numbers: 2^-127 and an m of less than 2.  Infinities and NaN are m's; their byte is a number, 255 being NaN.)
__device__ __forceinline__ unsigned scale_power(unsigned w) {
  const unsigned e = w >> 23 & 255;
  return e < 254 ? e : 254;
}
__device__ __forceinline__ float scale_mantissa(unsigned w) { return __builtin_amdgcn_ldexpf(__uint_as_float(w), 127 - (int)(w >> 23 & 255)); }
// A step's product with the scales of its block.  w: byte (of FLOATS: scale_power's).
template <int SCALES>
__device__ __forceinline__ floatx4 scaled_mfma(intx8 i, intx8 j, floatx4 acc, unsigned w, unsigned x) {
  if constexpr (SCALES == ROWS)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i, j, acc, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
  else if constexpr (SCALES == POWERS)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i, j, acc, 0, 0, 0, (int)w, 0, (int)x);
  else
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i, j, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, (int)w, 0, (int)x);
}
// The same with the rows of J as the first operand: four of them in a lane, of one row of I.
template <int SCALES>
__device__ __forceinline__ floatx4 turned_mfma(intx8 i, intx8 j, floatx4 acc, unsigned w, unsigned x) {
  if constexpr (SCALES == POWERS)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(j, i, acc, 0, 0, 0, (int)x, 0, (int)w);
  else
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(j, i, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, (int)x, 0, (int)w);
}
__device__ __forceinline__ floatx4 add_scaled(floatx4 acc, floatx4 part, float m) {
#pragma unroll
  for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(part[r], m, acc[r]);
  return acc;
}

// offsets[e] as the kernels take it: within [0, rows].
__device__ __forceinline__ int bound(const ProductArgs& a, int e) {
  const int v = a.offsets[e];
  return v < 0 ? 0 : (long long)v < a.rows ? v : (int)a.rows;
}

typedef __amdgpu_buffer_rsrc_t product_rsrc_t;

__device__ __forceinline__ product_rsrc_t product_rsrc(const void* p, unsigned bytes) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(size_t)p), hi = __builtin_amdgcn_readfirstlane((unsigned)((size_t)p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(((unsigned long long)hi << 32) | lo), 0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// Row tile t of all experts' (BJ rows each, the last of an expert may have fewer) -> its expert, first row and the expert's end.  Expert E: the rows that no
// expert has.  false: no such tile.  Every wave of a workgroup finds the same.
__device__ __forceinline__ bool find_rows(const ProductArgs& a, int BJ, int t, int& expert, int& first, int& end) {
  const int lane = (int)threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 <= a.E; e0 += 64) {
    const int e = e0 + lane;
    int lo = 0, hi = 0;
    if (e <= a.E) {
      lo = bound(a, e);
      hi = e < a.E ? bound(a, e + 1) : (int)a.rows;
    }
    const int v = hi > lo ? (hi - lo + BJ - 1) / BJ : 0;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(s, d);
      if (lane >= d) s += u;
    }
    const unsigned long long m = __ballot(t < before + s);
    if (m) {
      const int l = __ffsll((long long)m) - 1;
      expert = e0 + l;
      first = __shfl(lo + (t - (before + s - v)) * BJ, l);
      end = __shfl(hi, l);
      return true;
    }
    before += __shfl(s, 63);
  }
  return false;
}

// ---- LDS tiles: 128 (i or j) x 128 bytes of k by rows, 64 k x 128 by columns; 16 KiB either way ----
// By rows: piece (16 bytes) c of row r lies at r * 128 + (c ^ (r >> 1 & 7)) * 16, so that 16 rows' pieces c fill 256 bytes of banks.
// By columns: the 32 bytes u of row k lie at k * 256 + (u ^ turn(k)) * 32: the eight rows that two groups of 16 lanes read lie apart.
__device__ __forceinline__ int turn(int k) { return (k & 3) | (k >> 1 & 4); }

template <bool COLS>
struct Tile {
  // piece q (0 .. 1023) of the tile: its place in LDS, and its row and first byte in memory, relative to the tile
  static __device__ __forceinline__ int place(int q) {
    if constexpr (COLS) {
      const int k = q >> 4, c = q & 15;
      return k * 256 + (((c >> 1) ^ turn(k)) * 2 + (c & 1)) * 16;
    } else {
      const int r = q >> 3, c = q & 7;
      return r * 128 + (c ^ (r >> 1 & 7)) * 16;
    }
  }
  static __device__ __forceinline__ int row(int q) { return COLS ? q >> 4 : q >> 3; }
  static __device__ __forceinline__ int byte(int q) { return COLS ? (q & 15) * 16 : (q & 7) * 16; }
  // the MFMA operand of 16 rows (columns) from at0, half of the 128 bytes of k (32 k of 64)
  static __device__ __forceinline__ uint4_t fragment(const unsigned char* tile, int at0, int half, int lane) {
    if constexpr (COLS) {
      typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
      const int k = half * 32 + (lane >> 4) * 8 + (lane >> 2 & 3);
      const unsigned char* p = tile + k * 256 + ((at0 >> 4) ^ turn(k)) * 32 + (lane & 3) * 8;
      union { bf16x4_t h[2]; uint4_t u; } f;
      f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4_t*)p);
      f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4_t*)(p + 4 * 256));
      return f.u;
    } else {
      const int r = at0 + (lane & 15), c = half * 4 + (lane >> 4);
      return *(const uint4_t*)(tile + r * 128 + (c ^ (r >> 1 & 7)) * 16);
    }
  }
};

// Scales of e4m3 products.  sum * wscale * 2^(b - 127), without the product of the two scales, which may leave fp32's range where the result does not (2^127 times 4, or
// 2^-126 times 10^-6): the sum (2^-18 to 2^38 in size, or 0) times wscale's mantissa, from 1/2 to 1, then its exponent and the row's by v_ldexp, which rounds below the
// normal numbers alone.  A row's byte of 255 is NaN: it comes as the addend of the multiplication, -0 for any other row (which changes nothing, not even the sign of 0).
struct ColScale {
  float mantissa;
  int exponent;
};
__device__ __forceinline__ ColScale col_scale(float w) { return ColScale{__builtin_amdgcn_frexp_mantf(w), __builtin_amdgcn_frexp_expf(w)}; }
struct RowScale {
  int exponent;
  float addend;
};
__device__ __forceinline__ RowScale row_scale(unsigned byte) { return RowScale{(int)byte - 127, byte == 255 ? __uint_as_float(0x7fc00000u) : -0.f}; }
__device__ __forceinline__ float scaled(float sum, ColScale w, RowScale r) {
  return __builtin_amdgcn_ldexpf(__builtin_fmaf(sum, w.mantissa, r.addend), w.exponent + r.exponent);
}
// Two multiplications in this order give the same bits where sum * wscale is a normal number (or 0, infinite, NaN) whatever the sum: the streaming kernel's tiles take
// them where all of a wave's columns allow it (32768 rows, 4096 x 2048: 298 us; v_ldexp for every element 351; the other kernels take the same time either way).
__device__ __forceinline__ bool plain_scale(float w) {
  const int e = __builtin_amdgcn_frexp_expf(w);               // (0 of 0, infinities and NaN)
  return e >= -107 && e <= 89;
}
// 2^(b - 127); 255: NaN
__device__ __forceinline__ float scale_value(unsigned b) {
  return __uint_as_float(b == 255 ? 0x7fc00000u : b ? b << 23 : 0x00400000u);
}

// The 16 bytes of a row of `size` from byte b on, without a branch where every row has 16 bytes (WIDE): they may begin earlier, so as to end with the row
// (see cut_piece; what is before a shorter row is not kept, whatever it is).
template <bool WIDE>
__device__ __forceinline__ uint4_t row_piece(const unsigned char* row, int b, int size) {
  if (WIDE || size >= 16) return load16(row + (b < size - 16 ? b : size - 16));
  uint4_t v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i / 4] |= (unsigned)row[i > 16 - size ? i - (16 - size) : 0] << (8 * (i % 4));
  return v;
}
// ... of which n were left: moved to the front, zeros behind them.
__device__ __forceinline__ uint4_t cut_piece(uint4_t v, int n) {
  const int s = n <= 0 ? 16 : n < 16 ? 16 - n : 0;            // bytes to drop
#pragma unroll
  for (int w = 1; w <= 4; w *= 2) {
    uint4_t u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = i + w < 4 ? v[i + w] : 0u;
    if (s & 4 * w) v = u;
  }
  uint4_t u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_alignbyte(i < 3 ? v[i + 1] : 0u, v[i], s & 3);
  return u;
}

// The wave's NI x NJ blocks of 16 x 16, from column oi0 and row oj0 of the output on, scaled, rounded and stored.  Outputs whose columns and pitch are whole
// multiples of 4 elements go through a buffer that ends with row j_end, without a branch for each; others (and rows too far apart) element by element.
template <bool FP8, bool F32OUT, int NI, int NJ>
__device__ __forceinline__ void store_tile(const ProductArgs& a, unsigned char* out, int expert, int oi0, int oj0, int j_end, const floatx4 (&acc)[NI][NJ]) {
  constexpr int OB = F32OUT ? 4 : 2;
  const int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (made anew: no register holds it through the loop)
  const float floor = a.relu ? 0.f : -INFINITY;               // (NaN passes)
  RowScale up[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    up[j] = row_scale(127);
    if constexpr (FP8) {
      const int oj = oj0 + 16 * j + (lane & 15);
      if (a.scale && expert < a.E && oj < j_end) up[j] = row_scale(a.scale[oj]);
    }
  }
  if (oj0 >= j_end || oi0 >= a.ni) return;
  const bool fours = !((a.ni | (int)(a.out.pitch / OB)) & 3) && !((size_t)out & 3) && a.out.pitch < (1 << 22);
  const int rows = j_end - oj0 < 16 * NJ ? j_end - oj0 : 16 * NJ;
  const product_rsrc_t to = product_rsrc(out + (long long)oj0 * a.out.pitch + (long long)oi0 * OB,
                                         fours ? (unsigned)(rows - 1) * (unsigned)a.out.pitch + (unsigned)(a.ni - oi0) * OB : 0u);
  auto each = [&](auto store) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int oi = oi0 + 16 * i + (lane >> 4) * 4;
      float w[4] = {1.0f, 1.0f, 1.0f, 1.0f};
      if constexpr (FP8)
        if (a.wscale && expert < a.E) Elem<float>::widen(load_piece<float>((const unsigned char*)(a.wscale + (size_t)expert * a.ni + oi), a.ni - oi), w);
      ColScale ws[4];
      if constexpr (FP8)
#pragma unroll
        for (int r = 0; r < 4; ++r) ws[r] = col_scale(w[r]);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v[r] = acc[i][j][r];
          if constexpr (FP8) v[r] = scaled(v[r], ws[r], up[j]);
          v[r] = v[r] < floor ? floor : v[r];
        }
        store(i, j, oi, v);
      }
    }
  };
  if (fours) {
    each([&](int i, int j, int oi, const float (&v)[4]) {
      const int o = oi < a.ni ? (16 * j + (lane & 15)) * (int)a.out.pitch + (16 * i + (lane >> 4) * 4) * OB : -1;
      if constexpr (F32OUT)
        __builtin_amdgcn_raw_buffer_store_b128(Elem<float>::narrow(v), to, o, 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b64(uint2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}, to, o, 0, 0);
    });
  } else {
    each([&](int, int j, int oi, const float (&v)[4]) {
      const int oj = oj0 + 16 * j + (lane & 15);
      if (oj >= j_end) return;
      unsigned char* o = out + (long long)oj * a.out.pitch + (long long)oi * OB;
      if constexpr (F32OUT) {
        store_piece<float>(o, a.ni - oi, Elem<float>::narrow(v));
      } else if (oi + 4 <= a.ni) {
        *(uint2_any*)o = uint2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (oi + r < a.ni) Elem<__bf16>::put(o + 2 * r, bf16_pair(v[r], 0.f));
      }
    });
  }
}

// The same where the rows of J were the first operand and row 16 i + c of the wave's rows of I in LDS is row 4 c + i in memory: a lane has four columns next to each other of 4 NJ rows,
// 16 lanes a row's 128 bytes, a whole line.  (What a CU's 128 KiB of stores take goes by the lines that 16 lanes touch: 1.1 us of two whole ones, 7.1 of 16 by 8 bytes.)
template <int NJ>
__device__ __forceinline__ void store_turned_tile(const ProductArgs& a, int oi0, int oj0, int j_end, const floatx4 (&acc)[4][NJ]) {
  const int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  const float floor = a.relu ? 0.f : -INFINITY;               // (NaN passes)
  if (oj0 >= j_end || oi0 >= a.ni) return;
  const bool fours = !((a.ni | (int)(a.out.pitch / 2)) & 3) && !((size_t)a.out.data & 3) && a.out.pitch < (1 << 22);
  const int rows = j_end - oj0 < 16 * NJ ? j_end - oj0 : 16 * NJ, left = a.ni - oi0 - (lane & 15) * 4;
  unsigned char* out = a.out.data + (long long)oj0 * a.out.pitch + (long long)oi0 * 2;
  const product_rsrc_t to = product_rsrc(out, fours ? (unsigned)(rows - 1) * (unsigned)a.out.pitch + (unsigned)(a.ni - oi0) * 2 : 0u);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * j + (lane >> 4) * 4 + r;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = acc[i][j][r] < floor ? floor : acc[i][j][r];
      if (fours) {
        __builtin_amdgcn_raw_buffer_store_b64(uint2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}, to, left > 0 ? row * (int)a.out.pitch + (lane & 15) * 8 : -1, 0, 0);
      } else if (row < rows) {
        unsigned char* o = out + (long long)row * a.out.pitch + (lane & 15) * 8;
        if (left >= 4) {
          *(uint2_any*)o = uint2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < left) Elem<__bf16>::put(o + 2 * i, bf16_pair(v[i], 0.f));
        }
      }
    }
}

// Any alignment and width: 128 x 128 of the output by 4 waves, 64 x 64 each; rows and weights through registers into two LDS stages, the next step's loads in
// flight while this one's products run.  Bound by those loads: pieces that begin anywhere touch two lines of the caches.  16384 rows of 8 experts, 2047 x 2049:
// bf16 224 us, its gradients 256 and 266, 8 bits 141; a branch for each piece's end instead of row_piece: 222, 322, 421, 160, and with few columns up to five
// times as long (28473 rows, 2103 x 226, gradient of the weights 199 and 1010).
// FP8: e4m3, else bf16.  IC, JC: held by columns.  RAGGED: the reduction runs over an expert's rows (dW).  WIDE: see row_piece.
template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, bool WIDE, int SCALES = ROWS>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs a) {
  constexpr int BYTES = FP8 ? 1 : 2, KS = 128 / BYTES;
  __shared__ __attribute__((aligned(128))) unsigned char lds[2][2][16384];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ti = (int)(blockIdx.x % a.tiles_i);
  int expert, j0, j_end, k0, k_end;
  if constexpr (RAGGED) {
    const int rest = (int)(blockIdx.x / a.tiles_i);
    expert = rest / a.tiles_j;
    j0 = rest % a.tiles_j * 128;
    j_end = a.nj;
    k0 = bound(a, expert);
    k_end = bound(a, expert + 1);
  } else {
    if (!find_rows(a, 128, (int)(blockIdx.x / a.tiles_i), expert, j0, j_end)) return;
    k0 = 0;
    k_end = expert < a.E ? a.nk : 0;                          // (no reduction: zeros)
  }
  const int i0 = ti * 128;
  const unsigned char* I = a.I.data + (RAGGED ? 0 : (long long)(expert < a.E ? expert : 0) * a.i_expert);

  floatx4 acc[4][4] = {};
  uint4_t ri[4], rj[4];
  // Rows beyond the last are read as the last: of i or j, what comes of them is not stored; of k they are cut to nothing.
  const int row_i = (IC ? a.ni : a.nk) * BYTES, row_j = (JC ? a.nj : a.nk) * BYTES;
  const unsigned char *pi[4], *pj[4];                         // by rows: the rows of a thread's pieces
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int q = u * 256 + tid, i = i0 + Tile<IC>::row(q), j = j0 + Tile<JC>::row(q);
    pi[u] = I + (IC ? 0 : (long long)(i < a.ni ? i : a.ni - 1) * a.I.pitch);
    pj[u] = a.J.data + (JC ? 0 : (long long)(j < j_end ? j : j_end - 1) * a.J.pitch);
  }
  const int wi = (wave & 1) * 64, wj = (wave >> 1) * 64;
  // scales: of the step that is multiplied, and of the next
  unsigned sx[4], sw = 0, nx[4], nw = 0;
  auto fetch_scales = [&](int k) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = j0 + wj + 16 * j + (lane & 15);
      nx[j] = a.xblocks[(long long)(r < j_end ? r : j_end - 1) * a.kb + (k >> 7)];
    }
    const long long w = ((long long)expert * ((a.ni + 127) >> 7) + (i0 >> 7)) * a.kb + (k >> 7);
    nw = SCALES == POWERS ? ((const uint8_t*)a.wblocks)[w] : ((const unsigned*)a.wblocks)[w];
  };
  auto turn_scales = [&] {
#pragma unroll
    for (int j = 0; j < 4; ++j) sx[j] = nx[j];
    sw = nw;
  };
  auto fetch = [&](int k) {
    if constexpr (SCALES != ROWS) fetch_scales(k);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int q = u * 256 + tid, r = k + Tile<IC>::row(q);
      const unsigned char* row = IC ? I + (long long)(r < k_end ? r : k_end - 1) * a.I.pitch : pi[u];
      ri[u] = row_piece<WIDE>(row, (IC ? i0 : k) * BYTES + Tile<IC>::byte(q), row_i);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int q = u * 256 + tid, r = k + Tile<JC>::row(q);
      const unsigned char* row = JC ? a.J.data + (long long)(r < k_end ? r : k_end - 1) * a.J.pitch : pj[u];
      rj[u] = row_piece<WIDE>(row, (JC ? j0 : k) * BYTES + Tile<JC>::byte(q), row_j);
    }
  };
  auto stage = [&](int s, int k) {
    const bool whole_i = k + KS <= k_end && (!IC || i0 + 128 <= a.ni), whole_j = k + KS <= k_end && (!JC || j0 + 128 <= j_end);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int q = u * 256 + tid;
      if (!whole_i) {
        const int left = k_end - k, b = Tile<IC>::byte(q);
        ri[u] = cut_piece(ri[u], IC ? Tile<IC>::row(q) < left ? (a.ni - i0) * BYTES - b : 0 : left * BYTES - b);
      }
      if (!whole_j) {
        const int left = k_end - k, b = Tile<JC>::byte(q);
        rj[u] = cut_piece(rj[u], JC ? Tile<JC>::row(q) < left ? (j_end - j0) * BYTES - b : 0 : left * BYTES - b);
      }
      *(uint4_t*)(lds[s][0] + Tile<IC>::place(q)) = ri[u];
      *(uint4_t*)(lds[s][1] + Tile<JC>::place(q)) = rj[u];
    }
  };
  int s = 0;
  if (k0 < k_end) {
    fetch(k0);
    stage(0, k0);
    if constexpr (SCALES != ROWS) turn_scales();
  }
  __syncthreads();
  for (int k = k0; k < k_end; k += KS, s ^= 1) {
    if (k + KS < k_end) fetch(k + KS);
    if constexpr (FP8) {
      intx8 fi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        union { uint4_t u[2]; intx8 v; } f;
        f.u[0] = Tile<IC>::fragment(lds[s][0], wi + 16 * i, 0, lane);
        f.u[1] = Tile<IC>::fragment(lds[s][0], wi + 16 * i, 1, lane);
        fi[i] = f.v;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        union { uint4_t u[2]; intx8 v; } f;
        f.u[0] = Tile<JC>::fragment(lds[s][1], wj + 16 * j, 0, lane);
        f.u[1] = Tile<JC>::fragment(lds[s][1], wj + 16 * j, 1, lane);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 v = scaled_mfma<SCALES>(fi[i], f.v, acc[i][j], SCALES == FLOATS ? scale_power(sw) : sw, sx[j]);
          acc[i][j] = SCALES == FLOATS ? add_scaled(acc[i][j], v, scale_mantissa(sw)) : v;
        }
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        union F { uint4_t u; bf16x8 v; };
        F fi[4], fj[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) fi[i].u = Tile<IC>::fragment(lds[s][0], wi + 16 * i, h, lane);
#pragma unroll
        for (int j = 0; j < 4; ++j) fj[j].u = Tile<JC>::fragment(lds[s][1], wj + 16 * j, h, lane);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fi[i].v, fj[j].v, acc[i][j], 0, 0, 0);
      }
    }
    if (k + KS < k_end) {
      stage(s ^ 1, k + KS);
      if constexpr (SCALES != ROWS) turn_scales();
    }
    __syncthreads();
  }

  unsigned char* out = a.out.data + (RAGGED ? (long long)expert * a.out_expert : 0);
  store_tile<FP8 && SCALES == ROWS, F32OUT>(a, out, expert, i0 + wi, j0 + wj, j_end, acc);
}

// ---- whole pieces: rows, widths and addresses that are multiples of 16 bytes ----
// Tiles go from memory to LDS without passing registers, through buffers that end where the operand does: rows and k beyond come back as zeros, and nothing has
// to be clamped.  Every load is issued, those past the last step of an empty buffer, so that they can be counted.
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef int intx4 __attribute__((ext_vector_type(4)));
// Where an operand's loads are: the tile at the next step's k, and the buffer that ends with the operand (by rows: what there is of the tile's rows from there on;
// by columns: of the step's rows of k).  Kept to a few scalar instructions a step: the waves that share a SIMD have some 30 clocks for each pair of MFMAs.
template <bool COLS>
struct Feed {
  unsigned long long at;
  unsigned size;             // by rows: bytes from `at` to the end of the last row; by columns: of a row, from the tile's first column on
  __device__ __forceinline__ void start(const unsigned char* first, int rows, int most, long long pitch, unsigned row_bytes) {
    const unsigned long long f = (unsigned long long)first;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)f), hi = __builtin_amdgcn_readfirstlane((unsigned)(f >> 32));
    at = (unsigned long long)hi << 32 | lo;
    size = __builtin_amdgcn_readfirstlane(COLS ? row_bytes : (unsigned)((rows < most ? rows : most) - 1) * (unsigned)pitch + row_bytes);
  }
  // k: what is left of it (none: an empty buffer)
  __device__ __forceinline__ intx4 rsrc(int k, unsigned pitch) const {
    unsigned n = size;
    if constexpr (COLS) n += (unsigned)((k < 64 ? k : 64) - 1) * pitch;
    return intx4{(int)(unsigned)at, (int)(unsigned)(at >> 32), (int)(k > 0 ? n : 0u), 0x00020000};
  }
  __device__ __forceinline__ void move(unsigned by) {
    at += by;
    if constexpr (!COLS) size -= by;
  }
};
__device__ __forceinline__ void buffer_to_lds(intx4 rsrc, unsigned off, unsigned to) {                  // 64 x 16 bytes to 1 KiB
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "s"(to) : "memory");
}
// 64 bytes, or the same float 64 times, to 64 dwords.
template <bool BYTES>
__device__ __forceinline__ void scales_to_lds(intx4 rsrc, unsigned off, unsigned to) {
  if constexpr (BYTES)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_ubyte %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "s"(to) : "memory");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "s"(to) : "memory");
}
// All but the youngest VM memory operations of the wave have ended (they are counted off in the order they were issued in) and every LDS read has been
// answered; then all waves' have.  (The check build waits for all.)
template <int VM>
__device__ __forceinline__ void counted_barrier() {
  static_assert(VM >= 0 && VM < 64, "vmcnt is 6 bits");
  __builtin_amdgcn_sched_barrier(0);
#ifdef LASNET_DRAIN_AT_BARRIERS
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#else
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(VM) : "memory");
#endif
  __builtin_amdgcn_sched_barrier(0);
}

union Fragment { uint4_t h[2]; intx8 all; };

// A wave's scales of a step on their way through LDS, in a slot of its own (no other wave's barrier has to cover them): those of 64 rows of J from row0 on, a dword each, then
// that of I's rows from i0 on (which lie in one block of 128), 64 times.  Two loads a step, counted like the tiles'.
constexpr int kScaleSlot = 512, kScaleLoads = 2;
template <int SCALES>
struct ScaleFeed {
  intx4 x, w;
  unsigned off_x, off_w;
  int left;                                                   // steps with scales
  __device__ __forceinline__ void start(const ProductArgs& a, int expert, int i0, int row0, int j_end, int step, int lane) {
    constexpr int WB = SCALES == FLOATS ? 4 : 1;
    const int rows = j_end - row0 < 64 ? j_end - row0 : 64, nb = (a.ni + 127) >> 7, ib = i0 >> 7;
    const unsigned long long at_x = (unsigned long long)a.xblocks + (unsigned long long)((long long)row0 * a.kb);
    const unsigned long long at_w = (unsigned long long)a.wblocks + (unsigned long long)(((long long)expert * nb + ib) * a.kb * WB);
    auto uniform = [](unsigned v) { return (int)__builtin_amdgcn_readfirstlane(v); };
    x = intx4{uniform((unsigned)at_x), uniform((unsigned)(at_x >> 32)), uniform(rows > 0 ? (unsigned)(rows * a.kb) : 0u), 0x00020000};
    w = intx4{uniform((unsigned)at_w), uniform((unsigned)(at_w >> 32)), uniform(ib < nb ? (unsigned)(a.kb * WB) : 0u), 0x00020000};
    off_x = (unsigned)(lane * a.kb + step);
    off_w = (unsigned)(step * WB);
    left = a.kb - step;
  }
  // the next step's; past the last one zeros (not what the next row begins with: that may be NaN, and products of nothing would be, too)
  __device__ __forceinline__ void load(unsigned to) {
    scales_to_lds<true>(intx4{x[0], x[1], left > 0 ? x[2] : 0, x[3]}, off_x, to);
    --left;
    scales_to_lds<SCALES == POWERS>(w, off_w, to + 256);
    off_x += 1;
    off_w += SCALES == FLOATS ? 4 : 1;
  }
};
__device__ __forceinline__ unsigned read_dword(unsigned at) { return *(const __attribute__((address_space(3))) unsigned*)(size_t)at; }

// One operand's tile: B rows (columns), loaded by NW waves.
template <bool COLS, int B, int NW>
struct Stage {
  static constexpr int BYTES = B * 128, SEGS = B / 8 / NW;   // segments of 1 KiB, one load instruction each, of a wave
  static constexpr int PITCH = COLS ? B * 2 : 128;           // of the tile's rows in LDS
  static constexpr int TURNS = B / 16 < 8 ? B / 16 - 1 : 7;
  static_assert(B % (8 * NW) == 0, "whole segments");
  // of the piece that a lane loads for segment seg: its row (by columns: its k) and its first byte there
  static __device__ __forceinline__ int row(int seg, int lane) { return COLS ? seg * (1024 / PITCH) + lane / (PITCH / 16) : seg * 8 + (lane >> 3); }
  static __device__ __forceinline__ int byte(int seg, int lane) {
    const int r = row(seg, lane);
    if constexpr (COLS) {
      const int c = lane % (PITCH / 16);
      return (((c >> 1) ^ (turn(r) & TURNS)) * 2 + (c & 1)) * 16;
    } else {
      return ((lane & 7) ^ (r >> 1 & 7)) * 16;
    }
  }
  // Where a lane reads block 0 of the wave's from (w0: its first row or column); block i, half h lie at this address with some bits
  // turned over (a swizzle is an exclusive or) plus constants.
  static __device__ __forceinline__ unsigned lane_base(int w0, int lane) {
    if constexpr (COLS) {
      const int k = (lane >> 4) * 8 + (lane >> 2 & 3);
      return k * PITCH + ((w0 >> 4) ^ (turn(k) & TURNS)) * 32 + (lane & 3) * 8;
    } else {
      return (w0 + (lane & 15)) * 128 + ((lane >> 4) ^ (lane >> 1 & 7)) * 16;
    }
  }
  // Block i (16 rows or columns) of the tile: 128 bytes of k for two MFMAs of 32 (bf16) or one of 128 (e4m3).  at: lane_base() + the tile's first byte (whose low
  // ten bits are zero, so the bits may be turned over in the sum).
  static __device__ __forceinline__ void fragment(unsigned at, int i, Fragment& f) {
    if constexpr (COLS) {
      typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) bf16x4_t* p4;
      const lds_byte* p = (const lds_byte*)(size_t)(at ^ (i * 32));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        union { bf16x4_t h[2]; uint4_t u; } v;
        v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((p4)(p + h * 32 * PITCH));
        v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((p4)(p + (h * 32 + 4) * PITCH));
        f.h[h] = v.u;
      }
    } else {
      typedef const __attribute__((address_space(3))) uint4_t* p16;
      f.h[0] = *(p16)((const lds_byte*)(size_t)at + i * 2048);
      f.h[1] = *(p16)((const lds_byte*)(size_t)(at ^ 64) + i * 2048);
    }
  }
};

// Row tiles of all experts and of the rows without one.
template <int BJ>
__device__ __forceinline__ int row_tiles(const ProductArgs& a) {
  const int lane = (int)threadIdx.x & 63;
  int n = 0;
  for (int e = lane; e <= a.E; e += 64) {
    const int lo = bound(a, e), hi = e < a.E ? bound(a, e + 1) : (int)a.rows;
    n += hi > lo ? (hi - lo + BJ - 1) / BJ : 0;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  return __builtin_amdgcn_readfirstlane(n);
}
// Workgroup -> tile of `total`: each XCD (workgroups are dealt to the eight in turn) takes consecutive ones.  -1: none left.
__device__ __forceinline__ int xcd_tile(int total) {
  const int chunk = (total + 7) / 8, i = (int)blockIdx.x >> 3, t = ((int)blockIdx.x & 7) * chunk + i;
  return i < chunk && t < total ? t : -1;
}
// Tile t of ni x nj: four rows of tiles at a time, so that workgroups that run together share both operands.
__device__ __forceinline__ void tile_at(int t, int ni, int nj, int& i, int& j) {
  const int g = t / (4 * ni), r = t - g * 4 * ni, n = nj - 4 * g < 4 ? nj - 4 * g : 4;
  i = r / n;
  j = 4 * g + r % n;
}

// One tile: BI x BJ of the output by WI x WJ waves, through STAGES stages of 128 bytes of k of both operands.
//
// A wave holds the fragments of its J blocks for the whole step and walks its I blocks with a ring of four fragments, each read three blocks ahead, over the end of
// the step too: before the block second from last every read of the stage has been answered, so one barrier there frees the stage for the loads of STAGES
// steps on and opens the next, whose first fragments are read while the last two blocks' MFMAs run.  MFMAs come first behind the barrier, loads and
// reads between them: all waves are at the same place there.  The MFMAs of a block are independent of each other.
//
// WK > 1: so many groups of WI x WJ waves share the reduction, each a run of its steps through stages of its own; their sums are added in order.
template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1, int SCALES = ROWS>
__device__ __forceinline__ void tile_product(const ProductArgs& a, unsigned char* product_lds, int expert, int i0, int j0, int j_end, int k0, int k_end) {
  constexpr int BYTES = FP8 ? 1 : 2, KS = 128 / BYTES, NI = BI / WI / 16, NJ = BJ / WJ / 16;
  using SI = Stage<IC, BI, WI * WJ>;
  using SJ = Stage<JC, BJ, WI * WJ>;
  constexpr int STAGE = SI::BYTES + SJ::BYTES, LOADS = SI::SEGS + SJ::SEGS;
  constexpr int COUNTED = LOADS + (SCALES == ROWS ? 0 : kScaleLoads);
  static_assert(NI % 4 == 0, "a ring of four fragments");
  static_assert(SCALES == ROWS || (FP8 && !IC && !JC && !RAGGED && BI / WI == 64 && BJ / WJ <= 64), "a wave's columns in one block of 128, its rows in a load; see store_turned_tile");
  int lane = (int)threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) % (WI * WJ);
  const int group = WK > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) / (WI * WJ) : 0;
  const unsigned lds = (unsigned)(size_t)(lds_byte*)product_lds + group * STAGES * STAGE;
  asm volatile("" : "+v"(lane));                               // (nothing of this is worked out before its time and kept)
  const int steps = k_end > k0 ? (k_end - k0 + WK * KS - 1) / (WK * KS) : 0;
  if constexpr (WK > 1) {                                      // (a group whose run begins at the end or beyond loads nothing)
    k0 += group * steps * KS;
    if (k0 > k_end) k0 = k_end;
    if (k_end > k0 + steps * KS) k_end = k0 + steps * KS;
  }
  // where the tiles are in memory, and how far a step takes them
  const unsigned char* I = a.I.data + (RAGGED ? 0 : (long long)(expert < a.E ? expert : 0) * a.i_expert);
  const unsigned pitch_i = (unsigned)a.I.pitch, pitch_j = (unsigned)a.J.pitch, kb = (unsigned)a.nk * BYTES;
  Feed<IC> li;
  Feed<JC> lj;
  const unsigned skip = RAGGED ? 0 : (unsigned)k0 * BYTES;     // (by rows k0 is a place in the rows)
  li.start(I + (IC ? (long long)k0 * a.I.pitch + (long long)i0 * BYTES : (long long)i0 * a.I.pitch + skip), a.ni - i0, BI, a.I.pitch,
           IC ? (unsigned)(a.ni - i0) * BYTES : kb - skip);
  lj.start(a.J.data + (JC ? (long long)k0 * a.J.pitch + (long long)j0 * BYTES : (long long)j0 * a.J.pitch + skip), j_end - j0, BJ, a.J.pitch,
           JC ? (unsigned)(j_end - j0) * BYTES : kb - skip);
  const unsigned di = IC ? KS * pitch_i : 128, dj = JC ? KS * pitch_j : 128;
  unsigned off_i[SI::SEGS], off_j[SJ::SEGS];                  // of this lane's pieces from the tile
#pragma unroll
  for (int s = 0; s < SI::SEGS; ++s) {
    int row = SI::row(wave * SI::SEGS + s, lane);
    if constexpr (SCALES != ROWS) row = (row & ~63) + (row & 15) * 4 + (row >> 4 & 3);
    off_i[s] = (unsigned)row * pitch_i + (unsigned)SI::byte(wave * SI::SEGS + s, lane);
  }
#pragma unroll
  for (int s = 0; s < SJ::SEGS; ++s) off_j[s] = (unsigned)SJ::row(wave * SJ::SEGS + s, lane) * pitch_j + (unsigned)SJ::byte(wave * SJ::SEGS + s, lane);
  int l_k = k_end - k0;                                       // what is left of k to load
  unsigned l_to = lds;
  const int wi = wave % WI * (BI / WI), wj = wave / WI * (BJ / WJ);
  const unsigned slots = (unsigned)(size_t)(lds_byte*)product_lds + WK * STAGES * STAGE + (group * WI * WJ + wave) * STAGES * kScaleSlot;
  unsigned s_to = slots, s_at = slots;
  ScaleFeed<SCALES> ls;
  // (a group that begins at the end: behind the last block, whose scale times nothing would be NaN were it infinite)
  if constexpr (SCALES != ROWS) ls.start(a, expert < a.E ? expert : 0, i0 + wi, j0 + wj, j_end, (k0 + KS - 1) / KS, lane);
  // A step's loads, between the parts of `meanwhile` (which does what is due anyway, in LOADS parts).
  const unsigned to_i = wave * SI::SEGS * 1024, to_j = SI::BYTES + wave * SJ::SEGS * 1024;
  auto load = [&](auto meanwhile) {
    meanwhile(0);
    if constexpr (SCALES != ROWS) {
      ls.load(s_to);
      s_to = s_to == slots + (STAGES - 1) * kScaleSlot ? slots : s_to + kScaleSlot;
    }
    const intx4 ri = li.rsrc(l_k, pitch_i), rj = lj.rsrc(l_k, pitch_j);
    unsigned oi[SI::SEGS], oj[SJ::SEGS];
#pragma unroll
    for (int s = 0; s < SI::SEGS; ++s) oi[s] = off_i[s];
#pragma unroll
    for (int s = 0; s < SJ::SEGS; ++s) oj[s] = off_j[s];
    if ((!IC || !JC) && l_k < KS) {                           // by rows, what is beyond the end of k lies inside the buffer
#pragma unroll
      for (int s = 0; s < SI::SEGS; ++s)
        if (!IC && SI::byte(wave * SI::SEGS + s, lane) >= l_k * BYTES) oi[s] = 0xffffffffu;
#pragma unroll
      for (int s = 0; s < SJ::SEGS; ++s)
        if (!JC && SJ::byte(wave * SJ::SEGS + s, lane) >= l_k * BYTES) oj[s] = 0xffffffffu;
    }
#pragma unroll
    for (int s = 0; s < LOADS; ++s) {
      if (s) meanwhile(s);
      __builtin_amdgcn_sched_barrier(0);
      if (s < SI::SEGS)
        buffer_to_lds(ri, oi[s < SI::SEGS ? s : 0], l_to + to_i + s * 1024);
      else
        buffer_to_lds(rj, oj[s < SI::SEGS ? 0 : s - SI::SEGS], l_to + to_j + (s - SI::SEGS) * 1024);
      __builtin_amdgcn_sched_barrier(0);
    }
    l_to = l_to == lds + (STAGES - 1) * STAGE ? lds : l_to + STAGE;
    li.move(di);
    lj.move(dj);
    l_k -= KS;
  };

  floatx4 acc[NI][NJ] = {};
  Fragment fi[4], fj[2][NJ];
  unsigned sx[2][NJ], sw[2] = {0, 0};                         // scales of this step and the next
  constexpr int LAG = NJ > 1 ? 3 : 2;
  unsigned power = 0;                                         // FLOATS: this step's scale, and the m of the step before
  float m_now = 0.f, m_before = 0.f;
  floatx4 part[4] = {};                                       // FLOATS: sums of blocks, each added to its whole LAG MFMAs later
  const unsigned bi = SI::lane_base(wi, lane), bj = SJ::lane_base(wj, lane) + SI::BYTES;
  unsigned at = lds, at_i = bi + at;                          // at: the stage that is read
  auto read_i = [&](int i) { SI::fragment(at_i, i, fi[i % 4]); };
  auto read_j = [&](auto stage) {
    const unsigned at_j = bj + at;
#pragma unroll
    for (int j = 0; j < NJ; ++j) SJ::fragment(at_j, j, fj[stage.value][j]);
    if constexpr (SCALES != ROWS) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) sx[stage.value][j] = read_dword(s_at + (16 * j + (lane & 15)) * 4);
      sw[stage.value] = read_dword(s_at + 256);
    }
  };
  auto add_part = [&](int m, float w) { acc[m / NJ][m % NJ] = add_scaled(acc[m / NJ][m % NJ], part[m % 4], w); };
  constexpr int MFMAS = (FP8 ? 1 : 2) * NJ;                   // of a block
  auto multiply = [&](auto stage, int i, int m0, int m1) {
    constexpr int S = decltype(stage)::value;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = m0; m < m1; ++m) {
      const int j = m % NJ, h = m / NJ;
      if constexpr (SCALES == FLOATS) {
        constexpr int ALL = NI * NJ;
        const int at = i * NJ + j;
        part[at % 4] = turned_mfma<SCALES>(fi[i % 4].all, fj[S][j].all, floatx4{}, power, sx[S][j]);
        add_part(at >= LAG ? at - LAG : ALL + at - LAG, at >= LAG ? m_now : m_before);
      } else if constexpr (SCALES == POWERS) {
        acc[i][j] = turned_mfma<SCALES>(fi[i % 4].all, fj[S][j].all, acc[i][j], sw[S], sx[S][j]);
      } else if constexpr (FP8) {
        acc[i][j] = scaled_mfma<ROWS>(fi[i % 4].all, fj[S][j].all, acc[i][j], 0, 0);
      } else {
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fi[i % 4].h[h]), __builtin_bit_cast(bf16x8, fj[S][j].h[h]), acc[i][j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](auto stage) {
    constexpr int S = decltype(stage)::value;
    if constexpr (SCALES == FLOATS) {
      power = scale_power(sw[S]);
      m_before = m_now;
      m_now = scale_mantissa(sw[S]);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (i + 3 < NI) read_i(i + 3);
      if (i == NI - 2) {
        counted_barrier<(STAGES - 2) * COUNTED>();
        at = at == lds + (STAGES - 1) * STAGE ? lds : at + STAGE;
        if constexpr (SCALES != ROWS) s_at = s_at == slots + (STAGES - 1) * kScaleSlot ? slots : s_at + kScaleSlot;
        at_i = bi + at;
        asm volatile("" : "+v"(at_i));                         // (a sum in a register: reads add constants to it)
        load([&](int l) {
          multiply(stage, i, l * MFMAS / LOADS, (l + 1) * MFMAS / LOADS);
          if (l == 0) {
            read_j(std::integral_constant<int, S ^ 1>{});
            read_i(0);
            read_i(1);
          }
        });
      } else {
        if (i == NI - 1) read_i(2);
        multiply(stage, i, 0, MFMAS);
      }
    }
  };
  if (steps) {
    auto nothing = [](int) {};
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) load(nothing);
    counted_barrier<(STAGES - 2) * COUNTED>();
    load(nothing);
    read_j(std::integral_constant<int, 0>{});
    read_i(0);
    read_i(1);
    read_i(2);
    for (int s = 0; s < steps; s += 2) {
      step(std::integral_constant<int, 0>{});
      if (s + 1 < steps) step(std::integral_constant<int, 1>{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (the last loads write to this workgroup's LDS)
    if constexpr (SCALES == FLOATS)
#pragma unroll
      for (int m = NI * NJ - LAG; m < NI * NJ; ++m) add_part(m, m_now);
  }
  if constexpr (WK > 1) {
    floatx4* sums = (floatx4*)product_lds + wave * NI * NJ * 64 + lane;        // [group - 1][wave][block][lane]
    constexpr int GROUP = WI * WJ * NI * NJ * 64;
    static_assert((WK - 1) * GROUP * 16 <= WK * STAGES * STAGE, "room for the sums");
    __syncthreads();
    if (group) {
#pragma unroll
      for (int b = 0; b < NI * NJ; ++b) sums[(group - 1) * GROUP + b * 64] = acc[b / NJ][b % NJ];
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int g = 0; g < WK - 1; ++g)
#pragma unroll
      for (int b = 0; b < NI * NJ; ++b) acc[b / NJ][b % NJ] += sums[g * GROUP + b * 64];
  }
  unsigned char* out = a.out.data + (RAGGED ? (long long)expert * a.out_expert : 0);
  if constexpr (SCALES == ROWS)
    store_tile<FP8, F32OUT>(a, out, expert, i0 + wi, j0 + wj, j_end, acc);
  else
    store_turned_tile(a, i0 + wi, j0 + wj, j_end, acc);
}

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1, int SCALES = ROWS>
__global__ __launch_bounds__(64 * WI * WJ * WK, 2) void product_tile_kernel(ProductArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char product_lds[];
  int expert, ti, j0, j_end, k0, k_end;
  if constexpr (RAGGED) {
    const int per = a.tiles_i * a.tiles_j, t = xcd_tile(a.E * per);
    if (t < 0) return;
    int tj;
    expert = t / per;
    tile_at(t - expert * per, a.tiles_i, a.tiles_j, ti, tj);
    j0 = tj * BJ;
    j_end = a.nj;
    k0 = __builtin_amdgcn_readfirstlane(bound(a, expert));
    k_end = __builtin_amdgcn_readfirstlane(bound(a, expert + 1));
  } else {
    int tj;
    if (a.E <= 62) {                                          // an expert (and the rows without one, and their end) for each lane: looked up once
      const int lane = (int)threadIdx.x & 63;
      const int lo = lane <= a.E ? bound(a, lane) : (int)a.rows, hi = __shfl(lo, lane < 63 ? lane + 1 : 63);
      int upto = hi > lo ? (hi - lo + BJ - 1) / BJ : 0;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(upto, d);
        if (lane >= d) upto += u;
      }
      const int tiles = __builtin_amdgcn_readlane(upto, 63), t = xcd_tile(tiles * a.tiles_i);
      if (t < 0) return;
      tile_at(t, a.tiles_i, tiles, ti, tj);
      expert = __ffsll((long long)__ballot(tj < upto)) - 1;
      j0 = __builtin_amdgcn_readlane(lo, expert) + (tj - (expert ? __builtin_amdgcn_readlane(upto, expert - 1) : 0)) * BJ;
      j_end = __builtin_amdgcn_readlane(lo, expert + 1);
    } else {
      const int tiles = row_tiles<BJ>(a), t = xcd_tile(tiles * a.tiles_i);
      if (t < 0) return;
      tile_at(t, a.tiles_i, tiles, ti, tj);
      if (!find_rows(a, BJ, tj, expert, j0, j_end)) return;
      expert = __builtin_amdgcn_readfirstlane(expert);
      j0 = __builtin_amdgcn_readfirstlane(j0);
      j_end = __builtin_amdgcn_readfirstlane(j_end);
    }
    k0 = 0;
    k_end = expert < a.E ? a.nk : 0;
  }
  tile_product<FP8, IC, JC, RAGGED, F32OUT, BI, BJ, WI, WJ, STAGES, WK, SCALES>(a, product_lds, expert, ti * BI, j0, j_end, k0, k_end);
}

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1, int SCALES = ROWS>
hipError_t go_tile(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + BI - 1) / BI;
  a.tiles_j = (a.nj + BJ - 1) / BJ;
  const long long tiles = (RAGGED ? (long long)a.E * a.tiles_j : a.rows / BJ + a.E + 1) * a.tiles_i;     // (each expert and the rest may have one that is not full)
  constexpr int bytes = WK * STAGES * ((BI + BJ) * 128 + (SCALES == ROWS ? 0 : WI * WJ * kScaleSlot));
  static_assert(bytes <= 160 * 1024, "a CU's LDS");
  auto kernel = product_tile_kernel<FP8, IC, JC, RAGGED, F32OUT, BI, BJ, WI, WJ, STAGES, WK, SCALES>;
  static std::atomic<unsigned long long> allowed{0};
  const hipError_t e = allow_lds((const void*)kernel, bytes, allowed);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(64 * WI * WJ * WK), bytes, st>>>(a);
  return hipGetLastError();
}

// A tile with a reduction.
struct TileWork {
  int expert, i0, j0, j_end, k0, k_end, steps;
};

constexpr int kTileStores = 32;
// The wave's 128 x 64 of a tile: scaled, rounded, stored through a buffer that ends with the tile's last row.  Always kTileStores stores (by hand: they are
// counted, see unit_barrier).
template <bool FP8, bool F32OUT>
__device__ __forceinline__ void store_big_tile(const ProductArgs& a, unsigned char* out, const TileWork& t, int wi, int wj, int lane, const floatx4 (&acc)[8][4]) {
  constexpr int OB = F32OUT ? 4 : 2;
  asm volatile("" : "+v"(lane));
  const unsigned pitch = (unsigned)a.out.pitch;
  const int rows = t.j_end - t.j0 < 256 ? t.j_end - t.j0 : 256;
  const unsigned long long first = (unsigned long long)(out + (long long)t.j0 * a.out.pitch + (long long)t.i0 * OB);
  const intx4 to = {(int)(unsigned)first, (int)(unsigned)(first >> 32), (int)((unsigned)(rows - 1) * pitch + (unsigned)(a.ni - t.i0) * OB), 0x00020000};
  // the scales of the wave's 64 rows and 128 columns, one and two a lane, all asked for before the first store
  unsigned byte = 127;
  float col[2] = {1.f, 1.f};
  if constexpr (FP8) {
    if (a.scale) byte = __builtin_amdgcn_raw_buffer_load_b8(product_rsrc(a.scale + t.j0, (unsigned)rows), wj + lane, 0, 0);
    if (a.wscale) {
      const product_rsrc_t ws = product_rsrc(a.wscale + (size_t)t.expert * a.ni, (unsigned)a.ni * 4);
#pragma unroll
      for (int h = 0; h < 2; ++h) col[h] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ws, (t.i0 + wi + 64 * h + lane) * 4, 0, 0));
    }
  }
  const float row = FP8 ? scale_value(byte) : 1.f;
  float up[4] = {1.f, 1.f, 1.f, 1.f};
  if constexpr (FP8)
#pragma unroll
    for (int j = 0; j < 4; ++j) up[j] = __shfl(row, 16 * j + (lane & 15));
  auto each = [&](auto relu, auto plain) {
    const intx4 buffer = to;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int oi = wi + 16 * i + (lane >> 4) * 4;
      float w[4] = {1.f, 1.f, 1.f, 1.f};
      if constexpr (FP8)
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = __shfl(col[i / 4], 16 * (i % 4) + (lane >> 4) * 4 + r);
      // (ni is a multiple of 4: a lane's four are stored or, beyond the buffer's 2^31 bytes, not)
      unsigned o = t.i0 + oi < a.ni ? (unsigned)(wj + (lane & 15)) * pitch + (unsigned)oi * OB : 0x80000000u;
#pragma unroll
      for (int j = 0; j < 4; ++j, o += 16 * pitch) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v[r] = acc[i][j][r];
          if constexpr (FP8 && decltype(plain)::value) v[r] = v[r] * w[r] * up[j];
          if constexpr (!decltype(plain)::value) v[r] = scaled(v[r], col_scale(w[r]), row_scale((unsigned)__shfl((int)byte, 16 * j + (lane & 15))));
          if constexpr (decltype(relu)::value) v[r] = v[r] < 0.f ? 0.f : v[r];              // (NaN passes)
        }
        // (s_nop: the registers of a store of more than 8 bytes may not be written by the very next instruction)
        if constexpr (F32OUT)
          asm volatile("buffer_store_dwordx4 %0, %1, %2, 0 offen\n\ts_nop 1" ::"v"(Elem<float>::narrow(v)), "v"(o), "s"(buffer) : "memory");
        else
          asm volatile("buffer_store_dwordx2 %0, %1, %2, 0 offen" ::"v"(uint2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}), "v"(o), "s"(buffer) : "memory");
      }
    }
  };
  auto store = [&](auto plain) {
    if (a.relu)
      each(std::true_type{}, plain);
    else
      each(std::false_type{}, plain);
  };
  if constexpr (FP8)
    if (!__all(plain_scale(col[0]) && plain_scale(col[1]))) return store(std::false_type{});
  store(std::true_type{});
}

// ---- few rows an expert: bound by reading the weights once ----
// A workgroup takes 16 columns and up to 16 NJ rows of an expert.  Its four waves share the reduction, each a quarter of it, and read their weights straight into
// registers (nothing is used twice), DEPTH steps of 128 bytes ahead; the quarters' sums are added in order through LDS.  One row, 4096 x 4096: 8.2 us in bf16
// (4.1 TB/s), 6.2 in 8 bits.
template <bool FP8, int NJ, int SCALES = ROWS>
__global__ __launch_bounds__(256) void product_few_kernel(ProductArgs a) {
  constexpr int BYTES = FP8 ? 1 : 2, DEPTH = NJ == 1 ? 8 : 4;
  constexpr unsigned NONE = 0xffffffffu;
  __shared__ floatx4 sums[3][NJ][64];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int ti = (int)(blockIdx.x % a.tiles_i), i0 = ti * 16;
  int expert, j0, j_end;
  if (!find_rows(a, 16 * NJ, (int)(blockIdx.x / a.tiles_i), expert, j0, j_end)) return;
  expert = __builtin_amdgcn_readfirstlane(expert);
  j0 = __builtin_amdgcn_readfirstlane(j0);
  j_end = __builtin_amdgcn_readfirstlane(j_end);
  floatx4 acc[NJ] = {};
  if (expert < a.E) {
    const unsigned kb = (unsigned)a.nk * BYTES;
    const int rows = j_end - j0 < 16 * NJ ? j_end - j0 : 16 * NJ, cols = a.ni - i0 < 16 ? a.ni - i0 : 16;
    const product_rsrc_t I = product_rsrc(a.I.data + (long long)expert * a.i_expert + (long long)i0 * a.I.pitch, (unsigned)(cols - 1) * (unsigned)a.I.pitch + kb);
    const product_rsrc_t J = product_rsrc(a.J.data + (long long)j0 * a.J.pitch, (unsigned)(rows - 1) * (unsigned)a.J.pitch + kb);
    const int steps = (int)((kb + 127) / 128), mine = (steps + 3) / 4;
    unsigned k = (unsigned)(wave * mine) * 128 + (lane >> 4) * 32;            // this lane's 32 bytes of a step
    const unsigned k_end = (unsigned)(wave + 1) * mine * 128 < kb ? (unsigned)(wave + 1) * mine * 128 : kb;
    // (rows and columns beyond the last lie beyond the buffers: zeros)
    const unsigned at_i = (unsigned)(lane & 15) * (unsigned)a.I.pitch, at_j = (unsigned)(lane & 15) * (unsigned)a.J.pitch;
    Fragment fi[DEPTH], fj[DEPTH][NJ];
    unsigned sx[DEPTH][NJ], sw[DEPTH];                        // scales of blocks (of the steps beyond this wave's: 0, for products of nothing)
    const product_rsrc_t X = product_rsrc(a.xblocks + (long long)j0 * a.kb, SCALES == ROWS ? 0u : (unsigned)(rows * a.kb));
    const int WB = SCALES == FLOATS ? 4 : 1;
    const product_rsrc_t S = product_rsrc((const unsigned char*)a.wblocks + ((long long)expert * ((a.ni + 127) >> 7) + (i0 >> 7)) * a.kb * WB, SCALES == ROWS ? 0u : (unsigned)(a.kb * WB));
    auto fetch = [&](int d) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool there = k + h * 16 < k_end;
        fi[d].h[h] = __builtin_bit_cast(uint4_t, __builtin_amdgcn_raw_buffer_load_b128(I, (int)(there ? at_i + k + h * 16 : NONE), 0, 0));
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          fj[d][j].h[h] = __builtin_bit_cast(uint4_t, __builtin_amdgcn_raw_buffer_load_b128(
                                                          J, (int)(there ? at_j + (unsigned)(16 * j) * (unsigned)a.J.pitch + k + h * 16 : NONE), 0, 0));
      }
      if constexpr (SCALES != ROWS) {
        const unsigned step = k >> 7;
        const bool there = step * 128 < k_end;
        sw[d] = SCALES == FLOATS ? __builtin_amdgcn_raw_buffer_load_b32(S, (int)(there ? step * 4 : NONE), 0, 0) : __builtin_amdgcn_raw_buffer_load_b8(S, (int)(there ? step : NONE), 0, 0);
#pragma unroll
        for (int j = 0; j < NJ; ++j) sx[d][j] = __builtin_amdgcn_raw_buffer_load_b8(X, (int)(there ? (unsigned)((lane & 15) + 16 * j) * a.kb + step : NONE), 0, 0);
      }
      k += 128;
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(d);
    for (int s = 0; s < mine; s += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          if constexpr (SCALES == FLOATS)
            acc[j] = add_scaled(acc[j], scaled_mfma<SCALES>(fi[d].all, fj[d][j].all, acc[j], scale_power(sw[d]), sx[d][j]), scale_mantissa(sw[d]));
          else if constexpr (FP8)
            acc[j] = scaled_mfma<SCALES>(fi[d].all, fj[d][j].all, acc[j], sw[d], sx[d][j]);
          else
#pragma unroll
            for (int h = 0; h < 2; ++h)
              acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fi[d].h[h]), __builtin_bit_cast(bf16x8, fj[d][j].h[h]), acc[j], 0, 0, 0);
        fetch(d);
      }
  }
  if (wave)
#pragma unroll
    for (int j = 0; j < NJ; ++j) sums[wave - 1][j][lane] = acc[j];
  __syncthreads();
  if (wave) return;
  floatx4 whole[1][NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) whole[0][j] = ((acc[j] + sums[0][j][lane]) + sums[1][j][lane]) + sums[2][j][lane];
  store_tile<FP8 && SCALES == ROWS, false>(a, a.out.data, expert, i0, j0, j_end, whole);
}

template <bool FP8, int NJ, int SCALES = ROWS>
hipError_t go_few(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + 15) / 16;
  const long long groups = a.rows / (16 * NJ) + (a.rows < a.E ? a.rows : a.E) + 1;       // (experts with rows, one that is not full each, and the rest)
  product_few_kernel<FP8, NJ, SCALES><<<dim3((unsigned)(groups * a.tiles_i)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

// Whole pieces, and what the loads address with 32 bits.
template <bool IC, bool JC>
bool whole(const ProductArgs& a, int bytes, int B) {
  const unsigned long long low = (unsigned long long)a.I.data | (unsigned long long)a.J.data | (unsigned long long)a.I.pitch |
                                 (unsigned long long)a.J.pitch | (unsigned long long)a.i_expert;
  if (low & 15) return false;
  if ((!IC || !JC) && (long long)a.nk * bytes % 16) return false;
  if (IC && (long long)a.ni * bytes % 16) return false;
  if (JC && (long long)a.nj * bytes % 16) return false;
  return a.I.pitch < (1ll << 31) / B && a.J.pitch < (1ll << 31) / B;
}

}  // namespace
}  // namespace lasnet
