// The experts' products and their gradients on the matrix cores.
//
//   forward   out[p][i] = sum_c x[p][c] W[e][i][c]          rows p of expert e
//   dx        dx[p][c]  = sum_i dy[p][i] W[e][i][c]
//   dW        dW[e][i][c] = sum_p dy[p][i] x[p][c]          over the rows of expert e
//
// All three are D[j][i] = sum_k J[j][k] I[i][k] with i along the output's rows in memory: D comes out of the MFMA with four
// consecutive i in a lane.  An operand is held by ROWS (k is contiguous in memory: x, dy, and W in the forward product) or by COLUMNS (i or j
// is: W for dx, both for dW).  In LDS a tile by rows lies as it is read, 128 bytes of k a row; one by columns lies as it is in memory, and
// the transposing LDS read (ds_read_b64_tr_b16: 4 k x 16 columns for 16 lanes) turns it.
//
// Four kinds of kernel, from what bounds them: many tiles, the matrix cores (product_stream_kernel); fewer, the latency of a step and the loads to LDS, 64 bytes a clock
// for a CU (product_tile_kernel; dW from many rows in parts); few rows, the weights' bytes (product_few_kernel); rows of any alignment through registers
// (product_kernel).  go() says when which one runs.  Sums are held in 32 bits and rounded once, where they are stored.
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
};

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

// Any alignment and width: 128 x 128 of the output by 4 waves, 64 x 64 each; rows and weights through registers into two LDS stages, the next step's loads in
// flight while this one's products run.  Bound by those loads: pieces that begin anywhere touch two lines of the caches.  16384 rows of 8 experts, 2047 x 2049:
// bf16 224 us, its gradients 256 and 266, 8 bits 141; a branch for each piece's end instead of row_piece: 222, 322, 421, 160, and with few columns up to five
// times as long (28473 rows, 2103 x 226, gradient of the weights 199 and 1010).
// FP8: e4m3, else bf16.  IC, JC: held by columns.  RAGGED: the reduction runs over an expert's rows (dW).  WIDE: see row_piece.
template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, bool WIDE>
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
  auto fetch = [&](int k) {
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
  const int wi = (wave & 1) * 64, wj = (wave >> 1) * 64;
  int s = 0;
  if (k0 < k_end) {
    fetch(k0);
    stage(0, k0);
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
        for (int i = 0; i < 4; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fi[i], f.v, acc[i][j], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
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
    if (k + KS < k_end) stage(s ^ 1, k + KS);
    __syncthreads();
  }

  unsigned char* out = a.out.data + (RAGGED ? (long long)expert * a.out_expert : 0);
  store_tile<FP8, F32OUT>(a, out, expert, i0 + wi, j0 + wj, j_end, acc);
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
template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1>
__device__ __forceinline__ void tile_product(const ProductArgs& a, unsigned char* product_lds, int expert, int i0, int j0, int j_end, int k0, int k_end) {
  constexpr int BYTES = FP8 ? 1 : 2, KS = 128 / BYTES, NI = BI / WI / 16, NJ = BJ / WJ / 16;
  using SI = Stage<IC, BI, WI * WJ>;
  using SJ = Stage<JC, BJ, WI * WJ>;
  constexpr int STAGE = SI::BYTES + SJ::BYTES, LOADS = SI::SEGS + SJ::SEGS;
  static_assert(NI % 4 == 0, "a ring of four fragments");
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
  for (int s = 0; s < SI::SEGS; ++s) off_i[s] = (unsigned)SI::row(wave * SI::SEGS + s, lane) * pitch_i + (unsigned)SI::byte(wave * SI::SEGS + s, lane);
#pragma unroll
  for (int s = 0; s < SJ::SEGS; ++s) off_j[s] = (unsigned)SJ::row(wave * SJ::SEGS + s, lane) * pitch_j + (unsigned)SJ::byte(wave * SJ::SEGS + s, lane);
  int l_k = k_end - k0;                                       // what is left of k to load
  unsigned l_to = lds;
  // A step's loads, between the parts of `meanwhile` (which does what is due anyway, in LOADS parts).
  const unsigned to_i = wave * SI::SEGS * 1024, to_j = SI::BYTES + wave * SJ::SEGS * 1024;
  auto load = [&](auto meanwhile) {
    meanwhile(0);
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
  const int wi = wave % WI * (BI / WI), wj = wave / WI * (BJ / WJ);
  const unsigned bi = SI::lane_base(wi, lane), bj = SJ::lane_base(wj, lane) + SI::BYTES;
  unsigned at = lds, at_i = bi + at;                          // at: the stage that is read
  auto read_i = [&](int i) { SI::fragment(at_i, i, fi[i % 4]); };
  auto read_j = [&](auto stage) {
    const unsigned at_j = bj + at;
#pragma unroll
    for (int j = 0; j < NJ; ++j) SJ::fragment(at_j, j, fj[stage.value][j]);
  };
  constexpr int MFMAS = (FP8 ? 1 : 2) * NJ;                   // of a block
  auto multiply = [&](auto stage, int i, int m0, int m1) {
    constexpr int S = decltype(stage)::value;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = m0; m < m1; ++m) {
      const int j = m % NJ, h = m / NJ;
      if constexpr (FP8)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fi[i % 4].all, fj[S][j].all, acc[i][j], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
      else
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fi[i % 4].h[h]), __builtin_bit_cast(bf16x8, fj[S][j].h[h]), acc[i][j], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](auto stage) {
    constexpr int S = decltype(stage)::value;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (i + 3 < NI) read_i(i + 3);
      if (i == NI - 2) {
        counted_barrier<(STAGES - 2) * LOADS>();
        at = at == lds + (STAGES - 1) * STAGE ? lds : at + STAGE;
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
    counted_barrier<(STAGES - 2) * LOADS>();
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
  store_tile<FP8, F32OUT>(a, out, expert, i0 + wi, j0 + wj, j_end, acc);
}

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1>
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
  tile_product<FP8, IC, JC, RAGGED, F32OUT, BI, BJ, WI, WJ, STAGES, WK>(a, product_lds, expert, ti * BI, j0, j_end, k0, k_end);
}

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1>
hipError_t go_tile(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + BI - 1) / BI;
  a.tiles_j = (a.nj + BJ - 1) / BJ;
  const long long tiles = (RAGGED ? (long long)a.E * a.tiles_j : a.rows / BJ + a.E + 1) * a.tiles_i;     // (each expert and the rest may have one that is not full)
  constexpr int bytes = WK * STAGES * (BI + BJ) * 128;
  auto kernel = product_tile_kernel<FP8, IC, JC, RAGGED, F32OUT, BI, BJ, WI, WJ, STAGES, WK>;
  static std::atomic<unsigned long long> allowed{0};
  const hipError_t e = allow_lds((const void*)kernel, bytes, allowed);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(64 * WI * WJ * WK), bytes, st>>>(a);
  return hipGetLastError();
}

// ---- many tiles: 256 x 256 by eight waves, one workgroup a CU that goes from tile to tile without letting its loads run dry ----
// 8192 x 8192 x 8192 bf16 810 us, 1360 TFLOP/s (the library's product 745 to 757 us), 8 bits 412 us, 2660 TFLOP/s.  Reductions of 2048 leave the end of a
// tile more to say, some 9 to 11 us of each round of tiles beside the loop's rate (16384 x 2048 x 2048 128 to 137 us, 1000 to 1070 TFLOP/s; 32768 x 4096 x 2048 in 8 bits
// 295 to 302 us, 1830 TFLOP/s): 128 KiB of stores a CU, 8 bytes a lane in bf16, 32 of a row's bytes at a time.  That all CUs store at once is not what it
// costs: with every second workgroup at another place of its tile it was the same.
//
// LDS holds five units of 32 KiB, each the 128 bytes of k of one operand's tile, loaded in the order J0 I0 J1 I1 ... of the workgroup's steps, whatever
// tile they belong to.  In step s a wave multiplies the I fragments of its eight blocks, a ring of four read three blocks ahead, with the four J fragments it
// holds, and reads the J fragments of step s + 1 (behind Y, the last of them in block 7).  Two barriers a step, each of which waits for one unit, frees one and is followed
// by the loads of one into it:
//   Y, before block 1: J of s + 1 has landed, J of s has been read by all -> I of s + 2 where J of s was
//   X, before block 5: I of s + 1 has landed, I of s has been read by all -> J of s + 3 where I of s was (J of s + 1 is still being read, up to Y of s + 1)
// so each load has a step and a half (some 2 us) to arrive.  Behind a barrier MFMAs come first, loads and reads between them: all eight waves are at the
// same place there, and whatever came before the MFMAs would leave the matrix cores idle.
// The loop over a tile's steps has no branch but that at a tile's end.
constexpr int kUnit = 32768, kUnits = 5;

// The barriers X and Y: all but the youngest 8 loads of the wave, two units', have landed.  stored: a tile's stores are younger than what is waited for, too.
constexpr int kTileStores = 32;
__device__ __forceinline__ void unit_barrier(bool stored) {
  if (stored)
    counted_barrier<8 + kTileStores>();
  else
    counted_barrier<8>();
}

// A tile with a reduction.
struct TileWork {
  int expert, i0, j0, j_end, k0, k_end, steps;
};

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

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT>
__global__ __launch_bounds__(512, 2) void product_stream_kernel(ProductArgs a) {
  constexpr int BYTES = FP8 ? 1 : 2, KS = 128 / BYTES, OB = F32OUT ? 4 : 2;
  constexpr int PAIR = FP8 ? 1 : 2;                           // steps of the loop's body: bf16 holds the J fragments of two steps, which change places
  using SI = Stage<IC, 256, 8>;
  using SJ = Stage<JC, 256, 8>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char product_lds[];
  const unsigned lds = (unsigned)(size_t)(lds_byte*)product_lds;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wi = wave % 2 * 128, wj = wave / 2 * 64;

  // The experts' rows, one expert a lane (up to 63 of them; else they are looked up anew for each tile): first row, and tiles up to and with it (dW: the
  // number of experts with more rows).
  int lo = 0, upto = 0, tiles_j = a.tiles_j;
  const bool kept = a.E <= 63;
  if (kept) lo = bound(a, lane < a.E ? lane : a.E);
  const int hi = __shfl(lo, lane < 63 ? lane + 1 : 63);
  if constexpr (RAGGED) {
    if (kept)
      for (int e = 0; e < a.E; ++e) {
        const int n = __builtin_amdgcn_readlane(hi - lo, e);
        upto += n > hi - lo || (n == hi - lo && e < lane);
      }
    if (lane >= a.E) upto = 64;
  } else {
    if (kept) {
      upto = hi > lo ? (hi - lo + 255) / 256 : 0;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(upto, d);
        if (lane >= d) upto += u;
      }
      tiles_j = __builtin_amdgcn_readlane(upto, 63);
    } else {
      const int rest = (int)a.rows - __builtin_amdgcn_readfirstlane(bound(a, a.E));
      tiles_j = row_tiles<256>(a) - (rest + 255) / 256;
    }
    // the rows that no expert has
    const int width = a.ni * OB;
    for (long long r = bound(a, a.E) + (long long)blockIdx.x; r < a.rows; r += gridDim.x)
      for (int c = (int)threadIdx.x * 4 * OB; c < width; c += 512 * 4 * OB)
        if constexpr (F32OUT)
          *(uint4_t*)(a.out.data + r * a.out.pitch + c) = uint4_t{0, 0, 0, 0};
        else
          *(uint2_t*)(a.out.data + r * a.out.pitch + c) = uint2_t{0, 0};
  }
  // Workgroups are dealt to the eight XCDs in turn, each of which has an L2.  Products of rows: an XCD takes consecutive tiles.  dW: an XCD takes its eighth of
  // every expert's tiles (or, of few, every eighth tile), so that none is left with the longest reductions, and the experts with most rows come first.
  // Within the XCD its `stride` workgroups take a tile each in turn (dW: there and back, the longest with the shortest).
  const int xcd = (int)blockIdx.x & 7, slot = (int)blockIdx.x >> 3, stride = (int)gridDim.x >> 3;
  const int per = RAGGED ? a.tiles_i * a.tiles_j : 1;
  const bool eighths = RAGGED && per >= 64;
  const int per_first = eighths ? (int)((long long)per * xcd / 8) : 0, per_mine = eighths ? (int)((long long)per * (xcd + 1) / 8) - per_first : 1;
  const int total = RAGGED ? a.E * per : tiles_j * a.tiles_i;
  const int chunk = (total + 7) / 8;
  int end = RAGGED ? (eighths ? a.E * per_mine : (total - xcd + 7) / 8) : total - xcd * chunk < chunk ? total - xcd * chunk : chunk;      // this XCD's tiles
  // A last round that would leave half of the XCD idle or more is cut into quarters of tiles.
  const int rest = end > 0 && end % stride <= stride / 2 ? end % stride : 0;
  end -= rest;

  auto work = [&](int p) {                                    // the XCD's tile p
    TileWork w;
    int ti, tj;
    if constexpr (RAGGED) {
      int rank, u;
      if (eighths) {
        rank = p / per_mine;
        u = per_first + p - rank * per_mine;
      } else {
        rank = (p * 8 + xcd) / per;
        u = p * 8 + xcd - rank * per;
      }
      w.expert = kept ? __ffsll((long long)__ballot(upto == rank)) - 1 : rank;
      tile_at(u, a.tiles_i, a.tiles_j, ti, tj);
      w.j0 = tj * 256;
      w.j_end = a.nj;
      w.k0 = kept ? __builtin_amdgcn_readlane(lo, w.expert) : __builtin_amdgcn_readfirstlane(bound(a, w.expert));
      w.k_end = kept ? __builtin_amdgcn_readlane(hi, w.expert) : __builtin_amdgcn_readfirstlane(bound(a, w.expert + 1));
    } else {
      tile_at(xcd * chunk + p, a.tiles_i, tiles_j, ti, tj);
      if (kept) {
        const int l = __ffsll((long long)__ballot(tj < upto)) - 1;
        const int before = l ? __builtin_amdgcn_readlane(upto, l - 1) : 0;
        w.expert = l;
        w.j0 = __builtin_amdgcn_readlane(lo, l) + (tj - before) * 256;
        w.j_end = __builtin_amdgcn_readlane(lo, l + 1);
      } else {
        int e = 0, j0 = 0, j1 = 0;
        find_rows(a, 256, tj, e, j0, j1);
        w.expert = __builtin_amdgcn_readfirstlane(e);
        w.j0 = __builtin_amdgcn_readfirstlane(j0);
        w.j_end = __builtin_amdgcn_readfirstlane(j1);
      }
      w.k0 = 0;
      w.k_end = a.nk;
    }
    w.i0 = ti * 256;
    // four at least (so loads are never further ahead than the next tile), with zeros behind the end
    const int n = w.k_end > w.k0 ? (w.k_end - w.k0 + PAIR * KS - 1) / (PAIR * KS) * PAIR : 0;
    w.steps = n && n < 4 ? 4 : n;
    return w;
  };
  floatx4 acc[8][4];
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  };
  auto tile_of = [&](int round) { return round * stride + (RAGGED && (round & 1) ? stride - 1 - slot : slot); };
  // the tile of this round; dW: of the first round from this one on whose tile has a reduction (none left: round is past the end)
  auto next_work = [&](int& round) {
    TileWork w;
    w.steps = 0;
    for (; round * stride < end; ++round) {
      const int p = tile_of(round);
      if (p >= end) continue;
      w = work(p);
      if (!RAGGED || w.steps) break;
    }
    return w;
  };
  if constexpr (RAGGED) {                                      // dW of experts without rows: zeros, ahead of everything else
    clear();
    for (int round = 0; round * stride < end; ++round) {
      const int p = tile_of(round);
      if (p >= end) continue;
      const TileWork w = work(p);
      if (!w.steps) store_big_tile<FP8, F32OUT>(a, a.out.data + (long long)w.expert * a.out_expert, w, wi, wj, lane, acc);
    }
  }

  // ---- loads ----
  const unsigned pitch_i = (unsigned)a.I.pitch, pitch_j = (unsigned)a.J.pitch, kb = (unsigned)a.nk * BYTES;
  const unsigned di = IC ? KS * pitch_i : 128, dj = JC ? KS * pitch_j : 128;
  // Of this lane's first piece of a unit from the tile.  The next lies a segment's rows further with bit 6 of its byte turned over (both kinds of tile: the
  // bit is bit 2 of the lane), the other two likewise two segments further.
  unsigned off_i = (unsigned)SI::row(wave * 4, lane) * pitch_i + (unsigned)SI::byte(wave * 4, lane);
  unsigned off_j = (unsigned)SJ::row(wave * 4, lane) * pitch_j + (unsigned)SJ::byte(wave * 4, lane);
  auto feed_i = [&](const TileWork& w) {
    Feed<IC> v;
    v.start(a.I.data + (RAGGED ? 0 : (long long)w.expert * a.i_expert) + (IC ? (long long)w.k0 * a.I.pitch + (long long)w.i0 * BYTES : (long long)w.i0 * a.I.pitch),
            a.ni - w.i0, 256, a.I.pitch, IC ? (unsigned)(a.ni - w.i0) * BYTES : kb);
    return v;
  };
  auto feed_j = [&](const TileWork& w) {
    Feed<JC> v;
    v.start(a.J.data + (JC ? (long long)w.k0 * a.J.pitch + (long long)w.j0 * BYTES : (long long)w.j0 * a.J.pitch), w.j_end - w.j0, 256, a.J.pitch,
            JC ? (unsigned)(w.j_end - w.j0) * BYTES : kb);
    return v;
  };
  Feed<IC> li, ni;                                            // of the tile being loaded, and of the one after the tile being computed
  Feed<JC> lj, nj;
  int l_k = 0, l_steps = 0, n_k = 0, n_steps = 0;             // its k and steps left (past the last tile: no k)
  unsigned l_to = lds;
  const unsigned mine = lds + (kUnits - 1) * kUnit;           // the last unit
  auto turn_slot = [&](unsigned& s) { s = s == mine ? lds : s + kUnit; };
  auto nothing = [](int) {};
  // A unit of the load step, between the parts of `meanwhile` (which does what is due anyway, in four parts).
  auto issue = [&](auto j, auto meanwhile) {
    constexpr bool J = decltype(j)::value, C = J ? JC : IC;
    meanwhile(0);
    intx4 rsrc;
    if constexpr (J) rsrc = lj.rsrc(l_k, pitch_j);
    else rsrc = li.rsrc(l_k, pitch_i);
    unsigned o[4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
      o[s] = (J ? off_j : off_i) + (s & 1 ? 64u - ((unsigned)lane & 4) * 32 : 0u) + (unsigned)(s * (C ? 2 : 8)) * (J ? pitch_j : pitch_i);
    if (!FP8 && !C && l_k < KS) {                             // by rows, what is beyond the end of k lies inside the buffer (e4m3: whole steps only, registers lack for more)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if ((J ? SJ::byte(wave * 4 + s, lane) : SI::byte(wave * 4 + s, lane)) >= l_k * BYTES) o[s] = 0xffffffffu;
    }
    const unsigned to = l_to + wave * 4096;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s) meanwhile(s);
      __builtin_amdgcn_sched_barrier(0);
      buffer_to_lds(rsrc, o[s], to + s * 1024);
      __builtin_amdgcn_sched_barrier(0);
    }
    turn_slot(l_to);
    if constexpr (J) {
      lj.move(dj);
    } else {
      li.move(di);
      l_k -= KS;
      if (--l_steps == 0) {
        li = ni;
        lj = nj;
        l_k = n_k;
        l_steps = n_steps;
      }
    }
  };

  // ---- products ----
  // The next step's J fragments 2 and 3 take the place of this step's as the last block is done with them (every block begins with these two); 0 and 1
  // are held twice in bf16, and follow 2 and 3 in e4m3, whose fragments are whole octets of registers and leave no room for that.
  Fragment fi[4], fj[PAIR][2], fj2[2];
  const unsigned bi = SI::lane_base(wi, lane), bj = SJ::lane_base(wj, lane);
  unsigned c_j = lds, c_i = lds + kUnit;                      // the units that J and I fragments are read from
  unsigned at_i = bi + c_i;
  auto next_unit = [&](unsigned& c) { c = c >= mine - kUnit ? c - 3 * kUnit : c + 2 * kUnit; };
  auto read_i = [&](int i) { SI::fragment(at_i, i, fi[i % 4]); };
  auto read_j = [&](auto stage, int j) { SJ::fragment(bj + c_j, j, j < 2 ? fj[stage.value][j] : fj2[j - 2]); };
  auto multiply = [&](auto stage, int i, int part) {          // a quarter of block i's MFMAs
    constexpr int S = decltype(stage)::value;
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (FP8) {
      const int j = part ^ 2;
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fi[i % 4].all, (j < 2 ? fj[S][j] : fj2[j - 2]).all, acc[i][j], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
    } else {
      const int j0 = part < 2 ? 2 : 0, h = part & 1;
#pragma unroll
      for (int j = j0; j < j0 + 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fi[i % 4].h[h]),
                                                            __builtin_bit_cast(bf16x8, (j < 2 ? fj[S][j] : fj2[j - 2]).h[h]), acc[i][j], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  int young = 0;                                              // steps (Y to Y) for which the units waited for are older than the last tile's stores
  auto step = [&](auto stage) {
    constexpr int S = decltype(stage)::value;
    constexpr auto next = std::integral_constant<int, (S + 1) % PAIR>{};
    asm volatile("" : "+v"(off_i), "+v"(off_j));               // (what follows from them is made where it is used, not kept in registers throughout)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i == 1) {                                           // Y
        unit_barrier(young > 0);
        next_unit(c_j);
        issue(std::false_type{}, [&](int p) {
          multiply(stage, 1, p);
          if (p == 0) read_i(4);
          if (!FP8 && p == 1) read_j(next, 0);
        });
        --young;
      } else if (i == 5) {                                    // X
        unit_barrier(young > 0);
        next_unit(c_i);
        at_i = bi + c_i;
        asm volatile("" : "+v"(at_i));                         // (a sum in a register: reads add constants to it)
        issue(std::true_type{}, [&](int p) {
          multiply(stage, 5, p);
          if (p == 0) read_i(0);
        });
      } else {
        read_i((i + 3) % 8);
        if (!FP8 && i == 2) read_j(next, 1);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          multiply(stage, i, p);
          if (i == 7 && FP8) read_j(next, p ^ 2);
          if (i == 7 && !FP8 && p == 1) {
            read_j(next, 2);
            read_j(next, 3);
          }
        }
      }
    }
  };

  int round = 0;
  TileWork w = next_work(round);
  if (round * stride < end) {
    li = feed_i(w);
    lj = feed_j(w);
    l_k = w.k_end - w.k0;
    l_steps = w.steps;
    ni = li;
    nj = lj;
    issue(std::true_type{}, nothing);
    issue(std::false_type{}, nothing);
    issue(std::true_type{}, nothing);
    issue(std::false_type{}, nothing);
    unit_barrier(false);
    issue(std::true_type{}, nothing);
#pragma unroll
    for (int j = 0; j < 4; ++j) read_j(std::integral_constant<int, 0>{}, j);
#pragma unroll
    for (int i = 0; i < 3; ++i) read_i(i);
    while (true) {
      ++round;
      const TileWork after = next_work(round);
      const bool more = round * stride < end;
      if (more) {
        ni = feed_i(after);
        nj = feed_j(after);
        n_k = after.k_end - after.k0;
        n_steps = after.steps;
      } else {
        n_k = 0;
        n_steps = 0;
      }
      clear();
      for (int s = 0; s < w.steps; s += PAIR) {
        step(std::integral_constant<int, 0>{});
        if constexpr (PAIR == 2) step(std::integral_constant<int, 1>{});
      }
      store_big_tile<FP8, F32OUT>(a, a.out.data + (RAGGED ? (long long)w.expert * a.out_expert : 0), w, wi, wj, lane, acc);
      if (!more) break;
      young = 2;
      w = after;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (the last loads write to this workgroup's LDS)
  }
  for (int q = slot; q < 4 * rest; q += stride) {
    const TileWork v = work(end + q / 4);
    const int i0 = v.i0 + (q & 1) * 128, j0 = v.j0 + (q >> 1 & 1) * 128;
    if (i0 >= a.ni || j0 >= v.j_end) continue;
    __syncthreads();
    tile_product<FP8, IC, JC, RAGGED, F32OUT, 128, 128, 2, 4, 4>(a, product_lds, v.expert, i0, j0, v.j_end, v.k0, v.k_end);
  }
}

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT>
hipError_t go_stream(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + 255) / 256;
  a.tiles_j = (a.nj + 255) / 256;
  auto kernel = product_stream_kernel<FP8, IC, JC, RAGGED, F32OUT>;
  static std::atomic<unsigned long long> allowed{0};
  const hipError_t e = allow_lds((const void*)kernel, kUnits * kUnit, allowed);
  if (e != hipSuccess) return e;
  kernel<<<dim3(256), dim3(512), kUnits * kUnit, st>>>(a);
  return hipGetLastError();
}

// ---- dW of few tiles from many rows: parts of the rows, joined in order ----
// An expert's rows are cut into parts of part_rows (the last may have fewer), so that all parts' tiles fill the chip once whatever the experts' shares; each part's product
// is stored in 32 bits, and the second kernel sums an expert's parts in order.  Bound by the rows' bytes and the loads to LDS, then by the parts' 16 MB: one expert,
// 1024 x 256 from 32768 rows 32 us, 512 x 512 from 16384 rows 22 (groups of waves in one workgroup a tile: 95 and 48).
template <int BI, int BJ, int WI, int WJ, int STAGES, int WK>
__global__ __launch_bounds__(64 * WI * WJ * WK, 2) void product_part_kernel(ProductArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char product_lds[];
  const int per = a.tiles_i * a.tiles_j, t = xcd_tile(a.parts * per);
  if (t < 0) return;
  const int part = t / per;
  int expert, k0, k_end, ti, tj;
  if (!find_rows(a, a.part_rows, part, expert, k0, k_end)) return;
  if (__builtin_amdgcn_readfirstlane(expert) == a.E) return;
  k0 = __builtin_amdgcn_readfirstlane(k0);
  k_end = __builtin_amdgcn_readfirstlane(k_end);
  tile_at(t - part * per, a.tiles_i, a.tiles_j, ti, tj);
  tile_product<false, true, true, true, true, BI, BJ, WI, WJ, STAGES, WK>(a, product_lds, part, ti * BI, tj * BJ, a.nj, k0, k0 + a.part_rows < k_end ? k0 + a.part_rows : k_end);
}
// a.I: the parts; four elements a thread.
template <bool F32OUT>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a) {
  const int lane = (int)threadIdx.x & 63, expert = (int)blockIdx.y;
  int before = 0, mine = 0;
  for (int e = lane; e <= expert; e += 64) {
    const int n = bound(a, e + 1) - bound(a, e), parts = n > 0 ? (n + a.part_rows - 1) / a.part_rows : 0;
    if (e < expert) before += parts;
    else mine = parts;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    before += __shfl_xor(before, d);
    mine += __shfl_xor(mine, d);
  }
  if (before > a.parts) before = a.parts;                      // (offsets that do not ascend)
  if (mine > a.parts - before) mine = a.parts - before;
  const long long size = (long long)a.ni * a.nj, at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= size) return;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const unsigned char* part = a.I.data + ((long long)before * size + at) * 4;
#pragma unroll 8
  for (int i = 0; i < mine; ++i) {
    float v[4];
    Elem<float>::widen(load16(part + (long long)i * size * 4), v);
#pragma unroll
    for (int r = 0; r < 4; ++r) sum[r] += v[r];
  }
  unsigned char* out = a.out.data + (expert * size + at) * (F32OUT ? 4 : 2);
  if constexpr (F32OUT)
    store16(out, Elem<float>::narrow(sum));
  else
    *(uint2_any*)out = uint2_t{bf16_pair(sum[0], sum[1]), bf16_pair(sum[2], sum[3])};
}

// Whether and how dW is made in parts: parts == 0, not.
struct Parts {
  int rows;
  long long parts;
  bool narrow;                     // tiles of 64 x 64
};
// 6144 rows an expert: with 4096 (208 x 944) one workgroup a tile takes 17 us, two launches and the parts' way through memory are no less than 10.
Parts parts_for(long long rows, int E, int n, int k) {
  const bool narrow = n <= 64 || k <= 64;
  const int B = narrow ? 64 : 128;
  const long long per = (long long)((n + B - 1) / B) * ((k + B - 1) / B);
  if (n % 8 || k % 8 || rows / E < 6144 || E * per > 128) return Parts{0, 0, false};
  const long long want = 256 / per - E;                       // (2 E or more less E: every expert may have one that is not full)
  const long long each = (rows + want - 1) / want, part = (each < 512 ? 512 : each + 63) / 64 * 64;
  return Parts{(int)part, rows / part + E, narrow};
}

template <int BI, int BJ, int WI, int WJ, int STAGES, int WK>
hipError_t go_parts(ProductArgs a, const Parts& p, bool f32, void* workspace, hipStream_t st) {
  a.part_rows = p.rows;
  a.parts = (int)p.parts;
  a.tiles_i = (a.ni + BI - 1) / BI;
  a.tiles_j = (a.nj + BJ - 1) / BJ;
  ProductArgs b = a;
  b.out = RowsArg{(unsigned char*)workspace, (long long)a.ni * 4};
  b.out_expert = (long long)a.ni * a.nj * 4;
  constexpr int bytes = WK * STAGES * (BI + BJ) * 128;
  auto kernel = product_part_kernel<BI, BJ, WI, WJ, STAGES, WK>;
  static std::atomic<unsigned long long> allowed{0};
  hipError_t e = allow_lds((const void*)kernel, bytes, allowed);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)((p.parts * a.tiles_i * a.tiles_j + 7) / 8 * 8)), dim3(64 * WI * WJ * WK), bytes, st>>>(b);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.I = b.out;
  auto join = f32 ? product_join_kernel<true> : product_join_kernel<false>;
  join<<<dim3((unsigned)(((long long)a.ni * a.nj + 1023) / 1024), (unsigned)a.E), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

// ---- few rows an expert: bound by reading the weights once ----
// A workgroup takes 16 columns and up to 16 NJ rows of an expert.  Its four waves share the reduction, each a quarter of it, and read their weights straight into
// registers (nothing is used twice), DEPTH steps of 128 bytes ahead; the quarters' sums are added in order through LDS.  One row, 4096 x 4096: 8.2 us in bf16
// (4.1 TB/s), 6.2 in 8 bits.
template <bool FP8, int NJ>
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
      k += 128;
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(d);
    for (int s = 0; s < mine; s += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          if constexpr (FP8)
            acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fi[d].all, fj[d][j].all, acc[j], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
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
  store_tile<FP8, false>(a, a.out.data, expert, i0, j0, j_end, whole);
}

template <bool FP8, int NJ>
hipError_t go_few(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + 15) / 16;
  const long long groups = a.rows / (16 * NJ) + (a.rows < a.E ? a.rows : a.E) + 1;       // (experts with rows, one that is not full each, and the rest)
  product_few_kernel<FP8, NJ><<<dim3((unsigned)(groups * a.tiles_i)), dim3(256), 0, st>>>(a);
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

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT>
hipError_t go(ProductArgs a, hipStream_t st) {
  if (whole<IC, JC>(a, FP8 ? 1 : 2, 256)) {
    // Few rows, and not much more than one workgroup a CU: rows go straight to registers.  1 row, 1024 x 2048 5.7 us (tiles 7.8), 4096 x 4096 8.2 (11.2); 16 rows of
    // 4 experts, 1024 x 2048 6.4 (7.8).  768 workgroups (24 rows of 2 experts, 4096 x 4096) 19.2 (14.1); in bf16 with more than 16 rows an expert and a
    // longer reduction: 32 rows, 1024 x 2048 8.7 (7.9; 8 bits 6.2 and 6.7).
    if constexpr (!IC && !RAGGED) {
      const long long blocks = a.E < a.rows ? a.E : a.rows, units = (blocks > (a.rows + 15) / 16 ? blocks : (a.rows + 15) / 16) * ((a.ni + 15) / 16);
      if (a.rows <= 64 && units <= 384 && (FP8 || a.rows / a.E <= 16 || a.nk <= 1024))
        return a.rows <= 16 || a.rows / a.E <= 8 ? go_few<FP8, 1>(a, st) : go_few<FP8, 2>(a, st);
    }
    // Tiles of BI x BJ, about (how the rows are spread is not known here).
    const long long groups = a.E < a.rows ? a.E : a.rows;
    auto tiles = [&](int BI, int BJ) {
      const long long mean = a.rows / BJ + groups / 2, rows = mean > groups ? mean : groups;
      return (RAGGED ? (long long)a.E * ((a.nj + BJ - 1) / BJ) : rows) * ((a.ni + BI - 1) / BI);
    };
    const bool long_enough = RAGGED || (FP8 ? a.nk >= 256 && a.nk % 128 == 0 : a.nk >= 128);
    // Tiles of 256 x 256 where there are enough for the chip: 16384 rows of 4 experts, 2048 x 2048 bf16 128 us (128 x 128: 152), 8 bits 77 (99), dW of 8 experts 134
    // (223).  With 136 of them, 8192 rows of 4 experts, 1024 x 2048, evenly spread, 38 (34), unevenly 57 (60).  dW has few of them with long reductions: 128
    // tiles of 4096 rows 87 (125), of 2048 rows 45 (38).  Short reductions: 32768 x 2048 x 128 in bf16 66 (69), x 256 in 8 bits 70 (74); less does not
    // fill the steps that a tile has at least.
    if ((RAGGED ? tiles(256, 256) >= (a.rows / a.E >= 4096 ? 128 : 256) : (a.rows / 256 + groups / 2) * ((a.ni + 255) / 256) >= 200) && long_enough && a.ni % 4 == 0 &&
        !(((unsigned long long)a.out.data | (unsigned long long)a.out.pitch | (unsigned long long)a.out_expert) & 15) && a.out.pitch < (1ll << 31) / 256)
      return go_stream<FP8, IC, JC, RAGGED, F32OUT>(a, st);
    const long long steps = (RAGGED ? a.rows / a.E : a.nk) / (FP8 ? 128 : 64);
    // Tiles that all run at once, one workgroup a CU, with the reduction shared by groups of waves: a step of one wave a SIMD is 0.2 to 0.3 us of latency, whatever
    // the depth of the loads ahead.  64 x 32 by four groups: 64 rows, 1024 x 4096 11.2 us (128 x 64 by one group 23.3), 4096 x 1024 6.4 (9.1), 9 steps (300 rows
    // of 8 experts, 1024 x 520) 7.2 (6.9).  64 x 64 by two: 1024 x 1024 x 1024 8.0 (9.3), 2048 x 512 x 2048 10.5 (14.0), 4 steps 6.2 (5.8).
    // Shorter or more of them: 128 x 64 in three stages, two workgroups a CU; 1024 rows of 16 experts, 1024 x 2048 16.2 (128 x 128 in four stages 21.2, in two
    // 28.3), 8000 rows of 4, 512 x 2048 24.9 (39.7, 35.8).  128 x 128 by eight waves where one round does: 2048 rows of 16, 1024 x 2048 22.0 (25.5, 29.3).
    // Beyond, 128 x 128 by four waves, two workgroups a CU: dW of 3000 rows, 8 experts 1024 x 1024 18.7 (128 x 64 22.7).
    if (steps >= 12 && tiles(64, 32) <= 256) return go_tile<FP8, IC, JC, RAGGED, F32OUT, 64, 32, 1, 2, 3, 4>(a, st);
    if (steps >= 6 && tiles(64, 64) <= 256) return go_tile<FP8, IC, JC, RAGGED, F32OUT, 64, 64, 1, 4, 4, 2>(a, st);
    if (tiles(128, 64) <= 256) return go_tile<FP8, IC, JC, RAGGED, F32OUT, 128, 64, 2, 2, 3>(a, st);
    if (tiles(128, 128) <= 240) return go_tile<FP8, IC, JC, RAGGED, F32OUT, 128, 128, 2, 4, 4>(a, st);
    if (tiles(128, 64) <= 512) return go_tile<FP8, IC, JC, RAGGED, F32OUT, 128, 64, 2, 2, 3>(a, st);
    return go_tile<FP8, IC, JC, RAGGED, F32OUT, 128, 128, 2, 2, 2>(a, st);
  }
  a.tiles_i = (a.ni + 127) / 128;
  a.tiles_j = (a.nj + 127) / 128;
  const long long tiles = RAGGED ? (long long)a.E * a.tiles_j : a.rows / 128 + a.E + 1;     // (each expert and the rest may have one tile that is not full)
  const bool wide = (IC ? a.ni : a.nk) >= (FP8 ? 16 : 8) && (JC ? a.nj : a.nk) >= (FP8 ? 16 : 8);
  auto kernel = wide ? product_kernel<FP8, IC, JC, RAGGED, F32OUT, true> : product_kernel<FP8, IC, JC, RAGGED, F32OUT, false>;
  kernel<<<dim3((unsigned)(tiles * a.tiles_i)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_product(int dtype, long long rows, int E, int n, int k, RowsArg x, const uint8_t* scale, const int32_t* offsets,
                                 const void* W, const float* wscale, RowsArg out, bool relu, hipStream_t st) {
  const int b = dtype == LASNET_E4M3 ? 1 : 2;
  ProductArgs a{{(unsigned char*)W, (long long)k * b}, x, out, (long long)n * k * b, 0, offsets, scale, wscale, rows, E, n, 0, k, 0, 0, 0, 0, relu};
  return dtype == LASNET_E4M3 ? go<true, false, false, false, false>(a, st) : go<false, false, false, false, false>(a, st);
}

hipError_t launch_expert_product_dx(long long rows, int E, int n, int k, RowsArg dy, const int32_t* offsets, const void* W, RowsArg dx,
                                    hipStream_t st) {
  ProductArgs a{{(unsigned char*)W, (long long)k * 2}, dy, dx, (long long)n * k * 2, 0, offsets, nullptr, nullptr, rows, E, k, 0, n, 0, 0, 0, 0, false};
  return go<false, true, false, false, false>(a, st);
}

size_t product_dw_workspace_bytes(long long rows, int E, int n, int k) { return (size_t)parts_for(rows, E, n, k).parts * n * k * sizeof(float); }

hipError_t launch_expert_product_dw(long long rows, int E, int n, int k, RowsArg dy, RowsArg x, const int32_t* offsets, void* dW, bool f32,
                                    void* workspace, hipStream_t st) {
  const int b = f32 ? 4 : 2;
  ProductArgs a{x, dy, {(unsigned char*)dW, (long long)k * b}, 0, (long long)n * k * b, offsets, nullptr, nullptr, rows, E, k, n, 0, 0, 0, 0, 0, false};
  const Parts p = parts_for(rows, E, n, k);
  if (workspace && p.parts && whole<true, true>(a, 2, 256))
    return p.narrow ? go_parts<64, 64, 1, 4, 4, 2>(a, p, f32, workspace, st) : go_parts<128, 128, 2, 4, 4, 1>(a, p, f32, workspace, st);
  return f32 ? go<false, true, true, true, true>(a, st) : go<false, true, true, true, false>(a, st);
}

}  // namespace lasnet
