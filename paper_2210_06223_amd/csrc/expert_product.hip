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
  bool relu;
};

// offsets[e] as the kernels take it: within [0, rows].
__device__ __forceinline__ int bound(const ProductArgs& a, int e) {
  const int v = a.offsets[e];
  return v < 0 ? 0 : (long long)v < a.rows ? v : (int)a.rows;
}

// Row tile t of all experts' (BJ rows each, the last of an expert may have fewer) -> its expert, first row and end.  Expert E: the rows that no
// expert has.  false: no such tile.  Every wave of a workgroup finds the same.
template <int BJ>
__device__ __forceinline__ bool find_rows(const ProductArgs& a, int t, int& expert, int& first, int& end) {
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

// 2^(b - 127); 255: NaN
__device__ __forceinline__ float scale_value(unsigned b) {
  return __uint_as_float(b == 255 ? 0x7fc00000u : b ? b << 23 : 0x00400000u);
}

template <int BYTES>
__device__ __forceinline__ uint4_t load_some(const unsigned char* p, int n) {
  if constexpr (BYTES == 2) return load_piece<__bf16>(p, n);
  if (n >= 16) return load16(p);
  uint4_t v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < n) v[i / 4] |= (unsigned)p[i] << (8 * (i % 4));
  return v;
}

// 128 x 128 of the output by 4 waves, 64 x 64 each; rows and weights through registers into two LDS stages.
// FP8: e4m3, else bf16.  IC, JC: held by columns.  RAGGED: the reduction runs over an expert's rows (dW).
template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT>
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
    if (!find_rows<128>(a, (int)(blockIdx.x / a.tiles_i), expert, j0, j_end)) return;
    k0 = 0;
    k_end = expert < a.E ? a.nk : 0;                          // (no reduction: zeros)
  }
  const int i0 = ti * 128;
  const unsigned char* I = a.I.data + (RAGGED ? 0 : (long long)(expert < a.E ? expert : 0) * a.i_expert);

  floatx4 acc[4][4] = {};
  uint4_t ri[4], rj[4];
  auto fetch = [&](int k) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int q = u * 256 + tid;
      if constexpr (IC) {
        const int kk = k + Tile<true>::row(q), i = i0 + Tile<true>::byte(q) / BYTES;
        ri[u] = load_some<BYTES>(I + (long long)kk * a.I.pitch + (long long)i * BYTES, kk < k_end ? a.ni - i : 0);
      } else {
        const int i = i0 + Tile<false>::row(q), kk = k + Tile<false>::byte(q) / BYTES;
        ri[u] = load_some<BYTES>(I + (long long)i * a.I.pitch + (long long)kk * BYTES, i < a.ni ? k_end - kk : 0);
      }
      if constexpr (JC) {
        const int kk = k + Tile<true>::row(q), j = j0 + Tile<true>::byte(q) / BYTES;
        rj[u] = load_some<BYTES>(a.J.data + (long long)kk * a.J.pitch + (long long)j * BYTES, kk < k_end ? j_end - j : 0);
      } else {
        const int j = j0 + Tile<false>::row(q), kk = k + Tile<false>::byte(q) / BYTES;
        rj[u] = load_some<BYTES>(a.J.data + (long long)j * a.J.pitch + (long long)kk * BYTES, j < j_end ? k_end - kk : 0);
      }
    }
  };
  auto stage = [&](int s) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int q = u * 256 + tid;
      *(uint4_t*)(lds[s][0] + Tile<IC>::place(q)) = ri[u];
      *(uint4_t*)(lds[s][1] + Tile<JC>::place(q)) = rj[u];
    }
  };
  const int wi = (wave & 1) * 64, wj = (wave >> 1) * 64;
  int s = 0;
  if (k0 < k_end) {
    fetch(k0);
    stage(0);
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
    if (k + KS < k_end) stage(s ^ 1);
    __syncthreads();
  }

  unsigned char* out = a.out.data + (RAGGED ? (long long)expert * a.out_expert : 0);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int oj = j0 + wj + 16 * j + (lane & 15);
    if (oj >= j_end) continue;
    float up = 1.0f;
    if constexpr (FP8)
      if (a.scale && expert < a.E) up = scale_value(a.scale[oj]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int oi = i0 + wi + 16 * i + (lane >> 4) * 4;
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        v[r] = acc[i][j][r];
        if constexpr (FP8) {
          if (a.wscale && oi + r < a.ni && expert < a.E) v[r] *= a.wscale[(size_t)expert * a.ni + oi + r];
          v[r] *= up;
        }
        if (a.relu) v[r] = v[r] < 0.f ? 0.f : v[r];
      }
      unsigned char* o = out + (long long)oj * a.out.pitch + (long long)oi * (F32OUT ? 4 : 2);
      if constexpr (F32OUT) {
        store_piece<float>(o, a.ni - oi, Elem<float>::narrow(v));
      } else if (oi + 4 <= a.ni) {
        *(uint2_any*)o = uint2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (oi + r < a.ni) Elem<__bf16>::put(o + 2 * r, bf16_pair(v[r], 0.f));
      }
    }
  }
}

template <bool FP8, bool IC, bool JC, bool RAGGED, bool F32OUT>
hipError_t go(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + 127) / 128;
  a.tiles_j = (a.nj + 127) / 128;
  const long long tiles = RAGGED ? (long long)a.E * a.tiles_j : a.rows / 128 + a.E + 1;     // (each expert and the rest may have one tile that is not full)
  product_kernel<FP8, IC, JC, RAGGED, F32OUT><<<dim3((unsigned)(tiles * a.tiles_i)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_product(int dtype, long long rows, int E, int n, int k, RowsArg x, const uint8_t* scale, const int32_t* offsets,
                                 const void* W, const float* wscale, RowsArg out, bool relu, hipStream_t st) {
  const int b = dtype == LASNET_E4M3 ? 1 : 2;
  ProductArgs a{{(unsigned char*)W, (long long)k * b}, x, out, (long long)n * k * b, 0, offsets, scale, wscale, rows, E, n, 0, k, 0, 0, relu};
  return dtype == LASNET_E4M3 ? go<true, false, false, false, false>(a, st) : go<false, false, false, false, false>(a, st);
}

hipError_t launch_expert_product_dx(long long rows, int E, int n, int k, RowsArg dy, const int32_t* offsets, const void* W, RowsArg dx,
                                    hipStream_t st) {
  ProductArgs a{{(unsigned char*)W, (long long)k * 2}, dy, dx, (long long)n * k * 2, 0, offsets, nullptr, nullptr, rows, E, k, 0, n, 0, 0, false};
  return go<false, true, false, false, false>(a, st);
}

hipError_t launch_expert_product_dw(long long rows, int E, int n, int k, RowsArg dy, RowsArg x, const int32_t* offsets, void* dW, bool f32,
                                    hipStream_t st) {
  const int b = f32 ? 4 : 2;
  ProductArgs a{x, dy, {(unsigned char*)dW, (long long)k * b}, 0, (long long)n * k * b, offsets, nullptr, nullptr, rows, E, k, n, 0, 0, 0, false};
  return f32 ? go<false, true, true, true, true>(a, st) : go<false, true, true, true, false>(a, st);
}

}  // namespace lasnet
