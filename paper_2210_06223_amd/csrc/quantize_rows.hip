// Rows and matrices in 8 bits (e4m3) with a power-of-two scale for each block: 128 columns of a row, 128 x 128 of a matrix.
//
//   q = e4m3(x / 2^e), 2^e least with max|x| over the block <= 448 2^e (at least 2^-126)
//
// Bound by memory: everything is read once into registers, the maximum is a reduction over the lanes (the workgroup) that hold a block, and q is rounded once, to nearest
// even; the division by a power of two moves the exponent alone.  16384 x 2048 bf16 to four experts each 36 us (203 MB, 5.6 TB/s), 4099 x 1001 fp32 6.3; 16 matrices 4096 x 2048 with their
// transposes 95 us (537 MB, 5.6 TB/s), 8 of 1000 x 520 fp32 9.9: 320 workgroups, so one chain of loads, maximum, turn and stores; where a row ends inside a
// thread's eight columns its loads go by elements, a branch and a wait each (1368 x 158 bf16, 22 workgroups, 9.2 us; 704 x 848, 42, 5.7).
#include "row_ops.hpp"

namespace lasnet {
namespace {

typedef unsigned uint2_t __attribute__((ext_vector_type(2)));
typedef uint2_t uint2_any __attribute__((aligned(1)));
typedef unsigned uint_any __attribute__((aligned(1)));

// four floats, times `up`, to e4m3
__device__ __forceinline__ unsigned four(const float* f, float up) {
  const int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * up, f[1] * up, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[2] * up, f[3] * up, v, true);
}

struct QuantizeRowsArgs {
  RowsArg x, out;
  uint8_t* scale;                  // [rows of out][blocks]
  const int32_t* position;         // or null: row t of out is row t of x
  const int32_t* offsets;
  long long tokens;
  int k, E, cols, pieces, blocks, width;    // width: lanes of a row, a power of two, whole blocks
};

// The n (0 < n) elements of a piece that a row has left, in 8 bits.  PAST: past the caches.
template <class T, bool PAST>
__device__ __forceinline__ void store_eight(unsigned char* p, int n, const unsigned (&q)[2]) {
  constexpr int PER = Elem<T>::PER;
  if (n >= PER) {
    if constexpr (PER == 8 && PAST) __builtin_nontemporal_store(uint2_t{q[0], q[1]}, (uint2_any*)p);
    else if constexpr (PER == 8) *(uint2_any*)p = uint2_t{q[0], q[1]};
    else if constexpr (PAST) __builtin_nontemporal_store(q[0], (uint_any*)p);
    else *(uint_any*)p = q[0];
    return;
  }
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (j < n) p[j] = (uint8_t)(q[j / 4] >> (8 * (j % 4)));
}

// Large outputs go past the caches: by the time of this pass and the product that reads its rows next (six pairs of 2 to 8 copies, 1024 to 7168 columns, 16 and 64 experts, products of 256 to
// 4096 columns; three sets of inputs in turn).  Against ordinary stores the pair takes, in the mean of the six and at the worst, at 32 MiB +7 % (+15), 64 +2 (+4), 96 0 (+5), 112 -0.5 (+1),
// 128 -0.3 (+2), 144 -2 (0), 160 -2 (0), 320 -2 (-1).  The pass alone is as fast or faster from 64 MiB on (112 MiB: 4 copies of 2048 columns 40 -> 31 us, 2 of 4096 51 either way).
bool rows_past(long long bytes) { return bytes >= 112 << 20; }

template <class T, bool PAST>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeRowsArgs a) {
  using El = Elem<T>;
  constexpr int BL = 128 / El::PER;                            // lanes of a block
  const int lane = (int)threadIdx.x % a.width, per = 256 / a.width;
  const long long first = (long long)blockIdx.x * per + threadIdx.x / a.width, stride = (long long)gridDim.x * per;
  const long long slots = a.position ? a.tokens * a.k : a.tokens;
  const int part = (int)blockIdx.y, parts = (int)gridDim.y;    // workgroups that share a row
  for (long long t = first; t < a.tokens; t += stride) {
    const unsigned char* x = a.x.data + t * a.x.pitch;
    for (int c0 = part * a.width; c0 < a.pieces; c0 += parts * a.width) {                 // (every lane of a block comes along)
      const int c = c0 + lane, left = a.cols - c * El::PER;
      float f[El::PER];
      El::widen(load_piece<T>(x + (size_t)c * 16, left), f);
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < El::PER; ++j) top = fmaxf(top, fabsf(f[j]));
      top = lanes_max<BL>(top);
      const int byte = scale_byte(top);
      const float up = __uint_as_float((unsigned)(254 - byte) << 23);          // 2^-e, exact
      unsigned q[2];
#pragma unroll
      for (int j = 0; j < El::PER / 4; ++j) q[j] = four(f + 4 * j, up);
      if (left <= 0) continue;
      const int n = a.position ? a.k : 1;
      for (int j = 0; j < n; ++j) {
        const long long p = a.position ? a.position[t * a.k + j] : t;
        if (p < 0 || p >= slots) continue;
        store_eight<T, PAST>(a.out.data + p * a.out.pitch + (size_t)c * El::PER, left, q);
        if (c % BL == 0) a.scale[p * a.blocks + c / BL] = (uint8_t)byte;
      }
    }
  }
  if (!a.position) return;
  // the rows that no expert has
  const long long s = a.offsets[a.E], sent = s < 0 ? 0 : s < slots ? s : slots;
  const unsigned none[2] = {0, 0};
  for (long long p = sent + first; p < slots; p += stride)
    for (int c = part * a.width + lane; c < a.pieces; c += parts * a.width) {
      store_eight<T, PAST>(a.out.data + p * a.out.pitch + (size_t)c * El::PER, a.cols - c * El::PER, none);
      if (c % BL == 0) a.scale[p * a.blocks + c / BL] = 127;
    }
}

struct QuantizeMatricesArgs {
  const unsigned char* W;
  unsigned char *out, *out_t;      // out_t: or null
  uint8_t *scale, *scale_t;
  int n, k, nb, kb;
};

// A workgroup takes a block; thread (r, c) its rows 8 r .. 8 r + 7 and columns 8 c .. 8 c + 7.
template <class T, bool PAST>
__global__ __launch_bounds__(256) void quantize_matrices_kernel(QuantizeMatricesArgs a) {
  using El = Elem<T>;
  constexpr int P = 8 / El::PER;                               // pieces of eight elements
  __shared__ float join[4];
  __shared__ uint2_t turned[128][17];                          // [column][r], a unit to spare: eight rows of eight columns lie apart
  const int tid = (int)threadIdx.x, r = tid >> 4, c = tid & 15;
  const int ib = (int)(blockIdx.x / a.kb % a.nb), cb = (int)(blockIdx.x % a.kb);
  const long long expert = blockIdx.x / a.kb / a.nb;
  const int i0 = ib * 128 + r * 8, c0 = cb * 128 + c * 8, left = a.k - c0;
  const long long first = (expert * a.n + i0) * a.k + c0;      // element
  float f[8][8], top = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float v[El::PER];
      El::widen(load_piece<T>(a.W + (first + (long long)u * a.k + p * El::PER) * El::BYTES, i0 + u < a.n ? left - p * El::PER : 0), v);
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        f[u][p * El::PER + j] = v[j];
        top = fmaxf(top, fabsf(v[j]));
      }
    }
  top = row_join<256, true>(top, join);
  const int byte = scale_byte(top);
  const float up = __uint_as_float((unsigned)(254 - byte) << 23);
  if (tid == 0) {
    a.scale[(expert * a.nb + ib) * a.kb + cb] = (uint8_t)byte;
    if (a.out_t) a.scale_t[(expert * a.kb + cb) * a.nb + ib] = (uint8_t)byte;
  }
  unsigned q[8][2];
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    q[u][0] = four(f[u], up);
    q[u][1] = four(f[u] + 4, up);
    if (i0 + u < a.n && left > 0) store_eight<__bf16, PAST>(a.out + first + (long long)u * a.k, left, q[u]);
  }
  if (!a.out_t) return;
  // 4 x 4 bytes turned: pairs of rows, then pairs of pairs
#pragma unroll
  for (int h = 0; h < 2; ++h) {                                // columns 4 h .. 4 h + 3
    unsigned t[2][4];
#pragma unroll
    for (int g = 0; g < 2; ++g) {                              // rows 4 g .. 4 g + 3
      const unsigned a0 = q[4 * g][h], a1 = q[4 * g + 1][h], a2 = q[4 * g + 2][h], a3 = q[4 * g + 3][h];
      const unsigned lo01 = __builtin_amdgcn_perm(a1, a0, 0x05010400), hi01 = __builtin_amdgcn_perm(a1, a0, 0x07030602);     // (b0 of a0, b0 of a1, b1, b1); b2, b3
      const unsigned lo23 = __builtin_amdgcn_perm(a3, a2, 0x05010400), hi23 = __builtin_amdgcn_perm(a3, a2, 0x07030602);
      t[g][0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100);
      t[g][1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302);
      t[g][2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100);
      t[g][3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) turned[c * 8 + h * 4 + j][r] = uint2_t{t[0][j], t[1][j]};
  }
  __syncthreads();
  const int left_t = a.n - ib * 128 - c * 8;                   // (here c counts eights of the matrix' rows)
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int col = u * 16 + r;                                // of the block
    if (cb * 128 + col >= a.k || left_t <= 0) continue;
    const uint2_t v = turned[col][c];
    const unsigned w[2] = {v[0], v[1]};
    store_eight<__bf16, PAST>(a.out_t + (expert * a.k + cb * 128 + col) * a.n + ib * 128 + c * 8, left_t, w);
  }
}

}  // namespace

hipError_t launch_quantize_rows(int dtype, long long tokens, int k, int E, int cols, RowsArg x, const int32_t* position, const int32_t* offsets,
                                RowsArg out, uint8_t* scale, hipStream_t st) {
  const int per = dtype == LASNET_F32 ? 4 : 8, pieces = (cols + per - 1) / per;
  int width = 128 / per;
  while (width < 256 && width < pieces) width *= 2;
  const QuantizeRowsArgs a{x, out, scale, position, offsets, tokens, k, E, cols, pieces, (cols + 127) / 128, width};
  const long long b = (tokens + 256 / width - 1) / (256 / width);
  // (few wide rows are shared by workgroups, a thousand in all: 59 rows of 7520 fp32 to eight experts each 16.7 -> 4.6 us, 500 of 8192 bf16 to six 11.2 -> 8.7, 3 of 131072 fp32 50.5 -> 3.3)
  const long long shares = b >= 1024 ? 1 : 1024 / b, chunks = (pieces + width - 1) / width;
  const bool past = rows_past((position ? tokens * k : tokens) * cols);
  auto kernel = dtype == LASNET_F32 ? past ? quantize_rows_kernel<float, true> : quantize_rows_kernel<float, false>
                                    : past ? quantize_rows_kernel<__bf16, true> : quantize_rows_kernel<__bf16, false>;
  kernel<<<dim3((unsigned)(b < 1 << 20 ? b : 1 << 20), (unsigned)(chunks < shares ? chunks : shares)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_quantize_matrices(int dtype, int E, int n, int k, const void* W, void* out, uint8_t* scale, void* out_t, uint8_t* scale_t,
                                    hipStream_t st) {
  const QuantizeMatricesArgs a{(const unsigned char*)W, (unsigned char*)out, (unsigned char*)out_t, scale, scale_t, n, k, (n + 127) / 128, (k + 127) / 128};
  const bool past = writes_past((long long)E * n * k * (out_t ? 2 : 1));
  auto kernel = dtype == LASNET_F32 ? past ? quantize_matrices_kernel<float, true> : quantize_matrices_kernel<float, false>
                                    : past ? quantize_matrices_kernel<__bf16, true> : quantize_matrices_kernel<__bf16, false>;
  kernel<<<dim3((unsigned)((long long)E * a.nb * a.kb)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace lasnet
