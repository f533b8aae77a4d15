// What the row operators (norm_rows.hip, route_rows.hip, expert_product.hip) share: rows as kernels see them, and pieces of rows.
#pragma once
#include "common.hpp"

namespace lasnet {

// Rows by value into a kernel: row i starts at data + i * pitch BYTES.
struct RowsArg {
  unsigned char* data;
  long long pitch;
};

constexpr int kNormCols = 16384;          // most columns of a norm: a row lies in the registers of 16 waves

// ---- launchers of the row operators (row_api.hip checks their arguments) ----
hipError_t launch_norm_rows(int dtype, int out_dtype, long long rows, int cols, RowsArg x, RowsArg residual, const float* weight, float eps,
                            RowsArg sum, RowsArg out, uint8_t* scale, float* rstd, hipStream_t st);
size_t norm_backward_workspace_bytes(long long rows, int cols);
hipError_t launch_norm_rows_backward(int dtype, long long rows, int cols, RowsArg dy, RowsArg s, const float* weight, const float* rstd,
                                     RowsArg dsum, RowsArg dx, float* dweight, void* workspace, hipStream_t st);
size_t route_workspace_bytes(long long slots, int E);
hipError_t launch_route(const int32_t* experts, long long slots, int E, int32_t* offsets, int32_t* order, int32_t* position, void* workspace,
                        hipStream_t st);
hipError_t launch_dispatch(long long tokens, int k, int E, int row_bytes, RowsArg x, const uint8_t* scale, const int32_t* position,
                           const int32_t* offsets, RowsArg out, uint8_t* out_scale, hipStream_t st);
hipError_t launch_combine(int dtype, long long tokens, int k, int cols, RowsArg y, const float* weights, const int32_t* position, RowsArg base,
                          RowsArg out, hipStream_t st);
hipError_t launch_combine_backward(int dtype, long long tokens, int k, int E, int cols, RowsArg dout, RowsArg y, const float* weights,
                                   const int32_t* position, const int32_t* offsets, RowsArg dy, float* dweights, hipStream_t st);
hipError_t launch_expert_product(int dtype, long long rows, int E, int n, int k, RowsArg x, const uint8_t* scale, const int32_t* offsets,
                                 const void* W, const float* wscale, RowsArg out, bool relu, hipStream_t st);
hipError_t launch_expert_product_dx(long long rows, int E, int n, int k, RowsArg dy, const int32_t* offsets, const void* W, RowsArg dx,
                                    hipStream_t st);
hipError_t launch_expert_product_dw(long long rows, int E, int n, int k, RowsArg dy, RowsArg x, const int32_t* offsets, void* dW, bool f32,
                                    void* workspace, hipStream_t st);
size_t product_dw_workspace_bytes(long long rows, int E, int n, int k);

// Whether a call that writes so many bytes writes them past the caches: more than the 256 MB Infinity Cache would still hold when the next kernel reads them.
// Dispatch of 268 MB and the sum that reads it: 156 us with ordinary stores, 116 past the caches; of 134 MB 56 and 61, of 67 MB 31 and 33.
inline bool writes_past(long long bytes) { return bytes > (192ll << 20); }

namespace {

// A kernel that needs more than 64 KiB of dynamic LDS must be told so once per device.
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<unsigned long long>& done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;    // devices past 63: set every time
  if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// ---- pieces of 16 bytes, at any address: gfx950's global loads and stores take every alignment (one instruction either way), so
// rows that start anywhere need no variant of their own; only the end of a row, where less than a piece is left, goes by elements.
typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
typedef uint4_t uint4_any __attribute__((aligned(1)));

__device__ __forceinline__ uint4_t load16(const unsigned char* p) { return *(const uint4_any*)p; }
// PAST: past the caches (see writes_past)
template <bool PAST = false>
__device__ __forceinline__ void store16(unsigned char* p, uint4_t v) {
  if constexpr (PAST)
    __builtin_nontemporal_store(v, (uint4_any*)p);
  else
    *(uint4_any*)p = v;
}

__device__ __forceinline__ float bf16_lo(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(unsigned u) { return __uint_as_float(u & 0xffff0000u); }
// two floats to bf16, nearest even
__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  union { bf16x2 h; unsigned u; } c;
  c.h = bf16x2{(__bf16)a, (__bf16)b};
  return c.u;
}

// T: the element in memory.  PER elements are 16 bytes.
template <class T> struct Elem;
template <> struct Elem<float> {
  static constexpr int PER = 4, BYTES = 4;
  static __device__ __forceinline__ void widen(uint4_t v, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ uint4_t narrow(const float (&f)[4]) {
    return uint4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
  static __device__ __forceinline__ unsigned bits(const unsigned char* p) { return *(const unsigned*)p; }
  static __device__ __forceinline__ void put(unsigned char* p, unsigned b) { *(unsigned*)p = b; }
};
template <> struct Elem<__bf16> {
  static constexpr int PER = 8, BYTES = 2;
  static __device__ __forceinline__ void widen(uint4_t v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_lo(v[i]);
      f[2 * i + 1] = bf16_hi(v[i]);
    }
  }
  static __device__ __forceinline__ uint4_t narrow(const float (&f)[8]) {
    return uint4_t{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])};
  }
  static __device__ __forceinline__ unsigned bits(const unsigned char* p) { return *(const unsigned short*)p; }
  static __device__ __forceinline__ void put(unsigned char* p, unsigned b) { *(unsigned short*)p = (unsigned short)b; }
};

// The n elements (0 <= n; PER or more: a whole piece) that a row has left at p, zeros behind them.
template <class T>
__device__ __forceinline__ uint4_t load_piece(const unsigned char* p, int n) {
  using E = Elem<T>;
  if (n >= E::PER) return load16(p);
  uint4_t v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < E::PER; ++i)
    if (i < n) v[i * E::BYTES / 4] |= E::bits(p + i * E::BYTES) << (8 * (i * E::BYTES % 4));
  return v;
}
template <class T, bool PAST = false>
__device__ __forceinline__ void store_piece(unsigned char* p, int n, uint4_t v) {
  using E = Elem<T>;
  if (n >= E::PER) {
    store16<PAST>(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < E::PER; ++i)
    if (i < n) E::put(p + i * E::BYTES, v[i * E::BYTES / 4] >> (8 * (i * E::BYTES % 4)));
}

template <int L = 64>
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = L / 2; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
template <int L = 64>
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = L / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
// Sum (or maximum) over the L threads that share a row, the same bits in each.  at: L / 64 floats of LDS that nobody else writes before the next barrier but one.
template <int L, bool MAX>
__device__ __forceinline__ float row_join(float v, float* at) {
  v = MAX ? wave_max<(L < 64 ? L : 64)>(v) : wave_sum<(L < 64 ? L : 64)>(v);
  if constexpr (L <= 64) return v;
  const int wave = (int)(threadIdx.x >> 6) % (L / 64);
  if ((threadIdx.x & 63) == 0) at[wave] = v;
  __syncthreads();
  float r = at[0];
#pragma unroll
  for (int i = 1; i < L / 64; ++i) r = MAX ? fmaxf(r, at[i]) : r + at[i];
  return r;
}

}  // namespace
}  // namespace lasnet
