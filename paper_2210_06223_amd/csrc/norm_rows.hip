// Root-mean-square norm of rows with the residual's addition, and its gradients.
//
//   s = x + r;  rstd = (mean s^2 + eps)^-1/2;  y = s rstd g;  in 8 bits q = e4m3(y / 2^e), 2^e least with max|y| <= 448 2^e
//
// Bound by memory: a row is read once into the registers of L threads (16 to 1024), N pieces of 16 bytes each, and everything follows from
// there: the sum of squares and, for 8 bits, the maximum are two reductions over lanes.  Sums, s and y stay in 32 bits; s is rounded where it is
// stored (and y follows from what was not), y once, to its own type.
//
//   16384 x 4096 bf16 with a residual, out in e4m3 (470 MB): 84 us, 5.6 TB/s, where a large copy reaches 5.0.  4 rows of it: 3.7 us, a launch and one
//   row's chain of loads and reductions.  Gradients of 25088 x 1024 bf16 (206 MB): 45.0 us, 4.6 TB/s, of which joining the parts of g's takes 4.9.
#include <type_traits>

#include "row_ops.hpp"

namespace lasnet {
namespace {

struct NormArgs {
  RowsArg x, res, sum, out;
  const float* weight;
  uint8_t* scale;
  float* rstd;
  long long rows;
  int cols;
  float eps;
};

__device__ __forceinline__ void load_weights(const float* w, int n, float* f, int per) {
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    if (i >= per) break;
    const uint4_t v = load_piece<float>((const unsigned char*)(w + i), n - i);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[i + j] = __uint_as_float(v[j]);
  }
}

// T: the rows' type; E4M3: out has 8 bits.
template <class T, bool E4M3, int L, int N>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_rows_kernel(NormArgs a) {
  using E = Elem<T>;
  constexpr int ROWS = L < 256 ? 256 / L : 1;                 // rows of a workgroup
  __shared__ float join[2][L < 256 ? 4 : L / 64];
  const int tid = (int)threadIdx.x, lane = tid % L;
  const long long row = (long long)blockIdx.x * ROWS + tid / L;
  if (L <= 64 && row >= a.rows) return;                       // (beyond: a workgroup has one row, and there are as many)
  const unsigned char* x = a.x.data + row * a.x.pitch;
  float s[N][E::PER], g[N][E::PER], ss = 0.f;
  uint4_t px[N], pr[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * L + lane) * E::PER;
    px[i] = load_piece<T>(x + (size_t)c * E::BYTES, a.cols - c);
  }
  if (a.res.data) {
    const unsigned char* r = a.res.data + row * a.res.pitch;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      pr[i] = load_piece<T>(r + (size_t)c * E::BYTES, a.cols - c);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * L + lane) * E::PER;
    load_weights(a.weight + c, a.cols - c, g[i], E::PER);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    E::widen(px[i], s[i]);
    if (a.res.data) {
      float r[E::PER];
      E::widen(pr[i], r);
#pragma unroll
      for (int j = 0; j < E::PER; ++j) s[i][j] += r[j];
    }
#pragma unroll
    for (int j = 0; j < E::PER; ++j) ss += s[i][j] * s[i][j];
  }
  ss = row_join<L, false>(ss, join[0]);
  const float rstd = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
  if (a.sum.data) {
    unsigned char* o = a.sum.data + row * a.sum.pitch;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      if (c < a.cols) store_piece<T>(o + (size_t)c * E::BYTES, a.cols - c, E::narrow(s[i]));
    }
  }
  if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < E::PER; ++j) s[i][j] *= rstd * g[i][j];
  unsigned char* o = a.out.data + row * a.out.pitch;
  if constexpr (!E4M3) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      if (c < a.cols) store_piece<T>(o + (size_t)c * E::BYTES, a.cols - c, E::narrow(s[i]));
    }
  } else {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < E::PER; ++j) top = fmaxf(top, fabsf(s[i][j]));
    top = row_join<L, true>(top, join[1]);
    const int byte = scale_byte(top);
    const float up = __uint_as_float((unsigned)(254 - byte) << 23);            // 2^-e, exact
    if (lane == 0) a.scale[row] = (uint8_t)byte;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      unsigned q[E::PER / 4];
#pragma unroll
      for (int j = 0; j < E::PER / 4; ++j) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][4 * j] * up, s[i][4 * j + 1] * up, 0, false);
        q[j] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(s[i][4 * j + 2] * up, s[i][4 * j + 3] * up, v, true);
      }
      const int n = a.cols - c;
      if (n >= E::PER) {
        if constexpr (E::PER == 8) {
          typedef unsigned uint2_any __attribute__((ext_vector_type(2), aligned(1)));
          *(uint2_any*)(o + c) = uint2_any{q[0], q[1]};
        } else {
          typedef unsigned uint_any __attribute__((aligned(1)));
          *(uint_any*)(o + c) = q[0];
        }
      } else {
#pragma unroll
        for (int j = 0; j < E::PER; ++j)
          if (j < n) o[c + j] = (uint8_t)(q[j / 4] >> (8 * (j % 4)));
      }
    }
  }
}

template <class T, bool E4M3, int L, int N>
hipError_t go(const NormArgs& a, hipStream_t st) {
  constexpr int ROWS = L < 256 ? 256 / L : 1, THREADS = L < 256 ? 256 : L;
  constexpr long long most = (1ll << 31) / THREADS * ROWS;      // rows of a launch: one of 2^32 threads is an error
  for (long long done = 0; done < a.rows; done += most) {
    NormArgs b = a;
    b.rows = a.rows - done < most ? a.rows - done : most;
    for (RowsArg* r : {&b.x, &b.res, &b.sum, &b.out})
      if (r->data) r->data += done * r->pitch;
    if (b.scale) b.scale += done;
    if (b.rstd) b.rstd += done;
    norm_rows_kernel<T, E4M3, L, N><<<dim3((unsigned)((b.rows + ROWS - 1) / ROWS)), dim3(THREADS), 0, st>>>(b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Threads of a row, in us a call: 59300 x 122 bf16 7.9 by 16 threads, 20.0 by 64; 65536 x 256 12.2 by 32, 18.4 by 64; 16384 x 512 12.1 by 64, 17.9 by 256; 4096 x 4096 19.9 by
// 256, 22.0 by 1024; rows of up to 2048 elements in 16384 of them 68 by 1024.  A few rows take 3.5 to 3.8 either way, whatever their width.
template <class T, bool E4M3>
hipError_t pick(const NormArgs& a, hipStream_t st) {
  const int pieces = (a.cols + Elem<T>::PER - 1) / Elem<T>::PER;
  if (pieces <= 16) return go<T, E4M3, 16, 1>(a, st);
  if (pieces <= 32) return go<T, E4M3, 32, 1>(a, st);
  if (pieces <= 64) return go<T, E4M3, 64, 1>(a, st);
  if (pieces <= 128) return go<T, E4M3, 64, 2>(a, st);
  // (a wave alone needs no barrier: 4099 rows of 251 pieces 7.65 us a call, four waves 8.5; a few rows are better spread)
  if (pieces <= 256) return a.rows >= 1024 ? go<T, E4M3, 64, 4>(a, st) : go<T, E4M3, 256, 1>(a, st);
  if (pieces <= 512) return go<T, E4M3, 256, 2>(a, st);
  if (pieces <= 1024) return go<T, E4M3, 256, 4>(a, st);
  return go<T, E4M3, 1024, kNormCols / 1024 / Elem<T>::PER>(a, st);
}

// ---- the gradients ----
__host__ __device__ inline int part_pitch(int cols) { return (cols + 3) / 4 * 4; }     // floats of a workgroup's part: whole pieces

struct NormGradArgs {
  RowsArg dy, s, dsum, dx;
  const float* weight;
  const float* rstd;
  float* part;                     // [workgroups][part_pitch(cols)]
  long long rows;
  int cols;
};

// A workgroup takes the rows blockIdx.x, blockIdx.x + gridDim.x, ... (times ROWS) and keeps its columns' sums of dy s rstd in registers.
template <class T, int L, int N>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_grad_kernel(NormGradArgs a) {
  using E = Elem<T>;
  constexpr int ROWS = L < 256 ? 256 / L : 1;
  __shared__ float join[2][L < 256 ? 4 : L / 64];
  const int tid = (int)threadIdx.x, lane = tid % L, sub = tid / L;
  float dg[N][E::PER] = {};
  int turn = 0;
  for (long long row = (long long)blockIdx.x * ROWS + sub; row < a.rows; row += (long long)gridDim.x * ROWS, turn ^= 1) {
    const float rstd = a.rstd[row];
    uint4_t py[N], ps[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      py[i] = load_piece<T>(a.dy.data + row * a.dy.pitch + (size_t)c * E::BYTES, a.cols - c);
      ps[i] = load_piece<T>(a.s.data + row * a.s.pitch + (size_t)c * E::BYTES, a.cols - c);
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      float y[E::PER], s[E::PER], g[E::PER];
      E::widen(py[i], y);
      E::widen(ps[i], s);
      load_weights(a.weight + c, a.cols - c, g, E::PER);
#pragma unroll
      for (int j = 0; j < E::PER; ++j) {
        dg[i][j] += y[j] * (s[j] * rstd);
        dot += y[j] * g[j] * s[j];
      }
    }
    dot = row_join<L, false>(dot, join[turn]);
    const float pull = dot / (float)a.cols * rstd * rstd;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * E::PER;
      if (c >= a.cols) continue;
      float y[E::PER], s[E::PER], g[E::PER], d[E::PER] = {};
      E::widen(py[i], y);
      E::widen(ps[i], s);
      load_weights(a.weight + c, a.cols - c, g, E::PER);
      if (a.dsum.data) E::widen(load_piece<T>(a.dsum.data + row * a.dsum.pitch + (size_t)c * E::BYTES, a.cols - c), d);
#pragma unroll
      for (int j = 0; j < E::PER; ++j) d[j] += rstd * (y[j] * g[j] - s[j] * pull);
      store_piece<T>(a.dx.data + row * a.dx.pitch + (size_t)c * E::BYTES, a.cols - c, E::narrow(d));
    }
  }
  // the ROWS rows' sums of a column are added in order
  if constexpr (ROWS > 1) {
    __shared__ float rest[(ROWS - 1) * L * E::PER];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __syncthreads();
      if (sub)
#pragma unroll
        for (int j = 0; j < E::PER; ++j) rest[((sub - 1) * E::PER + j) * L + lane] = dg[i][j];
      __syncthreads();
      if (!sub)
#pragma unroll
        for (int j = 0; j < E::PER; ++j)
#pragma unroll
          for (int r = 0; r < ROWS - 1; ++r) dg[i][j] += rest[(r * E::PER + j) * L + lane];
    }
    if (sub) return;
  }
  float* part = a.part + (size_t)blockIdx.x * part_pitch(a.cols);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * L + lane) * E::PER;
#pragma unroll
    for (int j = 0; j < E::PER; j += 4)
      if (c + j < part_pitch(a.cols)) store16((unsigned char*)(part + c + j), Elem<float>::narrow({dg[i][j], dg[i][j + 1], dg[i][j + 2], dg[i][j + 3]}));
  }
}

// dweight[c] = sum of the workgroups' parts: a workgroup has 16 columns, four a thread, and 64 threads share the parts, each every 64th in order; then the 64 sums in
// order of a tree.  (One thread a column, 16 a workgroup, took 20 us for 1024 parts of 1024 columns: few loads in flight.)
__global__ __launch_bounds__(256) void norm_grad_join_kernel(const float* part, int groups, int pitch, int cols, float* dweight) {
  __shared__ float sum[64][20];
  const int four = (int)threadIdx.x & 3, share = (int)threadIdx.x >> 2;
  const int c = (int)blockIdx.x * 16 + four * 4;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < cols)
#pragma unroll 8
    for (int b = share; b < groups; b += 64) {
      float f[4];
      Elem<float>::widen(load16((const unsigned char*)(part + (size_t)b * pitch + c)), f);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += f[i];
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[share][four * 4 + i] = v[i];
  for (int d = 32; d >= 1; d >>= 1) {
    __syncthreads();
    if (share < d)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[share][four * 4 + i] += sum[share + d][four * 4 + i];
  }
  if (share == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < cols) dweight[c + i] = sum[0][four * 4 + i];
}

// Workgroups of the backward pass: as many as the chip runs at once, so that the parts stay few (25088 x 1024: 45.7 us a call; 512 of them
// 49.0, 2048 49.9), and of many rows at least two for each wave that has one at a time (1024 x 4096 15.5 us, one each 19.2; 4 x 4096 6.9, two each 8.2).
int grad_groups(long long rows, int cols) {
  const long long most = 1024, each = rows < (cols <= 1024 ? 2048 : 256) ? 1 : 2, at_once = cols <= 64 ? 16 : cols <= 128 ? 8 : cols <= 1024 ? 4 : 1;
  const long long need = (rows + at_once * each - 1) / (at_once * each);
  return (int)(need < most ? need : most);
}

template <class T, int L, int N>
hipError_t go_grad(const NormGradArgs& a, int groups, float* dweight, hipStream_t st) {
  norm_grad_kernel<T, L, N><<<dim3((unsigned)groups), dim3(L < 256 ? 256 : L), 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  norm_grad_join_kernel<<<dim3((unsigned)((a.cols + 15) / 16)), dim3(256), 0, st>>>(a.part, groups, part_pitch(a.cols), a.cols, dweight);
  return hipGetLastError();
}

template <class T>
hipError_t pick_grad(const NormGradArgs& a, int groups, float* dweight, hipStream_t st) {
  const int pieces = (a.cols + Elem<T>::PER - 1) / Elem<T>::PER;
  if (pieces <= 16) return go_grad<T, 16, 1>(a, groups, dweight, st);
  if (pieces <= 32) return go_grad<T, 32, 1>(a, groups, dweight, st);
  if (pieces <= 64) return go_grad<T, 64, 1>(a, groups, dweight, st);
  if (pieces <= 128) return go_grad<T, 64, 2>(a, groups, dweight, st);
  if (pieces <= 256) {
    // (32 bits: 16384 x 1001 40.4 us a call by one wave a row, four 45.1; bf16, twice as many elements for a lane: 16384 x 2048 45.4 and 41.9)
    if constexpr (std::is_same_v<T, float>) return go_grad<T, 64, 4>(a, groups, dweight, st);
    return go_grad<T, 256, 1>(a, groups, dweight, st);
  }
  if (pieces <= 512) return go_grad<T, 256, 2>(a, groups, dweight, st);
  if (pieces <= 1024) return go_grad<T, 256, 4>(a, groups, dweight, st);
  return go_grad<T, 1024, kNormCols / 1024 / Elem<T>::PER>(a, groups, dweight, st);
}

}  // namespace

hipError_t launch_norm_rows(int dtype, int out_dtype, long long rows, int cols, RowsArg x, RowsArg residual, const float* weight, float eps,
                            RowsArg sum, RowsArg out, uint8_t* scale, float* rstd, hipStream_t st) {
  const NormArgs a{x, residual, sum, out, weight, scale, rstd, rows, cols, eps};
  const bool q = out_dtype == LASNET_E4M3;
  if (dtype == LASNET_F32) return q ? pick<float, true>(a, st) : pick<float, false>(a, st);
  return q ? pick<__bf16, true>(a, st) : pick<__bf16, false>(a, st);
}

size_t norm_backward_workspace_bytes(long long rows, int cols) { return (size_t)grad_groups(rows, cols) * part_pitch(cols) * sizeof(float); }

hipError_t launch_norm_rows_backward(int dtype, long long rows, int cols, RowsArg dy, RowsArg s, const float* weight, const float* rstd,
                                     RowsArg dsum, RowsArg dx, float* dweight, void* workspace, hipStream_t st) {
  const NormGradArgs a{dy, s, dsum, dx, weight, rstd, (float*)workspace, rows, cols};
  const int groups = grad_groups(rows, cols);
  if (rows == 0) {                                             // no rows, no parts: dweight = 0
    norm_grad_join_kernel<<<dim3((unsigned)((cols + 15) / 16)), dim3(256), 0, st>>>(nullptr, 0, 0, cols, dweight);
    return hipGetLastError();
  }
  return dtype == LASNET_F32 ? pick_grad<float>(a, groups, dweight, st) : pick_grad<__bf16>(a, groups, dweight, st);
}

}  // namespace lasnet
