// The router of a layer of experts: which experts a token goes to and how they are weighted, the balance of the experts, and the logits' gradient of both.
//
//   choice     the k largest logits of a token; weights w = softmax over those k (or over all E); lse = log sum_e exp(l[e])
//   balance    counts[e], share[e] = mean_t p[t][e] with p = exp(l - lse), loss = (E sum_e counts[e] / (k T) share[e], mean_t lse[t]^2)
//   gradient   p (c - sum_e p c) + 2 lse p d1 / T + that of the weights, with c[e] = d0 E counts[e] / (k T^2)
//
// A token's logits lie in the registers of L lanes (16, 32 or 64), read once.  Exponentials, sums and statistics are held in 32 bits, sums over tokens in 64; only the
// gradient is rounded, once, to the logits' type.
#include "row_ops.hpp"

namespace lasnet {
namespace {

// ---- order: a key that is larger for what is chosen earlier.  NaN is above everything; 0: never chosen (-inf, and what is beyond the row). ----
__device__ __forceinline__ unsigned key_of(float v) {
  const unsigned u = __float_as_uint(v + 0.f);                 // (-0 + 0 = 0: equal values are equal keys)
  if (v != v) return 0xffffffffu;
  return u == 0xff800000u ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) {
  if (key == 0xffffffffu) return __uint_as_float(0x7fc00000u);
  return key == 0 ? -INFINITY : __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <int L>
__device__ __forceinline__ unsigned lanes_max(unsigned v) {
#pragma unroll
  for (int d = L / 2; d; d >>= 1) {
    const unsigned u = __shfl_xor(v, d);
    v = u > v ? u : v;
  }
  return v;
}

struct ChooseArgs {
  RowsArg logits;
  const uint8_t* mask;
  int32_t* experts;
  float* weights;
  float* lse;
  long long tokens;
  int E, k;
  bool all;
};

// L lanes a token, N pieces of 16 bytes each, one behind the other: a lower lane has the lower experts.  k <= L: lane j keeps the j-th choice.
template <class T, int L, int N>
__global__ __launch_bounds__(256) void choose_kernel(ChooseArgs a) {
  using El = Elem<T>;
  constexpr int C = N * El::PER;                               // logits of a lane
  const int lane = (int)threadIdx.x % L, base = (int)(threadIdx.x & 63) / L * L;
  for (long long t = (long long)blockIdx.x * (256 / L) + threadIdx.x / L; t < a.tokens; t += (long long)gridDim.x * (256 / L)) {
    const bool there = !a.mask || a.mask[t];
    float v[C];
    unsigned key[C];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (lane * N + i) * El::PER;
      float f[El::PER];
      El::widen(there ? load_piece<T>(a.logits.data + t * a.logits.pitch + (size_t)c * El::BYTES, a.E - c) : uint4_t{0, 0, 0, 0}, f);
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        const bool in = there && c + j < a.E;
        v[i * El::PER + j] = in ? f[j] : -INFINITY;
        key[i * El::PER + j] = in ? key_of(f[j]) : 0u;
      }
    }
    float top = 0.f, sum = 0.f, mine = -INFINITY;                // mine: the value of this lane's choice
    int expert = -1;
    for (int j = 0; j < a.k; ++j) {
      unsigned best = 0;
      int at = 0;
#pragma unroll
      for (int c = C - 1; c >= 0; --c)
        if (key[c] >= best) {
          best = key[c];
          at = c;
        }
      const unsigned m = lanes_max<L>(best);
      if (j == 0) {
        top = value_of(m);
        if (m) {
#pragma unroll
          for (int c = 0; c < C; ++c) sum += expf(v[c] - top);
        }
        sum = wave_sum<L>(sum);
      }
      const unsigned long long has = __ballot(best == m) >> base;
      const int first = __ffsll((long long)has) - 1;             // the lowest lane that has it
      const int e = __shfl(lane * C + at, base + first);
      if (lane == j && m) {
        expert = e;
        mine = value_of(m);
      }
      if (lane == first)
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (c == at) key[c] = 0;
    }
    const float lse = top + logf(sum);                           // (sum is 0 of a token without a candidate, with top = -inf)
    float w = expert >= 0 ? expf(mine - top) : 0.f;
    const float chosen = wave_sum<L>(lane < a.k ? w : 0.f);
    w = expert >= 0 ? w / (a.all ? sum : chosen) : 0.f;
    if (lane < a.k) {
      a.experts[t * a.k + lane] = expert;
      a.weights[t * a.k + lane] = w;
    }
    if (a.lse && lane == 0) a.lse[t] = lse;
  }
}

template <class T, int L, int N>
hipError_t go_choose(const ChooseArgs& a, hipStream_t st) {
  const long long b = (a.tokens + 256 / L - 1) / (256 / L);
  choose_kernel<T, L, N><<<dim3((unsigned)(b < 1 << 20 ? b : 1 << 20)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}
template <class T>
hipError_t pick_choose(const ChooseArgs& a, hipStream_t st) {
  const int pieces = (a.E + Elem<T>::PER - 1) / Elem<T>::PER;
  constexpr int MOST = 4096 / 64 / Elem<T>::PER;
  if (a.k <= 16 && pieces <= 16) return go_choose<T, 16, 1>(a, st);
  if (a.k <= 32 && pieces <= 32) return go_choose<T, 32, 1>(a, st);
  if (pieces <= 64) return go_choose<T, 64, 1>(a, st);
  if (pieces <= 128) return go_choose<T, 64, 2>(a, st);
  if (pieces <= 256) return go_choose<T, 64, 4>(a, st);
  return go_choose<T, 64, MOST>(a, st);
}

// ---- balance ----
struct BalanceArgs {
  RowsArg logits;
  const float* lse;
  const int32_t* experts;
  int32_t* counts;
  float* share;
  float* loss;
  double* part;                    // [workgroups][E + 2]: sums of p; of lse^2; tokens
  int32_t* part_counts;            // [workgroups][E]
  long long tokens, slots;
  int E, k, groups;
};

// The end of both kernels: from the sums over all tokens to the outputs, by one workgroup.  at(e), count(e): the sum of p and the number of rows of expert e.
template <class At, class Count>
__device__ __forceinline__ void finish_balance(const BalanceArgs& a, double squares, double tokens, double* join, At at, Count count) {
  const int tid = (int)threadIdx.x, n = (int)blockDim.x;
  const double T = tokens > 0. ? tokens : 1.;
  double loss = 0.;
  for (int e = tid; e < a.E; e += n) {
    const double share = at(e) / T;
    const int c = count(e);
    a.counts[e] = c;
    a.share[e] = (float)share;
    loss += (double)c * share;
  }
  __syncthreads();
  join[tid] = loss;
  __syncthreads();
  for (int d = n / 2; d; d >>= 1) {
    if (tid < d) join[tid] += join[tid + d];
    __syncthreads();
  }
  if (tid == 0) {
    a.loss[0] = (float)(join[0] * ((double)a.E / ((double)a.k * T)));
    a.loss[1] = (float)(squares / T);
    a.counts[a.E] = (int)tokens;
  }
}

// Workgroups take tokens in turn, L lanes each; a lane keeps its columns' sums.  One workgroup: finishes by itself.
template <class T, int L, int N>
__global__ __launch_bounds__(256) void balance_kernel(BalanceArgs a) {
  using El = Elem<T>;
  constexpr int G = 256 / L;                                   // tokens at a time
  extern __shared__ __attribute__((aligned(16))) double balance_lds[];
  double* sums = balance_lds;                                  // [E + 2]
  double* join = sums + a.E + 2;                               // [256]
  int* hist = (int*)(join + 256);                              // [E]
  const int tid = (int)threadIdx.x, lane = tid % L, group = tid / L;
  for (int e = tid; e < a.E; e += 256) hist[e] = 0;
  __syncthreads();
  for (long long s = (long long)blockIdx.x * 256 + tid; s < a.slots; s += (long long)gridDim.x * 256) {
    const int e = a.experts[s];
    if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);             // (whole numbers in LDS: any order gives the same)
  }
  double acc[N][El::PER] = {}, squares = 0., tokens = 0.;
  for (long long t = (long long)blockIdx.x * G + group; t < a.tokens; t += (long long)gridDim.x * G) {
    const float lse = a.lse[t];
    if (lse == -INFINITY) continue;
    squares += (double)lse * lse;
    tokens += 1.;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * L + lane) * El::PER;
      if (c >= a.E) continue;
      float f[El::PER];
      El::widen(load_piece<T>(a.logits.data + t * a.logits.pitch + (size_t)c * El::BYTES, a.E - c), f);
#pragma unroll
      for (int j = 0; j < El::PER; ++j) acc[i][j] += (double)expf(f[j] - lse);
    }
  }
  // the groups' sums, one group after the other
  for (int g = 0; g < G; ++g) {
    if (group == g) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < El::PER; ++j) {
          const int c = (i * L + lane) * El::PER + j;
          if (c < a.E) sums[c] = g ? sums[c] + acc[i][j] : acc[i][j];
        }
      if (lane == 0) {
        sums[a.E] = g ? sums[a.E] + squares : squares;
        sums[a.E + 1] = g ? sums[a.E + 1] + tokens : tokens;
      }
    }
    __syncthreads();
  }
  if (gridDim.x == 1) {
    finish_balance(a, sums[a.E], sums[a.E + 1], join, [&](int e) { return sums[e]; }, [&](int e) { return hist[e]; });
    return;
  }
  for (int e = tid; e < a.E + 2; e += 256) a.part[(long long)blockIdx.x * (a.E + 2) + e] = sums[e];
  for (int e = tid; e < a.E; e += 256) a.part_counts[(long long)blockIdx.x * a.E + e] = hist[e];
}

__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceArgs a) {
  __shared__ double join[1024];
  double squares = 0., tokens = 0.;
  for (int g = 0; g < a.groups; ++g) {
    squares += a.part[(long long)g * (a.E + 2) + a.E];
    tokens += a.part[(long long)g * (a.E + 2) + a.E + 1];
  }
  finish_balance(
      a, squares, tokens, join,
      [&](int e) {
        double s = 0.;
        for (int g = 0; g < a.groups; ++g) s += a.part[(long long)g * (a.E + 2) + e];
        return s;
      },
      [&](int e) {
        int c = 0;
        for (int g = 0; g < a.groups; ++g) c += a.part_counts[(long long)g * a.E + e];
        return c;
      });
}

// Workgroups of a call.
int balance_groups(long long tokens) {
  const long long g = (tokens + 63) / 64;
  return (int)(g < 1 ? 1 : g < 256 ? g : 256);
}

template <class T, int L, int N>
hipError_t go_balance(const BalanceArgs& a, hipStream_t st) {
  const int bytes = (a.E + 2 + 256) * 8 + a.E * 4;
  balance_kernel<T, L, N><<<dim3((unsigned)a.groups), dim3(256), bytes, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.groups == 1) return e;
  balance_join_kernel<<<dim3(1), dim3(1024), 0, st>>>(a);
  return hipGetLastError();
}
template <class T>
hipError_t pick_balance(const BalanceArgs& a, hipStream_t st) {
  const int pieces = (a.E + Elem<T>::PER - 1) / Elem<T>::PER;
  if (pieces <= 16) return go_balance<T, 16, 1>(a, st);
  if (pieces <= 32) return go_balance<T, 32, 1>(a, st);
  if (pieces <= 64) return go_balance<T, 64, 1>(a, st);
  if (pieces <= 256) return go_balance<T, 256, 1>(a, st);
  return go_balance<T, 256, 4>(a, st);
}

// ---- the gradient ----
struct ChooseGradArgs {
  RowsArg logits, dlogits;
  const float* lse;
  const int32_t* experts;
  const float* weights;
  const float* dweights;           // or null
  const int32_t* counts;           // with dloss
  const float* dloss;              // or null
  long long tokens;
  int E, k;
  bool all;
};

template <class T, int L, int N>
__global__ __launch_bounds__(256) void choose_grad_kernel(ChooseGradArgs a) {
  using El = Elem<T>;
  const int lane = (int)threadIdx.x % L, base = (int)(threadIdx.x & 63) / L * L;
  // what a probability of 1 would get from the balance loss, expert by expert
  float c[N][El::PER] = {}, z = 0.f;
  if (a.dloss) {
    const float T_ = (float)(a.counts[a.E] > 0 ? a.counts[a.E] : 1), unit = a.dloss[0] / T_ * ((float)a.E / ((float)a.k * T_));
    z = 2.f * a.dloss[1] / T_;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        const int e = (i * L + lane) * El::PER + j;
        if (e < a.E) c[i][j] = unit * (float)a.counts[e];
      }
  }
  for (long long t = (long long)blockIdx.x * (256 / L) + threadIdx.x / L; t < a.tokens; t += (long long)gridDim.x * (256 / L)) {
    const float lse = a.lse[t];
    const bool there = lse != -INFINITY;
    float d[N][El::PER], dot = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = (i * L + lane) * El::PER;
      float f[El::PER] = {};
      if (there && e < a.E) El::widen(load_piece<T>(a.logits.data + t * a.logits.pitch + (size_t)e * El::BYTES, a.E - e), f);
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        d[i][j] = there && e + j < a.E ? expf(f[j] - lse) : 0.f;
        dot += d[i][j] * c[i][j];
      }
    }
    // slot j of the token: lane j (and j + L ...)
    float pull = 0.f;
    if (a.dweights && there)
      for (int j = lane; j < a.k; j += L) pull += a.weights[t * a.k + j] * a.dweights[t * a.k + j];
    dot = wave_sum<L>(dot);
    pull = wave_sum<L>(pull);
    const float all = (there ? z * lse : 0.f) - dot - (a.all ? pull : 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < El::PER; ++j) d[i][j] *= c[i][j] + all;
    if (a.dweights && there)
      for (int j0 = 0; j0 < a.k; j0 += L) {
        int e = -1;
        float g = 0.f;
        if (j0 + lane < a.k) {
          const float w = a.weights[t * a.k + j0 + lane];
          e = a.experts[t * a.k + j0 + lane];
          g = w * a.dweights[t * a.k + j0 + lane] - (a.all ? 0.f : w * pull);
        }
        const int n = a.k - j0 < L ? a.k - j0 : L;
        for (int j = 0; j < n; ++j) {                          // (one after the other: an expert may be there twice)
          const int ej = __shfl(e, base + j);
          const float gj = __shfl(g, base + j);
#pragma unroll
          for (int i = 0; i < N; ++i)
#pragma unroll
            for (int r = 0; r < El::PER; ++r)
              if ((i * L + lane) * El::PER + r == ej) d[i][r] += gj;
        }
      }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = (i * L + lane) * El::PER;
      if (e < a.E) store_piece<T>(a.dlogits.data + t * a.dlogits.pitch + (size_t)e * El::BYTES, a.E - e, El::narrow(d[i]));
    }
  }
}

template <class T, int L, int N>
hipError_t go_choose_grad(const ChooseGradArgs& a, hipStream_t st) {
  const long long b = (a.tokens + 256 / L - 1) / (256 / L);
  choose_grad_kernel<T, L, N><<<dim3((unsigned)(b < 2048 ? b : 2048)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}
template <class T>
hipError_t pick_choose_grad(const ChooseGradArgs& a, hipStream_t st) {
  const int pieces = (a.E + Elem<T>::PER - 1) / Elem<T>::PER;
  constexpr int MOST = 4096 / 64 / Elem<T>::PER;
  if (pieces <= 16) return go_choose_grad<T, 16, 1>(a, st);
  if (pieces <= 32) return go_choose_grad<T, 32, 1>(a, st);
  if (pieces <= 64) return go_choose_grad<T, 64, 1>(a, st);
  if (pieces <= 256) return go_choose_grad<T, 64, 4>(a, st);
  return go_choose_grad<T, 64, MOST>(a, st);
}

}  // namespace

hipError_t launch_choose(int dtype, long long tokens, int E, int k, bool all, RowsArg logits, const uint8_t* mask, int32_t* experts, float* weights,
                         float* lse, hipStream_t st) {
  const ChooseArgs a{logits, mask, experts, weights, lse, tokens, E, k, all};
  return dtype == LASNET_F32 ? pick_choose<float>(a, st) : pick_choose<__bf16>(a, st);
}

size_t balance_workspace_bytes(long long tokens, int E) {
  const int g = balance_groups(tokens);
  return g == 1 ? 0 : (size_t)g * ((size_t)(E + 2) * sizeof(double) + (size_t)E * sizeof(int32_t));
}

hipError_t launch_balance(int dtype, long long tokens, int E, int k, RowsArg logits, const float* lse, const int32_t* experts, int32_t* counts,
                          float* share, float* loss, void* workspace, hipStream_t st) {
  const int g = balance_groups(tokens);
  double* part = (double*)workspace;
  const BalanceArgs a{logits, lse, experts, counts, share, loss, part, (int32_t*)(part + (size_t)g * (E + 2)), tokens, tokens * k, E, k, g};
  return dtype == LASNET_F32 ? pick_balance<float>(a, st) : pick_balance<__bf16>(a, st);
}

hipError_t launch_choose_grad(int dtype, long long tokens, int E, int k, bool all, RowsArg logits, const float* lse, const int32_t* experts,
                              const float* weights, const float* dweights, const int32_t* counts, const float* dloss, RowsArg dlogits,
                              hipStream_t st) {
  const ChooseGradArgs a{logits, dlogits, lse, experts, weights, dweights, counts, dloss, tokens, E, k, all};
  return dtype == LASNET_F32 ? pick_choose_grad<float>(a, st) : pick_choose_grad<__bf16>(a, st);
}

}  // namespace lasnet
