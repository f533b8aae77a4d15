// The router of a layer of experts: which experts a token goes to and how they are weighted, the balance of the experts, and the logits' gradient of both.
//
//   choice     the k largest logits of a token; weights w = softmax over those k (or over all E); lse = log sum_e exp(l[e])
//   balance    counts[e], share[e] = mean_t p[t][e] with p = exp(l - lse), loss = (E sum_e counts[e] / (k T) share[e], mean_t lse[t]^2)
//   gradient   p (c - sum_e p c) + 2 lse p d1 / T + that of the weights, with c[e] = d0 E counts[e] / (k T^2)
//
// A token's logits lie in the registers of L lanes (8 to 64), read once.  Exponentials, sums and statistics are held in 32 bits, sums over tokens in 64; only the
// gradient is rounded, once, to the logits' type.
#include <utility>

#include "row_ops.hpp"

namespace lasnet {
namespace {

// ---- order: a key that is larger for what is chosen earlier.  NaN is above everything; -inf (and what is beyond the row) is never chosen: kNone and less. ----
constexpr unsigned kNone = 0x007fffffu;
__device__ __forceinline__ unsigned key_of(float v) {
  unsigned u = __float_as_uint(v + 0.f);                       // (-0 + 0 = 0: equal values are equal keys)
  u = v != v ? 0x7fffffffu : u;
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu)); }

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

// The exchanges that sort C numbers: Batcher's odd-even merge sort.
template <int C>
struct Exchanges {
  int n = 0, a[64] = {}, b[64] = {};
  constexpr Exchanges() {
    for (int p = 1; p < C; p *= 2)
      for (int q = p; q >= 1; q /= 2)
        for (int j = q % p; j + q < C; j += 2 * q)
          for (int i = 0; i < q && i + j + q < C; ++i)
            if ((i + j) / (2 * p) == (i + j + q) / (2 * p)) {
              a[n] = i + j;
              b[n++] = i + j + q;
            }
  }
};
// The lane's C keys, largest first.
template <int C, int... I>
__device__ __forceinline__ void exchange_keys(unsigned (&key)[C], std::integer_sequence<int, I...>) {
  constexpr Exchanges<C> x;
  auto one = [&](auto a, auto b) {
    const unsigned u = key[a.value], v = key[b.value];
    key[a.value] = u > v ? u : v;
    key[b.value] = u > v ? v : u;
  };
  (one(std::integral_constant<int, x.a[I]>{}, std::integral_constant<int, x.b[I]>{}), ...);
}
template <int C>
__device__ __forceinline__ void sort_keys(unsigned (&key)[C]) {
  exchange_keys(key, std::make_integer_sequence<int, Exchanges<C>{}.n>{});
}

// L lanes a token, N pieces of 16 bytes each, one behind the other: a lower lane has the lower experts.  k <= L: lane j keeps the j-th choice.
//
// A choice is a maximum over the lanes.  bf16: the 16 bits of a value's key and those of its expert are one number, no two are equal, and one maximum gives both; up to 16 a lane
// are sorted once, so that a choice costs its lane a shift.  fp32: the maximum, then the lowest expert that has it.  Bound by these instructions (memory would take 1.9):
// 16384 tokens of 256 experts bf16, 8 each, 6.4 to 7.3 us.  Unsorted keys and maxima through LDS: 13.2.  8 tokens of 64 experts, 2.2: a launch and one token's chain.
template <class T, int L, int N>
__global__ __launch_bounds__(256) void choose_kernel(ChooseArgs a) {
  using El = Elem<T>;
  constexpr int C = N * El::PER;                               // logits of a lane
  constexpr bool PACKED = El::BYTES == 2, SORTED = PACKED && C <= 16;
  const int lane = (int)threadIdx.x % L;
  for (long long t = (long long)blockIdx.x * (256 / L) + threadIdx.x / L; t < a.tokens; t += (long long)gridDim.x * (256 / L)) {
    const bool there = !a.mask || a.mask[t];
    float v[C];
    unsigned key[C];
    uint4_t piece[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (lane * N + i) * El::PER;
      piece[i] = load_piece<T>(a.logits.data + t * a.logits.pitch + (size_t)c * El::BYTES, there ? a.E - c : 0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (lane * N + i) * El::PER, left = there ? a.E - c : 0;
      float f[El::PER];
      El::widen(piece[i], f);
      if (left < El::PER)
#pragma unroll
        for (int j = 0; j < El::PER; ++j) f[j] = j < left ? f[j] : -INFINITY;
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        v[i * El::PER + j] = f[j];
        key[i * El::PER + j] = PACKED ? (key_of(f[j]) & 0xffff0000u) | (0xffffu - (unsigned)(c + j)) : key_of(f[j]);
      }
    }
    // (a packed key's value: the 16 bits that the expert took were zeros of the value, so ones of a negative one's key)
    auto value = [](unsigned m) { return value_of(!PACKED ? m : m & 0x80000000u ? m & 0xffff0000u : m | 0xffffu); };
    if constexpr (SORTED) sort_keys(key);
    unsigned best = key[0];
    if constexpr (!SORTED)
#pragma unroll
      for (int c = 1; c < C; ++c) best = key[c] > best ? key[c] : best;
    unsigned m = lanes_max<L>(best);
    const float top = value(m);                                // (of a token without a candidate: -inf)
    // (NaN or +inf: nothing, which makes NaN of what follows; -inf less itself, too, which makes 0 of it)
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) sum += exp_below(v[c] - top);
    sum = lanes_sum<L>(sum);
    unsigned mine = 0;                                         // the key of this lane's choice
    int expert = -1;
    if constexpr (SORTED) {
      auto take = [&](auto most) {                             // most: keys that a lane may give up
        constexpr int M = decltype(most)::value;
        for (int j = 0; j < a.k; ++j) {
          m = lanes_max<L>(key[0]);
          if (lane == j) mine = m;
          const bool won = key[0] == m;
#pragma unroll
          for (int c = 0; c < M; ++c) {
            const unsigned next = c + 1 < C ? key[c + 1 < C ? c + 1 : c] : 0u, now = key[c];
            key[c] = won ? next : now;
          }
        }
      };
      if (a.k <= 4 && C > 4) take(std::integral_constant<int, 4>{});
      else if (a.k <= 8 && C > 8) take(std::integral_constant<int, 8>{});
      else take(std::integral_constant<int, C>{});
      if (mine > kNone) expert = (int)(0xffffu - (mine & 0xffffu));
    } else {
      for (int j = 0; j < a.k; ++j) {
        best = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) best = key[c] > best ? key[c] : best;
        m = lanes_max<L>(best);
        int e;
        if constexpr (PACKED) {
          e = (int)(0xffffu - (m & 0xffffu));
        } else {
          int at = 0;
#pragma unroll
          for (int c = C - 1; c >= 0; --c) at = key[c] == m ? c : at;
          e = (int)lanes_min<L>(best == m ? (unsigned)(lane * C + at) : 0xffffffffu);
        }
        if (lane == j) {
          mine = m;
          expert = m > kNone ? e : -1;
        }
        const int gone = e - lane * C;
#pragma unroll
        for (int c = 0; c < C; ++c) key[c] = gone == c ? 0u : key[c];
      }
    }
    const float lse = top + logf(sum);
    float w = expert >= 0 ? exp_below(value(mine) - top) : 0.f;
    const float chosen = lanes_sum<L>(lane < a.k ? w : 0.f);
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
// As few lanes a token as hold it: 65536 tokens of 60 experts bf16, 6 each, by 8 lanes 7.2 us, by 16 11.8.
template <class T>
hipError_t pick_choose(const ChooseArgs& a, hipStream_t st) {
  constexpr int PER = Elem<T>::PER, SIXTEEN = 16 / PER;        // pieces of sixteen logits
  const int pieces = (a.E + PER - 1) / PER;
  if (pieces <= 8 && a.k <= 8) return go_choose<T, 8, 1>(a, st);
  if (a.k <= 16) {
    if (pieces <= 16) return go_choose<T, 16, 1>(a, st);
    if (SIXTEEN == 4 && pieces <= 32) return go_choose<T, 16, 2>(a, st);
    if (a.E <= 256) return go_choose<T, 16, SIXTEEN>(a, st);
  }
  if (a.k <= 32 && a.E <= 512) return go_choose<T, 32, SIXTEEN>(a, st);
  if (pieces <= 64) return go_choose<T, 64, 1>(a, st);
  if (a.E <= 1024) return go_choose<T, 64, SIXTEEN>(a, st);
  return go_choose<T, 64, 64 / PER>(a, st);
}

// ---- balance ----
// Two launches: workgroups sum runs of tokens, others join the sums of 64 columns each; the last of those to end (a counter tells, which the first launch cleared) adds up the loss
// from their parts, in order.  One launch where one workgroup does.
//
// 32768 tokens of 256 experts fp32 (34 MB, 6.5 us from memory) 9.5 us and 6.0 for the join, 4099 of 60 bf16 6.6 and 4.7: what two launches, the second waiting for the first, take to begin, to read
// and to join their waves.  Of both calls' 15.8 and 11.7 us the count of the slots, which comes before the first logits, is 0.4, the exponentials 0.4 and 0.3 (16384 of 1000 bf16: 3.4 of 20.6).
// Workgroups of 256 or 512 threads, or loads further ahead, took as long.
constexpr int kBalance = 1024;                                 // threads of a workgroup
constexpr int kJoinCols = 64;                                  // columns of a workgroup of the second launch
constexpr int kBalanceUnits = 4098;                            // doubles of LDS: one unit's of the most experts

struct BalanceArgs {
  RowsArg logits;
  const float* lse;
  const int32_t* experts;
  int32_t* counts;
  float* share;
  float* loss;
  double* part;                    // [groups][E + 2]: sums of p; of lse^2; tokens
  double* part_loss;               // [workgroups of the second launch]
  int32_t* part_counts;            // [groups][E]
  unsigned* ended;
  long long tokens, slots;
  int E, k, groups;
};

// The loss from sum_e counts share and the sum of squares.
__device__ __forceinline__ void put_loss(const BalanceArgs& a, double sum, double squares, double tokens) {
  const double T = tokens > 0. ? tokens : 1.;
  a.loss[0] = (float)(sum * ((double)a.E / ((double)a.k * T)));
  a.loss[1] = (float)(squares / T);
  a.counts[a.E] = (int)tokens;
}
// The sum over lanes that lie D, 2 D ... apart (of 16 and 32), in each of them.
template <int D>
__device__ __forceinline__ double far_sum(double v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
  const unsigned lo = (unsigned)u, hi = (unsigned)(u >> 32);
  auto of = [](unsigned l, unsigned h) { return __builtin_bit_cast(double, (unsigned long long)h << 32 | l); };
  if constexpr (D == 16) {
    const auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    return of(l[0], h[0]) + of(l[1], h[1]);
  } else {
    const auto l = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return of(l[0], h[0]) + of(l[1], h[1]);
  }
}
// The sum over a wave, the same bits in each lane (see lanes_join).
__device__ __forceinline__ double lanes_sum(double v) {
  auto turned = [&](auto by) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, 0x120 + decltype(by)::value, 0xf, 0xf, true);           // row_ror
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), 0x120 + decltype(by)::value, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
  };
  v += turned(std::integral_constant<int, 8>{});
  v += turned(std::integral_constant<int, 4>{});
  v += turned(std::integral_constant<int, 2>{});
  v += turned(std::integral_constant<int, 1>{});
  return far_sum<32>(far_sum<16>(v));
}
// Sum of the workgroup's values, in every thread.  join: 16 doubles, one set for each call.
__device__ __forceinline__ double join_all(double v, double* join) {
  v = lanes_sum(v);
  if ((threadIdx.x & 63) == 0) join[threadIdx.x >> 6] = v;
  __syncthreads();
  double sum = 0.;
#pragma unroll
  for (int w = 0; w < kBalance / 64; ++w) sum += join[w];
  return sum;
}

// Groups of L lanes take tokens in turn, U at once; a lane keeps its columns' sums.
template <class T, int L>
__global__ __launch_bounds__(kBalance) void balance_kernel(BalanceArgs a) {
  using El = Elem<T>;
  constexpr int G = kBalance / L, U = 4, C = El::PER;
  __shared__ double join[kBalance / 64];
  __shared__ double units[kBalanceUnits];                      // [P][E + 2]: the sums of P units (waves, or groups of more)
  __shared__ int hist[4096];
  const int tid = (int)threadIdx.x, lane = tid % L, group = tid / L, c0 = lane * C;      // c0: the lane's first column
  if (blockIdx.x == 0 && tid == 0 && a.groups > 1) *a.ended = 0;
  for (int e = tid; e < a.E; e += kBalance) hist[e] = 0;
  __syncthreads();
  for (long long s0 = (long long)blockIdx.x * kBalance + tid; s0 < a.slots; s0 += 4ll * gridDim.x * kBalance) {
    int e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long s = s0 + (long long)i * gridDim.x * kBalance;
      e[i] = s < a.slots ? a.experts[s] : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e[i] >= 0 && e[i] < a.E) atomicAdd(&hist[e[i]], 1);  // (whole numbers in LDS: any order gives the same)
  }
  double acc[C] = {}, squares = 0., tokens = 0.;
  const long long stride = (long long)gridDim.x * G;
  for (long long t0 = (long long)blockIdx.x * G + group; t0 < a.tokens; t0 += U * stride) {
    float lse[U];
    uint4_t piece[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long t = t0 + u * stride;
      lse[u] = t < a.tokens ? a.lse[t] : -INFINITY;
      piece[u] = load_piece<T>(a.logits.data + t * a.logits.pitch + (size_t)c0 * El::BYTES, t < a.tokens ? a.E - c0 : 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (lse[u] == -INFINITY) continue;
      squares += (double)lse[u] * lse[u];
      tokens += 1.;
      float f[C];
      El::widen(piece[u], f);
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] += (double)exp_of(f[j] - lse[u]);
    }
  }
  // the sums of a wave's tokens (lanes with the same columns), then of all units: as many at a time as LDS has room for
  auto same_columns = [](double v) {
    if constexpr (L <= 16) v = far_sum<16>(v);
    if constexpr (L <= 32) v = far_sum<32>(v);
    return v;
  };
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = same_columns(acc[c]);
  squares = same_columns(squares);
  tokens = same_columns(tokens);
  const int all = a.E + 2;                                     // columns, squares and tokens behind them
  constexpr int UNIT = L < 64 ? 64 : L, UNITS = kBalance / UNIT, COLS = (C * L + 2 + kBalance - 1) / kBalance;
  const int P = kBalanceUnits / all < UNITS ? kBalanceUnits / all : UNITS;
  double sums[COLS] = {};                                      // of columns tid, tid + 1024 ...
  for (int u0 = 0; u0 < UNITS; u0 += P) {
    const int u = tid / UNIT - u0;
    if (u >= 0 && u < P && tid % UNIT < L) {
#pragma unroll
      for (int j = 0; j < C; ++j)
        if (c0 + j < a.E) units[u * all + c0 + j] = acc[j];
      if (lane == 0) {
        units[u * all + a.E] = squares;
        units[u * all + a.E + 1] = tokens;
      }
    }
    __syncthreads();
    const int n = UNITS - u0 < P ? UNITS - u0 : P;
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      const int e = tid + x * kBalance;
      if (e < all)
#pragma unroll 4
        for (int v = 0; v < n; ++v) sums[x] += units[v * all + e];
    }
    __syncthreads();
  }
  if (a.groups == 1) {
#pragma unroll
    for (int x = 0; x < COLS; ++x)
      if (tid + x * kBalance >= a.E && tid + x * kBalance < all) units[tid + x * kBalance - a.E] = sums[x];
    __syncthreads();
    squares = units[0];
    tokens = units[1];
    double loss = 0.;
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      const int e = tid + x * kBalance;
      if (e < a.E) {
        const double share = sums[x] / (tokens > 0. ? tokens : 1.);
        a.counts[e] = hist[e];
        a.share[e] = (float)share;
        loss += (double)hist[e] * share;
      }
    }
    loss = join_all(loss, join);
    if (tid == 0) put_loss(a, loss, squares, tokens);
    return;
  }
  double* part = a.part + (long long)blockIdx.x * all;
#pragma unroll
  for (int x = 0; x < COLS; ++x)
    if (tid + x * kBalance < all) part[tid + x * kBalance] = sums[x];
  for (int e = tid; e < a.E; e += kBalance) a.part_counts[(long long)blockIdx.x * a.E + e] = hist[e];
}

// A wave takes 64 columns of every 16th part.
__global__ __launch_bounds__(kBalance) void balance_join_kernel(BalanceArgs a) {
  constexpr int W = kBalance / 64;
  __shared__ double join[2][W];
  __shared__ double sums[W][kJoinCols];
  __shared__ int counts[W][kJoinCols];
  __shared__ int last;
  const int tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63, e = (int)blockIdx.x * kJoinCols + lane;
  double squares = 0., tokens = 0., sum = 0., loss = 0.;
  int count = 0;
  if (tid < a.groups) {
    squares = a.part[(long long)tid * (a.E + 2) + a.E];
    tokens = a.part[(long long)tid * (a.E + 2) + a.E + 1];
  }
  if (e < a.E)
#pragma unroll 8
    for (int g = wave; g < a.groups; g += W) {
      sum += a.part[(long long)g * (a.E + 2) + e];
      count += a.part_counts[(long long)g * a.E + e];
    }
  sums[wave][lane] = sum;
  counts[wave][lane] = count;
  squares = lanes_sum(squares);
  tokens = lanes_sum(tokens);
  if (lane == 0) {
    join[0][wave] = squares;
    join[1][wave] = tokens;
  }
  __syncthreads();
  if (wave == 0) {
    squares = tokens = 0.;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      squares += join[0][w];
      tokens += join[1][w];
    }
    sum = 0.;
    count = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      sum += sums[w][lane];
      count += counts[w][lane];
    }
    const double share = sum / (tokens > 0. ? tokens : 1.);
    if (e < a.E) {
      a.counts[e] = count;
      a.share[e] = (float)share;
      loss = (double)count * share;
    }
    loss = lanes_sum(loss);
    if (gridDim.x == 1) {
      if (lane == 0) put_loss(a, loss, squares, tokens);
    } else if (lane == 0) {
      a.part_loss[blockIdx.x] = loss;
      __threadfence();
      last = atomicAdd(a.ended, 1u) == gridDim.x - 1;
    }
  }
  if (gridDim.x == 1) return;
  __syncthreads();
  if (!last || wave) return;
  __threadfence();
  loss = lane < (int)gridDim.x ? __hip_atomic_load(a.part_loss + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.;
  loss = lanes_sum(loss);
  if (lane == 0) put_loss(a, loss, squares, tokens);
}

constexpr int kMostGroups = 256;
// Workgroups of a call: one for what it reads as soon as a second launch would start, else two logits a thread, and no more than there are CUs.
int balance_groups(long long tokens, int E) {
  const long long g = tokens * E / (2 * kBalance);
  return g <= 8 ? 1 : g < kMostGroups ? (int)g : kMostGroups;
}
int join_groups(int E) { return (E + kJoinCols - 1) / kJoinCols; }

template <class T, int L>
hipError_t go_balance(const BalanceArgs& a, hipStream_t st) {
  balance_kernel<T, L><<<dim3((unsigned)a.groups), dim3(kBalance), 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.groups == 1) return e;
  balance_join_kernel<<<dim3((unsigned)join_groups(a.E)), dim3(kBalance), 0, st>>>(a);
  return hipGetLastError();
}
// 23948 tokens of 340 experts fp32 by 128 lanes each 17.2 us, by 256 22.7.
template <class T>
hipError_t pick_balance(const BalanceArgs& a, hipStream_t st) {
  const int pieces = (a.E + Elem<T>::PER - 1) / Elem<T>::PER;
  if (pieces <= 16) return go_balance<T, 16>(a, st);
  if (pieces <= 32) return go_balance<T, 32>(a, st);
  if (pieces <= 64) return go_balance<T, 64>(a, st);
  if (pieces <= 128) return go_balance<T, 128>(a, st);
  if (pieces <= 256) return go_balance<T, 256>(a, st);
  return go_balance<T, 1024>(a, st);
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

// L lanes a token.  The weights' part lands on k of the E logits: each slot's lane writes its number to its expert's place in a row of LDS and reads it back, which tells whether any
// expert is there twice (then the slots add one after the other); its part goes the same way, and the lanes that hold the logits read the row.
// 32768 tokens of 256 experts fp32, 8 each, 15.6 us: memory (69 MB, 13.4 us); 4099 of 60 bf16, 5.4.
template <class T, int L, int N>
__global__ __launch_bounds__(256) void choose_grad_kernel(ChooseGradArgs a) {
  using El = Elem<T>;
  extern __shared__ __attribute__((aligned(16))) float grad_rows[];                       // [256 / L][pitch]
  const int lane = (int)threadIdx.x % L, pitch = (a.E + 3) / 4 * 4;
  float* row = grad_rows + (int)threadIdx.x / L * pitch;
  if (a.dweights)
    for (int e = lane; e < pitch; e += L) row[e] = 0.f;
  // what a probability of 1 would get from the balance loss, expert by expert
  float c[N][El::PER] = {}, z = 0.f;
  bool wild = false;
  if (a.dloss) {
    const float T_ = (float)(a.counts[a.E] > 0 ? a.counts[a.E] : 1), unit = a.dloss[0] / T_ * ((float)a.E / ((float)a.k * T_));
    z = 2.f * a.dloss[1] / T_;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        const int e = (i * L + lane) * El::PER + j;
        if (e < a.E) c[i][j] = unit * (float)a.counts[e];
        if (!(fabsf(c[i][j]) < INFINITY)) {
          wild = true;
          c[i][j] = 0.f;
        }
      }
    // An infinite or NaN dloss makes NaN of the tokens that take part, through a term that only they have: 0 times it would reach the others, which get zeros.
    if (__ballot(wild)) z = __uint_as_float(0x7fc00000u);
  }
  const unsigned long long group = (L == 64 ? ~0ull : (1ull << (L & 63)) - 1) << ((int)(threadIdx.x & 63) / L * L);     // the group's lanes
  // what is read of a token; the next one's is asked for before this one's is used.  Slot j: lane j (and j + L ...).
  struct Token {
    float lse, w, dw;
    int expert;
    uint4_t piece[N];
  };
  auto fetch = [&](long long t, Token& k) {
    k.lse = a.lse[t];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = (i * L + lane) * El::PER;
      k.piece[i] = load_piece<T>(a.logits.data + t * a.logits.pitch + (size_t)e * El::BYTES, a.E - e);
    }
    k.w = k.dw = 0.f;
    k.expert = -1;
    if (a.dweights && lane < a.k) {
      k.w = a.weights[t * a.k + lane];
      k.dw = a.dweights[t * a.k + lane];
      k.expert = a.experts[t * a.k + lane];
    }
  };
  auto weighed = [](float w, float dw) { return w == 0.f ? 0.f : dw; };         // (of a slot without weight: nothing, also of NaN)
  const long long stride = (long long)gridDim.x * (256 / L);
  long long t = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= a.tokens) return;
  Token now, next;
  fetch(t, now);
  for (; t < a.tokens; t += stride, now = next) {
    fetch(t + stride < a.tokens ? t + stride : t, next);
    const float lse = now.lse, w = now.w, dw = weighed(w, now.dw);
    const bool there = lse != -INFINITY, own = a.dweights && there;
    const int expert = now.expert;
    float pull = 0.f;
    if (own) {
      pull = w * dw;
      for (int j = lane + L; j < a.k; j += L) pull += a.weights[t * a.k + j] * weighed(a.weights[t * a.k + j], a.dweights[t * a.k + j]);
      pull = lanes_sum<L>(pull);
    }
    float d[N][El::PER], dot = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = (i * L + lane) * El::PER;
      float f[El::PER];
      El::widen(now.piece[i], f);
#pragma unroll
      for (int j = 0; j < El::PER; ++j) {
        d[i][j] = there && e + j < a.E ? exp_of(f[j] - lse) : 0.f;
        dot += d[i][j] * c[i][j];
      }
    }
    if (a.dloss) dot = lanes_sum<L>(dot);
    const float all = (there ? z * lse : 0.f) - dot - (a.all ? pull : 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < El::PER; ++j) d[i][j] *= c[i][j] + all;
    if (own) {
      auto part = [&](float v, float dv) { return v * dv - (a.all ? 0.f : v * pull); };
      auto fence = [] { asm volatile("" ::: "memory"); };      // (the compiler: LDS is written and read by other lanes of the wave, which it does in order)
      const bool sent = expert >= 0 && expert < a.E;
      if (sent) ((int*)row)[expert] = lane;
      fence();
      const bool twice = sent && ((volatile int*)row)[expert] != lane;
      const bool alone = a.k <= L && !(__ballot(twice) & group);
      fence();
      if (alone) {
        if (sent) row[expert] = part(w, dw);
      } else {
        if (sent) row[expert] = 0.f;
        fence();
        for (int j = 0; j < a.k; ++j) {                        // by the group's first lane, slot after slot
          const int e = a.experts[t * a.k + j];
          const float v = a.weights[t * a.k + j], dv = weighed(v, a.dweights[t * a.k + j]);
          if (lane == 0 && e >= 0 && e < a.E) row[e] += part(v, dv);
          fence();
        }
      }
      fence();
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < El::PER; j += 4) {
          const int e = (i * L + lane) * El::PER + j;
          if (e < a.E) {
            const floatx4 g = *(const floatx4*)(row + e);
#pragma unroll
            for (int r = 0; r < 4; ++r) d[i][j + r] += g[r];
          }
        }
      fence();
      if (sent) row[expert] = 0.f;
      for (int j = lane + L; j < a.k; j += L) {
        const int e = a.experts[t * a.k + j];
        if (e >= 0 && e < a.E) row[e] = 0.f;
      }
      fence();
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
  const int bytes = a.dweights ? 256 / L * ((a.E + 3) / 4 * 4) * 4 : 0;
  choose_grad_kernel<T, L, N><<<dim3((unsigned)(b < 2048 ? b : 2048)), dim3(256), bytes, st>>>(a);
  return hipGetLastError();
}
// 65536 tokens of 60 experts bf16 by 8 lanes 12.3 us, by 16 15.3; 23948 of 340 fp32 in two pieces a lane 17.3, in four 23.0.
template <class T>
hipError_t pick_choose_grad(const ChooseGradArgs& a, hipStream_t st) {
  const int pieces = (a.E + Elem<T>::PER - 1) / Elem<T>::PER;
  constexpr int MOST = 4096 / 64 / Elem<T>::PER;
  if (pieces <= 8 && a.k <= 8) return go_choose_grad<T, 8, 1>(a, st);
  if (pieces <= 16) return go_choose_grad<T, 16, 1>(a, st);
  if (pieces <= 32) return go_choose_grad<T, 32, 1>(a, st);
  if (pieces <= 64) return go_choose_grad<T, 64, 1>(a, st);
  if (pieces <= 128) return go_choose_grad<T, 64, 2>(a, st);
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
  const int g = balance_groups(tokens, E);
  return g == 1 ? 0 : ((size_t)g * (E + 2) + join_groups(E)) * sizeof(double) + ((size_t)g * E + 1) * sizeof(int32_t);
}

hipError_t launch_balance(int dtype, long long tokens, int E, int k, RowsArg logits, const float* lse, const int32_t* experts, int32_t* counts,
                          float* share, float* loss, void* workspace, hipStream_t st) {
  const int g = balance_groups(tokens, E);
  double *part = (double*)workspace, *part_loss = part + (size_t)g * (E + 2);
  int32_t* part_counts = (int32_t*)(part_loss + join_groups(E));
  const BalanceArgs a{logits, lse, experts, counts, share, loss, part, part_loss, part_counts, (unsigned*)(part_counts + (size_t)g * E), tokens, tokens * k, E, k, g};
  return dtype == LASNET_F32 ? pick_balance<float>(a, st) : pick_balance<__bf16>(a, st);
}

hipError_t launch_choose_grad(int dtype, long long tokens, int E, int k, bool all, RowsArg logits, const float* lse, const int32_t* experts,
                              const float* weights, const float* dweights, const int32_t* counts, const float* dloss, RowsArg dlogits,
                              hipStream_t st) {
  const ChooseGradArgs a{logits, dlogits, lse, experts, weights, dweights, counts, dloss, tokens, E, k, all};
  return dtype == LASNET_F32 ? pick_choose_grad<float>(a, st) : pick_choose_grad<__bf16>(a, st);
}

}  // namespace lasnet
