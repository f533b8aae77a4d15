// Rows to experts and back: slots sorted by expert, rows laid out in that order, weighted sums of them, and the gradients.
//
// The sort is a stable counting sort.  A wave takes a run of consecutive slots, 64 at a time: lanes with the same expert find each other
// by one ballot for each bit of its number, the first of them adds their count to the wave's table in LDS, and a lane's rank is the
// table's value before plus the lanes ahead of it.  What moves rows is bound by memory: each token's row is read once, the k copies are written
// (or read) once, and sums run over j in order, so nothing depends on timing.
//
//   sort: a chain of LDS and memory accesses: 32 slots of 64 experts 3 us, 65536 11, 4 Mi 67 (of 8 experts 56, of 256 115).  Rows, at the rate of large copies: dispatch of 16384 x 2048 bf16 to
//   four experts each (335 MB) with the sort 60 us, sum of them into the residual (386 MB) 74, its gradient (604 MB) 109.
#include "row_ops.hpp"

namespace lasnet {
namespace {

// ---- the sort ----
struct RouteArgs {
  const int32_t* experts;
  long long slots;
  int E, bits;                     // bits of E - 1
  int32_t* offsets;
  int32_t* order;
  int32_t* position;
  int32_t* counts;                 // [runs][E], several workgroups: a run's slots for each expert
  int runs;
  long long run;                   // slots of a run
};

// Lanes whose key is this lane's (valid lanes only).
__device__ __forceinline__ unsigned long long same_key(int key, bool valid, int bits) {
  unsigned long long m = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const bool one = (key >> b) & 1;
    const unsigned long long v = __ballot(one);
    m &= one ? v : ~v;
  }
  return m;
}
__device__ __forceinline__ unsigned long long lanes_before(int lane) { return (1ull << lane) - 1; }

// Keys of 256 slots from s on, four a lane, all requested at once.
struct Keys { int of[4]; };
__device__ __forceinline__ Keys load_keys(const RouteArgs& a, long long s, long long end) {
  const int lane = (int)threadIdx.x & 63;
  Keys k;
#pragma unroll
  for (int r = 0; r < 4; ++r) k.of[r] = s + 64 * r + lane < end ? a.experts[s + 64 * r + lane] : -1;
  return k;
}
// Counts of one wave's slots [first, end) into its table.
__device__ __forceinline__ void count_slots(const RouteArgs& a, long long first, long long end, int* table) {
  const int lane = (int)threadIdx.x & 63;
  for (long long s = first; s < end; s += 256) {
    const Keys k = load_keys(a, s, end);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (s + 64 * r >= end) break;
      const int key = k.of[r];
      const bool valid = (unsigned)key < (unsigned)a.E;
      const unsigned long long m = same_key(key, valid, a.bits);
      if (valid && !(m & lanes_before(lane))) atomicAdd(&table[key], __popcll(m));
    }
  }
}
// ... and their places, from the table of the first free row of each expert.
__device__ __forceinline__ void place_slots(const RouteArgs& a, long long first, long long end, int* table) {
  const int lane = (int)threadIdx.x & 63;
  for (long long s = first; s < end; s += 256) {
    const Keys k = load_keys(a, s, end);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const long long slot = s + 64 * r + lane;
      if (s + 64 * r >= end) break;
      const int key = k.of[r];
      const bool valid = (unsigned)key < (unsigned)a.E;
      const unsigned long long m = same_key(key, valid, a.bits);
      const int ahead = __popcll(m & lanes_before(lane));
      int at = 0;
      if (valid && !ahead) at = atomicAdd(&table[key], __popcll(m));
      at = __shfl(at, valid ? __ffsll((long long)m) - 1 : lane) + ahead;
      if (slot < end) a.position[slot] = valid ? at : -1;
      if (valid && a.order) a.order[at] = (int32_t)slot;
    }
  }
}

// Exclusive scan of f(0..n) over one wave, 64 at a time, g(i, sum before i); returns the total.
template <class F, class G>
__device__ __forceinline__ int wave_scan(int n, F f, G g) {
  const int lane = (int)threadIdx.x & 63;
  int before = 0;
  for (int i = lane; i - lane < n; i += 64) {
    const int v = i < n ? f(i) : 0;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(s, d);
      if (lane >= d) s += u;
    }
    if (i < n) g(i, before + s - v);
    before += __shfl(s, 63);
  }
  return before;
}

constexpr int kRouteTable = 8192;          // entries of LDS tables in a workgroup
__host__ __device__ inline int route_waves(int E) { return E <= kRouteTable / 16 ? 16 : kRouteTable / E; }      // E up to 4096: at least 2

// Places of a workgroup's slots [first, end): its waves' runs are counted, the counts summed over the waves before each, and the rows before the
// workgroup's first of each expert added: between() makes the tables' columns exclusive sums from there.
template <class Between>
__device__ __forceinline__ void place_run(const RouteArgs& a, long long first, long long end, int* table, Between between) {
  const int nw = (int)blockDim.x >> 6, wave = (int)threadIdx.x >> 6;
  const long long per = (end - first + 64 * nw - 1) / (64 * nw) * 64;
  const long long mine = first + per * wave, mine_end = mine + per < end ? mine + per : end;
  for (int i = (int)threadIdx.x; i < nw * a.E; i += blockDim.x) table[i] = 0;
  __syncthreads();
  count_slots(a, mine, mine_end, table + wave * a.E);
  __syncthreads();
  between();
  __syncthreads();
  place_slots(a, mine, mine_end, table + wave * a.E);
}
// Column e of the waves' tables, exclusively summed from `sum` on; returns the sum behind the last.
__device__ __forceinline__ int stack_column(const RouteArgs& a, int* table, int e, int sum) {
  const int nw = (int)blockDim.x >> 6;
  for (int w = 0; w < nw; ++w) {
    const int v = table[w * a.E + e];
    table[w * a.E + e] = sum;
    sum += v;
  }
  return sum;
}
// starts[e] <- the sum of starts before e, by wave 0; offsets too where `write`, and order beyond the last row.
__device__ __forceinline__ int scan_starts(const RouteArgs& a, int* starts, bool write) {
  const int sent = wave_scan(a.E, [&](int e) { return starts[e]; }, [&](int e, int v) {
    starts[e] = v;
    if (write) a.offsets[e] = v;
  });
  if (write && threadIdx.x == 0) a.offsets[a.E] = sent;
  return sent;
}

// Few slots: one workgroup does it all.
__global__ __launch_bounds__(1024) void route_one_kernel(RouteArgs a) {
  __shared__ int table[kRouteTable];
  __shared__ int starts[4096];
  const int nw = (int)blockDim.x >> 6, tid = (int)threadIdx.x;
  place_run(a, 0, a.slots, table, [&] {
    for (int e = tid; e < a.E; e += blockDim.x) starts[e] = stack_column(a, table, e, 0);
    __syncthreads();
    if (tid < 64) {
      const int sent = scan_starts(a, starts, true);
      if (a.order)
        for (long long p = sent + tid; p < a.slots; p += 64) a.order[p] = -1;
    }
    __syncthreads();
    for (int i = tid; i < nw * a.E; i += blockDim.x) table[i] += starts[i % a.E];
  });
}

// Many slots: a run of them for each workgroup.  Its counts first; then every workgroup adds up the counts of the runs before its own (and of all, for the
// offsets) and places its slots.  See route_run for how many there are.
__global__ __launch_bounds__(256) void route_count_kernel(RouteArgs a) {
  __shared__ int table[4096];
  for (int e = (int)threadIdx.x; e < a.E; e += 256) table[e] = 0;
  __syncthreads();
  const long long first = a.run * blockIdx.x, end = first + a.run < a.slots ? first + a.run : a.slots;
  const long long per = (end - first + 255) / 256 * 64, mine = first + per * ((int)threadIdx.x >> 6);
  count_slots(a, mine, mine + per < end ? mine + per : end, table);
  __syncthreads();
  for (int e = (int)threadIdx.x; e < a.E; e += 256) a.counts[(size_t)blockIdx.x * a.E + e] = table[e];
}
__global__ __launch_bounds__(256) void route_place_kernel(RouteArgs a) {
  __shared__ int table[kRouteTable];
  __shared__ int starts[4096], before[4096];                  // rows of each expert: of all runs, of those before this one
  const int tid = (int)threadIdx.x, nw = (int)blockDim.x >> 6, run = (int)blockIdx.x;
  const long long first = a.run * run, end = first + a.run < a.slots ? first + a.run : a.slots;
  for (int e = tid; e < a.E; e += blockDim.x) starts[e] = before[e] = 0;
  place_run(a, first, end, table, [&] {
    const int share = (a.runs + nw - 1) / nw, r0 = (tid >> 6) * share, r1 = r0 + share < a.runs ? r0 + share : a.runs;
    for (int e = tid & 63; e < a.E; e += 64) {
      int here = 0, all = 0;
#pragma unroll 16
      for (int r = r0; r < r1; ++r) {
        const int v = a.counts[(size_t)r * a.E + e];
        here += r < run ? v : 0;
        all += v;
      }
      atomicAdd(&starts[e], all);
      atomicAdd(&before[e], here);
    }
    __syncthreads();
    if (tid < 64) {
      const int sent = scan_starts(a, starts, run == 0);
      if (a.order)
        for (long long p = first + tid; p < end; p += 64)
          if (p >= sent) a.order[p] = -1;
    }
    __syncthreads();
    for (int e = tid; e < a.E; e += blockDim.x) stack_column(a, table, e, before[e] + starts[e]);
  });
}
// Up to so many slots one workgroup sorts (of 64 experts: 4096 slots 7.3 us, by two launches 9.4; 8192 slots 11.7 and 10.2).
constexpr long long kRouteOne = 6144;
// Slots of a workgroup: whole waves of 64.  Every workgroup adds up runs * E counts, so of many experts there are fewer runs: 4 Mi slots of 8 experts 57.8 us in
// 1024 runs, 71.7 in 256; of 256 experts 136.5 and 114.3 (64 runs 390).
long long route_run(long long slots, int E) {
  const long long most = E <= 64 ? 1024 : E <= 1024 ? 256 : 128;
  const long long least = 1024, run = (slots + most - 1) / most;
  return run < least ? least : (run + 255) / 256 * 256;
}

// ---- rows ----
// A group of `width` threads (a power of two from 16 to 256) takes a token; the groups of all workgroups go through the tokens.  16384 x 64 bf16, four each: groups
// of 16 threads 4.0 us, of 256 15.5; 16384 x 1024: 26 either way.
struct Groups {
  int width;                       // threads of a group
  int pieces;                      // of 16 bytes in a row, the last one may have less
  int part;                        // pieces of a row that a workgroup (blockIdx.y) takes
  __device__ __forceinline__ int first() const { return (int)blockIdx.y * part; }
  __device__ __forceinline__ int end() const { return first() + part < pieces ? first() + part : pieces; }
};
__device__ __forceinline__ long long first_group(int width) { return ((long long)blockIdx.x * 256 + threadIdx.x) / width; }
__device__ __forceinline__ long long group_count(int width) { return (long long)gridDim.x * (256 / width); }
Groups groups_for(long long tokens, int row_bytes, int least) {
  Groups g{least, (row_bytes + 15) / 16, 0};
  while (g.width < 256 && g.width < g.pieces) g.width *= 2;
  // Few tokens with wide rows: workgroups share a row.  Sum for 155 tokens of four rows of 7428 floats 5.1 us (one workgroup a token 16.3), for 500 of 4096 bf16 4.6 (5.8);
  // for 1000 of 4096 10.3 (9.6), so those are left whole.
  g.part = g.pieces;
  while (g.part > 256 && tokens * ((g.pieces + g.part - 1) / g.part) < 512) g.part = (g.part + 1) / 2;
  return g;
}
unsigned group_blocks(long long tokens, int width) {
  const long long b = (tokens + 256 / width - 1) / (256 / width);
  return (unsigned)(b < (1 << 20) ? b : 1 << 20);
}
__device__ __forceinline__ long long rows_sent(const int32_t* offsets, int E, long long n) {
  const long long s = offsets[E];
  return s < 0 ? 0 : s < n ? s : n;
}

struct DispatchArgs {
  RowsArg x, out;
  const uint8_t* scale;
  const int32_t* position;
  const int32_t* offsets;
  uint8_t* out_scale;
  long long tokens;
  int k, E, row_bytes;
  Groups g;
};

template <bool PAST>
__global__ __launch_bounds__(256) void dispatch_kernel(DispatchArgs a) {
  const int lane = (int)threadIdx.x % a.g.width;
  const long long slots = a.tokens * a.k, stride = group_count(a.g.width);
  const long long sent = rows_sent(a.offsets, a.E, slots);
  for (long long t = first_group(a.g.width); t < a.tokens; t += stride) {
    const int32_t* to = a.position + t * a.k;
    const unsigned char* x = a.x.data + t * a.x.pitch;
    for (int c = a.g.first() + lane; c < a.g.end(); c += a.g.width) {
      if (a.row_bytes >= 16) {
        // the last piece ends with the row: it may overlap the one before, which writes the same bytes
        const int at = c * 16 <= a.row_bytes - 16 ? c * 16 : a.row_bytes - 16;
        const uint4_t v = load16(x + at);
        for (int j0 = 0; j0 < a.k; j0 += 4) {                 // (four places requested at once)
          int p[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) p[j] = j0 + j < a.k ? to[j0 + j] : -1;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (p[j] >= 0 && p[j] < slots) store16<PAST>(a.out.data + p[j] * a.out.pitch + at, v);
        }
      } else {
        for (int j = 0; j < a.k; ++j) {
          const long long p = to[j];
          if (p >= 0 && p < slots)
            for (int i = 0; i < a.row_bytes; ++i) a.out.data[p * a.out.pitch + i] = x[i];
        }
      }
    }
    if (a.scale && blockIdx.y == 0)
      for (int j = lane; j < a.k; j += a.g.width) {
        const long long p = to[j];
        if (p >= 0 && p < slots) a.out_scale[p] = a.scale[t];
      }
  }
  for (long long p = sent + first_group(a.g.width); p < slots; p += stride) {
    for (int c = a.g.first() + lane; c < a.g.end(); c += a.g.width) {
      unsigned char* o = a.out.data + p * a.out.pitch;
      if (a.row_bytes >= 16)
        store16(o + (c * 16 <= a.row_bytes - 16 ? c * 16 : a.row_bytes - 16), uint4_t{0, 0, 0, 0});
      else
        for (int i = 0; i < a.row_bytes; ++i) o[i] = 0;
    }
    if (a.scale && lane == 0 && blockIdx.y == 0) a.out_scale[p] = 127;
  }
}

struct CombineArgs {
  RowsArg y, base, out;
  const float* weights;
  const int32_t* position;
  long long tokens;
  int k, cols;
  Groups g;
};

template <class T, bool PAST>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
  using E = Elem<T>;
  const int lane = (int)threadIdx.x % a.g.width;
  const long long slots = a.tokens * a.k, stride = group_count(a.g.width);
  for (long long t = first_group(a.g.width); t < a.tokens; t += stride) {
    const int32_t* from = a.position + t * a.k;
    for (int c = a.g.first() + lane; c < a.g.end(); c += a.g.width) {
      const int left = a.cols - c * E::PER;
      float sum[E::PER] = {};
      if (a.base.data) E::widen(load_piece<T>(a.base.data + t * a.base.pitch + (size_t)c * 16, left), sum);
      for (int j0 = 0; j0 < a.k; j0 += 4) {                    // (four rows requested at once)
        uint4_t v[4];
        float w[4];
        bool sent[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const long long p = j0 + j < a.k ? from[j0 + j] : -1;
          sent[j] = p >= 0 && p < slots;
          if (sent[j]) {
            w[j] = a.weights ? a.weights[t * a.k + j0 + j] : 1.0f;
            v[j] = load_piece<T>(a.y.data + p * a.y.pitch + (size_t)c * 16, left);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (sent[j]) {
            float f[E::PER];
            E::widen(v[j], f);
#pragma unroll
            for (int i = 0; i < E::PER; ++i) sum[i] += w[j] * f[i];
          }
      }
      store_piece<T, PAST>(a.out.data + t * a.out.pitch + (size_t)c * 16, left, E::narrow(sum));
    }
  }
}

struct CombineGradArgs {
  RowsArg dout, y, dy;
  const float* weights;
  const int32_t* position;
  const int32_t* offsets;
  float* dweights;
  long long tokens;
  int k, E, cols, pieces;
};

// W waves a token.  Four slots at a time: their rows are read, multiplied by dout for the weights' gradient, and written over.
template <class T, int W, bool PAST>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradArgs a) {
  using E = Elem<T>;
  constexpr int GROUPS = 4 / W;
  __shared__ float join[2][4][4];
  const int lane = (int)threadIdx.x % (64 * W), wave = (int)(threadIdx.x >> 6);
  const long long slots = a.tokens * a.k;
  int turn = 0;
  // (W == 4: every thread of a workgroup has the same t)
  for (long long t = (long long)blockIdx.x * GROUPS + threadIdx.x / (64 * W); t < a.tokens; t += (long long)gridDim.x * GROUPS) {
    for (int j0 = 0; j0 < a.k; j0 += 4, turn ^= 1) {
      long long p[4];
      float w[4], dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[j] = j0 + j < a.k ? a.position[t * a.k + j0 + j] : -1;
        if (p[j] >= slots) p[j] = -1;
        w[j] = p[j] >= 0 && a.weights ? a.weights[t * a.k + j0 + j] : 1.0f;
      }
      for (int c = lane; c < a.pieces; c += 64 * W) {
        const int left = a.cols - c * E::PER;
        const uint4_t d = load_piece<T>(a.dout.data + t * a.dout.pitch + (size_t)c * 16, left);
        uint4_t v[4];
        if (a.dweights)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (p[j] >= 0) v[j] = load_piece<T>(a.y.data + p[j] * a.y.pitch + (size_t)c * 16, left);
        float g[E::PER];
        E::widen(d, g);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (p[j] >= 0) {
            float o[E::PER];
#pragma unroll
            for (int i = 0; i < E::PER; ++i) o[i] = w[j] * g[i];
            store_piece<T, PAST>(a.dy.data + p[j] * a.dy.pitch + (size_t)c * 16, left, E::narrow(o));
            if (a.dweights) {
              float f[E::PER];
              E::widen(v[j], f);
#pragma unroll
              for (int i = 0; i < E::PER; ++i) dot[j] += g[i] * f[i];
            }
          }
      }
      if (!a.dweights) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) dot[j] = wave_sum(dot[j]);
      if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
          for (int j = 0; j < 4; ++j) join[turn][wave][j] = dot[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) dot[j] = join[turn][0][j] + join[turn][1][j] + join[turn][2][j] + join[turn][3][j];
      }
      if (lane < 4 && j0 + lane < a.k) {
        const float v = lane == 0 ? dot[0] : lane == 1 ? dot[1] : lane == 2 ? dot[2] : dot[3];
        a.dweights[t * a.k + j0 + lane] = v;
      }
    }
  }
  const long long group = (long long)blockIdx.x * GROUPS + threadIdx.x / (64 * W);
  for (long long r = rows_sent(a.offsets, a.E, slots) + group; r < slots; r += (long long)gridDim.x * GROUPS)
    for (int c = lane; c < a.pieces; c += 64 * W)
      store_piece<T>(a.dy.data + r * a.dy.pitch + (size_t)c * 16, a.cols - c * E::PER, uint4_t{0, 0, 0, 0});
}

template <class T, bool PAST>
hipError_t go_combine_grad(const CombineGradArgs& a, hipStream_t st) {
  // (16384 x 1024 bf16, four each: one wave a token 49.5 us, four 70.8; 16384 x 2048 122.6 and 109; 8 x 1024 4.3 and 3.6)
  if (a.pieces <= 64 || (a.pieces <= 128 && a.tokens >= 1024))
    combine_grad_kernel<T, 1, PAST><<<dim3(group_blocks(a.tokens, 64)), dim3(256), 0, st>>>(a);
  else
    combine_grad_kernel<T, 4, PAST><<<dim3(group_blocks(a.tokens, 256)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}
template <class T, bool PAST>
hipError_t go_combine(const CombineArgs& a, hipStream_t st) {
  combine_kernel<T, PAST><<<dim3(group_blocks(a.tokens, a.g.width), (unsigned)((a.g.pieces + a.g.part - 1) / a.g.part)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}
template <bool PAST>
hipError_t go_dispatch(const DispatchArgs& a, hipStream_t st) {
  dispatch_kernel<PAST><<<dim3(group_blocks(a.tokens, a.g.width), (unsigned)((a.g.pieces + a.g.part - 1) / a.g.part)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t route_workspace_bytes(long long slots, int E) {
  if (slots <= kRouteOne) return 0;
  return (size_t)((slots + route_run(slots, E) - 1) / route_run(slots, E)) * E * sizeof(int32_t);
}

hipError_t launch_route(const int32_t* experts, long long slots, int E, int32_t* offsets, int32_t* order, int32_t* position, void* workspace,
                        hipStream_t st) {
  RouteArgs a{experts, slots, E, 0, offsets, order, position, (int32_t*)workspace, 0, 0};
  while ((1 << a.bits) < E) ++a.bits;
  const int most = route_waves(E);
  if (slots <= kRouteOne) {
    const long long waves = (slots + 63) / 64;
    const int nw = waves < 1 ? 1 : waves < most ? (int)waves : most;
    route_one_kernel<<<dim3(1), dim3((unsigned)(64 * nw)), 0, st>>>(a);
    return hipGetLastError();
  }
  a.run = route_run(slots, E);
  a.runs = (int)((slots + a.run - 1) / a.run);
  route_count_kernel<<<dim3((unsigned)a.runs), dim3(256), 0, st>>>(a);
  route_place_kernel<<<dim3((unsigned)a.runs), dim3((unsigned)(64 * (most < 4 ? most : 4))), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_dispatch(long long tokens, int k, int E, int row_bytes, RowsArg x, const uint8_t* scale, const int32_t* position,
                           const int32_t* offsets, RowsArg out, uint8_t* out_scale, hipStream_t st) {
  const DispatchArgs a{x, out, scale, position, offsets, out_scale, tokens, k, E, row_bytes, groups_for(tokens, row_bytes, 16)};
  return writes_past(tokens * k * row_bytes) ? go_dispatch<true>(a, st) : go_dispatch<false>(a, st);
}

hipError_t launch_combine(int dtype, long long tokens, int k, int cols, RowsArg y, const float* weights, const int32_t* position, RowsArg base,
                          RowsArg out, hipStream_t st) {
  const int row_bytes = cols * (dtype == LASNET_F32 ? 4 : 2);
  const CombineArgs a{y, base, out, weights, position, tokens, k, cols, groups_for(tokens, row_bytes, 16)};
  if (writes_past(tokens * row_bytes)) return dtype == LASNET_F32 ? go_combine<float, true>(a, st) : go_combine<__bf16, true>(a, st);
  return dtype == LASNET_F32 ? go_combine<float, false>(a, st) : go_combine<__bf16, false>(a, st);
}

hipError_t launch_combine_backward(int dtype, long long tokens, int k, int E, int cols, RowsArg dout, RowsArg y, const float* weights,
                                   const int32_t* position, const int32_t* offsets, RowsArg dy, float* dweights, hipStream_t st) {
  const int per = dtype == LASNET_F32 ? 4 : 8;
  const CombineGradArgs a{dout, y, dy, weights, position, offsets, dweights, tokens, k, E, cols, (cols + per - 1) / per};
  if (writes_past(tokens * k * cols * (16 / per))) return dtype == LASNET_F32 ? go_combine_grad<float, true>(a, st) : go_combine_grad<__bf16, true>(a, st);
  return dtype == LASNET_F32 ? go_combine_grad<float, false>(a, st) : go_combine_grad<__bf16, false>(a, st);
}

}  // namespace lasnet
