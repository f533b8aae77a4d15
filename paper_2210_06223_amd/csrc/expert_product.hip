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
#include "expert_product.hpp"

namespace lasnet {
namespace {

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
__device__ __forceinline__ void unit_barrier(bool stored) {
  if (stored)
    counted_barrier<8 + kTileStores>();
  else
    counted_barrier<8>();
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
