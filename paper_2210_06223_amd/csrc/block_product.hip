// The experts' products of 8-bit rows and matrices whose scales belong to blocks of 128:
//
//   out[p][i] = sum_b 2^(scale[p][b] - 127) wscale[e][i / 128][b] sum_{c in block b} x[p][c] W[e][i][c]          rows p of expert e
//
// A step of the reduction is 128 bytes, a block: its two scales go with the step's products (see SCALES).  Kernels, by rows and tiles (see go_blocks, with both sides of each choice):
//   many tiles       256 x 256 by eight waves, streaming from tile to tile
//   fewer            64 x 16 to 128 x 128, a tile a workgroup, loads straight to LDS, the reduction shared by groups of waves where tiles are few
//   few rows         fragments straight to registers
//   odd rows         (not whole pieces of 16 bytes) words through registers; many tiles of them 128 x 128
// 8192 x 8192 x 8192: 392 to 400 us with bytes as scales (2750 to 2800 TFLOP/s; a product of that size without scales reaches 3260 here), 460 to 470 in fp32 (2340 to 2390).  A step reads 192 KiB from LDS and writes 64,
// about what its MFMAs take, too; but four waves of 128 x 128, which read 128, took 441 (eight 411 then): one wave a SIMD waits for itself.  fp32 scales add four multiply-adds an MFMA to the vector unit.
#include "expert_product.hpp"

namespace lasnet {
namespace {

// ---- many tiles: 256 x 256 by eight waves, one workgroup a CU that goes from tile to tile without letting its loads run dry ----
//
// LDS holds two steps, each 32 KiB of either operand, and each wave's scales of them in slots of its own.  In step s a wave multiplies the I fragments of its eight blocks, a ring of four
// read three blocks ahead, with the four J fragments it holds, and reads those of step s + 1 in block 7.  One barrier a step, before block 5, where all of I of step s has been read (and J, in block
// 7 of the step before): step s + 1 has landed, and the loads of step s + 2 go where step s was; they have a step, some 1.6 us, to arrive.
// FLOATS: the sum of a block of 128, four registers, is added to the whole kLag MFMAs later, when it is there.
constexpr int kBlockStage = 65536, kBlockSlots = 2 * kScaleSlot, kLag = 2;
constexpr int kBlockAside = 2 * kBlockStage + 8 * kBlockSlots, kBlockPieces = 6 * (24576 + 4 * kScaleSlot);
constexpr int kBlockTable = kBlockPieces, kBlockLds = kBlockTable + 512;                 // (behind what an eighth of a tile uses, which is more than a quarter or a stream does)
static_assert(kBlockAside + 8 * 64 <= kBlockTable && 4 * (32768 + 8 * kScaleSlot) <= kBlockTable && kBlockLds <= 160 * 1024, "a CU's LDS");
constexpr int kStepLoads = 8 + kScaleLoads;

// A workgroup's tile.
struct BlockTile {
  int expert, i0, j0, j_end;
};

// Where a wave's scales are: those of its rows of J (a byte each lane, kb apart) and that of its columns.
template <int SCALES>
struct ScaleStream {
  unsigned long long x, w;
  unsigned size_x;
  __device__ __forceinline__ void start(const ProductArgs& a, int expert, int i0, int row0, int j_end) {
    constexpr int WB = SCALES == FLOATS ? 4 : 1;
    const int rows = j_end - row0 < 64 ? j_end - row0 : 64, nb = (a.ni + 127) >> 7, ib = i0 >> 7 < nb ? i0 >> 7 : nb - 1;
    auto uniform = [](unsigned long long v) {
      return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((unsigned)v);
    };
    x = uniform((unsigned long long)a.xblocks + (unsigned long long)((long long)row0 * a.kb));
    w = uniform((unsigned long long)a.wblocks + (unsigned long long)(((long long)expert * nb + ib) * a.kb * WB));
    size_x = __builtin_amdgcn_readfirstlane(rows > 0 ? (unsigned)((rows - 1) * a.kb + 1) : 0u);
  }
  // a step's, of a tile that has any left (else zeros: NaN times nothing would be NaN)
  __device__ __forceinline__ void load(unsigned off_x, unsigned to, int left) {
    constexpr int WB = SCALES == FLOATS ? 4 : 1;
    const int there = ~((left - 1) >> 31);
    scales_to_lds<true>(intx4{(int)(unsigned)x, (int)(unsigned)(x >> 32), (int)__builtin_amdgcn_readfirstlane(size_x & (unsigned)there), 0x00020000}, off_x, to);
    scales_to_lds<SCALES == POWERS>(intx4{(int)(unsigned)w, (int)(unsigned)(w >> 32), (int)__builtin_amdgcn_readfirstlane((unsigned)(WB & there)), 0x00020000}, off_x & 0u, to + 256);
    x += 1;
    w += WB;
  }
};

// The wave's 64 x 128 of a tile, rounded and stored through a buffer that ends with the tile's last row.  Row 16 i + c of the wave's matrix rows in LDS is row 8 c + i in memory, and the rows of J
// are the MFMA's first operand: so a lane has 8 columns next to each other of 16 rows, 16 lanes a row's 256 bytes, and a store is 4 rows of two whole lines each.  What a CU's 128 KiB take by
// themselves goes by the lines that 16 lanes touch: 1.1 us so, 2.0 of 8 rows, 3.6 of 16 rows by 16 bytes, 7.1 of 16 by 8; 256 CUs at once, 5.3 (memory), 8.1 of 16 by 8.
// While memory takes what all CUs store at once the loads behind wait (32768 rows, 4096 x 2048: without the stores 209 us, with half of them 235, with all 262): whole lines of a large output
// go past the caches, 230 us (f32 scales 307 -> 261; with inputs from memory 288 -> 275, 338 -> 332); 67 MB, which stay in them, 107 us, past them 110.
// Always kBlockStores stores (by hand: they are counted).  ni: a multiple of 8.
constexpr int kBlockStores = 16;
__device__ __forceinline__ void store_block_tile(const ProductArgs& a, const BlockTile& t, int wi, int wj, int lane, const floatx4 (&acc)[8][4]) {
  asm volatile("" : "+v"(lane));
  const unsigned pitch = (unsigned)a.out.pitch;
  const int rows = t.j_end - t.j0 < 256 ? t.j_end - t.j0 : 256;
  const unsigned long long first = (unsigned long long)(a.out.data + (long long)t.j0 * a.out.pitch + (long long)t.i0 * 2);
  const intx4 to = {(int)(unsigned)first, (int)(unsigned)(first >> 32), (int)((unsigned)(rows - 1) * pitch + (unsigned)(a.ni - t.i0) * 2), 0x00020000};
  auto each = [&](auto relu, auto past) {
    const intx4 buffer = to;
    const int col = wi + (lane & 15) * 8;
    const bool there = t.i0 + col < a.ni;
    unsigned o = (unsigned)(wj + (lane >> 4) * 4) * pitch + (unsigned)col * 2;
#pragma unroll
    for (int j = 0; j < 4; ++j, o += 12 * pitch)
#pragma unroll
      for (int r = 0; r < 4; ++r, o += pitch) {
        uint4_t piece;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x = acc[2 * q][j][r], y = acc[2 * q + 1][j][r];
          if constexpr (decltype(relu)::value) {
            x = x < 0.f ? 0.f : x;                             // (NaN passes)
            y = y < 0.f ? 0.f : y;
          }
          piece[q] = bf16_pair(x, y);
        }
        // (beyond the buffer's 2^31 bytes: not stored; s_nop: the registers of a store of more than 8 bytes may not be written by the very next instruction)
        const unsigned at = there ? o : 0x80000000u;
        if constexpr (decltype(past)::value)
          asm volatile("buffer_store_dwordx4 %0, %1, %2, 0 offen nt\n\ts_nop 1" ::"v"(piece), "v"(at), "s"(buffer) : "memory");
        else
          asm volatile("buffer_store_dwordx4 %0, %1, %2, 0 offen\n\ts_nop 1" ::"v"(piece), "v"(at), "s"(buffer) : "memory");
      }
  };
  auto store = [&](auto past) {
    if (a.relu)
      each(std::true_type{}, past);
    else
      each(std::false_type{}, past);
  };
  if (a.past)
    store(std::true_type{});
  else
    store(std::false_type{});
}

template <int SCALES>
__global__ __launch_bounds__(512, 2) void block_stream_kernel(ProductArgs a) {
  // SPREAD: MFMAs among which a step's loads lie, of blocks 5 to 7.  8192 x 8192 x 8192, 8 and 12: 409 and 400 us, fp32 scales 463 and 479.
  constexpr int KS = 128, SPREAD = SCALES == POWERS ? 12 : 8;
  using S = Stage<false, 256, 8>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char product_lds[];
  const unsigned lds = (unsigned)(size_t)(lds_byte*)product_lds;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wi = wave % 2 * 128, wj = wave / 2 * 64;

  // The experts' rows, one expert a lane (up to 63 of them; else they are looked up anew for each tile): first row, and tiles up to and with it.  In LDS (every wave writes
  // the same), until a tile is looked up.
  typedef __attribute__((address_space(3))) unsigned lds_dword;
  int tiles_j;
  const bool kept = a.E <= 63;
  if (kept) {
    const int lo = bound(a, lane < a.E ? lane : a.E), hi = __shfl(lo, lane < 63 ? lane + 1 : 63);
    int upto = hi > lo ? (hi - lo + 255) / 256 : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(upto, d);
      if (lane >= d) upto += u;
    }
    tiles_j = __builtin_amdgcn_readlane(upto, 63);
    *(lds_dword*)(size_t)(lds + kBlockTable + lane * 8) = (unsigned)lo;
    *(lds_dword*)(size_t)(lds + kBlockTable + lane * 8 + 4) = (unsigned)upto;
  } else {
    const int rest = (int)a.rows - __builtin_amdgcn_readfirstlane(bound(a, a.E));
    tiles_j = row_tiles<256>(a) - (rest + 255) / 256;
  }
  // the rows that no expert has
  for (long long r = bound(a, a.E) + (long long)blockIdx.x; r < a.rows; r += gridDim.x)
    for (int c = (int)threadIdx.x * 8; c < a.ni * 2; c += 512 * 8) *(uint2_t*)(a.out.data + r * a.out.pitch + c) = uint2_t{0, 0};
  // Workgroups are dealt to the eight XCDs in turn, each of which has an L2: an XCD takes consecutive tiles, its workgroups one each in turn.  A last round that would
  // leave half of the XCD idle or more is cut into pieces of tiles.
  const int xcd = (int)blockIdx.x & 7, slot = (int)blockIdx.x >> 3, stride = (int)gridDim.x >> 3;
  const int total = tiles_j * a.tiles_i, chunk = (total + 7) / 8;
  int end = total - xcd * chunk < chunk ? total - xcd * chunk : chunk;
  const int rest = end > 0 && end % stride <= stride / 2 ? end % stride : 0;
  end -= rest;

  auto work = [&](int p) {                                    // the XCD's tile p
    BlockTile w;
    int ti, tj;
    tile_at(xcd * chunk + p, a.tiles_i, tiles_j, ti, tj);
    if (kept) {
      const int lo = (int)read_dword(lds + kBlockTable + lane * 8), upto = (int)read_dword(lds + kBlockTable + lane * 8 + 4);
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
    w.i0 = ti * 256;
    return w;
  };
  const int steps = (a.nk + KS - 1) / KS;                     // (two at least: nk >= 256, so that loads are never further ahead than the next tile)

  // ---- loads ----
  const unsigned pitch_i = (unsigned)a.I.pitch, pitch_j = (unsigned)a.J.pitch, kb = (unsigned)a.nk;
  struct Loads {
    Feed<false> i, j;
    ScaleStream<SCALES> s;
  };
  auto feed = [&](const BlockTile& w) {
    Loads l;
    l.i.start(a.I.data + (long long)w.expert * a.i_expert + (long long)w.i0 * a.I.pitch, a.ni - w.i0, 256, a.I.pitch, kb);
    l.j.start(a.J.data + (long long)w.j0 * a.J.pitch, w.j_end - w.j0, 256, a.J.pitch, kb);
    l.s.start(a, w.expert, w.i0 + wi, w.j0 + wj, w.j_end);
    return l;
  };
  Loads l;                                                    // of the tile being loaded
  int l_k = 0, after_k = 0;                                   // its k left, and that of the next (past the last tile: none)
  // Those of the next tile wait in LDS, where a wave has a place for them: registers are short.
  constexpr int WORDS = sizeof(Loads) / 4;
  const unsigned aside = lds + kBlockAside + wave * 64;
  union Words { Loads l; unsigned u[WORDS]; __device__ Words() {} };
  auto put_aside = [&](const Loads& v) {
    Words w;
    w.l = v;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) *(lds_dword*)(size_t)(aside + 4 * i) = w.u[i];
  };
  auto take_up = [&] {
    Words w;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w.u[i] = __builtin_amdgcn_readfirstlane(read_dword(aside + 4 * i));
    l = w.l;
  };
  const unsigned slots = lds + 2 * kBlockStage + wave * kBlockSlots;
  unsigned l_to = lds, l_slot = slots;
  auto nothing = [](int) {};
  // A step's loads, between the eight parts of `meanwhile`.
  auto issue = [&](auto meanwhile) {
    meanwhile(0);
    int at = lane;                                             // (made where it is used, not kept)
    asm volatile("" : "+v"(at));
    l.s.load((unsigned)(at * a.kb), l_slot, l_k);
    const unsigned to = l_to + wave * 4096;
#pragma unroll
    for (int h = 0; h < 2; ++h) {                             // J, I
      const intx4 rsrc = h ? l.i.rsrc(l_k, pitch_i) : l.j.rsrc(l_k, pitch_j);
      // this lane's first piece of the operand's tile; the next lies a segment's rows further with bit 6 of its byte turned over (bit 2 of the lane), the other two likewise two
      // segments further
      // (I: row 16 i + c of a wave's 128 in LDS is row 8 c + i in memory)
      const unsigned byte = (unsigned)S::byte(wave * 4, at);
      const unsigned first = (h ? (unsigned)(wave / 4 * 128 + wave % 4 * 2 + (at >> 3) * 8) * pitch_i : (unsigned)S::row(wave * 4, at) * pitch_j) + byte;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        unsigned o = first + (s & 1 ? 64u - ((unsigned)at & 4) * 32 : 0u) + (h ? (unsigned)(s % 2 * 64 + s / 2) * pitch_i : (unsigned)(s * 8) * pitch_j);
        if ((int)(byte ^ (s & 1 ? 64u : 0u)) >= l_k) o = 0xffffffffu;             // what is beyond the end of k lies inside the buffer
        if (h || s) meanwhile(h * 4 + s);
        __builtin_amdgcn_sched_barrier(0);
        buffer_to_lds(rsrc, o, to + h * 32768 + s * 1024);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    l_to = 2 * lds + kBlockStage - l_to;
    l_slot = 2 * slots + kScaleSlot - l_slot;
    l.i.move(KS);
    l.j.move(KS);
    l_k -= KS;
  };

  // ---- products ----
  floatx4 acc[8][4];
  Fragment fi[4], fj[4];
  unsigned sx[4], sw = 0, sw_next = 0;
  float m_now = 0.f, m_before = 0.f;                          // FLOATS: the scales' m, of this step and the one before; sw is their power
  floatx4 part[kLag];                                         // ... and the sums of a block of 128
  unsigned c = lds, c_slot = slots;                           // the step that fragments are read from
  unsigned at_i = S::lane_base(0, lane) + c + 32768 + wi * 128;                           // where a lane reads block 0 of I's from (and of J's, wi and wj apart)
  auto read_i = [&](int i) { S::fragment(at_i, i, fi[i % 4]); };
  auto read_j = [&](int j) {
    unsigned of = (unsigned)lane;
    asm volatile("" : "+v"(of));
    S::fragment(at_i + (unsigned)((wj - wi) * 128 - 32768), j, fj[j]);
    sx[j] = read_dword(c_slot + (of & 15) * 4 + 64 * j);
  };
  auto take_scale = [&](unsigned w) {
    if constexpr (SCALES == FLOATS) {
      m_now = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(scale_mantissa(w))));
      sw = scale_power(w);
    } else {
      sw = w;
    }
  };
  auto add_part = [&](int m, float w) {                       // that of the m-th MFMA of a step
    floatx4& sum = acc[m / 4][m % 4 ^ 2];
    sum = add_scaled(sum, part[m % kLag], w);
  };
  auto multiply = [&](int i, int p) {                         // the p-th MFMA of block i
    const int j = p ^ 2, m = 4 * i + p;
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (SCALES == FLOATS) {
      add_part(m >= kLag ? m - kLag : 32 + m - kLag, m >= kLag ? m_now : m_before);
      part[m % kLag] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fj[j].all, fi[i % 4].all, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, (int)sx[j], 0, (int)sw);
    } else {
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fj[j].all, fi[i % 4].all, acc[i][j], 0, 0, 0, (int)sx[j], 0, (int)sw);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  bool young = false;                                         // whether a tile's stores are younger than the loads waited for
  auto step = [&] {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i == 5) {
        if (young)
          counted_barrier<kBlockStores>();
        else
          counted_barrier<0>();
        young = false;
        at_i += 2 * (lds - c) + kBlockStage;
        c = 2 * lds + kBlockStage - c;
        c_slot = 2 * slots + kScaleSlot - c_slot;
        asm volatile("" : "+v"(at_i));                         // (a sum in a register: reads add constants to it)
        issue([&](int p) {
#pragma unroll
          for (int m = p * SPREAD / 8; m < (p + 1) * SPREAD / 8; ++m) {
            if (m == 8) read_i(2);
            multiply(5 + m / 4, m % 4);
            if (m == 0) read_i(0);
            if (m == 4) read_i(1);
            if (m == 5) sw_next = read_dword(c_slot + 256);
            if (m >= 8) read_j((m - 8) ^ 2);                   // (in place of the one that has been used up)
          }
        });
      } else if (i < 5 || (i == 7 && SPREAD == 8)) {
        read_i((i + 3) % 8);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          multiply(i, p);
          if (i == 7) read_j(p ^ 2);
        }
      }
    }
    m_before = m_now;
    take_scale(sw_next);
  };

  int round = 0;
  if (slot < end) {
    BlockTile w = work(slot);
    l = feed(w);
    l_k = a.nk;
    issue(nothing);
    issue(nothing);
    counted_barrier<kStepLoads>();
#pragma unroll
    for (int j = 0; j < 4; ++j) read_j(j);
    take_scale(read_dword(c_slot + 256));
#pragma unroll
    for (int i = 0; i < 3; ++i) read_i(i);
    while (true) {
      ++round;
      const bool more = round * stride + slot < end;
      BlockTile next = w;
      if (more) {
        next = work(round * stride + slot);
        put_aside(feed(next));
      }
      after_k = more ? a.nk : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
      if constexpr (SCALES == FLOATS) {
        m_before = 0.f;
#pragma unroll
        for (int r = 0; r < kLag; ++r) part[r] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      for (int s = 0; s < steps; ++s) {
        if (s == steps - 2) {                                  // (loads are two steps ahead)
          if (more) take_up();
          l_k = after_k;
        }
        step();
      }
      if constexpr (SCALES == FLOATS)
#pragma unroll
        for (int m = 32 - kLag; m < 32; ++m) add_part(m, m_before);
      store_block_tile(a, w, wi, wj, lane, acc);
      if (!more) break;
      young = true;
      w = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (the last loads write to this workgroup's LDS)
  }
  // What is left in pieces, two a workgroup at most.  Few: eighths of tiles, the reduction shared by two groups of waves (a step of a quarter is 0.6 us, whatever it does: 16640 rows, 2048 x
  // 4096 129 -> 122 us, with scales in 32 bits 149 -> 137).
  const int cut = 8 * rest <= stride ? 8 : 4;
  for (int q = slot; q < cut * rest; q += stride) {
    const BlockTile v = work(end + q / cut);
    const int i0 = v.i0 + (cut == 8 ? (q & 3) * 64 : (q & 1) * 128), j0 = v.j0 + (cut == 8 ? q >> 2 & 1 : q >> 1 & 1) * 128;
    if (i0 >= a.ni || j0 >= v.j_end) continue;
    __syncthreads();
    if (cut == 8)
      tile_product<true, false, false, false, false, 64, 128, 1, 4, 3, 2, SCALES>(a, product_lds, v.expert, i0, j0, v.j_end, 0, a.nk);
    else
      tile_product<true, false, false, false, false, 128, 128, 2, 4, 4, 1, SCALES>(a, product_lds, v.expert, i0, j0, v.j_end, 0, a.nk);
  }
}

template <int SCALES>
hipError_t go_block_stream(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + 255) / 256;
  auto kernel = block_stream_kernel<SCALES>;
  static std::atomic<unsigned long long> allowed{0};
  const hipError_t e = allow_lds((const void*)kernel, kBlockLds, allowed);
  if (e != hipSuccess) return e;
  kernel<<<dim3(256), dim3(512), kBlockLds, st>>>(a);
  return hipGetLastError();
}

template <int SCALES, int BI, int BJ, int WI, int WJ, int STAGES, int WK = 1>
hipError_t go_block_tile(const ProductArgs& a, hipStream_t st) {
  return go_tile<true, false, false, false, false, BI, BJ, WI, WJ, STAGES, WK, SCALES>(a, st);
}

// ---- rows that are not whole pieces of 16 bytes, and few tiles ----
// A piece that begins anywhere costs its load as much as several: these load whole words, the four that hold its first 16 bytes and the one behind them (no word but those that hold bytes of the
// row), and shift.  Straight to registers, 1 row, 4096 columns of 4095: 18.7 -> 10.4 us.
struct Words {
  uint4_t v;
  unsigned next;
};
// The words of 16 bytes of a row of `size` (16 or more) from byte b on, or of its last 16, where they end earlier (see cut_piece).
__device__ __forceinline__ Words row_words(const unsigned char* row, int b, int size) {
  typedef uint4_t four_words __attribute__((aligned(4)));
  const size_t first = ((size_t)row + (b < size - 16 ? b : size - 16)) & ~(size_t)3, last = ((size_t)row + size - 1) & ~(size_t)3;
  return Words{*(const four_words*)first, *(const unsigned*)(first + 16 < last ? first + 16 : last)};
}
__device__ __forceinline__ uint4_t word_piece(const Words& w, const unsigned char* row, int b, int size) {
  const unsigned shift = ((unsigned)(size_t)row + (unsigned)(b < size - 16 ? b : size - 16)) & 3;
  return uint4_t{__builtin_amdgcn_alignbyte(w.v[1], w.v[0], shift), __builtin_amdgcn_alignbyte(w.v[2], w.v[1], shift), __builtin_amdgcn_alignbyte(w.v[3], w.v[2], shift),
                 __builtin_amdgcn_alignbyte(w.next, w.v[3], shift)};
}

// A workgroup's tile is 16 x 16 NJ; its four waves share the reduction.  A wave's fragments come straight to registers, DEPTH steps ahead: no LDS and no barrier before the sums of the waves
// meet.  (The order of k in a step is the matrix core's own affair as long as both operands have the same: a load takes 64 bytes of each of 16 rows.)
template <int SCALES, int NJ, int DEPTH>
__global__ __launch_bounds__(256) void block_odd_kernel(ProductArgs a) {
  __shared__ floatx4 sums[4][NJ][64];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int ti = (int)(blockIdx.x % a.tiles_i), i0 = ti * 16;
  int expert, j0, j_end;
  if (!find_rows(a, 16 * NJ, (int)(blockIdx.x / a.tiles_i), expert, j0, j_end)) return;
  expert = __builtin_amdgcn_readfirstlane(expert);
  j0 = __builtin_amdgcn_readfirstlane(j0);
  j_end = __builtin_amdgcn_readfirstlane(j_end);
  floatx4 acc[NJ] = {};
  const int steps = (a.nk + 127) / 128, share = (steps + 3) / 4, first = wave * share, n = steps - first < share ? steps - first : share;
  if (expert < a.E && n > 0) {
    // (rows and columns beyond the last are read as the last, and not stored)
    const unsigned char* pj[NJ];
    const uint8_t* px[NJ];
    const int column = i0 + (lane & 15);
    const unsigned char* pi = a.I.data + (long long)expert * a.i_expert + (long long)(column < a.ni ? column : a.ni - 1) * a.I.pitch;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int r = j0 + 16 * j + (lane & 15);
      const long long row = r < j_end ? r : j_end - 1;
      pj[j] = a.J.data + row * a.J.pitch;
      px[j] = a.xblocks + row * a.kb;
    }
    const long long w0 = ((long long)expert * ((a.ni + 127) >> 7) + (i0 >> 7)) * a.kb;
    Words ri[DEPTH][2], rj[DEPTH][NJ][2];
    unsigned sx[DEPTH][NJ], sw[DEPTH];
    auto byte = [&](int s, int h) { return (first + s) * 128 + h * 64 + (lane >> 4) * 16; };
    auto fetch = [&](int d, int s) {                           // the wave's step s (past the last: the last again, for nothing)
      if (s >= n) s = n - 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        ri[d][h] = row_words(pi, byte(s, h), a.nk);
#pragma unroll
        for (int j = 0; j < NJ; ++j) rj[d][j][h] = row_words(pj[j], byte(s, h), a.nk);
      }
      sw[d] = SCALES == POWERS ? ((const uint8_t*)a.wblocks)[w0 + first + s] : ((const unsigned*)a.wblocks)[w0 + first + s];
#pragma unroll
      for (int j = 0; j < NJ; ++j) sx[d][j] = px[j][first + s];
    };
    auto multiply = [&](int d, int s) {
      const bool ends = (first + s + 1) * 128 > a.nk;
      auto piece = [&](const Words& w, const unsigned char* row, int h) {
        const uint4_t v = word_piece(w, row, byte(s, h), a.nk);
        return ends ? cut_piece(v, a.nk - byte(s, h)) : v;
      };
      Fragment fi;
#pragma unroll
      for (int h = 0; h < 2; ++h) fi.h[h] = piece(ri[d][h], pi, h);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        Fragment fj;
#pragma unroll
        for (int h = 0; h < 2; ++h) fj.h[h] = piece(rj[d][j][h], pj[j], h);
        const floatx4 v = scaled_mfma<SCALES>(fi.all, fj.all, acc[j], SCALES == FLOATS ? scale_power(sw[d]) : sw[d], sx[d][j]);
        acc[j] = SCALES == FLOATS ? add_scaled(acc[j], v, scale_mantissa(sw[d])) : v;
      }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(d, d);
    for (int s = 0; s < n; s += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (s + d < n) multiply(d, s + d);
        fetch(d, s + d + DEPTH);
      }
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) sums[wave][j][lane] = acc[j];
  __syncthreads();
  if (wave >= NJ) return;
  const floatx4 whole[1][1] = {{((sums[0][wave][lane] + sums[1][wave][lane]) + sums[2][wave][lane]) + sums[3][wave][lane]}};
  store_tile<false, false>(a, a.out.data, expert, i0, j0 + 16 * wave, j_end, whole);
}

template <int SCALES, int NJ, int DEPTH>
hipError_t go_block_odd(ProductArgs a, hipStream_t st) {
  static_assert(NJ <= 4, "a wave stores 16 rows");
  a.tiles_i = (a.ni + 15) / 16;
  const long long groups = a.rows / (16 * NJ) + (a.rows < a.E ? a.rows : a.E) + 1;       // (experts with rows, one that is not full each, and the rest)
  block_odd_kernel<SCALES, NJ, DEPTH><<<dim3((unsigned)(groups * a.tiles_i)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

// BI x BJ of the output by WK groups of WI x WJ waves that share the reduction: words go through registers, where they are shifted, into two LDS stages; the loads of the next DEPTH
// steps are in flight while a step's products run.
template <int SCALES, int BI, int BJ, int WI, int WJ, int WK, int DEPTH>
__global__ __launch_bounds__(64 * WI * WJ * WK) void block_odd_tile_kernel(ProductArgs a) {
  constexpr int G = 64 * WI * WJ, PI = BI * 8 / G, PJ = BJ * 8 / G, NI = BI / WI / 16, NJ = BJ / WJ / 16, STAGE = (BI + BJ) * 128;
  static_assert(PI >= 1 && PJ >= 1 && BI <= 128, "pieces of a thread; columns in one block of 128");
  extern __shared__ __attribute__((aligned(1024))) unsigned char product_lds[];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), group = wave / (WI * WJ), tid = (int)threadIdx.x - group * G;
  const int ti = (int)(blockIdx.x % a.tiles_i), i0 = ti * BI;
  int expert, j0, j_end;
  if (!find_rows(a, BJ, (int)(blockIdx.x / a.tiles_i), expert, j0, j_end)) return;
  expert = __builtin_amdgcn_readfirstlane(expert);
  j0 = __builtin_amdgcn_readfirstlane(j0);
  j_end = __builtin_amdgcn_readfirstlane(j_end);
  const int w = wave % (WI * WJ), wi = w % WI * (BI / WI), wj = w / WI * (BJ / WJ);
  floatx4 acc[NI][NJ] = {};
  if (expert < a.E) {
    const int steps = (a.nk + 127) / 128, share = (steps + WK - 1) / WK, first = group * share, n = steps - first < share ? steps - first : share;    // (n: this group's, maybe none)
    unsigned char* lds = product_lds + group * 2 * STAGE;
    // (rows and columns beyond the last are read as the last, and not stored)
    const unsigned char *pi[PI], *pj[PJ];
#pragma unroll
    for (int u = 0; u < PI; ++u) {
      const int r = i0 + (u * G + tid) / 8;
      pi[u] = a.I.data + (long long)expert * a.i_expert + (long long)(r < a.ni ? r : a.ni - 1) * a.I.pitch;
    }
#pragma unroll
    for (int u = 0; u < PJ; ++u) {
      const int r = j0 + (u * G + tid) / 8;
      pj[u] = a.J.data + (long long)(r < j_end ? r : j_end - 1) * a.J.pitch;
    }
    const uint8_t* px[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int r = j0 + wj + 16 * j + (lane & 15);
      px[j] = a.xblocks + (long long)(r < j_end ? r : j_end - 1) * a.kb;
    }
    const long long w0 = ((long long)expert * ((a.ni + 127) >> 7) + (i0 >> 7)) * a.kb;
    Words ri[DEPTH][PI], rj[DEPTH][PJ];
    unsigned nx[DEPTH + 1][NJ], nw[DEPTH + 1];                 // (the last: of the step that is multiplied)
    const int byte = tid % 8 * 16;
    auto fetch = [&](int d, int s) {                           // the group's step s (past the last: the last again, for nothing)
      int step = first + (s < n ? s : n - 1);
      step = step < 0 ? 0 : step < steps ? step : steps - 1;
#pragma unroll
      for (int u = 0; u < PI; ++u) ri[d][u] = row_words(pi[u], step * 128 + byte, a.nk);
#pragma unroll
      for (int u = 0; u < PJ; ++u) rj[d][u] = row_words(pj[u], step * 128 + byte, a.nk);
      nw[d] = SCALES == POWERS ? ((const uint8_t*)a.wblocks)[w0 + step] : ((const unsigned*)a.wblocks)[w0 + step];
#pragma unroll
      for (int j = 0; j < NJ; ++j) nx[d][j] = px[j][step];
    };
    auto stage = [&](int d, int s, int to) {
      const int b = (first + s) * 128 + byte;
      const bool ends = (first + s + 1) * 128 > a.nk;
      auto put = [&](const unsigned char* row, const Words& w, int q, unsigned char* tile) {
        const uint4_t v = word_piece(w, row, b, a.nk);
        *(uint4_t*)(tile + Tile<false>::place(q)) = ends ? cut_piece(v, a.nk - b) : v;
      };
#pragma unroll
      for (int u = 0; u < PI; ++u) put(pi[u], ri[d][u], u * G + tid, lds + to * STAGE);
#pragma unroll
      for (int u = 0; u < PJ; ++u) put(pj[u], rj[d][u], u * G + tid, lds + to * STAGE + BI * 128);
      nw[DEPTH] = nw[d];
#pragma unroll
      for (int j = 0; j < NJ; ++j) nx[DEPTH][j] = nx[d][j];
    };
    auto multiply = [&](int at) {
      const unsigned char* t = lds + at * STAGE;
      Fragment fi[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) fi[i].h[h] = Tile<false>::fragment(t, wi + 16 * i, h, lane);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        Fragment fj;
#pragma unroll
        for (int h = 0; h < 2; ++h) fj.h[h] = Tile<false>::fragment(t + BI * 128, wj + 16 * j, h, lane);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const floatx4 v = scaled_mfma<SCALES>(fi[i].all, fj.all, acc[i][j], SCALES == FLOATS ? scale_power(nw[DEPTH]) : nw[DEPTH], nx[DEPTH][j]);
          acc[i][j] = SCALES == FLOATS ? add_scaled(acc[i][j], v, scale_mantissa(nw[DEPTH])) : v;
        }
      }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(d, d);
    stage(0, 0, 0);
    fetch(0, DEPTH);
    __syncthreads();
    int at = 0;
    for (int s0 = 0; s0 < share; s0 += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int s = s0 + d;
        if (s >= share) break;
        if (s < n) multiply(at);                               // (a group without steps loads and waits along)
        stage((d + 1) % DEPTH, s + 1, at ^ 1);
        fetch((d + 1) % DEPTH, s + 1 + DEPTH);
        at ^= 1;
        __syncthreads();
      }
  }
  if constexpr (WK > 1) {
    floatx4* sums = (floatx4*)product_lds + w * 64 + lane;
    constexpr int EACH = WI * WJ * 64;
    if (group)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) sums[((group - 1) * NI * NJ + i * NJ + j) * EACH] = acc[i][j];
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int g = 0; g < WK - 1; ++g)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] += sums[(g * NI * NJ + i * NJ + j) * EACH];
  }
  store_tile<false, false>(a, a.out.data, expert, i0 + wi, j0 + wj, j_end, acc);
}

template <int SCALES, int BI, int BJ, int WI, int WJ, int WK, int DEPTH>
hipError_t go_block_odd_tile(ProductArgs a, hipStream_t st) {
  a.tiles_i = (a.ni + BI - 1) / BI;
  constexpr int stages = WK * 2 * (BI + BJ) * 128, sums = (WK - 1) * BI * BJ * 4, bytes = stages > sums ? stages : sums;
  const long long groups = a.rows / BJ + (a.rows < a.E ? a.rows : a.E) + 1;
  auto kernel = block_odd_tile_kernel<SCALES, BI, BJ, WI, WJ, WK, DEPTH>;
  static std::atomic<unsigned long long> allowed{0};
  const hipError_t e = allow_lds((const void*)kernel, bytes, allowed);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)(groups * a.tiles_i)), dim3(64 * WI * WJ * WK), bytes, st>>>(a);
  return hipGetLastError();
}

template <int SCALES>
hipError_t go_blocks(ProductArgs a, hipStream_t st) {
  const long long experts = a.E < a.rows ? a.E : a.rows, each = a.rows / experts;              // experts with rows at most, and rows of one
  const int steps = (a.nk + 127) / 128;
  // Tiles of BI x BJ, about (how the rows are spread is not known here).
  auto tiles = [&](int BI, int BJ) {
    const long long mean = a.rows / BJ + experts / 2, rows = mean > experts ? mean : experts;
    return rows * ((a.ni + BI - 1) / BI);
  };
  if (whole<false, false>(a, 1, 256)) {
    // us, bytes as scales, three sets of inputs in turn.
    // One workgroup a CU or little more, straight to registers: 1 row, 4096 x 4096 7.1 (64 x 16 by four groups of waves 8.5), 1024 x 2048 5.6 (6.5); 8 rows of 4 experts, 2048 x 4096 7.6
    // (8.6).  Of more of them or shorter reductions the loads of a few rows do not pay: 4 rows, 8192 x 2048 9.3 (7.2), 8 of 8, 1024 x 1024 7.6 (5.5).
    const long long units = tiles(16, 16);
    if (a.rows <= 64 && units <= (steps >= 32 ? 512 : 384)) return a.rows <= 16 || each <= 8 ? go_few<true, 1, SCALES>(a, st) : go_few<true, 2, SCALES>(a, st);
    // All at once, one workgroup a CU, the reduction shared by four groups of waves.  Rows of up to 16 an expert: 16 rows of 16 experts, 1024 x 2048 7.7 (64 x 32 8.1), 30 of 30,
    // 512 x 1024 5.6 (6.2), 32 of 4, 2048 x 2048 6.9 (7.4); beyond, tiles of 32 and 64 rows: 128 rows, 4096 x 4096 11.6 (64 x 64 13.1, 128 x 64 16.9), 512 rows, 2048 x 2048 14.5 (9.6, 11.1).
    if (steps >= 4 && each <= 16 && tiles(64, 16) <= 256) return go_block_tile<SCALES, 64, 16, 1, 1, 3, 4>(a, st);
    if (steps >= 12 && tiles(64, 32) <= 256) return go_block_tile<SCALES, 64, 32, 1, 2, 3, 4>(a, st);
    if (steps >= 6 && tiles(64, 64) <= 256) return go_block_tile<SCALES, 64, 64, 1, 4, 4, 2>(a, st);
    // Few rows an expert, more workgroups, three a CU: 64 rows of 64 experts, 1024 x 1024 10.9 (128 x 64 11.9), 64 of 8, 2048 x 2048 9.1 (10.7); 256 of 16, 2048 x 4096 39.3 (35.5).
    if (each <= 8 && tiles(64, 32) <= 1024) return go_block_tile<SCALES, 64, 32, 1, 2, 4>(a, st);
    // 256 x 256 where there are enough for the chip, or more of 128 x 128 than run at once (two a CU): 8000 rows of 8 experts, 2048 x 1024 29 (128 x 128 40), 8192 of 2, 1024 x 4096
    // 50 (67), 1024 x 512 14.8 (18.7), 3000 of 16, 2048 x 4096 62 (85).  Else not: 4096 rows, 2048 x 4096, 128 of them, 51 (41); 20000 of 2, 256 x 1024 19.9 (15.9).
    const long long halves = (a.rows / 128 + experts / 2 + experts / 4) * ((a.ni + 127) / 128);           // (rows are hardly ever spread evenly)
    if ((tiles(256, 256) >= 200 || halves > 512) && a.nk >= 256 && a.ni % 8 == 0 && !(((unsigned long long)a.out.data | (unsigned long long)a.out.pitch) & 15) &&
        a.out.pitch < (1ll << 31) / 256)
      return go_block_stream<SCALES>(a, st);
    // 128 x 64 in three stages, two a CU, up to two rounds, else 128 x 128: 1000 rows of 8 experts, 1024 x 1024 8.1 (128 x 128 11.9), 1500 of 4, 1024 x 8192 30 (56); 4096 rows, 2048 x 1024
    // 21.0 (17.9), 4001 of 8, 1000 x 528 13.7 (11.7).  128 x 128 by eight waves: 2048 rows, 2048 x 4096 26.6 (28.8 and 32.7), 2048 of 16, 4096 x 2048 55 (51, 57).
    // In two stages a step waits for the loads of that very step: 4224 rows, 1056 x 5024, a tile or two a CU, 50, 1.2 a step, of which its MFMAs take 0.2.  (More stages there: not tried.)
    if (tiles(128, 64) <= 512) return go_block_tile<SCALES, 128, 64, 2, 2, 3>(a, st);
    return go_block_tile<SCALES, 128, 128, 2, 2, 2>(a, st);
  }
  // Whole pieces or not.  us, bytes and fp32 as scales, three sets of inputs in turn, against 128 x 128 of the last kernel: 16 x 32 without LDS, 1 row, 4095 x 4095 10.5 and 10.4 (40.8, 54.6),
  // 16 of 4 experts, 1001 x 2047 8.4, 8.4 (23.9, 31.6); beyond that many tiles not: 300 of 4, 1001 x 1001 21.7.  64 x 32, the reduction shared by four groups: the latter 9.4, 9.4 (15.3, 18.8),
  // 64 of 8, 2047 x 4095 22.7, 22.8 (49.9, 65.0).  64 x 64, by four: 256 rows, 4095 x
  // 4095 28.4, 27.8 (56.4, 70.5; 128 x 64 35.1, 35.9).  128 x 64, by two: 1000 of 8, 1023 x 2049 21.4, 21.7 (31.8, 38.8), 2000 of 2, 1001 x 4001 36.2, 36.3 (55.2, 68.9).  128 x 128, by two: 30000
  // of 16, 100 x 8001 112, 114 (133, 159); with more than one a CU not: 4000 of 8, 1001 x 521 28.6, 28.7 (17.7, 18.7), 16384 of 8, 2047 x 2049 257, 260 (184, 202).
  if (a.nk >= 16) {
    if (tiles(16, 32) <= 320) return go_block_odd<SCALES, 2, 4>(a, st);
    if (steps >= 4 && tiles(64, 32) <= 256) return go_block_odd_tile<SCALES, 64, 32, 2, 1, 4, 2>(a, st);
    if (steps >= 4 && tiles(64, 64) <= 256) return go_block_odd_tile<SCALES, 64, 64, 2, 2, 4, 1>(a, st);
    if (steps >= 2 && tiles(128, 64) <= 256) return go_block_odd_tile<SCALES, 128, 64, 2, 2, 2, 1>(a, st);
    if (steps >= 2 && tiles(128, 128) <= 256) return go_block_odd_tile<SCALES, 128, 128, 2, 2, 2, 1>(a, st);
  }
  a.tiles_i = (a.ni + 127) / 128;
  const long long row_tiles = a.rows / 128 + a.E + 1;          // (each expert and the rest may have one tile that is not full)
  auto kernel = a.nk >= 16 ? product_kernel<true, false, false, false, false, true, SCALES> : product_kernel<true, false, false, false, false, false, SCALES>;
  kernel<<<dim3((unsigned)(row_tiles * a.tiles_i)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_product(long long rows, int E, int n, int k, RowsArg x, const uint8_t* scale, const int32_t* offsets, const void* W,
                                const void* wscale, bool f32_scales, RowsArg out, bool relu, hipStream_t st) {
  const ProductArgs a{{(unsigned char*)W, k}, x, out, (long long)n * k, 0, offsets, nullptr, nullptr, rows, E, n, 0, k, 0, 0, 0, 0, relu, scale, wscale, (k + 127) / 128, writes_past(rows * n * 2)};
  return f32_scales ? go_blocks<FLOATS>(a, st) : go_blocks<POWERS>(a, st);
}

}  // namespace lasnet
