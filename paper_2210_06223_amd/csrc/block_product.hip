// The experts' products of 8-bit rows and matrices whose scales belong to blocks of 128:
//
//   out[p][i] = sum_b 2^(scale[p][b] - 127) wscale[e][i / 128][b] sum_{c in block b} x[p][c] W[e][i][c]          rows p of expert e
//
// A step of the reduction is 128 bytes, a block: its two scales go with the step's products (see SCALES).
#include "expert_product.hpp"

namespace lasnet {
namespace {

template <int SCALES>
hipError_t go_blocks(ProductArgs a, hipStream_t st) {
  if (whole<false, false>(a, 1, 256)) {
    const long long blocks = a.E < a.rows ? a.E : a.rows, units = (blocks > (a.rows + 15) / 16 ? blocks : (a.rows + 15) / 16) * ((a.ni + 15) / 16);
    if (a.rows <= 64 && units <= 384) return a.rows <= 16 || a.rows / a.E <= 8 ? go_few<true, 1, SCALES>(a, st) : go_few<true, 2, SCALES>(a, st);
    auto tiles = [&](int BI, int BJ) {
      const long long mean = a.rows / BJ + blocks / 2, rows = mean > blocks ? mean : blocks;
      return rows * ((a.ni + BI - 1) / BI);
    };
    const int steps = a.nk / 128;
    if (steps >= 12 && tiles(64, 32) <= 256) return go_tile<true, false, false, false, false, 64, 32, 1, 2, 3, 4, SCALES>(a, st);
    if (steps >= 6 && tiles(64, 64) <= 256) return go_tile<true, false, false, false, false, 64, 64, 1, 4, 4, 2, SCALES>(a, st);
    if (tiles(128, 64) <= 256) return go_tile<true, false, false, false, false, 128, 64, 2, 2, 3, 1, SCALES>(a, st);
    if (tiles(128, 128) <= 240) return go_tile<true, false, false, false, false, 128, 128, 2, 4, 4, 1, SCALES>(a, st);
    if (tiles(128, 64) <= 512) return go_tile<true, false, false, false, false, 128, 64, 2, 2, 3, 1, SCALES>(a, st);
    return go_tile<true, false, false, false, false, 128, 128, 2, 2, 2, 1, SCALES>(a, st);
  }
  a.tiles_i = (a.ni + 127) / 128;
  const long long tiles = a.rows / 128 + a.E + 1;              // (each expert and the rest may have one tile that is not full)
  auto kernel = a.nk >= 16 ? product_kernel<true, false, false, false, false, true, SCALES> : product_kernel<true, false, false, false, false, false, SCALES>;
  kernel<<<dim3((unsigned)(tiles * a.tiles_i)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_product(long long rows, int E, int n, int k, RowsArg x, const uint8_t* scale, const int32_t* offsets, const void* W,
                                const void* wscale, bool f32_scales, RowsArg out, bool relu, hipStream_t st) {
  const ProductArgs a{{(unsigned char*)W, k}, x, out, (long long)n * k, 0, offsets, nullptr, nullptr, rows, E, n, 0, k, 0, 0, 0, 0, relu, scale, wscale, (k + 127) / 128};
  return f32_scales ? go_blocks<FLOATS>(a, st) : go_blocks<POWERS>(a, st);
}

}  // namespace lasnet
