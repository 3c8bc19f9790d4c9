// Which kernel computes a matrix product of the 8-bit layers and of the experts, and how its work is cut.
#include "common.cuh"

namespace bl {

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Row tiles of `tile` rows, as far as the host can tell: the lists' lengths are on the device.  Of lists longer than a tile
// half are taken to end inside one.
int64_t row_tiles(const MatmulArgs& a, int64_t tile) {
  if (!a.offsets) return ceil_div(a.R, tile);
  const int64_t met = a.experts < a.R ? a.experts : a.R, likely = a.R / tile + a.experts / 2;
  return likely > met ? likely : met;
}

}  // namespace

cudaError_t launch_matmul(const MatmulArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int64_t mean = a.offsets ? ceil_div(a.R, a.experts) : a.R;       // rows per list
  // The wide kernel's time is its rounds of tiles times the time of a block of K, which depends little on the rows of a tile
  // (0.28 us with 32 rows, 0.31 with 128, 0.40 with 256; with listed rows 0.31, 0.36, 0.48): the largest tiles, unless smaller
  // ones need no more rounds (1000 x 2048 x 2048: 10.3 us with 128 rows, 11.9 with 256; 509 x 2048 x 8192: 16.3 and 13.0).
  int wide = 64;
  int64_t wide_tiles = 0;
  double least = 0;
  for (int tile = 64; tile <= 256; tile += 64) {
    const int64_t tiles = row_tiles(a, tile) * ceil_div(a.N, 256), each = mean < tile ? mean : ceil_div(mean, ceil_div(mean, tile));
    const double cost = (double)ceil_div(tiles, sms / 2) * (a.rows ? 0.29 + 0.0007 * (double)each : 0.27 + 0.0005 * (double)each);
    if (tile == 64 || cost < least) { wide = tile; wide_tiles = tiles; least = cost; }
  }
  // Few rows: what counts is that every SM loads weights.  One list of up to 64 rows, or lists of up to 16 (64 experts of 2048 x 2048
  // with 16 rows each 48 us, the wide kernel 52; with 32 rows 57 and 51), or a product that leaves half of the SMs without a wide
  // tile (96 x 8192 x 2048: 12.4 us and 22.4).
  const bool narrow = a.offsets ? mean <= 16 || (mean <= 64 && 4 * wide_tiles < sms) : a.R <= 64 || 4 * wide_tiles < sms;
  if (!narrow) return launch_matmul_wide(a, wide, s);
  const int tokens = mean <= 16 ? 16 : mean <= 32 ? 32 : 64;
  const int64_t tiles = (a.offsets ? a.R / tokens + (a.experts < a.R ? a.experts : a.R) : ceil_div(a.R, tokens)) * ceil_div(a.N, 128);
  // K is shared as long as there are SMs for it and four blocks left for each (1 x 4096 x 4096: 12.6 us in one piece, 7.6 in four;
  // 1 x 4096 x 16384, 128 tiles: 13.6 in one, 15.4 in two).
  const int64_t blocks = ceil_div(a.K * (a.operand == BL_I8 ? 1 : 2), 128);
  int splits = 1;
  while (splits < 8 && tiles * splits * 2 <= sms && blocks >= 8 * splits) splits *= 2;
  // Two CTAs per SM where there is a tile or two for each (16 experts met, 2048 x 2048, 256 tiles: 16.1 us, one per SM 17.0), one
  // with twice the room for loads where there is only one tile, or one runs through many (1024 tiles: 48 and 50).
  const int per_sm = tiles * splits <= sms || tiles > 3 * sms ? 1 : 2;
  return launch_matmul_narrow(a, tokens, splits, per_sm, s);
}

}  // namespace bl
