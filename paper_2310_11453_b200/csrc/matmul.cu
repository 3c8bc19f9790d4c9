// Which kernel computes a matrix product of the 8-bit layers and of the experts, and how its work is cut: the way whose estimated time is
// least.  The estimates (microseconds) were fitted to measurements over 1 to 512 rows x 512 to 8192 x 1024 to 32001 and lists of 2 to 128
// rows, on a B200 with its weights in DRAM; what they decide is named with both sides measured.
#include <math.h>

#include "common.cuh"

namespace bl {

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Choice { bool narrow; int tokens, splits, per_sm, wide; };

Choice choose(const MatmulArgs& a, int64_t sms) {
  const int es = a.operand == BL_I8 ? 1 : 2;
  const int64_t blocks = ceil_div(a.K * es, 128), features = ceil_div(a.N, 128), pairs = ceil_div(a.N, 256);
  const int64_t met = a.experts < a.R ? a.experts : a.R;                 // experts with rows, at most
  const int64_t mean = a.offsets ? ceil_div(a.R, met) : a.R;             // rows of a list
  const double bytes = (double)met * (double)a.N * (double)a.K * es;     // of weights
  // Row tiles, as far as the host can tell: the lists' lengths are on the device, and taken to be spread exponentially.
  auto row_tiles = [&](int64_t tile) {
    if (!a.offsets) return ceil_div(a.R, tile);
    const int64_t likely = (int64_t)ceil((double)met / (1.0 - exp(-(double)tile / (double)mean))), most = a.R / tile + met;
    return likely < most ? likely : most;
  };
  auto rows_of_tile = [&](int64_t tile) { return mean <= tile ? mean : ceil_div(mean, ceil_div(mean, tile)); };

  // Wide: rounds of tiles over the pairs of SMs, 0.27 us a block of K and a little for each row; weights at 5.2 TB/s at most.  So large
  // tiles, unless smaller ones need no more rounds (1000 x 2048 x 2048: 9.5 us with 128 rows, 10.6 with 256; 509 x 2048 x 8192: 15.2 and 12.3).
  Choice c{false, 0, 1, 1, 64};
  double least = 0;
  for (int tile = 64; tile <= 256; tile += 64) {
    const double rows = (double)(mean < 64 ? 64 : rows_of_tile(tile)), rounds = (double)ceil_div(row_tiles(tile) * pairs, sms / 2);
    const double work = rounds * (double)blocks * (a.rows ? 0.29 + 0.0007 * rows : 0.27 + 0.0005 * rows), stream = bytes / 5.2e6;
    const double cost = 3.2 + 0.006 * rows + (work > stream ? work : stream);
    if (tile == 64 || cost < least) { c.wide = tile; least = cost; }
  }
  if (mean > 256) return c;
  // Narrow: 0.24 us a block of K (listed rows 0.035 more for every four), two CTAs on an SM 1.6 times that each; weights at 6.5 TB/s at
  // most.  K shared by a cluster: as much less of it for each CTA, and a join that grows with the rows (1 x 4096 x 4096 11.3 us in one
  // piece, 8.0 in four; 64 x 4096 x 4096 13.0 and 10.5; 40 x 2048 x 8192 8.8 in one, 10.3 in two).  Clusters of eight need GPCs with room
  // for them: one CTA per SM takes 16.2 us for 40 x 8192 x 2048, two per SM 9.5.
  for (int tokens = mean <= 16 ? 16 : 32; tokens <= (mean <= 16 ? 16 : 64); tokens *= 2) {
    const int64_t tiles = row_tiles(tokens) * features;
    const int64_t most = (a.offsets ? a.R / tokens + met : ceil_div(a.R, tokens)) * features;      // that there can be
    const double rows = (double)rows_of_tile(tokens);
    for (int splits = 1; splits <= 8; splits *= 2) {
      for (int per_sm = 1; per_sm <= 2; ++per_sm) {
        const int64_t room = splits == 8 && per_sm == 1 ? sms * 3 / 4 : sms * per_sm;
        if (splits > 1 && (most * splits > room || blocks < splits)) continue;
        // Two CTAs per SM where there are more than SMs (8 lists of 5 rows, 4096 x 4096: 24.8 us, one per SM 25.6), else one (some SMs
        // would get two and others none: 192 x 4096 x 4096 17.4, one per SM 14.0).
        if (splits == 1 ? per_sm != (tiles > sms ? 2 : 1) : per_sm == 2 && tiles * splits <= sms) continue;
        const double rounds = (double)ceil_div(tiles * splits, room);
        const double block = (a.rows ? 0.24 + 0.035 * (double)ceil_div((int64_t)rows, 4) : 0.24 + 0.0006 * tokens) * (per_sm == 2 ? 1.6 : 1.0);
        const double work = rounds * (double)ceil_div(blocks, splits) * block, stream = bytes / 6.5e6;
        const double cost = 3.6 + 0.012 * rows + (work > stream ? work : stream) + (splits > 1 ? 0.7 + 0.04 * rows : 0.0);
        if (cost < least) { c = Choice{true, tokens, splits, per_sm, c.wide}; least = cost; }
      }
    }
  }
  return c;
}

}  // namespace

cudaError_t launch_matmul(const MatmulArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const Choice c = choose(a, sms);
  return c.narrow ? launch_matmul_narrow(a, c.tokens, c.splits, c.per_sm, s) : launch_matmul_wide(a, c.wide, s);
}

}  // namespace bl
