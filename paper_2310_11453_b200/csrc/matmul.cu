// Which kernel computes a matrix product of the 8-bit layers and of the experts.
#include "common.cuh"

namespace bl {

cudaError_t launch_matmul(const MatmulArgs& a, cudaStream_t s) {
  const int64_t mean = a.offsets ? (a.R + a.experts - 1) / a.experts : a.R;
  if (mean > 160) return launch_matmul_wide(a, 256, s);
  if (mean > 64) return launch_matmul_wide(a, 128, s);
  const int tokens = mean <= 16 ? 16 : mean <= 32 ? 32 : 64;
  const int64_t token_tiles = a.offsets ? a.R / tokens + (a.experts < a.R ? a.experts : a.R) : (a.R + tokens - 1) / tokens;
  const int64_t tiles = token_tiles * ((a.N + 127) / 128);
  const int64_t blocks = (a.K * (a.operand == BL_I8 ? 1 : 2) + 127) / 128;
  int splits = 1;
  while (splits < 8 && tiles * splits * 2 <= 296 && blocks >= 8 * splits) splits *= 2;
  return launch_matmul_narrow(a, tokens, splits, s);
}

}  // namespace bl
