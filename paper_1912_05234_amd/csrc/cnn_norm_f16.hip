// The norms' kernels for one element type (a file to each, so that they compile side by side).
#include "cnn_norm.h"

void cnn::norm::launch_f16(const Args& a, int stream_type, Mode mode, bool backward, Cut cut, unsigned grid, hipStream_t st) {
  launch_type<_Float16>(a, stream_type, mode, backward, cut, grid, st);
}
