#include "cnn_norm.h"

namespace cnn {
namespace norm {
void launch_f32(const Args& a, int stream_type, Mode mode, bool backward, Cut cut, unsigned grid, hipStream_t st) {
  launch_type<float>(a, stream_type, mode, backward, cut, grid, st);
}
}  // namespace norm
}  // namespace cnn
