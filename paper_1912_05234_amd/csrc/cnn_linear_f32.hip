// Linear attention's kernels for one element type (a file to each, so that they compile side by side).
#include "cnn_linear.h"

int cnn::linear::run_scan_f32(const Args& a, int roles, bool state_only, hipStream_t st) { return run_scan<float>(a, roles, state_only, st); }
