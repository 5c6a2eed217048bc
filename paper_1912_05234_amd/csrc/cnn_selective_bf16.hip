// The selective scan's kernels for one element type (a file to each, so that they compile side by side).
#include "cnn_selective.h"

void cnn::selective::launch_bf16(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st) { launch_type<__bf16>(a, pass, f, grid, st); }
