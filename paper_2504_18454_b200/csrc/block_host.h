// Notes a CUDA error that no context owns (palsgd_last_cuda_error(NULL) returns it) and gives PALSGD_ECUDA.
#pragma once
__attribute__((visibility("hidden"))) int palsgd_block_cuda_fail(int cuda_error, const char* what);
