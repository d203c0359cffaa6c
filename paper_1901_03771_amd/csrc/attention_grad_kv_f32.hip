#include "attention_backward.h"
hipError_t gr::attn::grad_kv_f32(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream) { return grad_kv_all<float>(a, dp, mode, grid, stream); }
