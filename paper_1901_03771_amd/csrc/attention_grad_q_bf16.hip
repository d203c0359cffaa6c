#include "attention_backward.h"
hipError_t gr::attn::grad_q_bf16(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream) { return grad_q_all<__bf16>(a, dp, mode, grid, stream); }
