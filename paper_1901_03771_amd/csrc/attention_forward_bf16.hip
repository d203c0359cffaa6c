#include "attention_forward.h"
hipError_t gr::attn::forward_bf16(const Args& a, int dp, int mode, bool divided, unsigned grid, hipStream_t stream) { return forward_all<__bf16>(a, dp, mode, divided, grid, stream); }
