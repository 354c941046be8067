// Linear attention's walk forward in time, bfloat16: one source for each so that they compile side by side.
#include "linear_attention_walk.hpp"

template hipError_t ucd::attention::run_mix<ucd::seq::bf16_t, false>(ucd::attention::Mix &, bool, hipStream_t);
