// Linear attention's walk forward in time, fp32: one source for each so that they compile side by side.
#include "linear_attention_walk.hpp"

template hipError_t ucd::attention::run_mix<float, false>(ucd::attention::Mix &, bool, hipStream_t);
