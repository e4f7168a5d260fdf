// GEMM_Q4 with groups of 32 k.
#include "gemm_q4.hpp"

namespace lithos {

gemm_q4_fn gemm_q4_g32_fn(int rows, int blocks, bool a32) { return q4_table<1>(rows, blocks, a32); }

} // namespace lithos
