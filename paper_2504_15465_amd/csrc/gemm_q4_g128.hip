// GEMM_Q4 with groups of 128 k.
#include "gemm_q4.hpp"

namespace lithos {

gemm_q4_fn gemm_q4_g128_fn(int rows, int blocks, bool a32) { return q4_table<4>(rows, blocks, a32); }

} // namespace lithos
