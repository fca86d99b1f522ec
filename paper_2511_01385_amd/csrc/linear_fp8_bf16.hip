// linear_fp8_bf16.hip -- the 8-bit product's kernels of linear_fp8_kernels.hpp with bf16 results.
#include "linear_fp8_kernels.hpp"

namespace rdfft {

Linear8Table linear_fp8_table_bf16() { return make_linear_fp8_table<ElemBF16>(); }

}  // namespace rdfft
