// linear_fp8_f16.hip -- the 8-bit product's kernels of linear_fp8_kernels.hpp with f16 results.
#include "linear_fp8_kernels.hpp"

namespace rdfft {

Linear8Table linear_fp8_table_f16() { return make_linear_fp8_table<ElemF16>(); }

}  // namespace rdfft
