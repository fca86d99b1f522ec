// linear_fp8_f32.hip -- the 8-bit product's kernels of linear_fp8_kernels.hpp with float32 results.
#include "linear_fp8_kernels.hpp"

namespace rdfft {

Linear8Table linear_fp8_table_f32() { return make_linear_fp8_table<ElemF32>(); }

}  // namespace rdfft
