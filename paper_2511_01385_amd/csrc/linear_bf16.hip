// linear_bf16.hip -- the dense product's kernels of linear_kernels.hpp for bf16 storage.
#include "linear_kernels.hpp"

namespace rdfft {

LinearTable linear_table_bf16() { return make_linear_table<ElemBF16>(); }

}  // namespace rdfft
