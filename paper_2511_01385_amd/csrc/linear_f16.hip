// linear_f16.hip -- the dense product's kernels of linear_kernels.hpp for f16 storage.
#include "linear_kernels.hpp"

namespace rdfft {

LinearTable linear_table_f16() { return make_linear_table<ElemF16>(); }

}  // namespace rdfft
