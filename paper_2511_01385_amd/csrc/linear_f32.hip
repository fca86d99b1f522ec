// linear_f32.hip -- the dense product's kernels of linear_kernels.hpp for f32 storage.
#include "linear_kernels.hpp"

namespace rdfft {

LinearTable linear_table_f32() { return make_linear_table<ElemF32>(); }

}  // namespace rdfft
