// Attention over pages: queries of float (see ttc_attend.h).
#include "ttc_attend.h"

namespace ttc {

AttendKernel attend_kernel_f32(int cache_dtype, int dim, int rows) { return attend::kernel_of<float>(cache_dtype, dim, rows); }

}  // namespace ttc
