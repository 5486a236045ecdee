// Attention over pages: queries of _Float16 (see ttc_attend.h).
#include "ttc_attend.h"

namespace ttc {

AttendKernel attend_kernel_f16(int cache_dtype, int dim, int rows) { return attend::kernel_of<_Float16>(cache_dtype, dim, rows); }

}  // namespace ttc
