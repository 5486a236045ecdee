// Attention over pages: queries of __bf16 (see ttc_attend.h).
#include "ttc_attend.h"

namespace ttc {

AttendKernel attend_kernel_bf16(int cache_dtype, int dim, int rows) { return attend::kernel_of<__bf16>(cache_dtype, dim, rows); }

}  // namespace ttc
