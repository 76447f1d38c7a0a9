#include "linear_laid.h"

namespace sc {

int launch_laid_f16(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s) { return launch_kernel<_Float16>(kernel, turned, a, s); }

}  // namespace sc
