#include "linear_laid.h"

namespace sc {

int launch_laid_bf16(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s) { return launch_kernel<__bf16>(kernel, turned, a, s); }

}  // namespace sc
