#include "linear_laid.h"

namespace sc {

int launch_laid_f32(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s) { return launch_kernel<float>(kernel, turned, a, s); }

}  // namespace sc
