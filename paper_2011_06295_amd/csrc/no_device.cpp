// Stand-ins for the device side of the library in the host-only build that the sanitizer check links
// (build.py --sanitize): everything that would enqueue a kernel reports "not supported".
#include <hip/hip_runtime_api.h>

#include "internal.h"
#include "text_ops.h"

namespace sc {

int static_scratch(void**) { return (int)hipErrorNotSupported; }
int launch_tile_kernel(int, int, int, int, const KernelArgs&, int, int, int, void*) { return (int)hipErrorNotSupported; }
int launch_matrix_f32(const MatrixPlan&, const MatrixArgs&, void*) { return (int)hipErrorNotSupported; }
int launch_matrix_f16(const MatrixPlan&, const MatrixArgs&, void*) { return (int)hipErrorNotSupported; }
int launch_lds_read_probe(void*, int, int, void*, long long*) { return (int)hipErrorNotSupported; }
int launch_copy_probe(void*, const void*, long long, void*) { return (int)hipErrorNotSupported; }

int launch_embed(int, const EmbedArgs&, void*) { return (int)hipErrorNotSupported; }
int launch_embed_grad(int, int, const EmbedGradArgs&, char*, void*) { return (int)hipErrorNotSupported; }
int launch_int8_quantize(int, const void*, int8_t*, float*, int, int, long long, void*) { return (int)hipErrorNotSupported; }
int launch_int8_linear(int, int, const Int8Args&, char*, void*) { return (int)hipErrorNotSupported; }
// (some calls need scratch memory and some none)
long long embed_grad_workspace(const EmbedGradArgs& a, int) { return a.dim % 2 ? 16ll * a.sentences * a.words : 0; }
long long int8_workspace(int M, int, int K, int in_dtype, int) { return in_dtype < 3 && K % 2 ? (long long)M * K : 0; }

}  // namespace sc
