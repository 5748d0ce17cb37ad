// What the launchers of the tensor-core products share (host side; defined in gemm_tc.cu, which does not include this file: the measured
// DRAM traffic of the engine's products is tied to its text, and the linker checks the functions' and variables' names).
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>

namespace zl {
namespace tc {

// Whether the tensor-core kernels run on this machine; then g_encode and g_sms hold.
bool init();
extern PFN_cuTensorMapEncodeTiled_v12000 g_encode;
extern int g_sms;

}  // namespace tc
}  // namespace zl
