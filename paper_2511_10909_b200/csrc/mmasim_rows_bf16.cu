// Norms and quantisation of rows in BF16 (mmasim_rows.cuh).
#include "mmasim_rows.cuh"

namespace mmasim {
namespace rows {

cudaError_t launch_bf16(const Args& a, int out, bool norm, cudaStream_t stream) { return launch_type<EF_BF16>(a, out, norm, stream); }

}  // namespace rows
}  // namespace mmasim
