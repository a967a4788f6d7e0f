// Norms and quantisation of rows in F16 (mmasim_rows.cuh).
#include "mmasim_rows.cuh"

namespace mmasim {
namespace rows {

cudaError_t launch_f16(const Args& a, int out, bool norm, cudaStream_t stream) { return launch_type<EF_F16>(a, out, norm, stream); }

}  // namespace rows
}  // namespace mmasim
