// Norms and quantisation of rows in F32 (mmasim_rows.cuh).
#include "mmasim_rows.cuh"

namespace mmasim {
namespace rows {

cudaError_t launch_f32(const Args& a, int out, bool norm, cudaStream_t stream) { return launch_type<EF_F32>(a, out, norm, stream); }

}  // namespace rows
}  // namespace mmasim
