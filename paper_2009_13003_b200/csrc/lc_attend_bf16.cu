// The kernels of lc_attend_rows.cuh for queries of bf16.
#include "lc_attend_rows.cuh"

namespace lc {

cudaError_t launch_attend_bf16(const AttendArgs& a, int bits, bool overlap, cudaStream_t cs) { return bits == 4 ? launch_dim<4, 1>(a, overlap, cs) : launch_dim<8, 1>(a, overlap, cs); }

}  // namespace lc
