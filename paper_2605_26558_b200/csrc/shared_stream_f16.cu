// The streaming kernel for f16 caches, a translation unit of its own: its instances take the compiler longer than the rest of the library.
#include "shared_stream.cuh"

namespace cass {

int launch_shared_stream_f16(const SharedAttn& a, int mt, int levels, int32_t* d_status, cudaStream_t s) { return launch_shared_stream<CASS_F16>(a, mt, levels, d_status, s); }

}  // namespace cass
