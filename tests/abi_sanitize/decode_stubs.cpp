// Stand-ins for the launchers of the decode entry points (csrc/zo_decode_abi.cpp) in the CPU-only sanitizer build:
// nothing is launched, scratch pointers are checked against the workspace that the test passed.
#include "zo_internal.hpp"

extern int g_launches;

namespace zo {

hipError_t launch_cache_append(const AppendArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_attention_paged(const PagedAttnArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_sample(const SampleArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_embed_rows(const EmbedArgs&, hipStream_t) { ++g_launches; return hipSuccess; }

}  // namespace zo
