// Stand-ins for the launchers of the decode entry points (csrc/zo_decode_abi.cpp) in the CPU-only sanitizer build:
// nothing is launched, scratch pointers are checked against the workspace that the test passed.
#include "zo_internal.hpp"

#include <stdio.h>
#include <stdlib.h>

extern int g_launches;
extern const char* g_ws_lo;
extern const char* g_ws_hi;

static void inside(const void* p, size_t bytes, const char* what) {
  const char* c = (const char*)p;
  if (g_ws_lo && (c < g_ws_lo || c + bytes > g_ws_hi)) {
    fprintf(stderr, "stub: %s [%p, +%zu) outside the workspace [%p, %p)\n", what, p, bytes, (const void*)g_ws_lo, (const void*)g_ws_hi);
    abort();
  }
}

namespace zo {

hipError_t launch_cache_append(const AppendArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
int attention_paged_ranges(bool bf16, int max_len) { return max_len < (bf16 ? 16384 : 8192) ? (max_len + (bf16 ? 255 : 127)) / (bf16 ? 256 : 128) : 64; }
hipError_t launch_attention_paged(const PagedAttnArgs& a, hipStream_t) {
  ++g_launches;
  const size_t parts = (size_t)a.T * a.n_heads * a.ranges;
  if (a.ranges > 1) {
    inside(a.part_ml, parts * 8, "part_ml");
    inside(a.part_o, parts * a.c.dh * 4, "part_o");
  }
  return hipSuccess;
}
hipError_t launch_sample(const SampleArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_embed_rows(const EmbedArgs&, hipStream_t) { ++g_launches; return hipSuccess; }

}  // namespace zo
