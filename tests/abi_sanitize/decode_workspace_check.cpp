// Drives zo_attention_paged's workspace checks in a CPU-only build under AddressSanitizer and UndefinedBehaviorSanitizer: calls
// that need a workspace (rows of more than one range), with one that is missing, misaligned, too small by a byte, or just enough.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "../../include/zo.h"

extern int g_launches;
extern const char* g_ws_lo;
extern const char* g_ws_hi;

static int g_checks = 0, g_failed = 0;
#define EXPECT(call, want)                                                                    \
  do {                                                                                        \
    const int32_t got__ = (call);                                                             \
    ++g_checks;                                                                               \
    if (got__ != (want)) {                                                                    \
      fprintf(stderr, "line %d: %s -> %d, expected %d\n", __LINE__, #call, got__, (int)(want)); \
      ++g_failed;                                                                             \
    }                                                                                         \
  } while (0)

static char* const FAKE = (char*)(uintptr_t)0x7f0000000000ull;

int main() {
  for (zo_dtype dt : {ZO_F32, ZO_BF16})
    for (int T : {1, 7, 300})
      for (int max_pages : {17, 64, 5000}) {
        const int H = 4, dh = 128, P = 64;
        zo_batch b;
        memset(&b, 0, sizeof b);
        b.n_tokens = T; b.n_seqs = T; b.cu_seqlens = (const int32_t*)FAKE; b.seq_cand = (const int32_t*)FAKE;
        zo_cache c;
        memset(&c, 0, sizeof c);
        c.n_pages = 7; c.page_size = P; c.n_kv_heads = 2; c.head_dim = dh; c.dtype = dt; c.max_pages = max_pages;
        c.K = FAKE; c.V = FAKE; c.page_table = (const int32_t*)FAKE; c.kv_len = (const int32_t*)FAKE;
        const size_t need = zo_attention_paged_workspace_bytes(T, H, dh, max_pages * P, dt);
        ++g_checks;
        if (need == 0) { fprintf(stderr, "no workspace for %d pages\n", max_pages); ++g_failed; }
        auto attend = [&](void* ws, size_t bytes) {
          return zo_attention_paged(&b, FAKE, H * dh, H, 0.1f, &c, FAKE, H * dh, ws, bytes, nullptr);
        };
        const int before = g_launches;
        EXPECT(attend(nullptr, need), ZO_ERR_WORKSPACE);
        EXPECT(attend(FAKE + 128, need), ZO_ERR_WORKSPACE);
        EXPECT(attend(FAKE, need - 1), ZO_ERR_WORKSPACE);
        EXPECT(attend(FAKE, 0), ZO_ERR_WORKSPACE);
        EXPECT(attend(FAKE, zo_attention_paged_workspace_bytes(T, H, dh, 8 * P, dt)), ZO_ERR_WORKSPACE);   // of a narrower table
        EXPECT(g_launches, before);
        g_ws_lo = FAKE; g_ws_hi = FAKE + need;
        EXPECT(attend(FAKE, need), ZO_OK);
        g_ws_lo = g_ws_hi = nullptr;
        EXPECT(g_launches, before + 1);
      }
  printf("decode workspace check: %d checks, %d failed\n", g_checks, g_failed);
  return g_failed ? 1 : 0;
}
