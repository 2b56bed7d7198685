// Drives the host side of the decode entry points in a CPU-only build under AddressSanitizer and
// UndefinedBehaviorSanitizer: host tables of exactly the documented size, error paths, workspaces at the sizes of
// use.  Device pointers are fake addresses that nothing dereferences.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <vector>

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
      char msg[512];                                                                          \
      zo_last_error(msg, sizeof msg);                                                         \
      fprintf(stderr, "line %d: %s -> %d, expected %d (%s)\n", __LINE__, #call, got__, (int)(want), msg); \
      ++g_failed;                                                                             \
    }                                                                                         \
  } while (0)

static void* const FAKE = (void*)(uintptr_t)0x7f0000000000ull;

int main() {
  for (int S : {1, 3, 64}) {
    for (int P : {16, 64, 1024}) {
      const int max_pages = 5;
      std::vector<int32_t> cu(S + 1), kv(S), table((size_t)S * max_pages, -1);
      for (int s = 0; s <= S; ++s) cu[s] = s;
      for (int s = 0; s < S; ++s) kv[s] = 1 + (s * 37) % (max_pages * P);
      for (int s = 0; s < S; ++s)
        for (int j = 0; j < (kv[s] + P - 1) / P; ++j) table[(size_t)s * max_pages + j] = (s + j) % 7;
      zo_batch b;
      memset(&b, 0, sizeof b);
      b.n_tokens = S; b.n_seqs = S; b.cu_seqlens = (const int32_t*)FAKE; b.seq_cand = (const int32_t*)FAKE;
      b.host_cu_seqlens = cu.data();
      zo_cache c;
      memset(&c, 0, sizeof c);
      c.n_pages = 7; c.page_size = P; c.n_kv_heads = 2; c.head_dim = 64; c.dtype = ZO_BF16; c.max_pages = max_pages;
      c.K = FAKE; c.V = FAKE; c.page_table = (const int32_t*)FAKE; c.kv_len = (const int32_t*)FAKE;
      c.host_page_table = table.data(); c.host_kv_len = kv.data();
      auto append = [&] {
        return zo_cache_append(&b, FAKE, 512, FAKE, 512, FAKE, 512, 4, nullptr, nullptr, 0.f, 1e4f, &c, FAKE, 512, nullptr);
      };
      auto attend = [&] {
        const size_t need = zo_attention_paged_workspace_bytes(S, 4, 64, max_pages * P, ZO_BF16);
        g_ws_lo = (const char*)FAKE; g_ws_hi = g_ws_lo + need;
        const int32_t st = zo_attention_paged(&b, FAKE, 512, 4, 0.1f, &c, FAKE, 512, FAKE, need, nullptr);
        g_ws_lo = g_ws_hi = nullptr;
        return st;
      };
      EXPECT(append(), ZO_OK);
      EXPECT(attend(), ZO_OK);
      const int32_t keep = kv[S - 1];
      kv[S - 1] = 0;
      EXPECT(append(), ZO_ERR_INDEX);
      kv[S - 1] = max_pages * P + 1;
      EXPECT(attend(), ZO_ERR_INDEX);
      kv[S - 1] = keep;
      table[(size_t)(S - 1) * max_pages] = 7;
      EXPECT(append(), ZO_ERR_INDEX);
      c.page_size = 24;
      EXPECT(attend(), ZO_ERR_UNSUPPORTED);
    }
  }
  for (int T : {1, 4, 64, 256, 1000})
    for (int V : {1, 1000, 50272, 151936, 1 << 19})
      for (zo_dtype dt : {ZO_F32, ZO_BF16}) {
        const size_t need = zo_sample_workspace_bytes(T, V, dt);
        g_ws_lo = (const char*)FAKE; g_ws_hi = g_ws_lo + need;
        EXPECT(zo_sample(FAKE, V, T, V, dt, (float*)FAKE, nullptr, nullptr, nullptr, (float*)FAKE, (int32_t*)FAKE, nullptr, nullptr,
                         FAKE, need, nullptr), ZO_OK);
        if (need > 0) {
          EXPECT(zo_sample(FAKE, V, T, V, dt, (float*)FAKE, nullptr, nullptr, nullptr, (float*)FAKE, (int32_t*)FAKE, nullptr, nullptr,
                           FAKE, need - 1, nullptr), ZO_ERR_WORKSPACE);
          EXPECT(zo_sample(FAKE, V, T, V, dt, (float*)FAKE, nullptr, nullptr, nullptr, (float*)FAKE, (int32_t*)FAKE, nullptr, nullptr,
                           nullptr, need, nullptr), ZO_ERR_WORKSPACE);
        }
        g_ws_lo = g_ws_hi = nullptr;
      }
  EXPECT(zo_embed_rows((int32_t*)FAKE, nullptr, 4, FAKE, 64, 100, nullptr, 0, 0, 64, ZO_F32, FAKE, 64, nullptr, nullptr), ZO_OK);
  EXPECT(zo_embed_rows((int32_t*)FAKE, nullptr, 4, FAKE, 64, 100, nullptr, 0, 0, 64, ZO_F32, FAKE, 64, (int32_t*)FAKE, nullptr), ZO_ERR_NULL);
  printf("decode host check: %d checks, %d failed, %d stub launches\n", g_checks, g_failed, g_launches);
  return g_failed ? 1 : 0;
}
