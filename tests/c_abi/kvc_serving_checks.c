/*
 * Host-side checks of the packed-sequence plans, the pages and the attention
 * over a shared prefix, for a build of the library whose host code is
 * instrumented (tests/test_serving_sanitizers.py).  The "device" addresses are
 * fake, so it runs only where there is no GPU: a valid call then stops at the
 * device check with KVC_ERR_DEVICE.  Exit status: 0 all checks passed, 1 a
 * check failed, 77 skipped (a GPU is present).
 */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "kvc.h"

#define EXPECT(cond)                                                                                          \
  do {                                                                                                        \
    if (!(cond)) {                                                                                            \
      fprintf(stderr, "line %d: check failed: %s (last error: %s)\n", __LINE__, #cond, kvc_last_error());     \
      return 1;                                                                                               \
    }                                                                                                         \
  } while (0)

static uint64_t g_state = 88172645463325252ull;

/* xorshift64 (Marsaglia), a seeded stream of test parameters */
static uint64_t next_u64(void) {
  g_state ^= g_state << 13;
  g_state ^= g_state >> 7;
  g_state ^= g_state << 17;
  return g_state;
}
static int32_t uniform(int32_t lo, int32_t hi) { return lo + (int32_t)(next_u64() % (uint64_t)((int64_t)hi - lo + 1)); }

static void* fake(int i) { return (void*)(uintptr_t)((uint64_t)(i + 1) << 42); }

static int pack_round(int it) {
  enum { kMax = 500 };
  int32_t len[kMax];
  kvc_pack P;
  memset(&P, 0, sizeof(P));
  P.n_seqs = uniform(0, it % 4 ? 20 : kMax);
  for (int32_t i = 0; i < P.n_seqs; ++i)
    len[i] = next_u64() % 6 == 0 ? 0 : uniform(1, it % 5 == 0 ? 9000 : it % 2 ? 800 : 70);
  P.seq_len = len;
  P.n_kv_heads = it % 3 == 0 ? uniform(1, 64) : 1 << uniform(0, 3);
  P.n_q_heads = P.n_kv_heads * uniform(1, 16);
  P.head_dim = 128;
  int64_t rows = 0;
  for (int32_t i = 0; i < P.n_seqs; ++i) rows += len[i];
  size_t pb = 0, wb = 0;
  kvc_plan plan;
  memset(&plan, 0, sizeof(plan));
  EXPECT(kvc_pack_plan_bytes(&P, &pb) == KVC_OK && pb > 0);
  EXPECT(kvc_packed_attention_workspace(&P, &wb) == KVC_OK);
  EXPECT(kvc_pack_plan_upload(&P, fake(0), pb - 1, NULL, &plan, NULL) == KVC_ERR_WORKSPACE);
  EXPECT(kvc_pack_plan_upload(&P, fake(0), pb, NULL, &plan, NULL) == KVC_ERR_DEVICE && plan.device == NULL);
  void* staging = malloc(pb);
  const kvc_status st = kvc_pack_plan_upload(&P, fake(0), pb, staging, &plan, NULL);
  EXPECT(st == KVC_ERR_DEVICE);
  memcpy(&plan.layout_id, staging, sizeof(plan.layout_id)); /* the header starts with the id */
  free(staging);
  plan.device = fake(0);
  plan.bytes = pb;
  EXPECT(kvc_packed_attention(&P, &plan, fake(1), fake(2), fake(3), rows, 0.0f, fake(4), (float*)fake(5), fake(6), wb,
                              NULL) == (rows > 0 ? KVC_ERR_DEVICE : KVC_OK));
  if (rows > 0) {
    EXPECT(kvc_packed_attention(&P, &plan, fake(1), fake(2), fake(3), rows - 1, 0.0f, fake(4), NULL, fake(6), wb, NULL) ==
           KVC_ERR_INVALID_ARG);
    plan.layout_id ^= 2;
    EXPECT(kvc_packed_attention(&P, &plan, fake(1), fake(2), fake(3), rows, 0.0f, fake(4), NULL, fake(6), wb, NULL) ==
           KVC_ERR_INVALID_ARG);
  }
  return 0;
}

static int pages_round(int it) {
  kvc_pages P;
  memset(&P, 0, sizeof(P));
  P.page_rows = 8 << uniform(0, 7);
  P.n_pages = uniform(1, it % 3 ? 5000 : 2000000);
  P.n_slots = uniform(0, it % 4 ? 200 : KVC_PAGES_MAX_SLOTS);
  P.max_pages = uniform(0, it % 4 ? 3000 : 30);
  P.ref = (int32_t*)fake(0);
  P.table = (int32_t*)fake(1);
  P.len = (int32_t*)fake(2);
  size_t wb = 0, sb = 0;
  EXPECT(kvc_pages_workspace(&P, &wb) == KVC_OK && wb > 0);
  const kvc_status want = P.n_slots > 0 ? KVC_ERR_DEVICE : KVC_OK;
  EXPECT(kvc_pages_trim(&P, (int32_t*)fake(3), NULL) == want);
  EXPECT(kvc_pages_fork(&P, (int32_t*)fake(3), fake(4), wb, NULL) == want);
  EXPECT(kvc_pages_reserve(&P, (int32_t*)fake(3), uniform(1, 4000), (int32_t*)fake(5), (int32_t*)fake(6),
                           (int32_t*)fake(7), (int32_t*)fake(8), fake(4), wb, NULL) == KVC_ERR_DEVICE);
  EXPECT(kvc_pages_compact(&P, (int32_t*)fake(5), (int32_t*)fake(6), (int32_t*)fake(7), fake(4), wb, NULL) ==
         KVC_ERR_DEVICE);
  const int32_t hkv = 1 << uniform(0, 3), hq = hkv * uniform(1, 8), n_new = uniform(1, 6);
  const int64_t n_prefix = it % 5 == 0 ? ((int64_t)1 << 31) - 128 : uniform(0, 200000);
  const kvc_status sw = kvc_shared_prefix_workspace(&P, n_prefix, n_new, hq, hkv, 128, &sb);
  EXPECT(sw == KVC_OK || sw == KVC_ERR_INVALID_ARG); /* too much for one launch */
  if (sw == KVC_OK && it % 5) {
    EXPECT(kvc_shared_prefix_attention(fake(10), n_new, fake(11), fake(12), n_prefix, &P, fake(13), fake(14), hq, hkv, 128,
                                       0.0f, fake(15), (float*)fake(16), fake(17), sb, NULL) == want);
    if (P.n_slots > 0 && sb > 0)
      EXPECT(kvc_shared_prefix_attention(fake(10), n_new, fake(11), fake(12), n_prefix, &P, fake(13), fake(14), hq, hkv,
                                         128, 0.0f, fake(15), (float*)fake(16), fake(17), sb - 1,
                                         NULL) == KVC_ERR_WORKSPACE);
  }
  return 0;
}

int main(void) {
  int n_dev = 0;
  if (hipGetDeviceCount(&n_dev) == hipSuccess && n_dev > 0) {
    puts("skip: a GPU is present (these checks pass fake device addresses)");
    return 77;
  }
  for (int it = 0; it < 400; ++it)
    if (pack_round(it) || pages_round(it)) return 1;
  /* limits of a launch and of the row numbers */
  kvc_pack P;
  memset(&P, 0, sizeof(P));
  int32_t len[2] = {(int32_t)(((int64_t)1 << 31) - 128), 1};
  size_t b = 0;
  P.n_seqs = 2;
  P.seq_len = len;
  P.n_q_heads = P.n_kv_heads = 1;
  P.head_dim = 128;
  EXPECT(kvc_pack_plan_bytes(&P, &b) == KVC_ERR_INVALID_ARG);
  P.n_seqs = 1;
  EXPECT(kvc_pack_plan_bytes(&P, &b) == KVC_ERR_INVALID_ARG); /* 8.4 million blocks */
  len[0] = 1 << 29;
  EXPECT(kvc_pack_plan_bytes(&P, &b) == KVC_OK && b > 0);
  puts("serving checks ok");
  return 0;
}
