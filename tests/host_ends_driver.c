/* The argument checks of the operators at both ends of a model from plain C, host code under AddressSanitizer and
 * UndefinedBehaviorSanitizer (tests/test_ends_sanitizers.py).  Every call returns before anything is launched. */
#include <math.h>
#include <stdio.h>

#include "modse.h"

static int failures = 0;
#define EXPECT(call, want)                                                                        \
  do {                                                                                            \
    modse_status got_ = (call);                                                                   \
    if (got_ != (want)) {                                                                         \
      fprintf(stderr, "line %d: %s returned %d (%s), expected %d\n", __LINE__, #call, (int)got_,  \
              modse_status_string(got_), (int)(want));                                            \
      ++failures;                                                                                 \
    }                                                                                             \
  } while (0)

int main(void) {
  void* const p = (void*)0x10000; /* stands for device memory */
  float* const f = (float*)p;
  const int32_t* const t = (const int32_t*)p;
  const uint64_t* const g = (const uint64_t*)p;
  size_t bytes = 0, most = 0;
  const modse_dtype odd = (modse_dtype)9;

  EXPECT(modse_embed_fwd(0, 64, 9, MODSE_F32, NULL, NULL, 1.f, NULL, NULL), MODSE_OK);
  EXPECT(modse_embed_fwd(4, 64, 9, MODSE_F32, t, NULL, 1.f, p, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_embed_fwd(4, 64, 9, odd, t, p, 1.f, p, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_embed_fwd(INT64_MAX, 64, 9, MODSE_BF16, t, p, 1.f, p, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_embed_fwd(INT64_MIN, 64, 9, MODSE_BF16, t, p, 1.f, p, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_embed_fwd(4, INT32_MAX, INT32_MAX, MODSE_BF16, t, p, 1.f, p, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_embed_fwd(4, 64, INT32_MIN, MODSE_BF16, t, p, 1.f, p, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_embed_fwd(4, 64, 9, MODSE_BF16, t, p, INFINITY, p, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_embed_bwd_workspace_size(1, 1, 1, MODSE_BF16, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_embed_bwd_workspace_size(INT64_MAX, 16384, 1 << 20, MODSE_BF16, &bytes), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_embed_bwd_workspace_size((1 << 24) - 64, 16384, 1 << 20, MODSE_BF16, &bytes), MODSE_OK);
  EXPECT(modse_embed_bwd((1 << 24) - 64, 16384, 1 << 20, MODSE_BF16, t, p, 1.f, f, 0, p, bytes - 1, NULL), MODSE_ERR_WORKSPACE);
  EXPECT(modse_embed_bwd(5, 7, 9, MODSE_F32, t, p, 1.f, f, 1, NULL, 1 << 20, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_embed_bwd(5, 7, 9, MODSE_F32, t, p, 1.f, f, 1, (char*)p + 4, 1 << 20, NULL), MODSE_ERR_INVALID_ARG);

  for (int which = MODSE_WS_FWD; which <= MODSE_WS_BWD; ++which)
    for (int dt = MODSE_F32; dt <= MODSE_BF16; ++dt)
      for (int32_t d = 32; d <= 16384; d *= 8)
        for (int32_t v = 1; v <= 1 << 20; v = v * 7 + (v < 200000 ? 1 : 1 << 20)) {
          if (v > 1 << 20) v = 1 << 20;
          size_t last = 0;
          for (int64_t T = 1; T <= (int64_t)1 << 24; T = T * 5 + 3) {
            EXPECT(modse_head_workspace_size(T, d, v, (modse_dtype)dt, which, &bytes), MODSE_OK);
            if (bytes < last) ++failures, fprintf(stderr, "size falls at T = %lld, d = %d, vocab = %d\n", (long long)T, (int)d, (int)v);
            last = bytes;
            if (bytes > most) most = bytes;
            if (which == MODSE_WS_FWD) EXPECT(modse_head_fwd(T, d, v, (modse_dtype)dt, p, p, t, f, f, p, bytes - 1, NULL), MODSE_ERR_WORKSPACE);
            else EXPECT(modse_head_bwd(T, d, v, (modse_dtype)dt, p, p, t, f, f, p, f, 0, p, bytes - 1, NULL), MODSE_ERR_WORKSPACE);
          }
        }
  EXPECT(modse_head_workspace_size(1, 32, 1, MODSE_BF16, MODSE_WS_FWD_SAVED, &bytes), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_head_workspace_size(1, 32, 1, MODSE_BF16, 77, &bytes), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_head_workspace_size(1, 33, 1, MODSE_BF16, MODSE_WS_FWD, &bytes), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_head_workspace_size(INT64_MAX, 32, 1, MODSE_BF16, MODSE_WS_FWD, &bytes), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_head_fwd(0, 32, 1, odd, NULL, NULL, NULL, NULL, NULL, NULL, 0, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_head_fwd(0, 32, 1, MODSE_F32, NULL, NULL, NULL, NULL, NULL, NULL, 0, NULL), MODSE_OK);
  EXPECT(modse_head_bwd(1, 32, 1, MODSE_F32, p, p, t, NULL, f, p, f, 0, p, (size_t)-1, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_head_bwd(1, 32, 1, MODSE_F32, p, p, t, f, f, NULL, NULL, 0, p, (size_t)-1, NULL), MODSE_ERR_INVALID_ARG);

  EXPECT(modse_dropout_fwd(0, 64, MODSE_F32, NULL, NULL, 0.5, NULL, 0, NULL, NULL), MODSE_OK);
  EXPECT(modse_dropout_fwd(1, 64, MODSE_F32, p, NULL, NAN, g, 0, p, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_dropout_fwd(INT64_MAX, 16384, MODSE_F32, p, NULL, 0.5, g, 0, p, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_dropout_fwd(1 << 21, 16384, MODSE_F32, p, NULL, 0.5, g, 0, p, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_dropout_bwd(1, 64, MODSE_F32, p, 0.5, NULL, 0xffffffffu, p, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_dropout_bwd(1, 64, odd, p, 0.5, g, 0, p, NULL), MODSE_ERR_UNSUPPORTED);

  if (failures) return 1;
  printf("all checks passed (largest workspace %zu MiB)\n", most >> 20);
  return 0;
}
