/* The argument checks of the operators around the layer from plain C, host code under AddressSanitizer and
 * UndefinedBehaviorSanitizer (tests/test_ops_sanitizers.py).  Every call returns before anything is launched. */
#include <stdio.h>
#include <stdlib.h>

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
  int32_t* const t = (int32_t*)p;
  size_t bytes = 0;
  const modse_dtype odd = (modse_dtype)9;

  EXPECT(modse_norm_fwd(0, 64, MODSE_F32, NULL, NULL, NULL, 0.f, NULL, NULL, NULL, NULL, NULL, 0, NULL), MODSE_OK);
  EXPECT(modse_norm_fwd(3, 64, MODSE_F32, p, NULL, NULL, 0.f, p, NULL, NULL, NULL, NULL, 0, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_norm_fwd(3, 64, odd, p, NULL, p, 0.f, p, NULL, NULL, NULL, NULL, 0, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_norm_fwd(INT64_MAX, 64, MODSE_F32, p, NULL, p, 0.f, p, NULL, NULL, NULL, NULL, 0, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_norm_fwd(3, INT32_MAX, MODSE_F32, p, NULL, p, 0.f, p, NULL, NULL, NULL, NULL, 0, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_norm_fwd(3, 64, MODSE_F32, p, NULL, p, 0.f, p, NULL, NULL, p, f, -128, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_norm_bwd_workspace_size(1 << 20, 16384, MODSE_BF16, &bytes), MODSE_OK);
  EXPECT(modse_norm_bwd_workspace_size(1, 1, MODSE_BF16, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_norm_bwd(1 << 20, 16384, MODSE_BF16, p, p, f, p, NULL, p, f, 0, p, bytes - 1, NULL), MODSE_ERR_WORKSPACE);
  EXPECT(modse_norm_bwd(5, 7, MODSE_BF16, p, p, f, p, NULL, p, f, 0, NULL, 1 << 20, NULL), MODSE_ERR_INVALID_ARG);

  EXPECT(modse_logprobs_workspace_size(INT64_MAX, 5, MODSE_F32, 0, &bytes), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_logprobs_workspace_size(100, 1 << 30, MODSE_F32, 64, &bytes), MODSE_OK);
  EXPECT(modse_logprobs_workspace_size(100, INT32_MAX, MODSE_F32, 64, &bytes), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_logprobs_workspace_size(2, 140000, MODSE_BF16, INT32_MAX, &bytes), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_logprobs_workspace_size(2, 140000, MODSE_BF16, 5, &bytes), MODSE_OK);
  EXPECT(modse_logprobs_fwd(2, 140000, MODSE_BF16, p, 140000, t, f, f, f, 5, t, f, p, bytes - 1, NULL), MODSE_ERR_WORKSPACE);
  EXPECT(modse_logprobs_fwd(2, 140000, MODSE_BF16, p, -140000, t, f, f, f, 5, t, f, p, bytes, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_logprobs_fwd(0, 140000, odd, p, 0, t, f, f, f, 5, t, f, p, bytes, NULL), MODSE_ERR_UNSUPPORTED);
  EXPECT(modse_logprobs_bwd(2, 100, MODSE_F32, p, 100, t, NULL, f, f, f, p, 100, NULL), MODSE_ERR_INVALID_ARG);
  EXPECT(modse_logprobs_bwd(2, 100, MODSE_F32, p, 100, t, f, NULL, f, f, p, 100, NULL), MODSE_ERR_INVALID_ARG);

  { /* arrays of exactly n entries on the heap: a read past them is an error the sanitizer reports */
    const int n = 70;
    int32_t* rows = (int32_t*)malloc(n * sizeof *rows);
    int32_t* cols = (int32_t*)malloc(n * sizeof *cols);
    const float** G = (const float**)malloc(n * sizeof *G);
    void** U = (void**)malloc(n * sizeof *U);
    float* coeffs = (float*)malloc(3 * 32 * sizeof *coeffs);
    modse_matrix_set set;
    for (int i = 0; i < n; ++i) {
      rows[i] = 1 + 37 * i;
      cols[i] = 65536 - 900 * i;
      G[i] = f;
      U[i] = p;
    }
    for (int i = 0; i < 32; ++i) {
      coeffs[3 * i] = 3.4445f;
      coeffs[3 * i + 1] = -4.775f;
      coeffs[3 * i + 2] = 2.0315f;
    }
    set.n_matrices = n;
    set.rows = rows;
    set.cols = cols;
    set.G = G;
    set.U = U;
    set.dtype = MODSE_BF16;
    EXPECT(modse_orthogonalize_workspace_size(&set, &bytes), MODSE_OK);
    EXPECT(modse_orthogonalize(&set, coeffs, 32, 1e-7f, p, bytes - 1, NULL), MODSE_ERR_WORKSPACE);
    EXPECT(modse_orthogonalize(&set, coeffs, 33, 1e-7f, p, bytes, NULL), MODSE_ERR_UNSUPPORTED);
    EXPECT(modse_orthogonalize(&set, coeffs, 0, 1e-7f, p, bytes, NULL), MODSE_ERR_INVALID_ARG);
    EXPECT(modse_orthogonalize(&set, NULL, 5, 1e-7f, p, bytes, NULL), MODSE_ERR_INVALID_ARG);
    EXPECT(modse_orthogonalize(NULL, coeffs, 5, 1e-7f, p, bytes, NULL), MODSE_ERR_INVALID_ARG);
    U[n - 1] = NULL;
    EXPECT(modse_orthogonalize(&set, coeffs, 5, 1e-7f, p, bytes, NULL), MODSE_ERR_INVALID_ARG);
    cols[n - 1] = 0;
    EXPECT(modse_orthogonalize(&set, coeffs, 5, 1e-7f, p, bytes, NULL), MODSE_ERR_INVALID_ARG);
    EXPECT(modse_orthogonalize_workspace_size(&set, NULL), MODSE_ERR_INVALID_ARG);
    set.dtype = odd;
    EXPECT(modse_orthogonalize_workspace_size(&set, &bytes), MODSE_ERR_UNSUPPORTED);
    set.dtype = MODSE_F32;
    set.n_matrices = 0;
    set.rows = set.cols = NULL;
    EXPECT(modse_orthogonalize(&set, coeffs, 5, 1e-7f, NULL, 0, NULL), MODSE_OK);
    free(rows);
    free(cols);
    free(G);
    free(U);
    free(coeffs);
  }
  if (failures) fprintf(stderr, "%d check(s) failed\n", failures);
  else printf("host operators driver: all checks passed\n");
  return failures ? 1 : 0;
}
