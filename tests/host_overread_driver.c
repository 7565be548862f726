/* A set whose arrays are one entry shorter than it says, host memory under AddressSanitizer: the library reads n entries, and the
 * sanitizer has to see the read past them (tests/test_ops_sanitizers_reach.py).  argv[1]: rows, cols or coeffs.  Nothing is launched: the
 * workspace is too small, had the read been let through. */
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "modse.h"

int main(int argc, char** argv) {
  const int n = 9, steps = 5;
  const char* const which = argc > 1 ? argv[1] : "";
  int32_t* rows = (int32_t*)malloc((n - !strcmp(which, "rows")) * sizeof *rows);
  int32_t* cols = (int32_t*)malloc((n - !strcmp(which, "cols")) * sizeof *cols);
  float* coeffs = (float*)malloc((3 * steps - !strcmp(which, "coeffs")) * sizeof *coeffs);
  const float* G[9];
  void* U[9];
  modse_matrix_set set;
  for (int i = 0; i < n; ++i) {
    if (i < n - !strcmp(which, "rows")) rows[i] = 64;
    if (i < n - !strcmp(which, "cols")) cols[i] = 96;
    G[i] = (const float*)0x10000;
    U[i] = (void*)0x10000;
  }
  for (int i = 0; i < 3 * steps - !strcmp(which, "coeffs"); ++i) coeffs[i] = 0.25f; /* bounded: 0.75 after the first step */
  set.n_matrices = n;
  set.rows = rows;
  set.cols = cols;
  set.G = G;
  set.U = U;
  set.dtype = MODSE_F32;
  const modse_status got = modse_orthogonalize(&set, coeffs, steps, 1e-7f, (void*)0x10000, 16, NULL);
  printf("returned %d\n", (int)got);
  free(rows);
  free(cols);
  free(coeffs);
  return got == MODSE_ERR_WORKSPACE ? 0 : 1;
}
