/* The host side of the feed-forward calls under the address and undefined-behaviour sanitizers: sizes of workspaces over many shapes, calls with a workspace that is too small and
 * one that is enough, null and unaligned pointers.  For machines without a GPU, where the calls that are not refused end: the pointers are none. */
#include <stdio.h>
#include <string.h>

#include "eco.h"

static void *at(unsigned long p) { return (void *)p; }

static eco_linear_t linear(uint64_t rows, uint64_t in, uint64_t out, uint64_t group, int fmt) {
  eco_linear_t l;
  memset(&l, 0, sizeof l);
  l.codes = at(0x1000); l.code_scales = at(0x2000); l.weights = at(0x3000); l.scales = at(0x4000); l.out = at(0x5000); l.grad_out = at(0x6000); l.grad_input = at(0x7000);
  l.grad_weights = at(0x8000); l.rows = rows; l.in_dim = in; l.out_dim = out; l.group_size = group; l.fmt = fmt; l.out_dtype = rows % 3 ? ECO_DT_BF16 : ECO_DT_FP32;
  return l;
}
static eco_gated_t gated(uint64_t rows, uint64_t in, uint64_t width, uint64_t group, int fmt) {
  eco_gated_t g;
  memset(&g, 0, sizeof g);
  g.codes = at(0x1000); g.code_scales = at(0x2000); g.gate = g.up = at(0x3000); g.gate_scales = g.up_scales = at(0x4000); g.out = at(0x5000); g.out_scales = at(0x6000);
  g.grad_out = at(0x7000); g.grad_input = at(0x8000); g.grad_gate = at(0x9000); g.grad_up = at(0xA000); g.rows = rows; g.in_dim = in; g.width = width; g.group_size = group; g.fmt = fmt;
  return g;
}

int main(void) {
  const uint64_t rows[] = {0, 1, 16, 17, 64, 65, 300, 4097, 1u << 20, 1u << 23}, dims[] = {16, 128, 640, 1152, 6912, 65536}, widths[] = {1, 100, 2048, 65535};
  size_t n, small = 0, more = 0;
  int k, j, i, fmt, back;
  for (k = 0; k < 10; ++k)
    for (j = 0; j < 6; ++j)
      for (i = 0; i < 4; ++i)
        for (fmt = 0; fmt < 2; ++fmt) {
          eco_linear_t l = linear(rows[k], dims[j], widths[i], dims[j], fmt);
          eco_gated_t g = gated(rows[k], dims[j], widths[i], dims[j], fmt);
          for (back = 0; back < 2; ++back) {
            eco_status_t s = eco_linear_workspace(&l, back, &n);
            if (s == ECO_OK && n) small += (back ? eco_linear_backward : eco_linear)(&l, at(0x100000), 1, 0) == ECO_EINVAL;
            if (s == ECO_OK) more += (back ? eco_linear_backward : eco_linear)(&l, at(0x100000), n, 0) == ECO_EINVAL;
            s = eco_gated_workspace(&g, back, &n);
            if (s == ECO_OK && n) small += (back ? eco_gated_backward : eco_gated)(&g, at(0x100000), 1, 0) == ECO_EINVAL;
            if (s == ECO_OK) more += (back ? eco_gated_backward : eco_gated)(&g, at(0x100000), n, 0) == ECO_EINVAL;
          }
        }
  if (eco_linear(0, 0, 0, 0) != ECO_EINVAL || eco_gated(0, 0, 0, 0) != ECO_EINVAL || eco_norm(0, 0) != ECO_EINVAL || eco_linear_workspace(0, 0, &n) != ECO_EINVAL ||
      eco_norm_backward(0, 0, 0, 0) != ECO_EINVAL || eco_rows_quantize(0, 0, 1, 1, 0, 0, 0, 0, 0) != ECO_EINVAL) {
    printf("FAILED: null pointers\n");
    return 1;
  }
  {
    eco_linear_t l = linear(4, 128, 64, 128, 0);
    eco_norm_t r;
    l.weights = at(0x3008);
    if (eco_linear(&l, at(0x100000), 1 << 20, 0) != ECO_EALIGN) { printf("FAILED: alignment\n"); return 1; }
    memset(&r, 0, sizeof r);
    r.input = at(0x1000); r.out = at(0x2000); r.rstd = (float *)at(0x3000); r.grad_out = at(0x4000); r.grad_gain = at(0x5000); r.dim = 512; r.eps = 1e-6; r.rows = 1u << 23;
    if (eco_norm_backward_workspace(&r, &n) != ECO_OK || n != 4ull * 1024 * 512 || eco_norm_backward(&r, at(0x100000), n - 1, 0) != ECO_EINVAL) { printf("FAILED: norm\n"); return 1; }
  }
  if (small == 0 || more) { printf("FAILED: %zu too small, %zu refused with what was asked for\n", small, more); return 1; }
  printf("ok\n");
  return 0;
}
