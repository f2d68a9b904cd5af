// The dense products' rules of csrc/rows_plan.h as plain functions, for the tests to ask without
// a GPU.
#include "rows_plan.h"

extern "C" {

void plan_linear(int in_dt, int backward, int64_t n, int red, int cols, int whole, int* out) {
  const spc::LinearPlan p = spc::linear_plan(in_dt, backward, n, red, cols, whole);
  out[0] = static_cast<int>(p.kernel);
  out[1] = p.tile;
}

int plan_linear_short(int64_t n, int red, int cols, int residual) {
  return spc::linear_short(n, red, cols, residual);
}

void plan_linear_weight(int dt, int64_t n, int C_in, int C_out, int64_t* out) {
  const spc::DwPlan p = spc::linear_dw_plan(dt, n, C_in, C_out);
  out[0] = p.tile;
  out[1] = p.chunk;
  out[2] = p.jobs;
  out[3] = p.tiles;
  out[4] = static_cast<int64_t>(p.bytes);
}
}
