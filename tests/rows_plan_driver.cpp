// The rules of csrc/rows_plan.h as plain functions, for the tests to ask without a GPU.
#include "rows_plan.h"

extern "C" {

void plan_grouped(int in_dt, int out_dt, int backward, int64_t m, int E, int red, int cols,
                  int whole, int* out) {
  const spc::GroupedPlan p = spc::grouped_plan(in_dt, out_dt, backward, m, E, red, cols, whole);
  out[0] = static_cast<int>(p.kernel);
  out[1] = p.tile;
  out[2] = p.ring;
}

void plan_weight(int dt, int64_t m, int E, int C_in, int C_out, int whole, int64_t* out) {
  const spc::DwPlan p = spc::dw_plan(dt, m, E, C_in, C_out, whole);
  out[0] = p.tile;
  out[1] = p.chunk;
  out[2] = p.jobs;
  out[3] = p.chunk ? spc::dw_sum_runs(p, E, static_cast<int64_t>(C_in) * C_out) : 0;
  out[4] = static_cast<int64_t>(p.bytes);
}
}
