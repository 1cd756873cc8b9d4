// Prints what attention calls over pages plan and launch (csrc/dreams_api.hip and the launchers behind it) on a device of 256
// compute units.  The HIP calls that describe the device and that enqueue a kernel are this file's own: a launch is noted and
// answers success, so that nothing touches a device and no pointer is followed.  A line of standard input is a call
//     e4m3 prompt batch q_heads kv_heads head_dim rows page_size table_width max_kv_len num_splits window sinks
// and a line of output what it does
//     status launches workgroups rows_per_wg units row_groups splits spread_wgs half_ring key_groups workspace_bytes
// (workgroups: of the first launch).  Every plan is also offered to the other launcher of its type and, as one of spread keys, to
// the kernel of 128 rows, which have to refuse it.
#include <stdint.h>
#include <stdio.h>

#include "dreams.h"
#include "kernels.h"

static dreams::AttnArgs8 seen;
static bool eight;
static int launches;
static long long workgroups;
static dim3 grid_of_call, block_of_call;
static size_t lds_of_call;
static hipStream_t stream_of_call;

extern "C" {
hipError_t hipGetDevice(int* device) {
  *device = 0;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t attribute, int) {
  *value = attribute == hipDeviceAttributeMultiprocessorCount ? 256 : 0;
  return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t n, hipStream_t s) {
  grid_of_call = g;
  block_of_call = b;
  lds_of_call = n;
  stream_of_call = s;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* n, hipStream_t* s) {
  *g = grid_of_call;
  *b = block_of_call;
  *n = lds_of_call;
  *s = stream_of_call;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3, void** args, size_t, hipStream_t) {
  if (launches++ == 0) {
    workgroups = (long long)grid.x * grid.y * grid.z;
    if (eight) seen = *(const dreams::AttnArgs8*)args[0];
    else static_cast<dreams::AttnArgs&>(seen) = *(const dreams::AttnArgs*)args[0];
  }
  return hipSuccess;
}
}

static bool refuses(hipError_t (*launch)(const dreams::AttnArgs8&, hipStream_t), const dreams::AttnArgs8& a) {
  const int before = launches;
  return launch(a, nullptr) == hipErrorInvalidValue && launches == before;
}

int main() {
  int e4m3, prompt, batch, hq, hkv, dim, rows, page, width, bound, splits, window, sinks, n = 0;
  while (scanf("%d %d %d %d %d %d %d %d %d %d %d %d %d", &e4m3, &prompt, &batch, &hq, &hkv, &dim, &rows, &page, &width, &bound,
               &splits, &window, &sinks) == 13) {
    dreams_paged_desc_t d{};
    d.batch = batch;
    d.num_q_heads = hq;
    d.num_kv_heads = hkv;
    d.head_dim = dim;
    d.num_rows = rows;
    d.num_pages = 1 << 18;
    d.page_size = page;
    d.table_width = width;
    d.max_kv_len = bound;
    d.num_splits = splits;
    d.window = window;
    d.sinks = sinks;
    d.dtype = DREAMS_BF16;
    d.scale = 0.125f;
    const auto at = [](uint64_t i) { return (void*)(i << 40); };
    const int32_t* ints = (const int32_t*)at(1);
    const dreams_page_scales_t scales{(uint8_t*)at(2), (uint8_t*)at(3), 0, 0};
    seen = dreams::AttnArgs8{};
    eight = e4m3 != 0;
    launches = 0;
    workgroups = 0;
    size_t bytes = 0;
    dreams_status_t st;
    if (e4m3 && prompt) {
      st = dreams_paged_prompt_attn_e4m3_workspace_size(&d, &bytes);
      if (st == DREAMS_OK)
        st = dreams_paged_prompt_attn_e4m3(&d, at(4), at(5), at(6), &scales, ints, ints, nullptr, at(7), nullptr, at(8), bytes, nullptr);
    } else if (e4m3) {
      st = dreams_paged_verify_attn_e4m3_workspace_size(&d, &bytes);
      if (st == DREAMS_OK)
        st = dreams_paged_verify_attn_e4m3(&d, at(4), at(5), at(6), &scales, ints, ints, ints, nullptr, at(7), nullptr, at(8), bytes,
                                           nullptr);
    } else if (prompt) {
      st = dreams_paged_prompt_attn_workspace_size(&d, &bytes);
      if (st == DREAMS_OK)
        st = dreams_paged_prompt_attn(&d, at(4), at(5), at(6), ints, ints, nullptr, at(7), nullptr, at(8), bytes, nullptr);
    } else {
      st = dreams_paged_verify_attn_workspace_size(&d, &bytes);
      if (st == DREAMS_OK)
        st = dreams_paged_verify_attn(&d, at(4), at(5), at(6), ints, ints, ints, nullptr, at(7), nullptr, at(8), bytes, nullptr);
    }
    if (st != DREAMS_OK) fprintf(stderr, "%s\n", dreams_last_error_message());
    printf("%d %d %lld %d %d %d %d %d %d %d %zu\n", (int)st, launches, workgroups, seen.rows_per_wg, seen.units, seen.row_groups,
           seen.splits, seen.spread_wgs, seen.half_ring, seen.key_groups, bytes);
    if (st == DREAMS_OK && e4m3 && launches > 0) {
      const bool many = seen.rows_per_wg == 128;
      if (!refuses(many ? dreams::launch_paged_attn_e4m3 : dreams::launch_paged_rows_e4m3, seen)) {
        fprintf(stderr, "call %d: rows of another kernel are not refused\n", n);
        return 1;
      }
      if (many) {
        dreams::AttnArgs8 spread = seen;
        spread.splits = spread.row_groups = 1;
        spread.groups_per_head = 0;
        spread.spread_wgs = 256;
        if (!refuses(dreams::launch_paged_rows_e4m3, spread)) {
          fprintf(stderr, "call %d: spread keys are not refused for 128 rows\n", n);
          return 1;
        }
      }
    }
    ++n;
  }
  fprintf(stderr, "plan driver: ok (%d calls)\n", n);
  return 0;
}
