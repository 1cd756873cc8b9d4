// Drives the paged cache's host layer (csrc/dreams_api.hip: argument checks, work planning, workspace sizes) with ordinary
// and extreme arguments, for a build with the host address and undefined-behaviour sanitizers.  Nothing here touches a
// device: every call answers from the arguments alone or fails its checks (null pointers at the latest) before anything
// is enqueued.  Exit status 0 on success.
#include <stdint.h>
#include <stdio.h>

#include "dreams.h"

static uint64_t state = 88172645463325252ull;
static uint64_t next() {   // xorshift
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return state;
}
static int32_t pick(int32_t ordinary) {
  static const int32_t extreme[] = {0, 1, -1, 2, 3, 7, 16, 64, 127, 128, 129, 4096, 65535, 65536, 1 << 20, 1 << 27, 1 << 30,
                                    INT32_MAX, INT32_MAX - 1, INT32_MIN};
  return next() % 3 ? ordinary : extreme[next() % (sizeof(extreme) / sizeof(extreme[0]))];
}
static int64_t pick64(int64_t ordinary) {
  static const int64_t extreme[] = {0, 1, -1, 8, 1 << 20, (int64_t)1 << 40, (int64_t)1 << 59, INT64_MAX, INT64_MIN};
  return next() % 3 ? ordinary : extreme[next() % (sizeof(extreme) / sizeof(extreme[0]))];
}

int main() {
  int fine = 0, refused = 0;
  for (int i = 0; i < 200000; ++i) {
    dreams_paged_desc_t d{};
    const int32_t kv_heads = 1 << next() % 5, page = 16 << next() % 4, width = 1 + (int32_t)(next() % 3000);
    d.batch = pick(1 + (int32_t)(next() % 64));
    d.num_kv_heads = pick(kv_heads);
    d.num_q_heads = pick(kv_heads * (1 + (int32_t)(next() % 8)));
    d.head_dim = pick(next() % 2 ? 64 : 128);
    d.num_rows = pick(1 + (int32_t)(next() % 200));
    d.num_pages = pick(1 + (int32_t)(next() % 100000));
    d.page_size = pick(page);
    d.table_width = pick(width);
    d.max_kv_len = pick((int32_t)(next() % 4000));
    d.num_splits = pick(1 + (int32_t)(next() % 40));
    if (d.num_splits == 0) d.num_splits = 1;      // (0 asks the device for its size)
    d.window = pick((int32_t)(next() % 5000));
    d.sinks = pick((int32_t)(next() % 100));
    d.dtype = next() % 2 ? DREAMS_BF16 : DREAMS_F32;
    d.scale = 0.1f;
    d.page_stride = pick64(next() % 2 ? 0 : (int64_t)kv_heads * page * 256);
    size_t n = 0;
    for (int prompt = 0; prompt < 2; ++prompt) {
      const dreams_status_t st = prompt ? dreams_paged_prompt_attn_workspace_size(&d, &n)
                                        : dreams_paged_verify_attn_workspace_size(&d, &n);
      if (st != DREAMS_OK && st != DREAMS_ERR_INVALID_ARG && st != DREAMS_ERR_UNSUPPORTED) return 1;
      ++(st == DREAMS_OK ? fine : refused);
      if (st == DREAMS_OK && d.dtype == DREAMS_BF16 && d.batch > 0 && d.num_splits > 1 && n > (size_t)1 << 50) return 2;
      const dreams_status_t call =
          prompt ? dreams_paged_prompt_attn(&d, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                            nullptr, 0, nullptr)
                 : dreams_paged_verify_attn(&d, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                            nullptr, 0, nullptr);
      if ((call == DREAMS_OK) != (st == DREAMS_OK && d.batch == 0)) return 3;
    }
    dreams_page_pool_t p{};
    p.num_layers = pick(1 + (int32_t)(next() % 64));
    p.batch = pick(1 + (int32_t)(next() % 64));
    p.num_kv_heads = pick(kv_heads);
    p.head_dim = pick(128);
    p.num_pages = pick(1 + (int32_t)(next() % 100000));
    p.page_size = pick(page);
    p.table_width = pick(width);
    p.dtype = next() % 2 ? DREAMS_BF16 : DREAMS_F32;
    p.layer_stride = pick64(0);
    p.page_stride = pick64(0);
    const int64_t strides[4] = {pick64(0), pick64(8192), pick64(1024), pick64(128)};
    const int32_t rows = pick((int32_t)(next() % 300)), count = pick((int32_t)(next() % 64));
    dreams_status_t st[5] = {
        dreams_paged_append(&p, nullptr, nullptr, rows, strides, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr),
        dreams_paged_kv_commit(&p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, pick(5), nullptr, nullptr),
        dreams_pages_reserve(&p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr),
        dreams_pages_fork(&p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, count, nullptr, nullptr, nullptr, nullptr),
        dreams_pages_release(&p, nullptr, nullptr, nullptr, nullptr, count, nullptr, pick(0), nullptr)};
    for (const dreams_status_t s : st) {
      if (s != DREAMS_OK && s != DREAMS_ERR_INVALID_ARG && s != DREAMS_ERR_UNSUPPORTED) return 4;
      if (s == DREAMS_OK && p.batch != 0 && rows != 0) return 5;
      ++(s == DREAMS_OK ? fine : refused);
    }
  }
  if (fine < 10000 || refused < 10000) return 6;
  printf("paged driver: ok (%d fine, %d refused)\n", fine, refused);
  return 0;
}
