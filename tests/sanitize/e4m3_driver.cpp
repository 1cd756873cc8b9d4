// Drives the host layer of rotary positions and of pages in 8 bits (csrc/dreams_api.hip: argument checks, work planning,
// workspace sizes) with ordinary and extreme arguments, for a build with the host address and undefined-behaviour
// sanitizers.  Nothing here touches a device: every call answers from the arguments alone or fails its checks (null pointers
// at the latest) before anything is enqueued.  Exit status 0 on success.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "dreams.h"

static uint64_t state = 1181783497276652981ull;
static uint64_t next() {   // xorshift
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return state;
}
static int32_t pick(int32_t ordinary) {
  static const int32_t extreme[] = {0, 1, -1, 2, 3, 7, 16, 64, 127, 128, 129, 512, 4096, 65535, 65536, 1 << 20, 1 << 27,
                                    1 << 30, INT32_MAX, INT32_MAX - 1, INT32_MIN};
  return next() % 4 ? ordinary : extreme[next() % (sizeof(extreme) / sizeof(extreme[0]))];
}
static int64_t pick64(int64_t ordinary) {
  static const int64_t extreme[] = {0, 1, -1, 8, 1 << 20, (int64_t)1 << 40, (int64_t)1 << 59, INT64_MAX, INT64_MIN};
  return next() % 4 ? ordinary : extreme[next() % (sizeof(extreme) / sizeof(extreme[0]))];
}
static double pick_double(double ordinary) {
  static const double extreme[] = {0.0, -1.0, 1e-300, 1e300, INFINITY, -INFINITY, NAN};
  return next() % 4 ? ordinary : extreme[next() % (sizeof(extreme) / sizeof(extreme[0]))];
}

int main() {
  int fine = 0, refused = 0;
  for (int i = 0; i < 100000; ++i) {
    const int32_t kv_heads = 1 << next() % 5, page = 16 << next() % 4, width = 1 + (int32_t)(next() % 3000);
    dreams_page_scales_t sc{};
    sc.layer_stride = pick64(0);
    sc.page_stride = pick64(next() % 2 ? 0 : (int64_t)kv_heads * page);
    dreams_paged_desc_t d{};
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
    d.dtype = next() % 8 ? DREAMS_BF16 : next() % 2 ? DREAMS_F32 : DREAMS_E4M3;
    d.scale = 0.1f;
    d.page_stride = pick64(next() % 2 ? 0 : (int64_t)kv_heads * page * 128);
    size_t n = 0;
    for (int prompt = 0; prompt < 2; ++prompt) {
      const dreams_status_t st = prompt ? dreams_paged_prompt_attn_e4m3_workspace_size(&d, &n)
                                        : dreams_paged_verify_attn_e4m3_workspace_size(&d, &n);
      if (st != DREAMS_OK && st != DREAMS_ERR_INVALID_ARG && st != DREAMS_ERR_UNSUPPORTED) return 1;
      ++(st == DREAMS_OK ? fine : refused);
      if (st == DREAMS_OK && d.dtype != DREAMS_BF16) return 2;
      if (st == DREAMS_OK && d.batch > 0 && d.num_splits > 1 && n > (size_t)1 << 50) return 3;
      const dreams_status_t call =
          prompt ? dreams_paged_prompt_attn_e4m3(&d, nullptr, nullptr, nullptr, &sc, nullptr, nullptr, nullptr, nullptr,
                                                 nullptr, nullptr, 0, nullptr)
                 : dreams_paged_verify_attn_e4m3(&d, nullptr, nullptr, nullptr, &sc, nullptr, nullptr, nullptr, nullptr,
                                                 nullptr, nullptr, nullptr, 0, nullptr);
      if ((call == DREAMS_OK) != (st == DREAMS_OK && d.batch == 0)) return 4;
    }
    dreams_page_pool_t p{};
    p.num_layers = next() % 2 ? 1 : pick(1 + (int32_t)(next() % 64));
    p.batch = pick(1 + (int32_t)(next() % 64));
    p.num_kv_heads = pick(kv_heads);
    p.head_dim = pick(128);
    p.num_pages = pick(1 + (int32_t)(next() % 100000));
    p.page_size = pick(page);
    p.table_width = pick(width);
    p.layer_stride = pick64(0);
    p.page_stride = pick64(0);
    dreams_rope_t r{};
    double frequencies[256];
    const int32_t positions[1] = {0};
    r.rotary_dim = pick(16 << next() % 4);
    r.interleaved = next() % 8 ? (int32_t)(next() % 2) : pick(1);
    r.frequencies = next() % 4 ? frequencies : nullptr;
    r.positions = next() % 2 ? positions : nullptr;
    r.parent = next() % 2 ? positions : nullptr;
    r.amplitude = (float)pick_double(1.0);
    dreams_rope_queries_t q{};
    q.num_q_heads = pick(8);
    for (int64_t& s : q.strides) s = pick64(1024);
    const int64_t strides[4] = {pick64(0), pick64(8192), pick64(1024), pick64(128)};
    const int32_t rows = pick((int32_t)(next() % 300)), count = pick((int32_t)(next() % 64)), heads = pick(8);
    const dreams_rope_t* rope = next() % 8 ? &r : nullptr;
    const dreams_rope_queries_t* queries = next() % 2 ? &q : nullptr;
    const dreams_dtype_t type = next() % 2 ? DREAMS_BF16 : DREAMS_F32;
    p.dtype = type;
    dreams_status_t st[6];
    st[0] = dreams_paged_append_rope(&p, rope, queries, nullptr, nullptr, rows, strides, nullptr, nullptr, nullptr, nullptr,
                                     nullptr, nullptr);
    p.dtype = next() % 8 ? DREAMS_E4M3 : type;
    st[1] = dreams_paged_append_e4m3(&p, &sc, rope, queries, type, nullptr, nullptr, rows, strides, nullptr, nullptr, nullptr,
                                     nullptr, nullptr, nullptr);
    st[2] = dreams_paged_kv_commit_e4m3(&p, &sc, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, pick(5), nullptr, nullptr);
    const int32_t slots = pick(rows);
    st[3] = dreams_paged_read_e4m3(&p, &sc, nullptr, nullptr, nullptr, nullptr, slots, nullptr, nullptr, nullptr);
    st[4] = dreams_pages_fork_e4m3(&p, &sc, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, count, nullptr, nullptr,
                                   nullptr, nullptr);
    st[5] = dreams_rope(rope, p.batch, heads, rows, p.head_dim, type, nullptr, strides + 1, positions, nullptr, strides, nullptr);
    for (const dreams_status_t s : st) {
      if (s != DREAMS_OK && s != DREAMS_ERR_INVALID_ARG && s != DREAMS_ERR_UNSUPPORTED) return 5;
      if (s == DREAMS_OK && p.batch != 0 && rows != 0 && slots != 0 && count != 0) return 6;
      ++(s == DREAMS_OK ? fine : refused);
    }
    const int32_t pairs = next() % 4 ? 2 * (int32_t)(next() % 257) : (int32_t)(next() % 512);
    const dreams_status_t f = dreams_rope_frequencies(next() % 8 ? pairs : -pairs, pick_double(1e4),
                                                      (dreams_rope_scaling_t)(next() % 3), pick_double(4.0),
                                                      pick_double(4096.0), pick_double(1.0), pick_double(32.0), frequencies);
    if (f != DREAMS_OK && f != DREAMS_ERR_INVALID_ARG) return 7;
    ++(f == DREAMS_OK ? fine : refused);
  }
  if (fine < 10000 || refused < 10000) return 8;
  printf("e4m3 driver: ok (%d fine, %d refused)\n", fine, refused);
  return 0;
}
