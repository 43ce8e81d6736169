// Host-side driver over the argument checks of the paged token cache's calls, linked to the built library
// and run without a GPU (tests/test_pcache_abi_cpu.py): a context built by hand (no device buffers), every
// refusal with its status, byte ranges that 32 bits do not hold, and calls that pass the checks down to
// the first device call, which then fails cleanly.  Exit status 0: every expectation held.
#include <climits>
#include <cmath>
#include <cstdio>
#include <vector>

#include "../paper_2604_24391_amd/csrc/fc_internal.h"

static int g_fail = 0;

#define EXPECT(call, want)                                                                  \
  do {                                                                                      \
    const fc_status _s = (call);                                                            \
    if (_s != (want) || !*fc_last_error()) {                                                \
      std::printf("FAIL line %d: -> %d (want %d): %s\n", __LINE__, (int)_s, (int)(want), fc_last_error()); \
      ++g_fail;                                                                             \
    }                                                                                       \
  } while (0)
#define SAME(got, want)                                                                     \
  do {                                                                                      \
    if ((got) != (want)) {                                                                  \
      std::printf("FAIL line %d: %zu, not %zu\n", __LINE__, (size_t)(got), (size_t)(want)); \
      ++g_fail;                                                                             \
    }                                                                                       \
  } while (0)

int main() {
  fc_ctx ctx;
  ctx.caps = fc_caps{4, 224, 224, 256, 288, 256, 1024, 768};
  ctx.part_elems = 1 << 20;
  // stand-ins for distinct allocations, 1 TiB apart, never dereferenced
  auto at = [](int i) { return (uintptr_t)(i + 1) << 40; };
  auto u8 = [&](int i) { return reinterpret_cast<uint8_t *>(at(i)); };
  auto u16 = [&](int i) { return reinterpret_cast<uint16_t *>(at(i)); };
  auto i32 = [&](int i) { return reinterpret_cast<int32_t *>(at(i)); };
  const fc_pcache c{u16(0), u16(1), i32(2), 4, 128, 64, 300, 40};
  const fc_rope_axes rope{1e6, {16, 24, 24}};
  const fc_qkv_rows x{u16(10), u16(10) + 28 * 128, u16(10) + 32 * 128, 36 * 128, 36 * 128, 36 * 128, 36 * 128, 36 * 128, 36 * 128, 28};
  auto app = [&](const fc_pcache *cc, const fc_rope_axes *r, const fc_qkv_rows *rr, int B = 2, int n = 1, uint16_t *qo = nullptr, bool noq = false) {
    return fc_pcache_append(&ctx, cc, r, rr, i32(11), i32(12), i32(13), noq ? nullptr : (qo ? qo : u16(14)), B, n, nullptr);
  };
  auto att = [&](const fc_pcache *cc, int H = 28, float s = 0.1f, int B = 2, int n = 1) {
    return fc_pcache_attention(&ctx, cc, u16(14), i32(12), i32(13), u8(15), u16(16), H, s, B, n, nullptr);
  };
  auto step = [&](const fc_pcache *cc, int layers = 1, int n = 5, int B = 2, int32_t *granted = nullptr) {
    return fc_pcache_step(&ctx, cc, layers, i32(17), i32(12), i32(13), n, granted ? granted : i32(18), B, nullptr);
  };
  auto pack = [&](const fc_pcache *cc, int layers = 1, int B = 2, int32_t *live = nullptr) {
    return fc_pcache_compact(&ctx, cc, layers, live, B, nullptr);
  };
  auto init = [&](const fc_pcache *cc, int B = 2) { return fc_pcache_init(&ctx, cc, B, nullptr); };
  // what passes the checks reaches the device (none here)
  EXPECT(app(&c, &rope, &x), FC_ERR_HIP);
  EXPECT(att(&c), FC_ERR_HIP);
  EXPECT(step(&c), FC_ERR_HIP);
  EXPECT(step(&c, 1, 0), FC_ERR_HIP);
  EXPECT(step(&c, 1, INT_MAX), FC_ERR_HIP);
  EXPECT(pack(&c), FC_ERR_HIP);
  EXPECT(pack(&c, 1, 2, i32(18)), FC_ERR_HIP);
  EXPECT(init(&c), FC_ERR_HIP);
  EXPECT(fc_pcache_step(&ctx, &c, 1, nullptr, i32(12), nullptr, 5, i32(18), 2, nullptr), FC_ERR_HIP);
  EXPECT(fc_pcache_attention(&ctx, &c, u16(14), i32(12), nullptr, nullptr, u16(16), 28, -0.5f, 2, 1, nullptr), FC_ERR_HIP);
  // null
  EXPECT(fc_pcache_init(nullptr, &c, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_append(nullptr, &c, &rope, &x, i32(11), i32(12), nullptr, u16(14), 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_attention(nullptr, &c, u16(14), i32(12), nullptr, nullptr, u16(16), 28, 1.f, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_step(nullptr, &c, 1, nullptr, i32(12), nullptr, 5, i32(18), 2, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_compact(nullptr, &c, 1, nullptr, 2, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(init(nullptr), FC_ERR_INVALID_ARG);
  EXPECT(app(nullptr, &rope, &x), FC_ERR_INVALID_ARG);
  EXPECT(app(&c, nullptr, &x), FC_ERR_INVALID_ARG);
  EXPECT(app(&c, &rope, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(app(&c, &rope, &x, 2, 1, nullptr, true), FC_ERR_INVALID_ARG);
  EXPECT(att(nullptr), FC_ERR_INVALID_ARG);
  EXPECT(step(nullptr), FC_ERR_INVALID_ARG);
  EXPECT(pack(nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_append(&ctx, &c, &rope, &x, nullptr, i32(12), nullptr, u16(14), 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_append(&ctx, &c, &rope, &x, i32(11), nullptr, nullptr, u16(14), 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_attention(&ctx, &c, nullptr, i32(12), nullptr, nullptr, u16(16), 28, 1.f, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_attention(&ctx, &c, u16(14), nullptr, nullptr, nullptr, u16(16), 28, 1.f, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_attention(&ctx, &c, u16(14), i32(12), nullptr, nullptr, nullptr, 28, 1.f, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_step(&ctx, &c, 1, nullptr, nullptr, nullptr, 5, i32(18), 2, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_step(&ctx, &c, 1, nullptr, i32(12), nullptr, 5, nullptr, 2, nullptr), FC_ERR_INVALID_ARG);
  for (int i = 0; i < 3; ++i)
    for (int bad = 0; bad < 2; ++bad) {   // null, or not aligned
      fc_pcache y = c;
      if (i == 0) y.k = bad ? c.k + 4 : nullptr;
      if (i == 1) y.v = bad ? c.v + 4 : nullptr;
      if (i == 2) y.state = bad ? c.state + 2 : nullptr;
      EXPECT(app(&y, &rope, &x), FC_ERR_INVALID_ARG);
      EXPECT(att(&y), FC_ERR_INVALID_ARG);
      EXPECT(step(&y), FC_ERR_INVALID_ARG);
      EXPECT(pack(&y), FC_ERR_INVALID_ARG);
      EXPECT(init(&y), FC_ERR_INVALID_ARG);
    }
  // the cache's shape
  for (int hd : {0, 32, 80, 256, -128, INT_MAX}) {
    fc_pcache y = c;
    y.head_dim = hd;
    EXPECT(att(&y), FC_ERR_UNSUPPORTED);
    EXPECT(step(&y), FC_ERR_UNSUPPORTED);
  }
  for (int kv : {0, -4, INT_MIN, 65536, INT_MAX}) {
    fc_pcache y = c;
    y.n_kv_heads = kv;
    EXPECT(att(&y), FC_ERR_SHAPE);
    EXPECT(pack(&y), FC_ERR_SHAPE);
  }
  for (int r : {0, 8, 24, 48, 2048, -64, INT_MIN, INT_MAX}) {
    fc_pcache y = c;
    y.page_rows = r;
    EXPECT(att(&y), FC_ERR_SHAPE);
    EXPECT(app(&y, &rope, &x), FC_ERR_SHAPE);
  }
  for (int n : {0, -1, INT_MIN}) {
    fc_pcache y = c;
    y.n_pages = n;
    EXPECT(att(&y), FC_ERR_SHAPE);
    y = c;
    y.max_pages = n;
    EXPECT(att(&y), FC_ERR_SHAPE);
  }
  {
    fc_pcache y = c;
    y.max_pages = (1 << 24) + 1;                               // 2^30 rows and one page
    EXPECT(att(&y), FC_ERR_SHAPE);
    y.max_pages = 1 << 24;
    EXPECT(att(&y, 28, 0.1f, 16), FC_ERR_HIP);                 // 2^28 entries, 2^34 rows
    EXPECT(att(&y, 28, 0.1f, 17), FC_ERR_UNSUPPORTED);
    y.page_rows = 1024, y.max_pages = 1 << 20;
    EXPECT(att(&y, 28, 0.1f, 64), FC_ERR_HIP);                 // 2^36 rows
    EXPECT(att(&y, 28, 0.1f, 65), FC_ERR_UNSUPPORTED);
    y = c;
    y.n_pages = INT_MAX;                                       // beyond 2^42 bytes of keys
    EXPECT(att(&y), FC_ERR_UNSUPPORTED);
    y.n_kv_heads = 1, y.head_dim = 64, y.page_rows = 16;       // 4 TiB less a page: reaches over the next stand-in
    EXPECT(fc_pcache_attention(&ctx, &y, u16(14), i32(12), nullptr, nullptr, u16(16), 28, 1.f, 1, 1, nullptr), FC_ERR_HIP);
    EXPECT(fc_pcache_attention(&ctx, &y, u16(14), i32(12), nullptr, nullptr, u16(3), 28, 1.f, 1, 1, nullptr), FC_ERR_INVALID_ARG);
    EXPECT(step(&y), FC_ERR_INVALID_ARG);                      // (its keys lie over its values)
  }
  for (int B : {0, -1, INT_MIN, 16384, INT_MAX}) {
    EXPECT(app(&c, &rope, &x, B), FC_ERR_SHAPE);
    EXPECT(att(&c, 28, 0.1f, B), FC_ERR_SHAPE);
    EXPECT(step(&c, 1, 5, B), FC_ERR_SHAPE);
    EXPECT(pack(&c, 1, B), FC_ERR_SHAPE);
    EXPECT(init(&c, B), FC_ERR_SHAPE);
  }
  for (int n : {0, -1, INT_MIN, 40 * 64 + 1, INT_MAX}) {
    EXPECT(app(&c, &rope, &x, 2, n), FC_ERR_SHAPE);
    EXPECT(att(&c, 28, 0.1f, 2, n), FC_ERR_SHAPE);
  }
  for (int n : {-1, INT_MIN}) EXPECT(step(&c, 1, n), FC_ERR_SHAPE);
  for (int H : {0, -4, 3, 30, INT_MAX}) EXPECT(att(&c, H), FC_ERR_SHAPE);
  for (int H : {65536, 1 << 28}) EXPECT(att(&c, H), FC_ERR_UNSUPPORTED);
  {
    fc_pcache y = c;
    y.page_rows = 1024, y.max_pages = 1 << 20;
    EXPECT(att(&y, 28, 0.1f, 1, 1 << 26), FC_ERR_UNSUPPORTED);                 // 28 2^26 rows
    const fc_qkv_rows one{nullptr, u16(20), u16(21), 0, 0, 0, 0, 0, 0, 4};
    EXPECT(fc_pcache_append(&ctx, &y, &rope, &one, i32(22), i32(12), nullptr, nullptr, 1, (1 << 27) - 15, nullptr), FC_ERR_HIP);
    EXPECT(fc_pcache_append(&ctx, &y, &rope, &one, i32(22), i32(12), nullptr, nullptr, 1, (1 << 27) - 14, nullptr), FC_ERR_UNSUPPORTED);
    // positions that end where the keys begin, and a number further
    const long bytes = 3L * (1 << 26) * 4;
    EXPECT(fc_pcache_append(&ctx, &y, &rope, &one, reinterpret_cast<int32_t *>(at(0) - bytes), i32(12), nullptr, nullptr, 1, 1 << 26, nullptr), FC_ERR_HIP);
    EXPECT(fc_pcache_append(&ctx, &y, &rope, &one, reinterpret_cast<int32_t *>(at(0) - bytes + 4), i32(12), nullptr, nullptr, 1, 1 << 26, nullptr),
           FC_ERR_INVALID_ARG);
  }
  for (float s : {NAN, INFINITY, -INFINITY}) EXPECT(att(&c, 28, s), FC_ERR_INVALID_ARG);
  // rotary sections and theta
  for (fc_rope_axes r : {fc_rope_axes{1.0, {0, 0, 0}}, fc_rope_axes{NAN, {0, 0, 0}}, fc_rope_axes{INFINITY, {0, 0, 0}}, fc_rope_axes{1e6, {16, 24, 23}},
                         fc_rope_axes{1e6, {-1, 41, 24}}, fc_rope_axes{1e6, {INT_MAX, INT_MAX, INT_MAX}}})
    EXPECT(app(&c, &r, &x), FC_ERR_INVALID_ARG);
  // rows
  for (int64_t s : {(int64_t)-8, (int64_t)4, (int64_t)36 * 128 + 1, INT64_MAX - 7, INT64_MIN}) {
    fc_qkv_rows y = x;
    y.k_row = s;
    EXPECT(app(&c, &rope, &y), FC_ERR_INVALID_ARG);
    y = x;
    y.q_item = s;
    EXPECT(app(&c, &rope, &y), FC_ERR_INVALID_ARG);
  }
  {
    fc_qkv_rows y = x;
    y.v += 4;
    EXPECT(app(&c, &rope, &y), FC_ERR_INVALID_ARG);
    y = x;
    y.n_heads = 30;
    EXPECT(app(&c, &rope, &y), FC_ERR_SHAPE);
    EXPECT(app(&c, &rope, &x, 2, 1, u16(14) + 4), FC_ERR_INVALID_ARG);   // alignment
    EXPECT(app(&c, &rope, &x, 2, 1, u16(10)), FC_ERR_INVALID_ARG);       // over the rows
    EXPECT(app(&c, &rope, &x, 2, 1, u16(0) + 8), FC_ERR_INVALID_ARG);    // in the pool
    EXPECT(app(&c, &rope, &x, 2, 1, u16(2)), FC_ERR_INVALID_ARG);        // over the state
    y = x;
    y.q = u16(14), y.q_row = y.q_item = 28 * 128;
    EXPECT(app(&c, &rope, &y), FC_ERR_HIP);                              // in place
    y.k = c.v;
    EXPECT(app(&c, &rope, &y), FC_ERR_INVALID_ARG);                      // the pool's own rows
  }
  {
    fc_pcache y = c;
    y.v = y.k + 64;
    EXPECT(app(&y, &rope, &x), FC_ERR_INVALID_ARG);
    y = c;
    y.state = reinterpret_cast<int32_t *>(c.v);
    EXPECT(app(&y, &rope, &x), FC_ERR_INVALID_ARG);
  }
  // the attention's output
  for (void *o : {(void *)u16(14), (void *)u8(15), (void *)c.k, (void *)c.v, (void *)c.state, (void *)i32(12), (void *)i32(13)})
    EXPECT(fc_pcache_attention(&ctx, &c, u16(14), i32(12), i32(13), u8(15), (uint16_t *)o, 28, 0.1f, 2, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_attention(&ctx, &c, u16(14) + 4, i32(12), nullptr, nullptr, u16(16), 28, 0.1f, 2, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_pcache_attention(&ctx, &c, u16(14), i32(12), nullptr, u8(15) + 8, u16(16), 28, 0.1f, 2, 1, nullptr), FC_ERR_INVALID_ARG);
  // layers: their number, sizes, state, and memory of their own
  {
    std::vector<fc_pcache> l(70, c);
    for (int i = 0; i < 70; ++i) l[i].k = u16(100 + 2 * i), l[i].v = u16(101 + 2 * i);
    EXPECT(step(l.data(), 70), FC_ERR_HIP);
    EXPECT(pack(l.data(), 70), FC_ERR_HIP);
    for (int n : {0, -1, 65537, INT_MIN}) EXPECT(step(l.data(), n), FC_ERR_SHAPE);
    for (int i = 0; i < 8; ++i) {
      std::vector<fc_pcache> y = l;
      if (i == 0) y[69].state = i32(3);
      if (i == 1) y[3].n_pages = 299;
      if (i == 2) y[3].page_rows = 32;
      if (i == 3) y[3].head_dim = 64;
      if (i == 4) y[3].max_pages = 41;
      if (i == 5) y[3].n_kv_heads = 2;
      if (i == 6) y[69].v = y[5].k;
      if (i == 7) y[69].k = nullptr;
      EXPECT(step(y.data(), 70), i < 6 ? FC_ERR_SHAPE : FC_ERR_INVALID_ARG);
      EXPECT(pack(y.data(), 70), i < 6 ? FC_ERR_SHAPE : FC_ERR_INVALID_ARG);
    }
    EXPECT(step(l.data(), 70, 5, 2, reinterpret_cast<int32_t *>(l[33].v) + 8), FC_ERR_INVALID_ARG);
    EXPECT(pack(l.data(), 70, 2, reinterpret_cast<int32_t *>(l[69].k)), FC_ERR_INVALID_ARG);
    EXPECT(pack(l.data(), 70, 2, c.state), FC_ERR_INVALID_ARG);
    EXPECT(step(l.data(), 70, 5, 2, i32(12)), FC_ERR_INVALID_ARG);
    EXPECT(step(l.data(), 70, 5, 2, i32(13) + 1), FC_ERR_INVALID_ARG);
    EXPECT(step(l.data(), 70, 5, 2, i32(17)), FC_ERR_INVALID_ARG);
    EXPECT(fc_pcache_step(&ctx, l.data(), 70, c.state, i32(12), nullptr, 5, i32(18), 2, nullptr), FC_ERR_INVALID_ARG);
  }
  // the workspace
  {
    fc_pcache y = c;
    y.n_pages = 1 << 18;
    EXPECT(step(&y), FC_ERR_CAPACITY);
    EXPECT(pack(&y), FC_ERR_CAPACITY);
    EXPECT(att(&y), FC_ERR_HIP);
  }
  SAME(fc_pcache_state_bytes(2, 40, 300), (80 + 300) * 4);
  SAME(fc_pcache_state_bytes(3, 3, 5), (12 + 5) * 4);
  SAME(fc_pcache_state_bytes(0, 1, 1), 0);
  SAME(fc_pcache_state_bytes(1, 0, 1), 0);
  SAME(fc_pcache_state_bytes(1, 1, 0), 0);
  SAME(fc_pcache_state_bytes(1 << 14, 1 << 14, INT_MAX), ((1ull << 28) + INT_MAX) * 4);
  SAME(fc_pcache_state_bytes(1 << 14, (1 << 14) + 1, 1), 0);
  std::printf("OK (%d failed expectations)\n", g_fail);
  return g_fail != 0;
}
