// Host-side driver over the argument checks of the 8-bit token cache's calls, linked to the
// built library and run without a GPU (tests/test_qcache_abi_cpu.py): a context built by hand
// (no device buffers), every refusal with its status, and calls that pass the checks down to
// the first device call, which then fails cleanly.  Exit status 0: every expectation held.
#include <climits>
#include <cmath>
#include <cstdio>

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

int main() {
  fc_ctx ctx;
  ctx.caps = fc_caps{4, 224, 224, 256, 288, 256, 1024, 768};
  // stand-ins for distinct allocations, 1 TiB apart, never dereferenced
  auto at = [](int i) { return (uintptr_t)(i + 1) << 40; };
  auto u8 = [&](int i) { return reinterpret_cast<uint8_t *>(at(i)); };
  auto u16 = [&](int i) { return reinterpret_cast<uint16_t *>(at(i)); };
  auto f32 = [&](int i) { return reinterpret_cast<float *>(at(i)); };
  auto i32 = [&](int i) { return reinterpret_cast<int32_t *>(at(i)); };
  const fc_qcache c{u8(0), u8(1), f32(2), f32(3), f32(4), 4, 128, 4224};
  const fc_qcache d{u8(5), u8(6), f32(7), f32(8), f32(9), 4, 128, 2176};
  const fc_rope_axes rope{1e6, {16, 24, 24}};
  fc_qkv_rows x{u16(10), u16(10) + 28 * 128, u16(10) + 32 * 128, 36 * 128, 36 * 128, 36 * 128, 36 * 128, 36 * 128, 36 * 128, 28};
  auto app = [&](const fc_qcache *cc, const fc_rope_axes *r, const fc_qkv_rows *rr, int B = 2, int n = 1, uint16_t *qo = nullptr, bool noq = false) {
    return fc_qcache_append(&ctx, cc, r, rr, i32(11), i32(12), i32(13), noq ? nullptr : (qo ? qo : u16(14)), B, n, nullptr);
  };
  auto att = [&](const fc_qcache *cc, int H = 28, float s = 0.1f, int acc = 1, int B = 2, int n = 1) {
    return fc_qcache_attention(&ctx, cc, u16(14), i32(12), i32(13), u8(15), u16(16), H, s, acc, B, n, nullptr);
  };
  auto ev = [&](const fc_qcache *a, const fc_qcache *b, int keep = 2000, int sink = 4, int rec = 100, int B = 2, int32_t *kept = nullptr, int32_t *left = nullptr) {
    return fc_qcache_evict(&ctx, a, b, i32(12), keep, sink, rec, kept ? kept : i32(17), left, B, nullptr);
  };
  // what passes the checks reaches the device (none here)
  EXPECT(app(&c, &rope, &x), FC_ERR_HIP);
  EXPECT(att(&c), FC_ERR_HIP);
  EXPECT(ev(&c, &d), FC_ERR_HIP);
  // null
  EXPECT(fc_qcache_append(nullptr, &c, &rope, &x, i32(11), i32(12), nullptr, u16(14), 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_qcache_attention(nullptr, &c, u16(14), i32(12), nullptr, nullptr, u16(16), 28, 1.f, 0, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_qcache_evict(nullptr, &c, &d, i32(12), 1, 0, 0, i32(17), nullptr, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(app(nullptr, &rope, &x), FC_ERR_INVALID_ARG);
  EXPECT(app(&c, nullptr, &x), FC_ERR_INVALID_ARG);
  EXPECT(app(&c, &rope, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(app(&c, &rope, &x, 2, 1, nullptr, true), FC_ERR_INVALID_ARG);
  EXPECT(fc_qcache_append(&ctx, &c, &rope, &x, nullptr, i32(12), nullptr, u16(14), 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_qcache_append(&ctx, &c, &rope, &x, i32(11), nullptr, nullptr, u16(14), 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_qcache_attention(&ctx, &c, nullptr, i32(12), nullptr, nullptr, u16(16), 28, 1.f, 0, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  EXPECT(fc_qcache_evict(&ctx, &c, &d, nullptr, 1, 0, 0, i32(17), nullptr, 1, nullptr), FC_ERR_INVALID_ARG);
  for (int i = 0; i < 4; ++i) {
    fc_qcache y = c;
    if (i == 0) y.k = nullptr;
    if (i == 1) y.v = nullptr;
    if (i == 2) y.k_scale = nullptr;
    if (i == 3) y.v_scale = nullptr;
    EXPECT(app(&y, &rope, &x), FC_ERR_INVALID_ARG);
    EXPECT(att(&y), FC_ERR_INVALID_ARG);
    EXPECT(ev(&y, &d), FC_ERR_INVALID_ARG);
    EXPECT(ev(&c, &y), FC_ERR_INVALID_ARG);
  }
  // the cache's shape
  for (int cap : {0, 63, 100, -64, INT_MIN, (1 << 30) + 64, INT_MAX}) {
    fc_qcache y = c;
    y.capacity = cap;
    EXPECT(att(&y), FC_ERR_SHAPE);
  }
  for (int hd : {0, 32, 80, 256, -128, INT_MAX}) {
    fc_qcache y = c;
    y.head_dim = hd;
    EXPECT(att(&y), FC_ERR_UNSUPPORTED);
  }
  for (int kv : {0, -4, INT_MIN, 65536, INT_MAX}) {
    fc_qcache y = c;
    y.n_kv_heads = kv;
    EXPECT(att(&y), FC_ERR_SHAPE);
  }
  for (int B : {0, -1, INT_MIN, 16384, INT_MAX}) {
    EXPECT(app(&c, &rope, &x, B), FC_ERR_SHAPE);
    EXPECT(att(&c, 28, 0.1f, 1, B), FC_ERR_SHAPE);
    EXPECT(ev(&c, &d, 2000, 4, 100, B), FC_ERR_SHAPE);
  }
  for (int n : {0, -1, INT_MIN, 4225, INT_MAX}) {
    EXPECT(app(&c, &rope, &x, 2, n), FC_ERR_SHAPE);
    EXPECT(att(&c, 28, 0.1f, 1, 2, n), FC_ERR_SHAPE);
  }
  for (int H : {0, -4, 3, 30, INT_MAX}) EXPECT(att(&c, H), FC_ERR_SHAPE);
  for (int H : {65536, 1 << 28}) EXPECT(att(&c, H), FC_ERR_UNSUPPORTED);
  {
    fc_qcache big = c;
    big.capacity = 1 << 30;
    EXPECT(att(&big, 28, 0.1f, 0, 1, 1 << 29), FC_ERR_UNSUPPORTED);
    fc_qcache odd = c;
    odd.k = c.k + 8;
    EXPECT(att(&odd), FC_ERR_INVALID_ARG);
    odd = c;
    odd.weight = c.weight + 1;
    EXPECT(att(&odd), FC_ERR_INVALID_ARG);
    EXPECT(ev(&c, &odd), FC_ERR_INVALID_ARG);
  }
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
    y.v_item = s;
    EXPECT(app(&c, &rope, &y), FC_ERR_INVALID_ARG);
    y = x;
    y.q_row = s;
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
    y = x;
    y.q = u16(14), y.q_row = y.q_item = 28 * 128;
    EXPECT(app(&c, &rope, &y, 2, 1), FC_ERR_HIP);                        // in place
    y.q_item = 28 * 128 + 8;
    EXPECT(app(&c, &rope, &y, 2, 1), FC_ERR_INVALID_ARG);
    y = x;
    y.q = nullptr;
    EXPECT(app(&c, &rope, &y), FC_ERR_INVALID_ARG);
    EXPECT(app(&c, &rope, &y, 2, 1, nullptr, true), FC_ERR_HIP);
  }
  // attention
  for (float s : {NAN, INFINITY, -INFINITY}) EXPECT(att(&c, 28, s), FC_ERR_INVALID_ARG);
  for (int a : {-1, 2, INT_MAX}) EXPECT(att(&c, 28, 0.1f, a), FC_ERR_INVALID_ARG);
  {
    fc_qcache y = c;
    y.weight = nullptr;
    EXPECT(att(&y), FC_ERR_INVALID_ARG);
    EXPECT(att(&y, 28, 0.1f, 0), FC_ERR_HIP);
    EXPECT(ev(&y, &d), FC_ERR_INVALID_ARG);
    y = d;
    y.weight = nullptr;
    EXPECT(ev(&c, &y), FC_ERR_HIP);
    EXPECT(fc_qcache_attention(&ctx, &c, u16(14), i32(12), nullptr, nullptr, u16(14) + 8, 28, 1.f, 0, 1, 1, nullptr), FC_ERR_INVALID_ARG);
    EXPECT(fc_qcache_attention(&ctx, &c, u16(14), i32(12), nullptr, u8(15) + 1, u16(16), 28, 1.f, 0, 1, 1, nullptr), FC_ERR_INVALID_ARG);
  }
  // what is written shares memory with nothing else
  {
    const size_t k_bytes = (size_t)2 * 4 * 4224 * 128;
    auto to = [&](const void *out) {
      return fc_qcache_attention(&ctx, &c, u16(14), i32(12), i32(13), u8(15), reinterpret_cast<uint16_t *>((uintptr_t)out), 28, 1.f, 1, 2, 1, nullptr);
    };
    for (const void *p : {(const void *)(c.k + k_bytes - 16), (const void *)c.v, (const void *)c.k_scale, (const void *)c.v_scale, (const void *)c.weight,
                          (const void *)u8(15), (const void *)i32(12), (const void *)i32(13)})
      EXPECT(to(p), FC_ERR_INVALID_ARG);
    EXPECT(to(c.k + k_bytes), FC_ERR_HIP);
    EXPECT(fc_qcache_attention(&ctx, &c, u16(14), i32(12), i32(13), nullptr, reinterpret_cast<uint16_t *>(c.weight), 28, 1.f, 0, 2, 1, nullptr),
           FC_ERR_INVALID_ARG);                                      // nor over weights that stay as they are
    fc_qcache y = c;
    y.weight = reinterpret_cast<float *>(u8(15));
    EXPECT(att(&y), FC_ERR_INVALID_ARG);                                 // over the mask
    EXPECT(att(&y, 28, 0.1f, 0), FC_ERR_HIP);                            // not written
    y = c;
    y.v = c.k + k_bytes - 16;
    EXPECT(app(&y, &rope, &x), FC_ERR_INVALID_ARG);
    for (int i : {0, 1, 2, 3, 4, 11, 12, 13}) EXPECT(app(&c, &rope, &x, 2, 1, u16(i)), FC_ERR_INVALID_ARG);
    fc_qkv_rows z = x;
    z.k = reinterpret_cast<uint16_t *>(c.v);
    EXPECT(app(&c, &rope, &z), FC_ERR_INVALID_ARG);
  }
  // evict
  EXPECT(ev(&c, &d, 0, 0, 0), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, INT_MIN, 0, 0), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, 100, 60, 41), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, INT_MAX, INT_MAX, INT_MAX), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, 100, -1, 0), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, 2177), FC_ERR_SHAPE);
  EXPECT(ev(&c, &c), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, 2000, 4, 100, 2, i32(17), i32(12)), FC_ERR_INVALID_ARG);
  EXPECT(ev(&c, &d, 2000, 4, 100, 2, i32(17), i32(17) + 5), FC_ERR_INVALID_ARG);
  {
    fc_qcache y = d;
    y.n_kv_heads = 2;
    EXPECT(ev(&c, &y), FC_ERR_SHAPE);
    y = d;
    y.head_dim = 64;
    EXPECT(ev(&c, &y), FC_ERR_SHAPE);
    y = d;
    y.v = c.k + (size_t)2 * 4 * 4224 * 128 - 16;      // its first bytes are the other's last
    EXPECT(ev(&c, &y), FC_ERR_INVALID_ARG);
    y.v = c.k + (size_t)2 * 4 * 4224 * 128;
    EXPECT(ev(&c, &y), FC_ERR_HIP);
    y = d;
    y.weight = reinterpret_cast<float *>(y.k);
    EXPECT(ev(&c, &y), FC_ERR_INVALID_ARG);
  }
  std::printf(g_fail ? "%d failed\n" : "OK (%d failed expectations)\n", g_fail);
  return g_fail != 0;
}
