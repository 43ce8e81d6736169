// Host-side driver over the 8-bit token cache's argument checks at the largest sizes, built with
// the host sanitizers and run without a GPU (tests/test_qcache_abi_sanitize.py): a context built by
// hand, byte ranges that 32 bits do not hold.  Exit status 0: every expectation held.
#include <climits>
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
  constexpr int kRows = 1 << 30;
  const fc_qcache c{u8(0), u8(1), f32(2), f32(3), f32(4), 1, 64, kRows};
  const fc_qcache d{u8(5), u8(6), f32(7), f32(8), f32(9), 1, 64, kRows};
  const fc_rope_axes axes{1e6, {8, 8, 16}};
  // one row for every token (stride 0)
  const fc_qkv_rows x{nullptr, u16(10), u16(11), 0, 0, 0, 0, 0, 0, 1};
  auto app = [&](const fc_qkv_rows &rows, const int32_t *pos, int n) {
    return fc_qcache_append(&ctx, &c, &axes, &rows, pos, i32(13), nullptr, nullptr, 1, n, nullptr);
  };
  // positions of three axes: 3 n numbers, more than an int counts
  for (int n : {715827883, 1 << 29, kRows - 200}) {
    EXPECT(app(x, i32(12), n), FC_ERR_HIP);                                   // passes the checks: no device here
    const long bytes = 3L * n * 4;
    EXPECT(app(x, reinterpret_cast<int32_t *>(at(0) - bytes), n), FC_ERR_HIP);       // end where the keys begin
    EXPECT(app(x, reinterpret_cast<int32_t *>(at(0) - bytes + 4), n), FC_ERR_INVALID_ARG);   // their last one is the keys' first
    EXPECT(app(x, reinterpret_cast<int32_t *>(at(0) + (64L << 30) - 4), n), FC_ERR_INVALID_ARG);
  }
  // strides whose rows end beyond 64 bits: (n - 1) k_row is 2^64 elements here, and 2^63 bytes
  for (int n : {(1 << 24) + 1, (1 << 22) + 1, kRows - 200}) {
    for (int64_t s : {(int64_t)1 << 40, ((int64_t)1 << 40) - 8}) {
      fc_qkv_rows y = x;
      y.k_row = s;
      EXPECT(app(y, i32(12), n), FC_ERR_INVALID_ARG);
      y = x;
      y.v_row = s;
      EXPECT(app(y, i32(12), n), FC_ERR_INVALID_ARG);
    }
    fc_qkv_rows y = x;
    y.k_row = y.v_row = 64;
    EXPECT(app(y, i32(12), n), FC_ERR_HIP);
  }
  // a stride that no token takes says nothing
  fc_qkv_rows one = x;
  one.k_row = one.v_row = one.k_item = one.v_item = (int64_t)1 << 40;
  EXPECT(app(one, i32(12), 1), FC_ERR_HIP);
  // a grid holds fewer than 2^32 threads: 2^24 - 1 workgroups of 256, 64 rows each, one more block
  // where the rows start inside one
  for (int n : {kRows, kRows - 64, kRows - 126}) EXPECT(app(x, i32(12), n), FC_ERR_UNSUPPORTED);
  EXPECT(app(x, i32(12), kRows - 127), FC_ERR_HIP);
  auto ev = [&](int keep) { return fc_qcache_evict(&ctx, &c, &d, i32(13), keep, 0, 0, i32(14), nullptr, 1, nullptr); };
  for (int keep : {kRows, kRows - 63}) EXPECT(ev(keep), FC_ERR_UNSUPPORTED);
  EXPECT(ev(kRows - 64), FC_ERR_HIP);
  std::printf(g_fail ? "%d failed\n" : "OK (%d failed expectations)\n", g_fail);
  return g_fail != 0;
}
