// Drives the host side of the calls for chunks with extreme and ordinary arguments; launchers are stubs that check what they are given.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../include/akvq.h"
#include "../../paper_2501_15021_amd/csrc/akvq_kernels.h"

namespace akvq {
static int launches = 0;
static void check(bool ok, const char *what) {
  if (!ok) { std::printf("failed: %s\n", what); std::exit(1); }
}
static void check_pages(const PagedArgs &c) {
  check(c.max_rows > 0 && c.max_rows <= c.n_rows && c.max_len >= 0 && c.max_len <= c.row_cap, "bounds of the chunk");
  check((1 << c.page_shift) >= 32 && (long long)c.max_pages << c.page_shift == c.row_cap, "pages");
}
hipError_t launch_rope_axes(AxesArgs a, hipStream_t) { check(a.n_rows > 0 && a.Hq + a.Hkv > 0, "rows"); ++launches; return hipSuccess; }
hipError_t launch_rope_axes_table(const AxesArgs &a, hipStream_t) { check(a.n_rows > 0, "rows"); ++launches; return hipSuccess; }
hipError_t launch_paged_append(const PagedAppendArgs &a, int, hipStream_t) { check_pages(a.c); ++launches; return hipSuccess; }
hipError_t launch_paged_attention(const PagedAttentionArgs &a, int, hipStream_t) {
  check_pages(a.c);
  const long units = (long)a.c.B * a.c.Hkv, R = a.Hq / a.c.Hkv, per = paged_tile_rows(units, a.c.max_rows, R, a.c.max_len);
  check(per == 16 || per == 32 || per == kPagedManyRows, "tile");
  check((a.c.max_rows * R + per - 1) / per <= 65535, "grid");
  check(per != 16 || a.c.max_rows <= 32, "a tile of 16 rows sees one block of the chunk");
  check(a.n_split >= 1 && a.n_split <= 1024 && (a.n_split == 1 || a.partial), "splits");
  ++launches;
  return hipSuccess;
}
int launch_status(hipError_t e) { return e == hipSuccess ? AKVQ_OK : -3; }
}  // namespace akvq

int main() {
  const int ints[] = {INT_MIN, -1, 0, 1, 2, 17, 31, 32, 33, 64, 96, 128, 1000, 65535, 65536, 1 << 20, 1 << 25, (1 << 25) + 1, 1 << 30, INT_MAX};
  const int64_t strides[] = {INT64_MIN, -8, 0, 8, 128, 4096, 4100, INT64_MAX};
  void *const p = reinterpret_cast<void *>(uintptr_t{1} << 20);
  int32_t *const i32 = static_cast<int32_t *>(p);
  uint32_t *const u32 = static_cast<uint32_t *>(p);
  uint16_t *const u16 = static_cast<uint16_t *>(p);
  long calls = 0;
  auto paged = [&](int B, int Hkv, int G, int rows, int n, int max, int S, int len) {
    return akvq_paged{B, Hkv, G, rows, n, max, S, len, u32, u32, u32, u32, u16, u16, i32, i32, i32, i32};
  };
  const akvq_paged good = paged(3, 4, 128, 64, 50, 20, 64, 1000);
  size_t sizes[8];
  auto drive = [&](const akvq_paged &c, const akvq_chunk &r, int Hq, int64_t stride, int n_split, size_t bytes) {
    ++calls;
    akvq_paged_bytes(&c, sizes);
    const int n = akvq_paged_default_splits(&c, Hq, r.max_rows);
    akvq::check(n >= 1 && n <= 64, "default splits");
    akvq_paged_workspace_bytes(r.n_rows, Hq, n_split);
    akvq_paged_append(&c, &r, p, stride, p, stride, 0.8f, 0, nullptr);
    akvq_paged_attention(&c, &r, p, stride, Hq, p, stride, p, stride, 0.1f, p, stride, nullptr, n_split, p, bytes, 0, nullptr);
  };
  for (int x : ints)
    for (int y : ints) {
      drive(good, {i32, x, y}, 8, 4096, 0, SIZE_MAX);
      drive(good, {i32, x, y}, 28, 4096, 3, SIZE_MAX);
      drive(good, {i32, 5, 5}, x, 4096, y, SIZE_MAX);
      drive(paged(x, y, 64, 32, 9, 9, 64, 100), {i32, 40, 40}, y, 1 << 20, 0, SIZE_MAX);
      drive(paged(1, 1, 128, x, y, 5, 64, 100), {i32, 300, 70}, 8, 4096, 0, 0);
      drive(paged(1, 2, 128, 64, x, y, 64, INT_MAX), {i32, 1 << 25, 1 << 25}, 16, 4096, 0, SIZE_MAX);
      drive(paged(2, 1, 64, 32, 4, 1 << 20, x, y), {i32, 33, 9}, 7, 4096, 1024, 1);
      akvq_axes axes{x, {}, {}};
      for (int a = 0; a < 64; ++a) axes.axis[a] = (uint8_t)(a % 4);
      for (int64_t s : strides) {
        drive(good, {i32, 70, 70}, 8, s, 0, SIZE_MAX);
        akvq_rope_axes(&axes, i32, s, y, p, s, 2, p, s, 1, p, s, p, s, 0, nullptr);
        axes.n_axes = 4;
        akvq_rope_axes(&axes, i32, INT64_MAX, y, p, 8192, x, p, 8192, y, p, 8192, p, 8192, 0, nullptr);
        akvq_rope_axes_table(&axes, i32, s, x, p, p, nullptr);
      }
    }
  std::printf("ok %d launches of %ld\n", akvq::launches, calls);
  return 0;
}
