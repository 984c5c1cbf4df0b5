// What the entry points of mpic_q4.h do when the host has no memory left for an error message (built by
// tests/test_q4_refusals.py with g++ and linked with the library): they return their status and throw nothing.
#include <cstdio>
#include <cstdlib>
#include <new>

#include "mpic_q4.h"

static bool none_left = false;
void* operator new(std::size_t n) {
  if (none_left) throw std::bad_alloc();
  return std::malloc(n ? n : 1);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

static int bad = 0;
template <typename F>
void expect(const char* what, int status, F call) {
  int rc = 1;
  none_left = true;
  try {
    rc = call();
  } catch (...) {
    rc = 2;
  }
  none_left = false;
  if (rc != status) {
    std::printf("%s: %s, expected status %d\n", what, rc == 2 ? "threw" : "wrong status", status);
    ++bad;
  }
}

int main() {
  mpic_config c{};
  c.n_q_heads = 4;
  c.n_kv_heads = 2;
  c.head_dim = 128;
  c.dtype = MPIC_BF16;
  c.rope_theta = 1e4;
  mpic_ctx* ctx = nullptr;
  if (mpic_create(&ctx, &c) != MPIC_OK) return 2;
  void* const at = reinterpret_cast<void*>(1 << 20);  // nothing is read from it
  const int32_t* const i32 = static_cast<const int32_t*>(at);
  expect("position_rows", MPIC_ERR_INVALID, [&] { return mpic_position_rows(ctx, at, 512, at, 256, -1, i32, 1, nullptr, nullptr, nullptr, -1.0, at, 512, at, 256, nullptr); });
  expect("position_rows, too many", MPIC_ERR_UNSUPPORTED, [&] { return mpic_position_rows(ctx, at, 512, at, 256, 1 << 30, i32, 1, nullptr, nullptr, nullptr, -1.0, at, 512, at, 256, nullptr); });
  expect("q4_write", MPIC_ERR_INVALID, [&] { return mpic_q4_write(ctx, at, 8, at, 256, 4, i32, at, 1 << 20, 64, nullptr); });
  expect("q4_write, too many", MPIC_ERR_UNSUPPORTED, [&] { return mpic_q4_write(ctx, at, 256, at, 256, 1 << 30, i32, at, 1 << 20, 64, nullptr); });
  expect("q4_read", MPIC_ERR_INVALID, [&] { return mpic_q4_read(ctx, at, 8, 64, i32, 4, at, 256, at, 256, nullptr); });
  expect("q4_attn", MPIC_ERR_INVALID, [&] { return mpic_q4_attn(ctx, at, 512, 3, nullptr, 1, at, 1 << 20, 64, i32, 4, 24, i32, 3, 64, 0.1, at, nullptr, nullptr, 0, nullptr); });
  expect("q4_attn, too many", MPIC_ERR_UNSUPPORTED, [&] { return mpic_q4_attn(ctx, at, 512, 70000, nullptr, 1, at, 1 << 20, 64, i32, 4, 16, i32, 70000, 64, 0.1, at, nullptr, nullptr, 0, nullptr); });
  // the message of the call that had memory again
  if (mpic_q4_write(ctx, at, 8, at, 256, 4, i32, at, 1 << 20, 64, nullptr) != MPIC_ERR_INVALID || !*mpic_last_error(ctx)) ++bad;
  mpic_destroy(ctx);
  if (!bad) std::printf("refused without memory\n");
  return bad ? 1 : 0;
}
