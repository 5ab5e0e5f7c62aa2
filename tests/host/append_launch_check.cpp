// What vq_cache_append launches (tests/test_append_launches.py): this program is linked against libvq.so and its own definitions of the HIP runtime's
// calls come first in the lookup, so nothing reaches the real runtime.  Batches up to the limits of vq_attn_batch: one launch each, every dimension of
// the grid within the threads and workgroups that a launch may have, and, for pages in 8 bits, a workgroup for every token and head, or for every tile.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <string>

#include <hip/hip_runtime_api.h>
#include "../../include/vq.h"

#define REQUIRE(cond)                                                                       \
  do {                                                                                      \
    if (!(cond)) {                                                                          \
      std::fprintf(stderr, "%s:%d: %s violated\n", __FILE__, __LINE__, #cond);              \
      std::abort();                                                                         \
    }                                                                                       \
  } while (0)

namespace {
std::map<const void*, std::string>& names() {   // filled while libvq's initialisers run
  static std::map<const void*, std::string> n;
  return n;
}
dim3 g_grid, g_block;
size_t g_shared;
hipStream_t g_stream;
std::string g_kernel;
int g_launches = 0;
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* device, unsigned, void*, void*, void*, void*, int*) { names()[host] = device; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t s) {
  g_grid = grid; g_block = block; g_shared = shared; g_stream = s;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* s) {
  *grid = g_grid; *block = g_block; *shared = g_shared; *s = g_stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  ++g_launches;
  g_kernel = names()[f];
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

int main() {
  std::mt19937 rng(7);
  auto below = [&](long long most) { return 1 + (int)((long long)(rng() % (1u << (1 + rng() % 31))) % most); };   // 1 .. most, small ones often
  auto at = [](uintptr_t i) { return reinterpret_cast<void*>(i << 45); };                                          // never read
  const int dims[] = {64, 96, 128, 256}, pages[] = {16, 32, 64, 128};
  int few = 0, tiles = 0, largest = 0;
  for (int i = 0; i < 200000; ++i) {
    vq_attn_desc d = {};
    d.kv_heads = rng() % 2 ? below(1024) : 1 << rng() % 11;
    d.heads = d.kv_heads * (rng() % 2 ? 1 : below(1024 / d.kv_heads));
    d.head_dim = dims[rng() % 4];
    d.page_size = pages[rng() % 4];
    d.n_pages = below(2147483647);
    d.dtype = rng() % 2 ? VQ_F16 : VQ_BF16;
    d.cache_dtype = rng() % 4 ? VQ_E4M3 : 0;
    vq_attn_batch b = {};
    b.n_seqs = rng() % 2 ? below(65535) : below(300);
    const long long most = (((1ll << 20) - (long long)b.n_seqs * d.heads) * 128 + 127) / d.heads;                  // tokens that a batch may have
    b.n_tokens = most < 1 || rng() % 4 == 0 ? b.n_seqs : (int)(rng() % 3 ? below(most < 2147483647 ? most : 2147483647) : (most < 2147483647 ? most : 2147483647));
    b.table_width = (1 << 29) / d.page_size;
    b.max_len = below(1 << 29);
    b.q_start = rng() % 8 || b.n_tokens != b.n_seqs ? (const int32_t*)at(3) : nullptr;
    b.kv_len = (const int32_t*)at(1);
    b.page_table = (const int32_t*)at(2);
    const vq_strides features = {1, (int64_t)d.head_dim << 28, 1 << 28};
    const vq_strides* s = rng() % 2 ? &features : nullptr;
    g_launches = 0;
    const int st = vq_cache_append(&d, &b, at(4), s, at(5), s, at(6), at(7), nullptr);
    if (st != VQ_OK) {
      REQUIRE(st == VQ_ERR_BAD_ARG && g_launches == 0);   // more rows than a batch may have
      REQUIRE((long long)b.n_tokens * d.heads / 128 + (long long)b.n_seqs * d.heads > 1 << 20);
      continue;
    }
    REQUIRE(g_launches == 1);
    REQUIRE(g_block.x <= 1024 && g_block.y == 1 && g_block.z == 1);
    REQUIRE(g_grid.x >= 1 && (uint64_t)g_grid.x * g_block.x < 1ull << 32);
    REQUIRE(g_grid.y >= 1 && g_grid.y <= 65535 && g_grid.z >= 1 && g_grid.z <= 65535);
    largest += (long long)b.n_tokens * d.heads / 128 + (long long)b.n_seqs * d.heads > (1 << 20) - 1024;
    if (!d.cache_dtype) {
      REQUIRE(g_kernel.find("append8") == std::string::npos);
      continue;
    }
    if (g_kernel.find("append8_few_kernel") != std::string::npos) {
      ++few;
      const int lanes = d.head_dim == 64 ? 8 : d.head_dim == 256 ? 32 : 16;
      REQUIRE(g_block.x == 256 && g_grid.x == (unsigned)b.n_tokens && (long long)g_grid.y * 256 >= (long long)d.kv_heads * lanes);
    } else {
      REQUIRE(g_kernel.find("append8_kernel") != std::string::npos);
      ++tiles;
      REQUIRE(g_block.x == 128u * ((d.head_dim + 63) / 64));
      REQUIRE(g_grid.x == (uint64_t)(b.n_tokens / 64 + 2ll * b.n_seqs) * d.kv_heads);
    }
  }
  REQUIRE(few > 10000 && tiles > 10000 && largest > 100);
  std::printf("append launches ok\n");
  return 0;
}
