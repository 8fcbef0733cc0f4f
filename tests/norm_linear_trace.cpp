// norm_linear_trace.cpp - walks the host side of the layers in front of the LM head without a GPU: the HIP runtime's entry points are defined here, ahead of the real ones, and a
// launch is a line of output: grid and block (three numbers each) and the kernel's mangled name.
//   norm_linear_trace LIBRARY CALL..     for each call its launches, then "status S workspace BYTES"
//     matmul M N K DTYPE | forward M N K DTYPE KEEP | backward M N K DTYPE DX DW | norm R H DTYPE KEPT (forward, then backward from x or its checkpoint) | rows R K DTYPE (pack, unpack)
//     | weight N K DTYPE | formats X W (of the calls that follow) | kernels (the names of those that the library holds)
#include <dlfcn.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>

#include "../include/rl_norm_linear.h"

struct dim3 { unsigned x, y, z; };

static std::map<const void*, std::string> g_names;
static dim3 g_grid, g_block;

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* h; return &h; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { g_names[host] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, void*) { g_grid = grid; g_block = block; return 0; }
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, void** stream) { *grid = g_grid; *block = g_block; *lds = 0; *stream = nullptr; return 0; }
int hipLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t, void*) {
  printf("%u %u %u %u %u %u %s\n", g.x, g.y, g.z, b.x, b.y, b.z, g_names.at(f).c_str());
  return 0;
}
int hipGetLastError() { return 0; }
}

int main(int argc, char** argv) {
  void* lib = argc > 1 ? dlopen(argv[1], RTLD_NOW | RTLD_LOCAL) : nullptr;
  if (!lib) { fprintf(stderr, "%s\n", argc > 1 ? dlerror() : "usage: norm_linear_trace LIBRARY CALL.."); return 2; }
  if (g_names.empty()) { fprintf(stderr, "the library registered no kernel here\n"); return 2; }
  auto at = [](int i) { return reinterpret_cast<void*>((uintptr_t)(i + 1) << 48); };          // addresses that nothing follows, far apart
#define GET(name) const auto name = reinterpret_cast<decltype(&::name)>(dlsym(lib, #name))
  GET(rl_f8_matmul_workspace_bytes); GET(rl_f8_matmul); GET(rl_f8_linear_forward_workspace_bytes); GET(rl_f8_linear_forward);
  GET(rl_f8_linear_backward_workspace_bytes); GET(rl_f8_linear_backward);
  GET(rl_layer_norm_forward); GET(rl_layer_norm_backward_workspace_bytes); GET(rl_layer_norm_backward); GET(rl_f8_pack); GET(rl_f8_unpack); GET(rl_f8_pack_weight);
  int fx = 0, fw = 0;
  for (int i = 2; i < argc;) {
    const std::string call = argv[i++];
    auto next = [&] { return i < argc ? atoll(argv[i++]) : 0; };
    if (call == "formats") { fx = (int)next(); fw = (int)next(); continue; }
    if (call == "kernels") { for (auto& k : g_names) printf("kernel %s\n", k.second.c_str()); continue; }
    size_t n = 0;
    int st;
    const int64_t M = next();
    const int N = (int)next();
    if (call == "norm" || call == "rows" || call == "weight") {
      const int dtype = (int)next();
      if (call == "norm") {
        const bool kept = next();
        st = rl_layer_norm_forward(at(0), N, dtype, M, N, at(1), at(2), 0, 1e-5f, at(3), N, (float*)at(4), kept ? at(5) : nullptr, kept ? at(6) : nullptr, fx, nullptr);
        if (st == RL_OK) st = rl_layer_norm_backward_workspace_bytes(M, N, &n);
        if (st == RL_OK) st = rl_layer_norm_backward(at(7), N, kept ? nullptr : at(0), N, kept ? at(5) : nullptr, kept ? at(6) : nullptr, fx, dtype, M, N, at(1), 0, (const float*)at(4),
                                                     at(8), N, (float*)at(9), (float*)at(10), at(11), n, nullptr);
      } else if (call == "rows") {
        st = rl_f8_pack(at(0), N, dtype, M, N, fx, at(1), at(2), nullptr);
        if (st == RL_OK) st = rl_f8_unpack(at(1), at(2), fx, M, N, at(3), N, dtype, nullptr);
      } else st = rl_f8_pack_weight(at(0), N, dtype, (int)M, N, fw, at(1), at(2), at(3), at(4), nullptr);
      printf("status %d workspace %zu\n", st, n);
      continue;
    }
    const int K = (int)next(), dtype = (int)next();
    if (call == "matmul") {
      st = rl_f8_matmul_workspace_bytes(M, N, K, &n);
      if (st == RL_OK) st = rl_f8_matmul(at(0), at(1), fx, at(2), at(3), fw, M, N, K, at(4), N, dtype, at(9), n, nullptr);
    } else if (call == "forward") {
      const bool keep = next();
      st = rl_f8_linear_forward_workspace_bytes(M, N, K, keep, &n);
      if (st == RL_OK) st = rl_f8_linear_forward(at(0), K, dtype, M, K, fx, at(2), at(3), fw, N, at(4), N, keep ? at(5) : nullptr, keep ? at(6) : nullptr, at(9), n, nullptr);
    } else {
      const bool dx = next(), dW = next();
      st = rl_f8_linear_backward_workspace_bytes(M, N, K, dtype, &n);
      if (st == RL_OK) st = rl_f8_linear_backward(at(0), N, dtype, M, N, K, fx, at(1), at(2), fx, at(3), at(4), fw, dx ? at(5) : nullptr, K, dW ? (float*)at(6) : nullptr, K, 0, at(9), n, nullptr);
    }
    printf("status %d workspace %zu\n", st, n);
  }
  return 0;
}
