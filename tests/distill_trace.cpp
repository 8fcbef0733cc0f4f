// distill_trace.cpp - walks the host side of scoring with alternatives and of distillation without a GPU: the HIP runtime's entry points are defined here, ahead of the real ones, and a
// launch is a line of output: grid and block (three numbers each) and the kernel's mangled name.
//   distill_trace LIBRARY CALL..     for each call its launches, then "status S workspace BYTES"
//     score R H V B DTYPE K CHUNK OFF | distill R H V B DTYPE K CHUNK OFF BACKWARD DWEIGHT      (OFF: bytes that weight and hidden start behind a 256-byte boundary)
//     kernels (the names of those that the library holds)
#include <dlfcn.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>

#include "../include/rl_distill.h"

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
  if (!lib) { fprintf(stderr, "%s\n", argc > 1 ? dlerror() : "usage: distill_trace LIBRARY CALL.."); return 2; }
  if (g_names.empty()) { fprintf(stderr, "the library registered no kernel here\n"); return 2; }
  auto at = [](int i) { return reinterpret_cast<void*>((uintptr_t)(i + 1) << 48); };          // addresses that nothing follows, far apart
#define GET(name) const auto name = reinterpret_cast<decltype(&::name)>(dlsym(lib, #name))
  GET(rl_token_top_logprobs_workspace_bytes); GET(rl_token_top_logprobs); GET(rl_distill_workspace_bytes); GET(rl_distill_loss_fwd_bwd);
  for (int i = 2; i < argc;) {
    const std::string call = argv[i++];
    auto next = [&] { return i < argc ? atoll(argv[i++]) : 0; };
    if (call == "kernels") { for (auto& k : g_names) printf("kernel %s\n", k.second.c_str()); continue; }
    rl_batch b{};
    b.R = next(); b.H = (int)next(); b.V = (int)next(); b.B = (int)next(); b.P = 1; b.dtype = (int)next();
    const int K = (int)next(), chunk = (int)next(), off = (int)next();
    b.hidden = static_cast<char*>(at(0)) + off; b.weight = static_cast<char*>(at(1)) + off;
    b.token_ids = (const int*)at(2); b.mask = (const uint8_t*)at(3); b.cu_seqlens = (const int*)at(4);
    size_t n = 0;
    int st;
    if (call == "score") {
      const rl_top_params p{K, chunk, 1.f};
      const rl_top_outputs o{(float*)at(5), (float*)at(6), (float*)at(7), (int*)at(8), (float*)at(9)};
      st = rl_token_top_logprobs_workspace_bytes(&b, &p, &n);
      if (st == RL_OK) st = rl_token_top_logprobs(&b, &p, &o, at(20), n, nullptr);
    } else {
      const bool bwd = next();
      const rl_distill_params p{K, 0, 0, chunk, 1.f, 1.f, (int)next()};
      rl_distill_outputs o{(float*)at(5), (float*)at(6), (float*)at(7), bwd ? at(8) : nullptr, bwd ? at(9) : nullptr, (rl_distill_stats*)at(10)};
      st = rl_distill_workspace_bytes(&b, &p, bwd, &n);
      if (st == RL_OK) st = rl_distill_loss_fwd_bwd(&b, (const int*)at(11), (const float*)at(12), &p, &o, at(20), n, nullptr);
    }
    printf("status %d workspace %zu\n", st, n);
  }
  return 0;
}
