// Runs, on the host alone, the choice of a product's kernel: launches are recorded here instead of
// reaching a GPU.  Each argument is a product, "M N K epilogue residual result" (epilogue as in
// launch.h, the types 0 for bf16 and 1 for fp32), and gives a line with the launch:
//   <workgroups> <threads each> <kernel>
#include "k_int_gemm.hip"

#include <stdio.h>
#include <string.h>

using namespace ardit;

static bool is(const void* f, const void* kernel, const char* name) {
  if (f == kernel) printf("%s", name);
  return f == kernel;
}
#define IS(NAME, ...) is(f, reinterpret_cast<const void*>(&__VA_ARGS__), NAME)

template <int BM>
static bool large(const void* f, const char* name) {
  char full[64];
#define IS_LARGE(E, R, O) (snprintf(full, sizeof(full), "%s:" #E ":" #R ":" #O, name), IS(full, int_gemm_kernel<BM, E, R, O>))
#define IS_RES(E) (IS_LARGE(E, float, float) || IS_LARGE(E, float, bf16_t) || IS_LARGE(E, bf16_t, float) || IS_LARGE(E, bf16_t, bf16_t))
  return IS_LARGE(kEpiBias, bf16_t, float) || IS_LARGE(kEpiBias, bf16_t, bf16_t) || IS_LARGE(kEpiBiasGelu, bf16_t, bf16_t) ||
         IS_RES(kEpiBiasRes) || IS_RES(kEpiBiasGateRes);
}

// Nothing is registered (there is no device code), and launches are taken over from the runtime.
extern "C" void** __hipRegisterFatBinary(const void*) { return nullptr; }
extern "C" void __hipUnregisterFatBinary(void**) {}
extern "C" void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
static dim3 g_grid, g_block;
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = g_grid;
  *block = g_block;
  *lds = 0;
  *stream = nullptr;
  return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }
extern "C" hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  printf("%u %u ", grid.x, block.x);
  const bool known = large<128>(f, "128x256") || large<192>(f, "192x256") || large<256>(f, "256x256") ||
                     IS("32x64", int_gemm_small<2, 2, 1, 2, 3, 4>) || IS("64x64", int_gemm_small<2, 2, 2, 2, 5, 1>) ||
                     IS("64x64/2", int_gemm_small<2, 2, 2, 2, 5, 2>) || IS("64x128/2", int_gemm_small<2, 2, 2, 4, 3, 2>) ||
                     IS("128x128", int_gemm_small<2, 4, 4, 2, 5, 1>);
  printf("%s\n", known ? "" : "few");
  return hipSuccess;
}

int main(int argc, char** argv) {
  for (int i = 1; i < argc; ++i) {
    IntGemmArgs a = {};
    int epi, res, out;
    if (sscanf(argv[i], "%d %d %d %d %d %d", &a.M, &a.N, &a.K, &epi, &res, &out) != 6) return 2;
    a.ldx = a.ldw = (a.K + 15) / 16 * 16;
    a.ldr = a.ldy = a.N;
    a.res_f32 = res;
    a.y_f32 = out;
    a.rows_per_stream = make_fastdiv(1);
    if (launch_int_gemm(nullptr, epi, a) != hipSuccess) return 3;
  }
  return 0;
}
