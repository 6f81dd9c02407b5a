// Attainable rate of v_mfma_scale_f32_32x32x64_f8f6f4 on this chip by the operands' formats, for the floors of the attention over block
// caches (not part of the library: a stand-alone program).
//
//   hipcc --offload-arch=gfx950 -O3 -std=c++17 -Xclang -target-feature -Xclang -packed-fp32-ops mfma_scale_rate_probe.hip -o mfma_scale_rate_probe
//   ./mfma_scale_rate_probe
//
// As in mfma_rate_probe.hip: one wavefront per SIMD, one workgroup per compute unit, four independent accumulators, on 256 compute units and
// on 32.  Operands are random bytes (those that would be NaN or among the largest as E4M3 are replaced), all scales 1.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <vector>

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

#define CHECK(x)                                                                   \
    do {                                                                           \
        hipError_t e_ = (x);                                                       \
        if (e_ != hipSuccess) {                                                    \
            fprintf(stderr, "%s failed: %s\n", #x, hipGetErrorString(e_));         \
            exit(1);                                                               \
        }                                                                          \
    } while (0)

// FA, FB: the instruction's format codes of A and B (0: E4M3, 2: E2M3, 4: E2M1)
template <int FA, int FB>
__global__ __launch_bounds__(256) void probe(const i32x8* __restrict__ in, float* out, int iters) {
    i32x8 a[4], b[4];
    for (int i = 0; i < 4; ++i) {
        a[i] = in[threadIdx.x * 8 + i];
        b[i] = in[threadIdx.x * 8 + 4 + i];
    }
    f32x16 acc[4];
    for (int c = 0; c < 4; ++c) acc[c] = f32x16{};
    for (int it = 0; it < iters; ++it) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[s], b[(s + c) & 3], acc[c], FA, FB, 0, 127, 0, 127);
    }
    float s = 0.f;
    for (int c = 0; c < 4; ++c)
        for (int v = 0; v < 16; ++v) s += acc[c][v];
    out[blockIdx.x * blockDim.x + threadIdx.x] = s;
}

template <int FA, int FB>
void run(const char* label, const i32x8* in, int blocks, int iters) {
    float* out;
    CHECK(hipMalloc(&out, sizeof(float) * blocks * 256));
    hipEvent_t e0, e1;
    CHECK(hipEventCreate(&e0));
    CHECK(hipEventCreate(&e1));
    CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(probe<FA, FB>), hipFuncAttributeMaxDynamicSharedMemorySize, 100 * 1024));
    float ms = 0;
    for (int rep = 0; rep < 4; ++rep) {
        CHECK(hipEventRecord(e0));
        hipLaunchKernelGGL((probe<FA, FB>), dim3(blocks), dim3(256), 100 * 1024, 0, in, out, iters);
        CHECK(hipEventRecord(e1));
        CHECK(hipEventSynchronize(e1));
        CHECK(hipEventElapsedTime(&ms, e0, e1));
    }
    const double n_mfma = (double)iters * 16;                // per wavefront = per SIMD
    printf("%-18s compute units %3d: %7.1f us, %5.2f ns per instruction and SIMD, %6.0f TFLOP/s\n", label, blocks, ms * 1e3, ms * 1e6 / n_mfma,
           n_mfma * 131072.0 * blocks * 4 / (ms * 1e-3) / 1e12);
    CHECK(hipFree(out));
}

int main() {
    std::vector<unsigned char> h(256 * 8 * sizeof(i32x8));
    srand(1);
    for (auto& x : h) {
        x = rand() & 0xff;
        if ((x & 0x7f) >= 0x70) x = (x & 0x80) | 0x38;
    }
    unsigned char* d;
    CHECK(hipMalloc(&d, h.size()));
    CHECK(hipMemcpy(d, h.data(), h.size(), hipMemcpyHostToDevice));
    for (int blocks : {256, 32}) {
        run<4, 0>("E2M1 x E4M3", (const i32x8*)d, blocks, 1000);
        run<0, 0>("E4M3 x E4M3", (const i32x8*)d, blocks, 1000);
        run<4, 2>("E2M1 x E2M3", (const i32x8*)d, blocks, 1000);
    }
    return 0;
}
