// Sweep of the W8A8 product: times every shape of kernel, with every K split that the library may choose, on each problem given, under HIP-graph
// replay, launches rotating over some 800 MB of weights (random bytes), and compares each launch's results with the first one's, which are the same bits
// where the kernels are right.
//   build:  hipcc -O3 -std=c++17 --offload-arch=gfx950 -Xclang -target-feature -Xclang -packed-fp32-ops -o w8a8_sweep w8a8_sweep.hip
//   run:    w8a8_sweep PROBLEMS [seconds]     (a file with "M N K" a line; stops at the next problem after so many seconds)
// Writes "M N K | shape/split us | ..." a problem, the shape by its place in kShapes (rtn_w8a8_plan.h), * behind the library's own choice.  w8a8_fit.py fits the
// plan's constants to that.
#include "../csrc/rtn_w8a8.hip"
#include <stdio.h>
#include <stdlib.h>
#include <time.h>
#include <vector>
using namespace rtn;
#define CK(x) do { hipError_t e = (x); if (e != hipSuccess) { printf("HIP error %s at %d\n", hipGetErrorString(e), __LINE__); fflush(stdout); exit(1); } } while (0)

__global__ void fill(uint32_t* p, int64_t n, uint32_t seed) {
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        uint32_t v = (uint32_t)i * 2654435769u + seed;
        v = (v ^ v >> 15) * 0x85EBCA6Bu;
        p[i] = v ^ v >> 13;
    }
}
__global__ void set_halves(half_t* p, int n, half_t v) { for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) p[i] = v; }
__global__ void set_floats(float* p, int n, float v) { for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) p[i] = v; }
__global__ void count_differences(const uint32_t* a, const uint32_t* b, int64_t n, int* count) {
    int here = 0;
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) here += a[i] != b[i];
    if (here) atomicAdd(count, here);
}

static hipStream_t st;
static hipEvent_t e0, e1;

int main(int argc, char** argv) {
    if (argc < 2) { printf("usage: w8a8_sweep PROBLEMS [seconds]\n"); return 1; }
    const double limit = argc > 2 ? atof(argv[2]) : 1e9;
    const int64_t kWeights = (int64_t)1 << 30, kRows = (int64_t)1 << 28, kOut = (int64_t)1 << 29;      // bytes of weights (a matrix may be larger), activations, results
    CK(hipStreamCreate(&st)); CK(hipEventCreate(&e0)); CK(hipEventCreate(&e1));
    uint8_t *W, *A, *C, *C0, *ws;
    half_t* scales; float* row_scales; int* wrong;
    const int64_t most = (int64_t)0x7FFF0000;
    CK(hipMalloc(&W, most + kWeights)); CK(hipMalloc(&A, kRows)); CK(hipMalloc(&C, kOut)); CK(hipMalloc(&C0, kOut)); CK(hipMalloc(&ws, kW8A8Workspace));
    CK(hipMalloc(&scales, (size_t)2 << 20)); CK(hipMalloc(&row_scales, (size_t)4 << 20)); CK(hipMalloc(&wrong, 4));
    fill<<<4096, 256, 0, st>>>((uint32_t*)W, (most + kWeights) / 4, 1); fill<<<4096, 256, 0, st>>>((uint32_t*)A, kRows / 4, 2);
    set_halves<<<64, 256, 0, st>>>(scales, 1 << 20, (half_t)1e-4f); set_floats<<<64, 256, 0, st>>>(row_scales, 1 << 20, 1e-3f);
    CK(hipStreamSynchronize(st));
    FILE* f = fopen(argv[1], "r");
    if (!f) { printf("no %s\n", argv[1]); return 1; }
    const time_t begin = time(nullptr);
    long M, N, K;
    while (fscanf(f, "%ld %ld %ld", &M, &N, &K) == 3) {
        if (difftime(time(nullptr), begin) > limit) { printf("# stopped before %ld %ld %ld\n", M, N, K); break; }
        if (check_w8a8(M, N, K) != RTN_OK || M * K > kRows || M * N * 2 > kOut || N > 1 << 20) { printf("# left out: %ld %ld %ld\n", M, N, K); continue; }
        const int sets = (int)std::max<int64_t>(1, std::min<int64_t>(24, (int64_t)800000000 / (N * K)));
        const W8A8Plan own = w8a8_plan(M, N, K, kW8A8Workspace);
        std::vector<W8A8Plan> plans = {own};
        for (int i = 0; i < kShapeCount; ++i) {
            const W8A8Shape& k = kShapes[i];
            const W8A8Cover& c = kCovers[i];
            const int64_t XB = (N + (1 << c.columns) - 1) >> c.columns, YB = (M + (1 << c.rows) - 1) >> c.rows, units = K >> c.unit;
            if (c.rows > 5 && ((int64_t)1 << c.rows) >= 2 * ((M + 15) / 16 * 16)) continue;
            if (k.kind == W8A8_STREAM && YB > 8) continue;
            if (k.kind == W8A8_BLOCK && XB * YB > 4096) continue;
            for (int split = 1; split <= kMostSplits; split += split < 4 ? 1 : 2) {
                if (split > 1 && (((int64_t)split << c.along) > units || XB * YB * split > 800 || (size_t)(M * N * 4 * split) > kW8A8Workspace)) break;
                if (i != own.shape || split != own.split) plans.push_back({i, split, XB, YB});
            }
        }
        printf("%ld %ld %ld", M, N, K);
        for (size_t n = 0; n < plans.size(); ++n) {
            const W8A8Plan& plan = plans[n];
            W8A8Params p = {(const int8_t*)A, row_scales, W, scales, n ? C : C0, (int*)ws, (int)M, (int)N, (int)(K / 64), (int)plan.XB, (int)plan.YB, plan.split};
            CK(launch_w8a8<RTN_TYPE_BF16>(p, plan, st));
            if (n) {
                int none = 0, count;
                CK(hipMemcpyAsync(wrong, &none, 4, hipMemcpyHostToDevice, st));
                count_differences<<<2048, 256, 0, st>>>((const uint32_t*)C, (const uint32_t*)C0, M * N / 2, wrong);
                CK(hipMemcpyAsync(&count, wrong, 4, hipMemcpyDeviceToHost, st)); CK(hipStreamSynchronize(st));
                if (count) { printf(" WRONG %d/%d: %d\n", plan.shape, plan.split, count); fflush(stdout); return 1; }
            }
            CK(hipEventRecord(e0, st)); CK(launch_w8a8<RTN_TYPE_BF16>(p, plan, st)); CK(hipEventRecord(e1, st)); CK(hipEventSynchronize(e1));
            float ms;
            CK(hipEventElapsedTime(&ms, e0, e1));
            const int launches = (int)std::max(4.f, std::min(24.f, 2.f / ms));
            hipGraph_t g; hipGraphExec_t ge;
            CK(hipStreamBeginCapture(st, hipStreamCaptureModeGlobal));
            p.C = C;
            for (int i = 0; i < launches; ++i) {
                p.B = W + (int64_t)(i % sets) * N * K;
                CK(launch_w8a8<RTN_TYPE_BF16>(p, plan, st));
            }
            CK(hipStreamEndCapture(st, &g)); CK(hipGraphInstantiate(&ge, g, nullptr, nullptr, 0));
            CK(hipGraphLaunch(ge, st));
            std::vector<float> ts;
            for (int r = 0; r < 5; ++r) {
                CK(hipEventRecord(e0, st)); CK(hipGraphLaunch(ge, st)); CK(hipEventRecord(e1, st)); CK(hipEventSynchronize(e1));
                CK(hipEventElapsedTime(&ms, e0, e1));
                ts.push_back(ms * 1e3f / launches);
            }
            std::sort(ts.begin(), ts.end());
            printf(" | %d/%d %.2f%s", plan.shape, plan.split, ts[2], n ? "" : "*");
            CK(hipGraphExecDestroy(ge)); CK(hipGraphDestroy(g));
        }
        printf("\n");
        fflush(stdout);
    }
    fclose(f);
    return 0;
}
