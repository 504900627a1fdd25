// launch_host.cu -- the launches of the 8-bit products without a GPU: the library's host code as it is, on a runtime made here that knows several
// devices, holds shared-memory attributes for each, and writes down every launch.  Built in three pieces (PIECE: the tokens' products, the
// layers, and the program that reads calls from its input).
#include <cuda.h>
#include <cuda_runtime.h>

#include <stdio.h>
#include <string.h>

#include <map>
#include <utility>

namespace fake {
struct Device {
    std::map<const void*, int> smem;  // attribute of each kernel
};
inline std::map<int, Device>& devices() {
    static std::map<int, Device> d;
    return d;
}
inline int& device() {
    static int d = 0;
    return d;
}
inline cudaError_t& error() {
    static cudaError_t e = cudaSuccess;
    return e;
}
inline int room(const void* kernel) {
    const auto& s = devices()[device()].smem;
    return s.count(kernel) ? s.at(kernel) : 48 * 1024;
}
inline cudaError_t get_device(int* d) { return *d = device(), cudaSuccess; }
inline cudaError_t last_error() {
    const cudaError_t e = error();
    error() = cudaSuccess;
    return e;
}
template <typename K>
cudaError_t set_attribute(K* kernel, cudaFuncAttribute a, int bytes) {
    if (a != cudaFuncAttributeMaxDynamicSharedMemorySize || bytes > 227 * 1024) return error() = cudaErrorInvalidValue;
    devices()[device()].smem[(const void*)kernel] = bytes;
    return cudaSuccess;
}
template <typename K>
cudaError_t get_attributes(cudaFuncAttributes* a, K*) {
    memset(a, 0, sizeof *a);
    a->numRegs = 80;
    return cudaSuccess;
}
inline int cluster(const cudaLaunchConfig_t& c) {
    int n = 1;
    for (unsigned i = 0; i < c.numAttrs; ++i)
        if (c.attrs[i].id == cudaLaunchAttributeClusterDimension) n = c.attrs[i].val.clusterDim.x;
    return n;
}
// (one CTA an SM, 152 SMs in groups of 19)
template <typename K>
cudaError_t most_clusters(int* n, K* kernel, const cudaLaunchConfig_t* c) {
    if ((int)c->dynamicSmemBytes > room((const void*)kernel)) return error() = cudaErrorInvalidValue;
    *n = 8 * (19 / cluster(*c));
    return cudaSuccess;
}
template <typename K, typename... A>
cudaError_t launch(const cudaLaunchConfig_t* c, K* kernel, A&&...) {
    const bool fits = (int)c->dynamicSmemBytes <= room((const void*)kernel) && c->gridDim.x >= 1 && c->gridDim.y >= 1 && c->gridDim.z >= 1 &&
                      c->gridDim.x <= 0x7fffffffu && c->gridDim.y <= 65535 && c->gridDim.z <= 65535 && cluster(*c) <= 8 && c->gridDim.x % cluster(*c) == 0;
    printf(" %s[%u %u %u; %u; %zu; %d]", fits ? "" : "REFUSED", c->gridDim.x, c->gridDim.y, c->gridDim.z, c->blockDim.x, c->dynamicSmemBytes, cluster(*c));
    return fits ? cudaSuccess : error() = cudaErrorInvalidValue;
}
}  // namespace fake

#if PIECE == 0
#include "fxpq_layer.cuh"

namespace fxpq {
int num_sms() { return 152; }
int* status_ptr() { return nullptr; }
void note_launch() {}
fxpq_status after_launch(const char*) { return fake::last_error() == cudaSuccess ? FXPQ_OK : FXPQ_ERR_CUDA; }
typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                           CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// What the driver refuses: extents and boxes of none, boxes past 256, strides that are not whole 16 bytes.
static CUresult encode(CUtensorMap*, CUtensorMapDataType type, cuuint32_t rank, void* at, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
                       const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    const unsigned bytes = type == CU_TENSOR_MAP_DATA_TYPE_FLOAT16 ? 2 : 1;
    const bool ok = rank == 2 && (size_t)at % 16 == 0 && dims[0] >= 1 && dims[0] <= 0xffffffffull && dims[1] >= 1 && dims[1] <= 0xffffffffull && strides[0] % 16 == 0 &&
                    strides[0] >= dims[0] * bytes && strides[0] < (1ull << 40) && box[0] * bytes == 128 && box[1] >= 1 && box[1] <= 256;
    return ok ? CUDA_SUCCESS : CUDA_ERROR_INVALID_VALUE;
}
Encode encode_tiled() { return encode; }
namespace llm {
fxpq_status grad_rows(const GradRows&, int, int, cudaStream_t) {
    printf(" rows");
    return FXPQ_OK;
}
}  // namespace llm
}  // namespace fxpq

// "device D", "linear M N K", "layer M N K x_type norm gated kept", "grad M N K dx_type act": the launches of each, and its status.
int main() {
    char what[16];
    void* p = reinterpret_cast<void*>(size_t(1) << 40);  // (nothing reads it)
    float* f = static_cast<float*>(p);
    while (scanf("%15s", what) == 1) {
        int rc = 0;
        long long M;
        int N, K, a, b, c, d;
        if (!strcmp(what, "device")) {
            if (scanf("%d", &fake::device()) != 1) return 1;
            continue;
        }
        if (scanf("%lld %d %d", &M, &N, &K) != 3) return 1;
        const int64_t pitch = ((int64_t)K + 15) / 16 * 16, t_pitch = ((int64_t)N + 15) / 16 * 16;
        if (!strcmp(what, "linear")) {
            rc = fxpq_linear_tokens(p, FXPQ_FT_BF16, K, (int8_t*)p, pitch, f, nullptr, M, N, K, FXPQ_FT_BF16, p, N, p, fxpq_linear_tokens_workspace(M, N, K), nullptr);
        } else if (!strcmp(what, "layer")) {
            if (scanf("%d %d %d %d", &a, &b, &c, &d) != 4) return 1;
            const fxpq_layer l = {p, K, b ? f : nullptr, (int8_t*)p, pitch, f, nullptr, nullptr, 0, p, N, d ? p : nullptr, d ? f : nullptr, M, N, K, a, FXPQ_FT_BF16,
                                  FXPQ_ACT_SILU, c, FXPQ_FT_F32, 0.0f};
            rc = fxpq_layer_forward(&l, p, fxpq_layer_workspace(&l), nullptr);
        } else if (!strcmp(what, "grad")) {
            if (scanf("%d %d", &a, &b) != 2) return 1;
            const fxpq_layer_grad g = {p, N, p, f, f, nullptr, (int8_t*)p, t_pitch, p, K, M, N, K, FXPQ_FT_BF16, a, b, 0, FXPQ_FT_F32, 0};
            rc = fxpq_layer_gradient(&g, p, fxpq_layer_gradient_workspace(&g), nullptr);
        } else {
            return 1;
        }
        printf(" = %d\n", rc);
    }
    return 0;
}
#else
#define cudaGetDevice fake::get_device
#define cudaGetLastError fake::last_error
#define cudaFuncSetAttribute fake::set_attribute
#define cudaFuncGetAttributes fake::get_attributes
#define cudaOccupancyMaxActiveClusters fake::most_clusters
#define cudaLaunchKernelEx fake::launch
#if PIECE == 1
#include "fxpq_linear.cu"
#else
#include "fxpq_layer.cu"
#endif
#endif
