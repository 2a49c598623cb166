// Linear layers as products of 8-bit integers for MI355X (gfx950): y = residual + gate * act(x_scale w_scale (x w^T) + bias).
// C ABI: include/rapid_packed.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "rapid_packed.h"
#include "rapid_tiles.h"

namespace {

struct Linear8Params {
    const signed char* x;
    const signed char* w;
    const float* x_scale;
    const float* w_scale;
    const __bf16* bias;
    const __bf16* gate;
    const __bf16* residual;
    const int* document;
    __bf16* y;
    long long x_sb, y_sb, r_sb, g_s;
    int x_sn, y_sn, r_sn, w_sn;
    int documents;
    int M, n, N, K;          // M rows in samples of n (n = M where samples make no difference)
    int activation;
};

// The sample and row of row m.
__device__ __forceinline__ void sample_of(const Linear8Params& p, int m, int& b, int& r)
{
    if (p.n == p.M) { b = 0; r = m; return; }
    b = (int)((unsigned)m / (unsigned)p.n);
    r = m - b * p.n;
}

// A wavefront: 16 rows by 64 outputs, operands straight from memory.
__global__ __launch_bounds__(256) void linear8_simple_kernel(Linear8Params p)
{
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int m0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 16, j0 = blockIdx.y * 64;
    if (m0 >= p.M) return;
    const int m = min(m0 + i, p.M - 1);
    int b, r;
    sample_of(p, m, b, r);
    const signed char* x = p.x + b * p.x_sb + (long long)r * p.x_sn;
    const signed char* w[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) w[f] = p.w + (long long)min(j0 + 16 * f + i, p.N - 1) * p.w_sn;
    i32x4 acc[4] = {};
    for (int k = 16 * g; k < p.K + 16 * g; k += 64) {
        const i32x4 none = {0, 0, 0, 0};
        const i32x4 xv = k < p.K ? *(const i32x4*)(x + k) : none;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            const i32x4 wv = k < p.K ? *(const i32x4*)(w[f] + k) : none;
            acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc[f], 0, 0, 0);
        }
    }
    if (m0 + i >= p.M) return;
    int d = b;
    if (p.document) {
        d = p.document[m];
        if ((unsigned)d >= (unsigned)p.documents) return;
    }
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int j = j0 + 16 * f + 4 * g + q;
            if (j >= p.N) continue;
            float z = (float)acc[f][q] * p.x_scale[m] * p.w_scale[j];
            if (p.bias) z += (float)p.bias[j];
            z = activated(z, p.activation);
            if (p.gate) z *= (float)p.gate[d * p.g_s + j];
            if (p.residual) z += (float)p.residual[b * p.r_sb + (long long)r * p.r_sn + j];
            p.y[b * p.y_sb + (long long)r * p.y_sn + j] = (__bf16)z;
        }
}

constexpr int MOST_INPUTS = (1 << 17) - 16;            // 2^14 times as many fit 32 bits

}  // namespace

extern "C" {

size_t rapid_linear_int8_workspace_bytes(long long M, int N, int K)
{
    return 0;
}

int rapid_linear_int8(const rapid_rows* x, const float* x_scale, const void* w, long long w_stride, const float* w_scale, const void* bias,
                      const rapid_rows* y, int activation, const void* gate, long long gate_stride, const rapid_rows* residual,
                      const int* document, int documents, int B, int n, int N, int K, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !x_scale || !y || !w || !w_scale || !x->ptr || !y->ptr || (residual && !residual->ptr)) return RAPID_ERR_NULL;
    if (B <= 0 || n <= 0 || N <= 0 || K <= 0 || N > MAX_STRIDE || K > MAX_STRIDE || (document && documents < 1)) return RAPID_ERR_SHAPE;
    const long long M = (long long)B * n;
    if (M >= (1LL << 31) - 256) return RAPID_ERR_SHAPE;
    if (K % 16 != 0 || K > MOST_INPUTS || activation < RAPID_ACT_NONE || activation > RAPID_ACT_GELU_TANH) return RAPID_ERR_UNSUPPORTED;
    Linear8Params p = {};
    if (!rows_ok(*x, B, n, K, false, p.x_sb, p.x_sn) || !rows_ok(*y, B, n, N, true, p.y_sb, p.y_sn)) return RAPID_ERR_SHAPE;
    if (residual && !rows_ok(*residual, B, n, N, false, p.r_sb, p.r_sn)) return RAPID_ERR_SHAPE;
    if (w_stride < K || w_stride > MAX_STRIDE) return RAPID_ERR_SHAPE;
    p.g_s = gate && (document ? documents : B) > 1 ? gate_stride : 0;
    if (p.g_s < 0 || p.g_s > (1LL << 40)) return RAPID_ERR_SHAPE;
    if (!aligned(x->ptr, 16) || !aligned(w, 16) || p.x_sb % 16 != 0 || p.x_sn % 16 != 0 || w_stride % 16 != 0) return RAPID_ERR_ALIGN;
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(document, 4)) return RAPID_ERR_ALIGN;
    if (!aligned(y->ptr, 2) || !aligned(bias, 2) || !aligned(gate, 2) || (residual && !aligned(residual->ptr, 2))) return RAPID_ERR_ALIGN;
    // rows of one tile are addressed from its first sample by 32 bits
    if (B > 1 && (255 / n + 1) * p.x_sb + (long long)(n - 1) * p.x_sn + K > (1LL << 30)) return RAPID_ERR_SHAPE;
    for (const void* in : {(const void*)x->ptr, (const void*)x_scale, w, (const void*)w_scale, bias, gate, (const void*)document})
        if (in == y->ptr) return RAPID_ERR_ALIAS;
    if (residual && y->ptr == residual->ptr && (p.y_sb != p.r_sb || p.y_sn != p.r_sn)) return RAPID_ERR_ALIAS;
    const size_t need = workspace ? rapid_linear_int8_workspace_bytes(M, N, K) : 0;
    if (workspace && (workspace_bytes < need || !aligned(workspace, 16))) return RAPID_ERR_WORKSPACE;
    p.x = (const signed char*)x->ptr;
    p.w = (const signed char*)w;
    p.x_scale = x_scale;
    p.w_scale = w_scale;
    p.bias = (const __bf16*)bias;
    p.gate = (const __bf16*)gate;
    p.residual = residual ? (const __bf16*)residual->ptr : nullptr;
    p.document = document;
    p.documents = documents;
    p.y = (__bf16*)y->ptr;
    p.w_sn = (int)w_stride;
    p.M = (int)M;
    p.n = B == 1 ? (int)M : n;
    p.N = N;
    p.K = K;
    p.activation = activation;
    if ((N + 63) / 64 > 65535) return RAPID_ERR_SHAPE;
    hipLaunchKernelGGL(linear8_simple_kernel, dim3((unsigned)((M + 63) / 64), (unsigned)((N + 63) / 64)), dim3(256), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

}  // extern "C"
