// Linear layers of an MM-DiT layer for MI355X (gfx950): y = residual + gate * act(x w^T + bias).
// C ABI: include/rapid_layer.h.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rapid_layer.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f;

struct LinearParams {
    const __bf16* x;
    const __bf16* w;
    const __bf16* bias;
    const __bf16* gate;
    const __bf16* residual;
    __bf16* y;
    long long x_sb, x_sn, y_sb, y_sn, r_sb, r_sn, w_sn, g_sb;
    int M, n, N, K;          // M rows in samples of n (n = M where samples make no difference)
    int activation;
    bool wide;               // N and everything the epilogue touches can be taken four elements at a time
};

// The sample and row of row m.
__device__ __forceinline__ void sample_of(const LinearParams& p, int m, int& b, int& r)
{
    if (p.n == p.M) { b = 0; r = m; return; }
    b = (int)((unsigned)m / (unsigned)p.n);
    r = m - b * p.n;
}

__device__ __forceinline__ float activated(float z, int activation)
{
    if (activation == RAPID_ACT_NONE) return z;
    // z / (1 + exp(-t)): t = z, or, with 1 + tanh(u) = 2 / (1 + exp(-2u)), t = 2u.  exp overflows to inf and the quotient to -0.
    const float t = activation == RAPID_ACT_SILU ? z : 1.5957691216057308f * z * __builtin_fmaf(0.044715f * z, z, 1.0f);
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * t));
}

// Outputs j0 .. j0 + 3 of row m from their sums: everything in fp32, rounded once.
__device__ __forceinline__ void finish(const LinearParams& p, int m, int j0, f32x4 sum)
{
    int b, r;
    sample_of(p, m, b, r);
    __bf16* y = p.y + b * p.y_sb + r * p.y_sn + j0;
    const __bf16* gate = p.gate ? p.gate + b * p.g_sb + j0 : nullptr;
    const __bf16* res = p.residual ? p.residual + b * p.r_sb + r * p.r_sn + j0 : nullptr;
    if (p.wide) {
        bf16x4 out;
        if (p.bias) {
            const bf16x4 c = *(const bf16x4*)(p.bias + j0);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += (float)c[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = activated(sum[i], p.activation);
        if (gate) {
            const bf16x4 c = *(const bf16x4*)gate;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] *= (float)c[i];
        }
        if (res) {
            const bf16x4 c = *(const bf16x4*)res;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += (float)c[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (__bf16)sum[i];
        *(bf16x4*)y = out;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (j0 + i >= p.N) break;
        float z = sum[i] + (p.bias ? (float)p.bias[j0 + i] : 0.f);
        z = activated(z, p.activation);
        if (gate) z *= (float)gate[i];
        if (res) z += (float)res[i];
        y[i] = (__bf16)z;
    }
}

constexpr int TILE = 64, STEP = 32, PITCH = STEP + 8;

// 64 x 64 outputs per workgroup, 32 x 32 per wavefront, the operands staged through registers into LDS.  The product is computed
// transposed (A = rows of w, B = rows of x), so that a lane holds four consecutive outputs of one row.
__global__ __launch_bounds__(256) void linear_kernel(LinearParams p)
{
    __shared__ __align__(16) __bf16 xs[TILE * PITCH], ws[TILE * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int m0 = blockIdx.x * TILE, j0 = blockIdx.y * TILE;
    const int row = tid >> 2, chunk = tid & 3;
    int b, r;
    sample_of(p, min(m0 + row, p.M - 1), b, r);
    const __bf16* xr = p.x + b * p.x_sb + r * p.x_sn;
    const __bf16* wr = p.w + (long long)min(j0 + row, p.N - 1) * p.w_sn;
    f32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < p.K; k0 += STEP) {
        const int k = k0 + 8 * chunk;
        const u32x4 none = {0u, 0u, 0u, 0u};
        const u32x4 xv = k < p.K ? *(const u32x4*)(xr + k) : none;
        const u32x4 wv = k < p.K ? *(const u32x4*)(wr + k) : none;
        __syncthreads();
        *(u32x4*)(xs + row * PITCH + 8 * chunk) = xv;
        *(u32x4*)(ws + row * PITCH + 8 * chunk) = wv;
        __syncthreads();
        bf16x8 a[2], c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = *(const bf16x8*)(ws + ((wave & 1) * 32 + i * 16 + (lane & 15)) * PITCH + 8 * (lane >> 4));
            c[i] = *(const bf16x8*)(xs + ((wave >> 1) * 32 + i * 16 + (lane & 15)) * PITCH + 8 * (lane >> 4));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], c[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int m = m0 + (wave >> 1) * 32 + j * 16 + (lane & 15), n = j0 + (wave & 1) * 32 + i * 16 + 4 * (lane >> 4);
            if (m < p.M && n < p.N) finish(p, m, n, acc[i][j]);
        }
}

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr long long MAX_STRIDE = 1LL << 22;            // elements, of a row

// Strides of dimensions of size 1 replaced by what changes no address; false: out of range.
bool rows_ok(const rapid_rows& a, int B, int n, int width, bool written, long long& sb, long long& sn)
{
    sn = n == 1 ? width : a.stride_n;
    sb = B == 1 ? 0 : a.stride_b;
    if (sn < 0 || sn > MAX_STRIDE || sb < 0 || sb > (1LL << 40)) return false;
    if (!written) return true;
    // apart: rows behind each other and samples behind each other, or samples within the rows' distance
    const long long rows = (n - 1) * sn + width, samples = (B - 1) * sb + width;
    if (n > 1 && B > 1) return (sn >= width && sb >= rows) || (sb >= width && sn >= samples);
    return n > 1 ? sn >= width : B == 1 || sb >= width;
}

inline bool by_four(const void* p, long long sb, long long sn) { return p == nullptr || (aligned(p, 8) && sb % 4 == 0 && sn % 4 == 0); }

}  // namespace

extern "C" {

size_t rapid_linear_workspace_bytes(long long M, int N, int K)
{
    (void)M; (void)N; (void)K;
    return 0;
}

int rapid_linear(const rapid_rows* x, const void* w, long long w_stride, const void* bias, const rapid_rows* y, int activation,
                 const void* gate, long long gate_stride, const rapid_rows* residual, int B, int n, int N, int K, void* workspace,
                 size_t workspace_bytes, void* stream)
{
    if (!x || !y || !w || !x->ptr || !y->ptr || (residual && !residual->ptr)) return RAPID_ERR_NULL;
    if (B <= 0 || n <= 0 || N <= 0 || K <= 0 || N > MAX_STRIDE || K > MAX_STRIDE) return RAPID_ERR_SHAPE;
    const long long M = (long long)B * n;
    if (M >= (1LL << 31) - 256) return RAPID_ERR_SHAPE;
    if (K % 8 != 0 || activation < RAPID_ACT_NONE || activation > RAPID_ACT_GELU_TANH) return RAPID_ERR_UNSUPPORTED;
    LinearParams p = {};
    if (!rows_ok(*x, B, n, K, false, p.x_sb, p.x_sn) || !rows_ok(*y, B, n, N, true, p.y_sb, p.y_sn)) return RAPID_ERR_SHAPE;
    if (residual && !rows_ok(*residual, B, n, N, false, p.r_sb, p.r_sn)) return RAPID_ERR_SHAPE;
    if (w_stride < K || w_stride > MAX_STRIDE) return RAPID_ERR_SHAPE;
    const long long gs = gate && B > 1 ? gate_stride : 0;
    if (gs < 0 || gs > (1LL << 40)) return RAPID_ERR_SHAPE;
    if (!aligned(x->ptr, 16) || !aligned(w, 16) || p.x_sb % 8 != 0 || p.x_sn % 8 != 0 || w_stride % 8 != 0) return RAPID_ERR_ALIGN;
    if (!aligned(y->ptr, 2) || !aligned(bias, 2) || !aligned(gate, 2) || (residual && !aligned(residual->ptr, 2))) return RAPID_ERR_ALIGN;
    // rows of one tile are addressed from its first sample by 32 bits
    if (B > 1 && (255 / n + 1) * p.x_sb + (n - 1) * p.x_sn + K > (1LL << 30)) return RAPID_ERR_SHAPE;
    if (y->ptr == x->ptr || y->ptr == w) return RAPID_ERR_ALIAS;
    const size_t need = rapid_linear_workspace_bytes(M, N, K);
    if (workspace && (workspace_bytes < need || !aligned(workspace, 16))) return RAPID_ERR_WORKSPACE;
    p.x = (const __bf16*)x->ptr;
    p.w = (const __bf16*)w;
    p.bias = (const __bf16*)bias;
    p.gate = (const __bf16*)gate;
    p.residual = residual ? (const __bf16*)residual->ptr : nullptr;
    p.y = (__bf16*)y->ptr;
    p.w_sn = w_stride;
    p.g_sb = gs;
    p.M = (int)M;
    p.n = n;
    p.N = N;
    p.K = K;
    p.activation = activation;
    p.wide = N % 4 == 0 && by_four(p.bias, 0, 0) && by_four(p.gate, p.g_sb, 0) && by_four(p.residual, p.r_sb, p.r_sn) &&
             by_four(p.y, p.y_sb, p.y_sn);
    if (B == 1) p.n = p.M;
    const long long mt = (M + TILE - 1) / TILE, nt = (N + TILE - 1) / TILE;
    if (nt > 65535) return RAPID_ERR_SHAPE;
    hipLaunchKernelGGL(linear_kernel, dim3((unsigned)mt, (unsigned)nt), dim3(256), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

}  // extern "C"
