// Attention of documents packed into one joint sequence, for MI355X (gfx950).  C ABI: include/rapid_packed.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rapid_internal.h"
#include "rapid_packed.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f;

struct Side {                                          // of a segment
    const char *q, *k, *v;
    char* o;
    long long in_sb, in_sh, out_sb, out_sh;            // bytes
    int in_sn, out_sn;                                 // bytes
};
struct PackedParams {
    Side side[2];
    const int* document;
    const int* order;                                  // or null
    long long document_sb, order_sb;
    int n0, N, B, H;                                   // tokens of the first segment, of both
    float scale;                                       // of a score: capped / log2(e), else as exponent of 2
    float cap;                                         // as exponent of 2; 0: none
};

__device__ __forceinline__ float most_of_lanes(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ float sum_of_lanes(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}

// The exponent of 2 that a product q k stands for.
__device__ __forceinline__ float exponent(float s, float scale, float cap)
{
    if (cap == 0.f) return s * scale;
    // cap tanh(u) = cap - 2 cap / (1 + exp(2 u)), scale = 2 log2(e) scale' / cap'
    return cap - 2.f * cap / (1.f + __builtin_amdgcn_exp2f(s * scale));
}

// One row of the output by one wavefront, key by key: a lane a key for the scores, D / 64 elements of the output a lane.
template <int D>
__device__ void row_by_keys(const PackedParams& p, int b, int h, int t, int lane)
{
    const int* document = p.document + b * p.document_sb;
    const int* order = p.order ? p.order + b * p.order_sb : nullptr;
    const Side& at = p.side[t >= p.n0];
    const int row = t >= p.n0 ? t - p.n0 : t;
    const char* q = at.q + b * at.in_sb + h * at.in_sh + (long long)row * at.in_sn;
    const int own = document[t], turn = order ? order[t] : 0;
    constexpr int EACH = D / 64;
    float acc[EACH] = {}, m = -INFINITY, l = 0.f;
    for (int first = 0; own >= 0 && first < p.N; first += 64) {
        const int j = min(first + lane, p.N - 1);
        const bool seen = first + lane < p.N && document[j] == own && (!order || order[j] <= turn);
        unsigned long long keys = __builtin_amdgcn_ballot_w64(seen);
        if (keys == 0ull) continue;
        const Side& from = p.side[j >= p.n0];
        const char* k = from.k + b * from.in_sb + h * from.in_sh + (long long)(j >= p.n0 ? j - p.n0 : j) * from.in_sn;
        float s = 0.f;
        for (int c = 0; c < D / 8; ++c) {
            const bf16x8 kv = *(const bf16x8*)(k + 16 * c), qv = *(const bf16x8*)(q + 16 * c);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)kv[i], (float)qv[i], s);
        }
        s = exponent(s, p.scale, p.cap);
        const float higher = fmaxf(m, most_of_lanes(seen ? s : -INFINITY));
        const float lower = m == higher ? 1.f : __builtin_amdgcn_exp2f(m - higher);
        m = higher;
        const float e = seen ? __builtin_amdgcn_exp2f(s - m) : 0.f;
        l = l * lower + sum_of_lanes(e);
#pragma unroll
        for (int i = 0; i < EACH; ++i) acc[i] *= lower;
        while (keys != 0ull) {
            const int i = __builtin_ctzll(keys), key = first + i;
            keys &= keys - 1ull;
            const Side& from = p.side[key >= p.n0];
            const char* v = from.v + b * from.in_sb + h * from.in_sh + (long long)(key >= p.n0 ? key - p.n0 : key) * from.in_sn;
            const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(e), i));
            const __bf16* of = (const __bf16*)v + EACH * lane;
#pragma unroll
            for (int c = 0; c < EACH; ++c) acc[c] = __builtin_fmaf(by, (float)of[c], acc[c]);
        }
    }
    __bf16* o = (__bf16*)(at.o + b * at.out_sb + h * at.out_sh + (long long)row * at.out_sn) + EACH * lane;
#pragma unroll
    for (int c = 0; c < EACH; ++c) o[c] = (__bf16)(own >= 0 ? acc[c] / l : 0.f);
}

template <int D>
__global__ __launch_bounds__(256) void attn_packed_simple_kernel(PackedParams p)
{
    const long long rows = (long long)p.B * p.H * p.N;
    for (long long row = blockIdx.x * 4LL + (threadIdx.x >> 6); row < rows; row += gridDim.x * 4LL) {
        const int head = (int)(row / p.N);
        row_by_keys<D>(p, head / p.H, head % p.H, (int)(row - (long long)head * p.N), threadIdx.x & 63);
    }
}

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

extern "C" {

size_t rapid_attn_packed_workspace_bytes(int B, int H, int N, int D)
{
    if (B <= 0 || H <= 0 || N <= 0 || N > (1 << 22) || (long long)B * H > 524287 || (D != 64 && D != 128)) return 0;
    return 16;
}

int rapid_attn_packed(const rapid_attn_segment* segments, int n_segments, int B, int H, int D, const int* document,
                      long long document_stride_b, const int* order, long long order_stride_b, float cap, float scale, void* workspace,
                      size_t workspace_bytes, void* stream)
{
    if (!segments || n_segments < 1 || !document || !workspace) return RAPID_ERR_NULL;
    if (n_segments > 2 || B <= 0 || H <= 0 || (long long)B * H > 524287) return RAPID_ERR_SHAPE;
    if (D != 64 && D != 128) return RAPID_ERR_UNSUPPORTED;
    if (!(cap >= 0.f) || isinf(cap) || isnan(scale) || isinf(scale)) return RAPID_ERR_UNSUPPORTED;
    PackedParams p = {};
    long long N = 0;
    for (int i = 0; i < n_segments; ++i) {
        const rapid_attn_segment& g = segments[i];
        if (!g.q || !g.k || !g.v || !g.o) return RAPID_ERR_NULL;
        if (g.n <= 0 || g.n > (1 << 22)) return RAPID_ERR_SHAPE;
        N += g.n;
        long long in[3] = {B == 1 ? 0 : g.in_stride_b, H == 1 ? 0 : g.in_stride_h, g.n == 1 ? D : g.in_stride_n};
        long long out[3] = {B == 1 ? 0 : g.out_stride_b, H == 1 ? 0 : g.out_stride_h, g.n == 1 ? D : g.out_stride_n};
        for (long long* s : {in, out}) {
            if (s[0] < 0 || s[0] > (1LL << 40) || s[1] < 0 || s[1] > (1LL << 40) || s[2] < D || s[2] > (1 << 23)) return RAPID_ERR_SHAPE;
            if ((s[0] | s[1] | s[2]) % 8 != 0) return RAPID_ERR_ALIGN;
        }
        if (!aligned(g.q, 16) || !aligned(g.k, 16) || !aligned(g.v, 16) || !aligned(g.o, 16)) return RAPID_ERR_ALIGN;
        p.side[i] = {(const char*)g.q, (const char*)g.k, (const char*)g.v, (char*)g.o, 2 * in[0], 2 * in[1], 2 * out[0], 2 * out[1], (int)(2 * in[2]), (int)(2 * out[2])};
    }
    if (N > (1 << 22) || (long long)B * H * ((N + 63) / 64) >= (1LL << 30)) return RAPID_ERR_SHAPE;
    for (int i = 0; i < n_segments; ++i)
        for (int j = 0; j < n_segments; ++j) {
            const char* o = p.side[i].o;
            if (o == p.side[j].q || o == p.side[j].k || o == p.side[j].v || (i != j && o == p.side[j].o)) return RAPID_ERR_ALIAS;
        }
    p.document_sb = B == 1 ? 0 : document_stride_b;
    p.order_sb = B == 1 || !order ? 0 : order_stride_b;
    if (p.document_sb < 0 || p.document_sb > (1LL << 40) || p.order_sb < 0 || p.order_sb > (1LL << 40)) return RAPID_ERR_SHAPE;
    if (!aligned(document, 4) || !aligned(order, 4) || !aligned(workspace, 16)) return RAPID_ERR_ALIGN;
    if (workspace_bytes < rapid_attn_packed_workspace_bytes(B, H, (int)N, D)) return RAPID_ERR_WORKSPACE;
    p.document = document;
    p.order = order;
    p.n0 = segments[0].n;
    p.N = (int)N;
    p.B = B;
    p.H = H;
    if (!(scale > 0.f)) scale = 1.0f / sqrtf((float)D);
    p.cap = cap * LOG2E;
    p.scale = cap > 0.f ? 2.f * LOG2E * scale / cap : scale * LOG2E;
    const long long groups = ((long long)B * H * N + 3) / 4;
    const dim3 grid((unsigned)(groups < (1 << 20) ? groups : 1 << 20));
    if (D == 64) hipLaunchKernelGGL(attn_packed_simple_kernel<64>, grid, dim3(256), 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL(attn_packed_simple_kernel<128>, grid, dim3(256), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

}  // extern "C"
