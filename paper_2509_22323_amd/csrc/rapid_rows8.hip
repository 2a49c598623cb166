// Rows as 8-bit integers with a scale for each, for MI355X (gfx950): of a bf16 tensor, and of the norm under the conditioning's scale and
// shift.  C ABI: include/rapid_packed.h.
//
// Both are bound by memory: two bytes read and one written an element.  A row stays in the registers of the lanes that read it, 16 bytes an
// access, until its largest magnitude is known.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rapid_packed.h"
#include "rapid_tiles.h"

namespace {

struct RowsParams {
    const __bf16* x;
    signed char* q;
    float* q_scale;
    const __bf16* scale;
    const __bf16* shift;
    const int* document;
    long long x_sb, q_sb, scale_s, shift_s;
    int x_sn, q_sn;
    int documents, M, n, C;
    float eps;
};

__device__ __forceinline__ float low(unsigned pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(unsigned pair) { return __uint_as_float(pair & 0xffff0000u); }

template <class T>
__device__ __forceinline__ T other(T v, int lane_xor)
{
    return __shfl_xor(v, lane_xor, 64);
}
// The largest value of the wavefront, in every lane.
template <class T>
__device__ __forceinline__ T most_of_lanes(T v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const T w = other(v, d);
        v = w > v ? w : v;
    }
    return v;
}
__device__ __forceinline__ double sum_of_lanes(double v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += other(v, d);
    return v;
}

// v in every wavefront of a row -> f over them, in all of them
template <int WAVES, class T, class F>
__device__ __forceinline__ T over_waves(T v, T* part, int wave, int own, F f)
{
    if constexpr (WAVES > 1) {
        if (threadIdx.x % 64 == 0) part[wave] = v;
        __syncthreads();
        v = part[own * WAVES];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = f(v, part[own * WAVES + w]);
    }
    return v;
}

// Four whole numbers, the low bytes of a, b, c, d
__device__ __forceinline__ unsigned bytes(unsigned a, unsigned b, unsigned c, unsigned d)
{
    const unsigned ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return ab | cd;
}

// The quotient 127 v / m of a row whose largest magnitude is m, rounded once.  With m = a 2^e, a in [1, 2): t = 127 v 2^-e is exact (15 bits; what
// is lost of tiny elements is far below the smallest quotient that does not round to 0), and so is the remainder t - q a of a quotient
// q = t (1/a) that is off by a step or two; one correction by it gives the quotient rounded to 24 bits, which is a tie between two
// integers only where the exact one is: v and a have 8 bits each, so any other quotient is 2^-17 or more away from one.
struct Divided {
    float a, inverse;
    int e;
};
__device__ __forceinline__ Divided divided_by(float m)
{
    Divided d;
    d.e = __builtin_amdgcn_frexp_expf(m);              // m = a 2^e, a in [0.5, 1)
    d.a = __builtin_amdgcn_frexp_mantf(m);
    d.inverse = 1.0f / d.a;
    return d;
}
// (the integer in the low byte: 1.5 * 2^23 leaves no bits behind the point)
__device__ __forceinline__ unsigned whole(float v, const Divided& d)
{
    const float t = 127.0f * __builtin_ldexpf(v, -d.e);
    const float q = t * d.inverse;
    return __float_as_uint(__builtin_fmaf(__builtin_fmaf(-q, d.a, t), d.inverse, q) + 12582912.0f);
}

// WAVES wavefronts a row, CHUNKS accesses a lane.
template <int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void quantize_rows_kernel(RowsParams p)
{
    constexpr int BLOCK = WAVES < 4 ? 256 : WAVES * 64, ROWS = BLOCK / 64 / WAVES, LANES = WAVES * 64;
    __shared__ unsigned part[BLOCK / 64];
    const int lane = threadIdx.x % LANES, wave = threadIdx.x / 64, own = threadIdx.x / LANES;
    const int row = blockIdx.x * ROWS + own;
    const bool there = row < p.M;
    const int m = there ? row : p.M - 1;
    const int b = p.n == p.M ? 0 : (int)((unsigned)m / (unsigned)p.n), r = m - b * p.n;
    const __bf16* x = p.x + b * p.x_sb + (long long)r * p.x_sn;
    u32x4 raw[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        const u32x4 none = {0u, 0u, 0u, 0u};
        raw[c] = at < p.C ? *(const u32x4*)(x + at) : none;
    }
    // magnitudes as bits: infinities and NaN are the largest
    unsigned most = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, max(raw[c][i] & 0x7fff0000u, raw[c][i] << 17 >> 1));
    most = most_of_lanes(most);
    most = over_waves<WAVES>(most, part, wave, own, [](unsigned a, unsigned b) { return max(a, b); });
    if (!there) return;
    const bool plain = most < 0x7f800000u && most != 0u;
    const Divided d = divided_by(plain ? __uint_as_float(most) : 1.0f);
    signed char* q = p.q + b * p.q_sb + (long long)r * p.q_sn;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        if (at >= p.C) continue;
        unsigned w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[2 * i] = whole(low(raw[c][i]), d);
            w[2 * i + 1] = whole(high(raw[c][i]), d);
        }
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        u32x2 out = {bytes(w[0], w[1], w[2], w[3]), bytes(w[4], w[5], w[6], w[7])};
        if (!plain) out = u32x2{0u, 0u};
        *(u32x2*)(q + at) = out;
    }
    if (lane == 0) p.q_scale[m] = most > 0x7f7fffffu ? __uint_as_float(0x7fc00000u) : __uint_as_float(most) / 127.0f;
}

// Rows longer than a workgroup's registers hold: a workgroup a row, read twice.
__global__ __launch_bounds__(512) void quantize_long_rows_kernel(RowsParams p)
{
    __shared__ unsigned part[8];
    const int m = blockIdx.x, b = p.n == p.M ? 0 : (int)((unsigned)m / (unsigned)p.n), r = m - b * p.n;
    const __bf16* x = p.x + b * p.x_sb + (long long)r * p.x_sn;
    unsigned most = 0;
    for (int at = 8 * threadIdx.x; at < p.C; at += 4096) {
        const u32x4 raw = *(const u32x4*)(x + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, max(raw[i] & 0x7fff0000u, raw[i] << 17 >> 1));
    }
    most = most_of_lanes(most);
    most = over_waves<8>(most, part, threadIdx.x / 64, 0, [](unsigned a, unsigned b) { return max(a, b); });
    const bool plain = most < 0x7f800000u && most != 0u;
    const Divided d = divided_by(plain ? __uint_as_float(most) : 1.0f);
    signed char* q = p.q + b * p.q_sb + (long long)r * p.q_sn;
    for (int at = 8 * threadIdx.x; at < p.C; at += 4096) {
        const u32x4 raw = *(const u32x4*)(x + at);
        unsigned w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[2 * i] = whole(low(raw[i]), d);
            w[2 * i + 1] = whole(high(raw[i]), d);
        }
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        u32x2 out = {bytes(w[0], w[1], w[2], w[3]), bytes(w[4], w[5], w[6], w[7])};
        if (!plain) out = u32x2{0u, 0u};
        *(u32x2*)(q + at) = out;
    }
    if (threadIdx.x == 0) p.q_scale[m] = most > 0x7f7fffffu ? __uint_as_float(0x7fc00000u) : __uint_as_float(most) / 127.0f;
}

// The norm, in fp64: what it ends in are whole numbers, and a result in 32 bits would be on another side of a border between two of them than
// the formula's about once in 10^5 elements, at another place for every order of the sums.  (The card adds and multiplies as fast
// in 64 bits as in 32.)
template <int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void norm_rows8_kernel(RowsParams p)
{
    constexpr int BLOCK = WAVES < 4 ? 256 : WAVES * 64, ROWS = BLOCK / 64 / WAVES, LANES = WAVES * 64;
    __shared__ double part[3][BLOCK / 64];
    const int lane = threadIdx.x % LANES, wave = threadIdx.x / 64, own = threadIdx.x / LANES;
    const int row = blockIdx.x * ROWS + own;
    const bool there = row < p.M;
    const int m = there ? row : p.M - 1;
    const int b = p.n == p.M ? 0 : (int)((unsigned)m / (unsigned)p.n), r = m - b * p.n;
    const __bf16* x = p.x + b * p.x_sb + (long long)r * p.x_sn;
    u32x4 raw[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        const u32x4 none = {0u, 0u, 0u, 0u};
        raw[c] = at < p.C ? *(const u32x4*)(x + at) : none;
    }
    const int d = p.document ? p.document[m] : b;
    const bool written = there && (!p.document || (unsigned)d < (unsigned)p.documents);
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum += (double)low(raw[c][i]);
            sum += (double)high(raw[c][i]);
        }
    auto add = [](double a, double b) { return a + b; };
    const double mean = over_waves<WAVES>(sum_of_lanes(sum), part[0], wave, own, add) / (double)p.C;
    double y[CHUNKS][8], square = 0.0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const bool in = 8 * (c * LANES + lane) < p.C;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[c][i] = in ? (double)(i % 2 ? high(raw[c][i / 2]) : low(raw[c][i / 2])) - mean : 0.0;
            square = __builtin_fma(y[c][i], y[c][i], square);
        }
    }
    const double inv = 1.0 / sqrt(over_waves<WAVES>(sum_of_lanes(square), part[1], wave, own, add) / (double)p.C + (double)p.eps);
    double most = 0.0, number = 0.0;                   // number: NaN where an element is none
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        if (at >= p.C) continue;
        if (p.scale && written) {
            const u32x4 scale = *(const u32x4*)(p.scale + d * p.scale_s + at), shift = *(const u32x4*)(p.shift + d * p.shift_s + at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double by = 1.0 + (double)(i % 2 ? high(scale[i / 2]) : low(scale[i / 2]));
                y[c][i] = __builtin_fma(y[c][i] * inv, by, (double)(i % 2 ? high(shift[i / 2]) : low(shift[i / 2])));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[c][i] *= inv;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            most = fmax(most, fabs(y[c][i]));
            number = __builtin_fma(y[c][i], 0.0, number);
        }
    }
    most = fmax(most, number != 0.0 ? INFINITY : 0.0);
    most = most_of_lanes(most);
    most = over_waves<WAVES>(most, part[2], wave, own, [](double a, double b) { return a > b ? a : b; });
    if (!written) return;
    const bool plain = most < INFINITY && most > 0.0;
    const double by = 127.0 / (plain ? most : 1.0);
    signed char* q = p.q + b * p.q_sb + (long long)r * p.q_sn;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        if (at >= p.C) continue;
        unsigned w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = (unsigned)__double2loint(__builtin_fma(y[c][i], by, 6755399441055744.0));   // 1.5 * 2^52
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        u32x2 out = {bytes(w[0], w[1], w[2], w[3]), bytes(w[4], w[5], w[6], w[7])};
        if (!plain) out = u32x2{0u, 0u};
        *(u32x2*)(q + at) = out;
    }
    if (lane == 0) p.q_scale[m] = plain || most == 0.0 ? (float)(most / 127.0) : __uint_as_float(0x7fc00000u);
}

int launched() { return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE; }

template <int WAVES, int CHUNKS>
int launch_quantize(const RowsParams& p, void* stream)
{
    constexpr int BLOCK = WAVES < 4 ? 256 : WAVES * 64, ROWS = BLOCK / 64 / WAVES;
    hipLaunchKernelGGL((quantize_rows_kernel<WAVES, CHUNKS>), dim3((unsigned)((p.M + ROWS - 1) / ROWS)), dim3(BLOCK), 0, (hipStream_t)stream, p);
    return launched();
}
template <int WAVES, int CHUNKS>
int launch_norm(const RowsParams& p, void* stream)
{
    constexpr int BLOCK = WAVES < 4 ? 256 : WAVES * 64, ROWS = BLOCK / 64 / WAVES;
    hipLaunchKernelGGL((norm_rows8_kernel<WAVES, CHUNKS>), dim3((unsigned)((p.M + ROWS - 1) / ROWS)), dim3(BLOCK), 0, (hipStream_t)stream, p);
    return launched();
}

constexpr long long MOST_ROWS = 1LL << 22;             // (a grid has fewer than 2^32 lanes)

// What both entries check of rows, and the parameters from them.
int rows_of(const rapid_rows* x, const rapid_rows* q, float* scale, int B, int n, int C, int most, RowsParams& p)
{
    if (!x || !q || !scale || !x->ptr || !q->ptr) return RAPID_ERR_NULL;
    if (B <= 0 || n <= 0 || C <= 0) return RAPID_ERR_SHAPE;
    const long long M = (long long)B * n;
    if (M > MOST_ROWS) return RAPID_ERR_SHAPE;
    if (C % 8 != 0 || C > most) return RAPID_ERR_UNSUPPORTED;
    if (!rows_ok(*x, B, n, C, false, p.x_sb, p.x_sn) || !rows_ok(*q, B, n, C, true, p.q_sb, p.q_sn)) return RAPID_ERR_SHAPE;
    if (!aligned(x->ptr, 16) || !aligned(q->ptr, 8) || !aligned(scale, 4) || (p.x_sb | p.x_sn | p.q_sb | p.q_sn) % 8 != 0) return RAPID_ERR_ALIGN;
    if (q->ptr == x->ptr || (void*)scale == x->ptr || (void*)scale == q->ptr) return RAPID_ERR_ALIAS;
    p.x = (const __bf16*)x->ptr;
    p.q = (signed char*)q->ptr;
    p.q_scale = scale;
    p.M = (int)M;
    p.n = B == 1 ? (int)M : n;
    p.C = C;
    return RAPID_OK;
}

}  // namespace

extern "C" {

int rapid_quantize_rows(const rapid_rows* x, const rapid_rows* q, float* scale, int B, int n, int K, void* stream)
{
    RowsParams p = {};
    const int rc = rows_of(x, q, scale, B, n, K, 1 << 17, p);
    if (rc != RAPID_OK) return rc;
    if (K <= 512) return launch_quantize<1, 1>(p, stream);
    if (K <= 1024) return launch_quantize<1, 2>(p, stream);
    if (K <= 2048) return launch_quantize<1, 4>(p, stream);
    if (K <= 4096) return launch_quantize<2, 4>(p, stream);
    if (K <= 8192) return launch_quantize<4, 4>(p, stream);
    if (K <= 16384) return launch_quantize<8, 4>(p, stream);
    hipLaunchKernelGGL(quantize_long_rows_kernel, dim3((unsigned)p.M), dim3(512), 0, (hipStream_t)stream, p);
    return launched();
}

int rapid_norm_modulate_int8(const rapid_rows* x, const rapid_rows* q, float* q_scale, const void* scale, long long scale_stride,
                             const void* shift, long long shift_stride, const int* document, int documents, int B, int n, int C,
                             float eps, void* stream)
{
    RowsParams p = {};
    if (!scale != !shift) return RAPID_ERR_NULL;
    if (!(eps >= 0.f) || (document && documents < 1)) return RAPID_ERR_SHAPE;
    const int rc = rows_of(x, q, q_scale, B, n, C, 16384, p);
    if (rc != RAPID_OK) return rc;
    const int vectors = document ? documents : B;
    p.scale_s = scale && vectors > 1 ? scale_stride : 0;
    p.shift_s = shift && vectors > 1 ? shift_stride : 0;
    if (p.scale_s < 0 || p.shift_s < 0 || p.scale_s > (1LL << 40) || p.shift_s > (1LL << 40)) return RAPID_ERR_SHAPE;
    if (!aligned(scale, 16) || !aligned(shift, 16) || (p.scale_s | p.shift_s) % 8 != 0 || !aligned(document, 4)) return RAPID_ERR_ALIGN;
    for (const void* in : {scale, shift, (const void*)document})
        if (in && (in == q->ptr || in == (const void*)q_scale)) return RAPID_ERR_ALIAS;
    p.scale = (const __bf16*)scale;
    p.shift = (const __bf16*)shift;
    p.document = document;
    p.documents = documents;
    p.eps = eps;
    if (C <= 512) return launch_norm<1, 1>(p, stream);
    if (C <= 1024) return launch_norm<1, 2>(p, stream);
    if (C <= 2048) return launch_norm<1, 4>(p, stream);
    if (C <= 4096) return launch_norm<2, 4>(p, stream);
    if (C <= 8192) return launch_norm<4, 4>(p, stream);
    return launch_norm<8, 4>(p, stream);
}

}  // extern "C"
