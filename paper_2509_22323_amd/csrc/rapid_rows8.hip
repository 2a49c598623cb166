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
    double share;            // 1 / C
};

__device__ __forceinline__ float low(unsigned pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(unsigned pair) { return __uint_as_float(pair & 0xffff0000u); }

template <int CTRL>
__device__ __forceinline__ unsigned moved(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ double moved(double v)
{
    return __hiloint2double((int)moved<CTRL>((unsigned)__double2hiint(v)), (int)moved<CTRL>((unsigned)__double2loint(v)));
}
// f over the values of the wavefront, in every lane.
template <class T, class F>
__device__ __forceinline__ T over_lanes(T v, F f)
{
    v = f(v, moved<0xB1>(v));                          // lane ^ 1
    v = f(v, moved<0x4E>(v));                          // lane ^ 2
    v = f(v, moved<0x141>(v));                         // 7 - lane of every 8
    v = f(v, moved<0x140>(v));                         // 15 - lane of every 16
    auto swapped = [&](auto swap) {
        if constexpr (sizeof(T) == 8) {
            const auto l = swap((unsigned)__double2loint(v)), h = swap((unsigned)__double2hiint(v));
            return f(__hiloint2double((int)h[0], (int)l[0]), __hiloint2double((int)h[1], (int)l[1]));
        } else {
            const auto w = swap(v);
            return f((T)w[0], (T)w[1]);
        }
    };
    v = swapped([](unsigned w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false); });
    return swapped([](unsigned w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false); });
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

// The quotient 127 v / m of a row whose largest magnitude is m, rounded once.  With m = a 2^e, a in [0.5, 1): t = 127 v 2^-e is exact (15 bits; what
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

// WAVES wavefronts a row, CHUNKS accesses a lane.  At the rate of a large copy: 2 x 4096 rows of 6144 28.3 us, 5.3 TB/s.
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
    auto larger = [](unsigned a, unsigned b) { return max(a, b); };
    most = over_waves<WAVES>(over_lanes(most, larger), part, wave, own, larger);
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
    auto larger = [](unsigned a, unsigned b) { return max(a, b); };
    most = over_waves<8>(over_lanes(most, larger), part, threadIdx.x / 64, 0, larger);
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

// 1 / v and 1 / sqrt(v) from the instructions' 2^-23 by two steps of Newton's, within some 2^-51.  (Divisions and a root to the last place
// are half as many instructions again as the rest of a row of 1536.)
__device__ __forceinline__ double one_by(double v)
{
    double r = __builtin_amdgcn_rcp(v);
    r = __builtin_fma(__builtin_fma(-v, r, 1.0), r, r);
    return __builtin_fma(__builtin_fma(-v, r, 1.0), r, r);
}
__device__ __forceinline__ double one_by_root(double v)
{
    double r = __builtin_amdgcn_rsq(v);
    r = __builtin_fma(0.5 * r, __builtin_fma(-v * r, r, 1.0), r);
    return __builtin_fma(0.5 * r, __builtin_fma(-v * r, r, 1.0), r);
}
// The larger of a and |b| (neither signals; a NaN is not taken).  Assembly: the compiler's form takes another instruction to quiet what cannot signal.
__device__ __forceinline__ double larger_of(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, |%2|" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// The norm, in fp64: what it ends in are whole numbers, and a result in 32 bits would be on another side of a border between two of them than
// the formula's about once in 10^5 elements, at another place for every order of the sums.  (The card adds and multiplies as fast
// in 64 bits as in 32.  Sums here are 58 additions deep at most, which the bound in include/rapid_packed.h counts on.)
// Bound by the vector instructions, 25 an element, 15 of which are the formula's: 8 x 4096 rows of 1536 46.8 us, 3.2 TB/s.
// FULL: every access of every lane is one of the row's; the form for any width takes 7 % more instructions.
template <int WAVES, int CHUNKS, bool FULL>
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
        raw[c] = FULL || at < p.C ? *(const u32x4*)(x + at) : none;
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
    auto larger = [](double a, double b) { return larger_of(a, b); };
    // (the mean rounded once: that of equal elements is their value)
    const double all = over_waves<WAVES>(over_lanes(sum, add), part[0], wave, own, add), near = all * p.share;
    const double mean = __builtin_fma(__builtin_fma(-near, (double)p.C, all), p.share, near);
    double y[CHUNKS][8], square = 0.0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const double off = FULL || 8 * (c * LANES + lane) < p.C ? mean : 0.0;         // (beyond the row: zeros)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[c][i] = (double)(i % 2 ? high(raw[c][i / 2]) : low(raw[c][i / 2])) - off;
            square = __builtin_fma(y[c][i], y[c][i], square);
        }
    }
    const double inv = one_by_root(__builtin_fma(over_waves<WAVES>(over_lanes(square, add), part[1], wave, own, add), p.share, (double)p.eps));
    double most = 0.0, number = inv * 0.0;             // number: NaN where an element is none
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        if (!FULL && at >= p.C) continue;
        if (p.scale && written) {
            const u32x4 scale = *(const u32x4*)(p.scale + d * p.scale_s + at), shift = *(const u32x4*)(p.shift + d * p.shift_s + at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double by = 1.0 + (double)(i % 2 ? high(scale[i / 2]) : low(scale[i / 2]));
                y[c][i] = __builtin_fma(y[c][i] * inv, by, (double)(i % 2 ? high(shift[i / 2]) : low(shift[i / 2])));
                number = __builtin_fma(y[c][i], 0.0, number);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[c][i] *= inv;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) most = larger(most, y[c][i]);
    }
    most = larger(most, number != 0.0 ? INFINITY : 0.0);
    most = over_waves<WAVES>(over_lanes(most, larger), part[2], wave, own, larger);
    if (!written) return;
    const bool plain = most < INFINITY && most > 0.0;
    const double by = 127.0 * one_by(plain ? most : 1.0);
    signed char* q = p.q + b * p.q_sb + (long long)r * p.q_sn;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        if (!FULL && at >= p.C) continue;
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
    const auto kernel = p.C == WAVES * CHUNKS * 512 ? norm_rows8_kernel<WAVES, CHUNKS, true> : norm_rows8_kernel<WAVES, CHUNKS, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.M + ROWS - 1) / ROWS)), dim3(BLOCK), 0, (hipStream_t)stream, p);
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
    // As few wavefronts a row as hold it with four accesses a lane.  Memory is the bound, so that it matters little: us for 8192 rows of 1536 by
    // 1 / 2 / 4 wavefronts 7.8 / 7.8 / 8.5, of 6144 by 2 / 4 / 8 29.5 / 28.4 / 27.8; any few hundred rows 3.7 to 4.4.
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
    if (!(eps >= 0.f) || isinf(eps) || (document && documents < 1)) return RAPID_ERR_SHAPE;      // (Newton's step on a root of 0 is no number)
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
    p.share = 1.0 / C;
    // As few wavefronts a row as hold it (joining sums of several costs three barriers a row) in a form that there is: five accesses take that of
    // six, seven that of eight over two wavefronts, where the last access of every lane, or of one wavefront, is empty (forms of five and
    // seven have not been measured); and four wavefronts rather than two or eight of a longer row.  us, rows of 1536 by 1 / 2 / 4 wavefronts: 8192 of them 14.1 / 15.7 / 19.2; of 2432 by
    // 1 x 6, 2 x 3, 4 x 2 accesses 21.1 / 21.7 / 25.8 (2 x 4: 23.9); of 6144 by 2 x 6, 4 x 3, 4 x 4, 8 x 2 51.4 / 47.5 / 52.5 / 55.6; 4096
    // of 9728 by 4 x 6, 8 x 3, 8 x 4 42.7 / 47.6 / 51.7.  A few hundred rows take 5.3 to 6.3 us by any.
    const int accesses = (C + 511) / 512;              // of a wavefront
    if (accesses == 1) return launch_norm<1, 1>(p, stream);
    if (accesses == 2) return launch_norm<1, 2>(p, stream);
    if (accesses == 3) return launch_norm<1, 3>(p, stream);
    if (accesses == 4) return launch_norm<1, 4>(p, stream);
    if (accesses <= 6) return launch_norm<1, 6>(p, stream);
    if (accesses <= 8) return launch_norm<2, 4>(p, stream);
    if (accesses <= 12) return launch_norm<4, 3>(p, stream);
    if (accesses <= 16) return launch_norm<4, 4>(p, stream);
    if (accesses <= 24) return launch_norm<4, 6>(p, stream);
    return launch_norm<8, 4>(p, stream);
}

}  // extern "C"
