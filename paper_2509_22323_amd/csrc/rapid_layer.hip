// What an MM-DiT layer does to rows around its products, for MI355X (gfx950): the norm under the conditioning's scale and shift,
// the norm of every head's queries and keys with their rotation by position, and the table of the rotation.
// C ABI: include/rapid_layer.h.
//
// All are bound by memory: every element is read once and written once, a row lives in the registers of the lanes that
// read it (16 bytes = 8 elements a lane and access), sums go over lanes by DPP moves, arithmetic is fp32 and each
// result is rounded once.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rapid_layer.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;

struct Eight {
    float v[8];
};
__device__ __forceinline__ Eight widened(u32x4 raw)
{
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e.v[2 * i] = __uint_as_float(raw[i] << 16);
        e.v[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
    return e;
}
__device__ __forceinline__ u32x4 rounded(const Eight& e)
{
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)e.v[i];
    return __builtin_bit_cast(u32x4, r);
}

template <int CTRL>
__device__ __forceinline__ float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// The sum over every run of LANES lanes (8, 16 or 64), in all of them; all lanes have to be there.
template <int LANES>
__device__ __forceinline__ float sum_over(float v)
{
    v += moved<0xB1>(v);                               // lane ^ 1
    v += moved<0x4E>(v);                               // lane ^ 2
    v += moved<0x141>(v);                              // 7 - lane of every 8: the other four
    if constexpr (LANES >= 16) v += moved<0x140>(v);   // 15 - lane of every 16: the other eight
    if constexpr (LANES == 64) {
        auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
        auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
    }
    return v;
}

// ---------------------------------------------------------------------------
// y = (x - mean) / sqrt(variance + eps) * (1 + scale) + shift
// ---------------------------------------------------------------------------
struct ModulateParams {
    const __bf16* x;
    __bf16* y;
    const __bf16* scale;
    const __bf16* shift;
    long long x_sb, x_sn, y_sb, y_sn, scale_sb, shift_sb;
    int M, n, C;
    float eps;
};

// WAVES wavefronts a row, CHUNKS accesses a lane: the row stays in registers between the mean, the mean square deviation from it
// (two passes over registers, so that a mean far from zero costs no digits) and the result.  8 samples of 4096 rows of 1536 (201 MB): 39 us
// = 5.1 TB/s, what a large copy reaches; 333 rows of 2432: 3.7 us, a launch.
template <int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void norm_modulate_kernel(ModulateParams p)
{
    constexpr int BLOCK = WAVES < 4 ? 256 : WAVES * 64, ROWS = BLOCK / 64 / WAVES, LANES = WAVES * 64;
    __shared__ float part[2][BLOCK / 64];
    const int lane = threadIdx.x % LANES, wave = threadIdx.x / 64, own = threadIdx.x / LANES;
    const int row = blockIdx.x * ROWS + own;
    const bool there = row < p.M;
    const int m = there ? row : p.M - 1;
    const int b = p.n == p.M ? 0 : (int)((unsigned)m / (unsigned)p.n), r = m - b * p.n;
    const __bf16* x = p.x + b * p.x_sb + r * p.x_sn;
    Eight e[CHUNKS];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        const u32x4 none = {0u, 0u, 0u, 0u};
        e[c] = widened(at < p.C ? *(const u32x4*)(x + at) : none);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += e[c].v[i];
    auto over_row = [&](float v, int turn) {
        v = sum_over<64>(v);
        if constexpr (WAVES == 1) return v;
        if (threadIdx.x % 64 == 0) part[turn][wave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += part[turn][own * WAVES + w];
        return v;
    };
    const float mean = over_row(sum, 0) / (float)p.C;
    float square = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const bool in = 8 * (c * LANES + lane) < p.C;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[c].v[i] -= mean;
            square += in ? e[c].v[i] * e[c].v[i] : 0.f;
        }
    }
    const float inv = 1.0f / sqrtf(over_row(square, 1) / (float)p.C + p.eps);
    if (!there) return;
    __bf16* y = p.y + b * p.y_sb + r * p.y_sn;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = 8 * (c * LANES + lane);
        if (at >= p.C) continue;
        if (p.scale) {
            const Eight scale = widened(*(const u32x4*)(p.scale + b * p.scale_sb + at));
            const Eight shift = widened(*(const u32x4*)(p.shift + b * p.shift_sb + at));
#pragma unroll
            for (int i = 0; i < 8; ++i) e[c].v[i] = __builtin_fmaf(e[c].v[i] * inv, 1.0f + scale.v[i], shift.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[c].v[i] *= inv;
        }
        *(u32x4*)(y + at) = rounded(e[c]);
    }
}

// ---------------------------------------------------------------------------
// Norm and rotation of queries and keys
// ---------------------------------------------------------------------------
struct QkSide {
    const __bf16* in[2];     // of the two segments
    __bf16* out[2];
    const __bf16* weight[2];
};
struct QkParams {
    QkSide side[2];          // queries, keys
    long long in_sb[2], in_sh[2], in_sn[2], out_sb[2], out_sh[2], out_sn[2];    // of the two segments
    const float* table;
    long long table_sb;
    int n0, N, H, rot, parts;          // parts: a token's heads are taken by that many lane groups
    long long tokens;                  // B * N
    float eps;
    bool heads_first;                  // neighbouring lane groups take neighbouring heads (else tokens)
};

// Heads of a lane group: 4 rows (queries and keys) in flight.  One head: 34 us at 4608 tokens of 24 heads of 128, two 29.5, four
// 30.5 (fewer workgroups, the last of them alone); small calls are faster the more workgroups there are.  Loads past the caches
// would gain 6 % where the rows come from memory and cost 20 % where the projection has just left them in the caches.  28 us at 4608
// tokens of 24 heads of 128 in a fused projection (115 MB, 4.1 TB/s; 22.6 from the caches), 88 us at 16896 head after head (424 MB,
// 4.8 TB/s; the table is fetched once a part, 80 MB more: workgroups in an order that keeps its rows in one L2 took 94).
// In halves 4 to 9 % more (eight angles a lane, four moves between lanes for 16 bytes, six wavefronts a SIMD for eight): 31.7 us for 29.3 at
// the first size, 99.6 for 92.4 at the second with the norm, 89.7 for 85.6 without.
constexpr int HEADS = 2;

// A group of D / 8 lanes takes one token: its row of the table, and heads part, part + parts, .. of queries and keys.
template <int D, bool NORM, int LAYOUT>            // LAYOUT -1: no rotation
__global__ __launch_bounds__(THREADS) void qk_rows_kernel(QkParams p)
{
    constexpr int LANES = D / 8, GROUPS = THREADS / LANES;
    const int lane = threadIdx.x % LANES;
    const unsigned item = blockIdx.x * GROUPS + threadIdx.x / LANES, items = (unsigned)(p.tokens * p.parts);
    const bool there = item < items;
    const unsigned it = there ? item : items - 1;
    unsigned token, part;
    if (p.heads_first) {
        token = it / (unsigned)p.parts;
        part = it - token * p.parts;
    } else {
        part = it / (unsigned)p.tokens;
        token = it - part * (unsigned)p.tokens;
    }
    const int b = (int)(token / (unsigned)p.N), t = (int)(token - b * (unsigned)p.N);
    const int s = t >= p.n0, r = s ? t - p.n0 : t;
    const bool turns = LAYOUT >= 0 && 8 * lane < p.rot;

    u32x4 raw[2][HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int h = min((int)(part + i * p.parts), p.H - 1);
        const long long at = b * p.in_sb[s] + h * p.in_sh[s] + r * p.in_sn[s] + 8 * lane;
#pragma unroll
        for (int j = 0; j < 2; ++j) raw[j][i] = *(const u32x4*)(p.side[j].in[s] + at);
    }
    // cosines and sines of this lane's elements (interleaved: of its four pairs; halves: of its eight, all in one half)
    constexpr int ANGLES = LAYOUT == RAPID_ROPE_HALVES ? 8 : 4;
    float co[ANGLES], si[ANGLES];
    bool upper = false;
    int other = lane;
    if constexpr (LAYOUT >= 0) {
        const int half = p.rot / 16;                   // lanes
        upper = LAYOUT == RAPID_ROPE_HALVES && lane >= half;
        const int first = turns ? (LAYOUT == RAPID_ROPE_HALVES ? 8 * (upper ? lane - half : lane) : 4 * lane) : 0;
        other = !turns ? lane : upper ? lane - half : lane + half;
        const f32x4* row = (const f32x4*)(p.table + b * p.table_sb + (long long)t * p.rot + 2 * first);
#pragma unroll
        for (int i = 0; i < ANGLES / 2; ++i) {
            const f32x4 two = row[i];
            co[2 * i] = two[0]; si[2 * i] = two[1]; co[2 * i + 1] = two[2]; si[2 * i + 1] = two[3];
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        Eight w, ow;                                   // weights of this lane's elements and of those they turn with
        if constexpr (NORM) {
            const __bf16* weight = p.side[j].weight[s];
#pragma unroll
            for (int i = 0; i < 8; ++i) w.v[i] = ow.v[i] = 1.0f;
            if (weight) {
                w = widened(*(const u32x4*)(weight + 8 * lane));
                if (LAYOUT == RAPID_ROPE_HALVES) ow = widened(*(const u32x4*)(weight + 8 * other));
            }
        }
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            Eight e = widened(raw[j][i]), o;
            if constexpr (LAYOUT == RAPID_ROPE_HALVES) {
                u32x4 from;
#pragma unroll
                for (int q = 0; q < 4; ++q) from[q] = (unsigned)__shfl((int)raw[j][i][q], other, LANES);
                o = widened(from);
            }
            if constexpr (NORM) {
                float square = 0.f;
#pragma unroll
                for (int q = 0; q < 8; ++q) square = __builtin_fmaf(e.v[q], e.v[q], square);
                const float inv = __builtin_amdgcn_rsqf(__builtin_fmaf(sum_over<LANES>(square), 1.0f / D, p.eps));
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    e.v[q] *= inv * w.v[q];
                    if (LAYOUT == RAPID_ROPE_HALVES) o.v[q] *= inv * ow.v[q];
                }
            }
            if (turns) {
                if constexpr (LAYOUT == RAPID_ROPE_INTERLEAVED) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float a = e.v[2 * q], c = e.v[2 * q + 1];
                        e.v[2 * q] = a * co[q] - c * si[q];
                        e.v[2 * q + 1] = c * co[q] + a * si[q];
                    }
                } else if constexpr (LAYOUT == RAPID_ROPE_HALVES) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) e.v[q] = e.v[q] * co[q] + (upper ? o.v[q] : -o.v[q]) * si[q];
                }
            }
            const int h = (int)(part + i * p.parts);
            if (there && h < p.H)
                *(u32x4*)(p.side[j].out[s] + (b * p.out_sb[s] + h * p.out_sh[s] + r * p.out_sn[s] + 8 * lane)) = rounded(e);
        }
    }
}

// ---------------------------------------------------------------------------
// The table
// ---------------------------------------------------------------------------
constexpr int MAX_PAIRS = 64, TABLE_GROUPS = 4096;
struct TableParams {
    const int* positions;
    float* table;
    long long tokens;
    double magnitude;
    int axes, pairs;
    double turns[MAX_PAIRS];           // of a pair per position: frequency / 2 pi
    unsigned char axis[MAX_PAIRS];
};

// magnitude * (cos, sin) of a number of turns, in fp64 as far as fp32 can tell: taken to the nearest quarter, where Taylor's sums of
// six and five terms are off by 1.1e-10 (cosine) and 1.8e-9 (sine) at most, 0.06 of half a step of fp32.  (With the library's
// fp64 sincospi 264 K tokens of 64 pairs take 62 us, stores of 8 bytes and a 64-bit division a pair included.)
__device__ __forceinline__ float2 turned(double turns, double magnitude)
{
    constexpr double WHOLE = 6755399441055744.0;            // 1.5 * 2^52: a sum with it is rounded to a whole number, in its low bits
    const double shifted = fma(4.0, turns, WHOLE);
    const double a = fma(-0.25, shifted - WHOLE, turns) * (2.0 * M_PI), q = a * a;
    double s = a * fma(q, fma(q, fma(q, fma(q, 1.0 / 362880, -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
    double c = fma(q, fma(q, fma(q, fma(q, fma(q, -1.0 / 3628800, 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
    if (magnitude != 1.0) { s *= magnitude; c *= magnitude; }
    const unsigned k = (unsigned)__double2loint(shifted);   // quarters: cos, sin = (c, s), (-s, c), (-c, -s), (s, -c)
    const float fs = (float)s, fc = (float)c, x = k & 1u ? fs : fc, y = k & 1u ? fc : fs;
    return make_float2(__uint_as_float(__float_as_uint(x) ^ ((k + 1u & 2u) << 30)), __uint_as_float(__float_as_uint(y) ^ ((k & 2u) << 30)));
}

// A lane stays with two neighbouring pairs and goes over tokens; 16 bytes a store, past the caches (264 K tokens of 64 pairs, 138 MB:
// 38 -> 25 us; 17 K tokens 5.4 -> 5.1).
__global__ __launch_bounds__(THREADS) void rope_table_kernel(TableParams p)
{
    const int lanes = p.pairs / 2, tokens = THREADS / lanes, own = threadIdx.x / lanes, i = 2 * (threadIdx.x - own * lanes);
    if (own >= tokens) return;
    const double f0 = p.turns[i], f1 = p.turns[i + 1];
    const int a0 = p.axis[i], a1 = p.axis[i + 1];
    for (long long t = (long long)blockIdx.x * tokens + own; t < p.tokens; t += (long long)gridDim.x * tokens) {
        const int* at = p.positions + t * p.axes;
        const float2 one = turned(at[a0] * f0, p.magnitude), two = turned(at[a1] * f1, p.magnitude);
        __builtin_nontemporal_store(f32x4{one.x, one.y, two.x, two.y}, (f32x4*)(p.table + 2 * (t * p.pairs + i)));
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE; }

constexpr long long MAX_ROW_STRIDE = 1LL << 22, MAX_STRIDE = 1LL << 40;

bool rows_ok(const rapid_rows& a, int B, int n, int width, bool written, long long& sb, long long& sn)
{
    sn = n == 1 ? width : a.stride_n;
    sb = B == 1 ? 0 : a.stride_b;
    if (sn < 0 || sn > MAX_ROW_STRIDE || sb < 0 || sb > MAX_STRIDE) return false;
    if (!written) return true;
    // apart: rows behind each other and samples behind each other, or samples within the rows' distance (sb <= sn <= 2^22 there:
    // of larger ones a product by B could leave 64 bits)
    if (n > 1 && B > 1) return (sn >= width && sb >= (n - 1) * sn + width) || (sb >= width && sb <= sn && sn >= (B - 1) * sb + width);
    return n > 1 ? sn >= width : B == 1 || sb >= width;
}

// Whether no two rows of D elements of an output share one: the dimensions by their strides, each at least as far as those within reach.
bool rows_apart(const int (&sizes)[3], const long long (&strides)[3], int D)
{
    int order[3] = {0, 1, 2};
    for (int i = 1; i < 3; ++i)
        for (int j = i; j > 0 && strides[order[j]] < strides[order[j - 1]]; --j) {
            const int k = order[j];
            order[j] = order[j - 1];
            order[j - 1] = k;
        }
    long long reach = D;
    for (int i : order) {
        if (sizes[i] == 1) continue;
        if (strides[i] < reach) return false;
        reach += (sizes[i] - 1) * strides[i];
    }
    return true;
}

template <int WAVES, int CHUNKS>
int launch_modulate(const ModulateParams& p, void* stream)
{
    constexpr int BLOCK = WAVES < 4 ? 256 : WAVES * 64, ROWS = BLOCK / 64 / WAVES;
    const long long blocks = ((long long)p.M + ROWS - 1) / ROWS;
    if (blocks * BLOCK >= (1LL << 32)) return RAPID_ERR_SHAPE;
    hipLaunchKernelGGL((norm_modulate_kernel<WAVES, CHUNKS>), dim3((unsigned)blocks), dim3(BLOCK), 0, (hipStream_t)stream, p);
    return launched();
}

template <int D, bool NORM>
int launch_qk(const QkParams& p, int layout, void* stream)
{
    constexpr int GROUPS = THREADS / (D / 8);
    const long long blocks = (p.tokens * p.parts + GROUPS - 1) / GROUPS;
    if (p.tokens * p.parts >= (1LL << 32) || blocks * THREADS >= (1LL << 32)) return RAPID_ERR_SHAPE;
    const dim3 grid((unsigned)blocks), block(THREADS);
    hipStream_t s = (hipStream_t)stream;
    if (layout < 0) {
        if constexpr (NORM) hipLaunchKernelGGL((qk_rows_kernel<D, NORM, -1>), grid, block, 0, s, p);
    } else if (layout == RAPID_ROPE_INTERLEAVED) {
        hipLaunchKernelGGL((qk_rows_kernel<D, NORM, RAPID_ROPE_INTERLEAVED>), grid, block, 0, s, p);
    } else {
        hipLaunchKernelGGL((qk_rows_kernel<D, NORM, RAPID_ROPE_HALVES>), grid, block, 0, s, p);
    }
    return launched();
}

int qk_rows(const rapid_qk_segment* segments, int n_segments, int B, int H, int D, bool norm, float eps, const float* table,
            long long table_stride_b, int rot, int layout, void* stream)
{
    if (!segments || n_segments < 1) return RAPID_ERR_NULL;
    if (n_segments > 2 || B <= 0 || H <= 0 || (long long)B * H > 524287) return RAPID_ERR_SHAPE;
    if (D != 64 && D != 128) return RAPID_ERR_UNSUPPORTED;
    if (norm && !(eps >= 0.f)) return RAPID_ERR_SHAPE;
    if (!norm && !table) return RAPID_ERR_NULL;
    QkParams p = {};
    long long N = 0;
    bool heads_first = true;
    for (int i = 0; i < n_segments; ++i) {
        const rapid_qk_segment& g = segments[i];
        if (!g.q || !g.k || !g.q_out || !g.k_out) return RAPID_ERR_NULL;
        if (g.n <= 0 || g.n > (1 << 22)) return RAPID_ERR_SHAPE;
        const long long in[3] = {B == 1 ? 0 : g.in_stride_b, H == 1 ? 0 : g.in_stride_h, g.n == 1 ? 0 : g.in_stride_n};
        const long long out[3] = {B == 1 ? 0 : g.out_stride_b, H == 1 ? 0 : g.out_stride_h, g.n == 1 ? 0 : g.out_stride_n};
        const int sizes[3] = {B, H, g.n};
        for (int j = 0; j < 3; ++j) {
            if (in[j] < 0 || in[j] > MAX_STRIDE || out[j] < 0 || out[j] > MAX_STRIDE) return RAPID_ERR_SHAPE;
            if (sizes[j] > 1 && out[j] < D) return RAPID_ERR_SHAPE;
            if (in[j] % 8 != 0 || out[j] % 8 != 0) return RAPID_ERR_ALIGN;
        }
        if (!aligned(g.q, 16) || !aligned(g.k, 16) || !aligned(g.q_out, 16) || !aligned(g.k_out, 16)) return RAPID_ERR_ALIGN;
        if (norm && (!aligned(g.q_weight, 16) || !aligned(g.k_weight, 16))) return RAPID_ERR_ALIGN;
        const bool same = in[0] == out[0] && in[1] == out[1] && in[2] == out[2];
        if (g.q_out == g.k_out || g.q_out == g.k || g.k_out == g.q) return RAPID_ERR_ALIAS;
        if (!same && (g.q_out == g.q || g.k_out == g.k)) return RAPID_ERR_ALIAS;
        p.in_sb[i] = in[0]; p.in_sh[i] = in[1]; p.in_sn[i] = in[2];
        p.out_sb[i] = out[0]; p.out_sh[i] = out[1]; p.out_sn[i] = out[2];
        p.side[0].in[i] = (const __bf16*)g.q; p.side[1].in[i] = (const __bf16*)g.k;
        p.side[0].out[i] = (__bf16*)g.q_out; p.side[1].out[i] = (__bf16*)g.k_out;
        p.side[0].weight[i] = (const __bf16*)g.q_weight; p.side[1].weight[i] = (const __bf16*)g.k_weight;
        if (i == 0) heads_first = g.n == 1 || in[1] <= in[2];
        N += g.n;
    }
    if (N > (1 << 22)) return RAPID_ERR_SHAPE;
    for (int i = 0; i < n_segments; ++i) {
        const int sizes[3] = {B, H, segments[i].n};
        const long long strides[3] = {p.out_sb[i], p.out_sh[i], p.out_sn[i]};
        if (!rows_apart(sizes, strides, D)) return RAPID_ERR_SHAPE;
        if (n_segments == 1) break;
        const rapid_qk_segment &g = segments[i], &o = segments[1 - i];
        for (const void* out : {g.q_out, g.k_out})
            if (out == o.q || out == o.k || out == o.q_out || out == o.k_out) return RAPID_ERR_ALIAS;
    }
    if (table) {
        if (rot <= 0 || rot > D || rot % 16 != 0 || layout < RAPID_ROPE_INTERLEAVED || layout > RAPID_ROPE_HALVES) return RAPID_ERR_UNSUPPORTED;
        p.table_sb = B == 1 ? 0 : table_stride_b;
        if (p.table_sb < 0 || p.table_sb > MAX_STRIDE) return RAPID_ERR_SHAPE;
        if (!aligned(table, 16) || p.table_sb % 4 != 0) return RAPID_ERR_ALIGN;
        p.table = table;
        p.rot = rot;
    }
    p.n0 = segments[0].n;
    p.N = (int)N;
    p.H = H;
    p.parts = (H + HEADS - 1) / HEADS;
    p.tokens = (long long)B * N;
    p.eps = eps;
    p.heads_first = heads_first;
    const int l = table ? layout : -1;
    if (D == 64) return norm ? launch_qk<64, true>(p, l, stream) : launch_qk<64, false>(p, l, stream);
    return norm ? launch_qk<128, true>(p, l, stream) : launch_qk<128, false>(p, l, stream);
}

}  // namespace

extern "C" {

int rapid_norm_modulate(const rapid_rows* x, const rapid_rows* y, const void* scale, long long scale_stride, const void* shift,
                        long long shift_stride, int B, int n, int C, float eps, void* stream)
{
    if (!x || !y || !x->ptr || !y->ptr || !scale != !shift) return RAPID_ERR_NULL;
    if (B <= 0 || n <= 0 || C <= 0 || !(eps >= 0.f)) return RAPID_ERR_SHAPE;
    const long long M = (long long)B * n;
    if (M >= (1LL << 31) - 256) return RAPID_ERR_SHAPE;
    if (C % 8 != 0 || C > 16384) return RAPID_ERR_UNSUPPORTED;
    ModulateParams p = {};
    if (!rows_ok(*x, B, n, C, false, p.x_sb, p.x_sn) || !rows_ok(*y, B, n, C, true, p.y_sb, p.y_sn)) return RAPID_ERR_SHAPE;
    if (scale && B > 1) { p.scale_sb = scale_stride; p.shift_sb = shift_stride; }
    if (p.scale_sb < 0 || p.scale_sb > MAX_STRIDE || p.shift_sb < 0 || p.shift_sb > MAX_STRIDE) return RAPID_ERR_SHAPE;
    if (!aligned(x->ptr, 16) || !aligned(y->ptr, 16) || !aligned(scale, 16) || !aligned(shift, 16)) return RAPID_ERR_ALIGN;
    if ((p.x_sb | p.x_sn | p.y_sb | p.y_sn | p.scale_sb | p.shift_sb) % 8 != 0) return RAPID_ERR_ALIGN;
    if (y->ptr == x->ptr && (p.x_sb != p.y_sb || p.x_sn != p.y_sn)) return RAPID_ERR_ALIAS;
    if (y->ptr == scale || y->ptr == shift) return RAPID_ERR_ALIAS;
    p.x = (const __bf16*)x->ptr;
    p.y = (__bf16*)y->ptr;
    p.scale = (const __bf16*)scale;
    p.shift = (const __bf16*)shift;
    p.M = (int)M;
    p.n = B == 1 ? (int)M : n;
    p.C = C;
    p.eps = eps;
    if (C <= 512) return launch_modulate<1, 1>(p, stream);
    if (C <= 1024) return launch_modulate<1, 2>(p, stream);
    if (C <= 2048) return launch_modulate<1, 4>(p, stream);
    if (C <= 4096) return launch_modulate<2, 4>(p, stream);
    if (C <= 8192) return launch_modulate<4, 4>(p, stream);
    return launch_modulate<8, 4>(p, stream);
}

int rapid_rope_table(const int* positions, long long tokens, int n_axes, const rapid_rope_axis* axes, double magnitude, float* table,
                     void* stream)
{
    if (!positions || !axes || !table) return RAPID_ERR_NULL;
    if (tokens <= 0 || tokens > (1LL << 28) || n_axes < 1 || n_axes > 8) return RAPID_ERR_SHAPE;
    TableParams p = {};
    for (int a = 0; a < n_axes; ++a) {
        const rapid_rope_axis& x = axes[a];
        if (x.dim < 2 || x.dim % 2 != 0 || p.pairs + x.dim / 2 > MAX_PAIRS || !(x.theta > 0.0) || !isfinite(x.theta)) return RAPID_ERR_UNSUPPORTED;
        if (x.scaling < RAPID_ROPE_PLAIN || x.scaling > RAPID_ROPE_BY_PARTS) return RAPID_ERR_UNSUPPORTED;
        if (x.scaling != RAPID_ROPE_PLAIN && (!(x.factor > 0.0) || !isfinite(x.factor))) return RAPID_ERR_UNSUPPORTED;
        if (x.scaling == RAPID_ROPE_NTK && x.dim < 4) return RAPID_ERR_UNSUPPORTED;
        if (x.scaling == RAPID_ROPE_BY_PARTS && (!(x.original_length > 0.0) || !(x.beta_fast > x.beta_slow))) return RAPID_ERR_UNSUPPORTED;
        // (in 64 bits of mantissa, one power an axis and a product a pair: with a power a pair a call took 0.5 us more, and its exponent,
        // rounded in 53 bits, cost the slow pairs up to three bits)
        constexpr long double TURN = 6.283185307179586476925286766559L;
        const int pairs = x.dim / 2;
        const long double dim = x.dim, theta = x.scaling == RAPID_ROPE_NTK ? x.theta * powl(x.factor, dim / (dim - 2)) : (long double)x.theta;
        // theta^(-1/pairs): a power in 53 bits, and a step of Newton's towards ratio^pairs = 1 / theta
        const long double near = pow((double)theta, -1.0 / pairs);
        long double power = 1, square = near;
        for (int bits = pairs; bits != 0; bits >>= 1, square *= square)
            if (bits & 1) power *= square;
        const long double ratio = near + near * (1 / (theta * power) - 1) / pairs;
        long double plain = 1;
        for (int i = 0; i < pairs; ++i, plain *= ratio) {
            long double f = plain;
            if (x.scaling == RAPID_ROPE_LINEAR) f /= x.factor;
            if (x.scaling == RAPID_ROPE_BY_PARTS) {
                const double r = (double)(x.original_length * f / TURN);
                const double g = fmin(fmax((r - x.beta_slow) / (x.beta_fast - x.beta_slow), 0.0), 1.0);
                f *= g + (1.0 - g) / x.factor;
            }
            p.turns[p.pairs] = (double)(f * (1 / TURN));
            if (!(p.turns[p.pairs] < 65536.0)) return RAPID_ERR_UNSUPPORTED;       // (reduction takes 2^50 turns)
            p.axis[p.pairs++] = (unsigned char)a;
        }
    }
    if (p.pairs % 8 != 0 || !isfinite(magnitude)) return RAPID_ERR_UNSUPPORTED;
    if (!aligned(positions, 4) || !aligned(table, 16)) return RAPID_ERR_ALIGN;
    p.positions = positions;
    p.table = table;
    p.tokens = tokens;
    p.magnitude = magnitude;
    p.axes = n_axes;
    const long long each = THREADS / (p.pairs / 2), blocks = (tokens + each - 1) / each;
    hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)(blocks < TABLE_GROUPS ? blocks : TABLE_GROUPS)), dim3(THREADS), 0, (hipStream_t)stream, p);
    return launched();
}

int rapid_qk_norm_rope(const rapid_qk_segment* segments, int n_segments, int B, int H, int D, float eps, const float* table,
                       long long table_stride_b, int rot, int layout, void* stream)
{
    return qk_rows(segments, n_segments, B, H, D, true, eps, table, table_stride_b, rot, layout, stream);
}

int rapid_rope(const rapid_qk_segment* segments, int n_segments, int B, int H, int D, const float* table, long long table_stride_b,
               int rot, int layout, void* stream)
{
    return qk_rows(segments, n_segments, B, H, D, false, 0.f, table, table_stride_b, rot, layout, stream);
}

}  // extern "C"
