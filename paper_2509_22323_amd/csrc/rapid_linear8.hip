// Linear layers as products of 8-bit integers for MI355X (gfx950): y = residual + gate * act(x_scale w_scale (x w^T) + bias).
// C ABI: include/rapid_packed.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "rapid_packed.h"
#include "rapid_wide.h"

namespace {

constexpr int STEP = 128;                              // inputs per step
constexpr int CUS = 256;
constexpr int MOST_PIECES = 8;                         // along K
static_assert(STEP == INPUTS<signed char>, "");

// The row of the gate that row m takes (sample b); below 0: the row is not written.
__device__ __forceinline__ int vector_of(const Linear8Params& p, int m, int b)
{
    if (!p.document) return b;
    const int d = p.document[m];
    return (unsigned)d < (unsigned)p.documents ? d : -1;
}

// The sums of a product's pieces, and the epilogue: eight outputs a lane.
__global__ __launch_bounds__(256) void linear8_join_kernel(Linear8Params p)
{
    const unsigned per_row = (unsigned)p.pitch / 8, at = blockIdx.x * 256 + threadIdx.x, m = at / per_row;
    const int n = 8 * (int)(at - m * per_row);
    if (m >= (unsigned)p.M || n >= p.N) return;
    int b, r;
    sample_of(p, (int)m, b, r);
    const int d = vector_of(p, (int)m, b);
    if (d < 0) return;
    bf16x8 bias = {}, gate = {}, residual = {};
    if (p.bias) bias = eight_of(p.bias, n, p.N, p.even);
    if (p.gate) gate = eight_of(p.gate + d * p.g_sb, n, p.N, p.even);
    if (p.residual) residual = eight_of(p.residual + b * p.r_sb + (long long)r * p.r_sn, n, p.N, p.even);
    const float by = p.x_scale[m];
    float scale[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) scale[i] = p.w_scale[min(n + i, p.N - 1)];
    const int* from = (const int*)p.partial + (long long)m * p.pitch + n;
    i32x4 part[MOST_PIECES][2];                        // all of them on their way before the first is added
#pragma unroll
    for (int s = 0; s < MOST_PIECES; ++s)
        if (s < p.pieces) {
            part[s][0] = *(const i32x4*)(from + s * (long long)p.M * p.pitch);
            part[s][1] = *(const i32x4*)(from + s * (long long)p.M * p.pitch + 4);
        }
    int sum[8] = {};
#pragma unroll
    for (int s = 0; s < MOST_PIECES; ++s)
        if (s < p.pieces)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += part[s][i / 4][i % 4];
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = scaled(sum[i], by, scale[i], (float)bias[i]);
    store_eight(p.y + b * p.y_sb + (long long)r * p.y_sn, n, p.N, finished(p, z, gate, residual), p.even);
}

__device__ __forceinline__ int sum_of_lanes(int v)
{
    auto moved = [](int v, auto how) { return __builtin_amdgcn_update_dpp(0, v, how.value, 0xf, 0xf, true); };
    v += moved(v, std::integral_constant<int, 0xB1>());
    v += moved(v, std::integral_constant<int, 0x4E>());
    v += moved(v, std::integral_constant<int, 0x141>());
    v += moved(v, std::integral_constant<int, 0x140>());
    auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = (int)a[0] + (int)a[1];
    auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (int)b[0] + (int)b[1];
}

// A handful of rows (the conditioning's projections): a wavefront takes OUT outputs of all rows and reads their rows of w end to end, 1 KB an
// access, four products an instruction.  Bound by the bytes of w and the launch: 2 rows, 1536 to 9216, 4.9 us (14 MB: 2.9 TB/s).
constexpr int OUT = 2, DOT_WAVES = 2;

template <int MAX_M>
__global__ __launch_bounds__(DOT_WAVES * 64) void linear8_dot_kernel(Linear8Params p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = (blockIdx.x * DOT_WAVES + wave) * OUT;
    if (j0 >= p.N) return;
    const signed char *x[MAX_M], *w[OUT];
#pragma unroll
    for (int m = 0; m < MAX_M; ++m) {
        int b, r;
        sample_of(p, min(m, p.M - 1), b, r);
        x[m] = p.x + b * p.x_sb + (long long)r * p.x_sn;
    }
#pragma unroll
    for (int j = 0; j < OUT; ++j) w[j] = p.w + (long long)min(j0 + j, p.N - 1) * p.w_sn;
    int acc[OUT][MAX_M] = {};
    auto some = [&](int k, auto count) {               // count times 1024 inputs from k on
        constexpr int COUNT = decltype(count)::value;
        i32x4 wv[COUNT][OUT], xv[COUNT][MAX_M];
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            const int at = k + 1024 * c + 16 * lane;
            const i32x4 none = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < OUT; ++j) wv[c][j] = at < p.K ? *(const i32x4*)(w[j] + at) : none;
#pragma unroll
            for (int m = 0; m < MAX_M; ++m) xv[c][m] = at < p.K ? *(const i32x4*)(x[m] + at) : none;
        }
        __builtin_amdgcn_sched_barrier(0);             // all of them are on their way before the first product
#pragma unroll
        for (int c = 0; c < COUNT; ++c)
#pragma unroll
            for (int j = 0; j < OUT; ++j)
#pragma unroll
                for (int m = 0; m < MAX_M; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][m] = __builtin_amdgcn_sdot4(wv[c][j][i], xv[c][m][i], acc[j][m], false);
    };
    int k = 0;
    for (; k + 1024 < p.K; k += 2048) some(k, std::integral_constant<int, 2>());
    if (k < p.K) some(k, std::integral_constant<int, 1>());
    // lane j * MAX_M + m keeps the sum of output j of row m
    int mine = 0;
#pragma unroll
    for (int j = 0; j < OUT; ++j)
#pragma unroll
        for (int m = 0; m < MAX_M; ++m) {
            const int sum = sum_of_lanes(acc[j][m]);
            mine = lane == j * MAX_M + m ? sum : mine;
        }
    const int j = lane / MAX_M, m = lane - j * MAX_M, n = j0 + j;
    if (j >= OUT || m >= p.M || n >= p.N) return;
    int b, r;
    sample_of(p, m, b, r);
    const int d = vector_of(p, m, b);
    if (d < 0) return;
    const float z = activated(scaled(mine, p.x_scale[m], p.w_scale[n], p.bias ? (float)p.bias[n] : 0.f), p.activation);
    const float gate = p.gate ? (float)p.gate[d * p.g_sb + n] : 1.f, residual = p.residual ? (float)p.residual[b * p.r_sb + (long long)r * p.r_sn + n] : 0.f;
    p.y[b * p.y_sb + (long long)r * p.y_sn + n] = (__bf16)ended(z, gate, residual);
}

// A wavefront's dot products, or tiles of matrix instructions.  us: 3 rows, 1536 by 1536 3.9 / 8.8, 6144 by 12288 13.7 / 17.7; 5 to 8 rows, 1536 by 9216 8.4 / 8.7,
// 4096 by 8192 10.6 / 13.6, 6144 by 12288 18.0 / 17.6.
bool by_dots(long long M, int N, int K) { return M <= 4 || (M <= 8 && (long long)N * K <= 1 << 25); }

// (as rapid_linear.hip has it)
bool even_rows(const Linear8Params& p)
{
    const uintptr_t starts = (uintptr_t)p.y | (uintptr_t)p.residual | (uintptr_t)p.gate | 2 * (uintptr_t)(p.y_sb | p.y_sn | p.r_sb | p.r_sn | p.g_sb);
    return starts % 4 == 0 || (long long)p.M * p.N < 1 << 21;
}

template <int MAX_M>
int launch_dot(const Linear8Params& p, void* stream)
{
    constexpr int EACH = OUT * DOT_WAVES;
    hipLaunchKernelGGL((linear8_dot_kernel<MAX_M>), dim3((unsigned)((p.N + EACH - 1) / EACH)), dim3(DOT_WAVES * 64), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

template <int WR, int FN, bool SPLIT>
int launch_wide(const Linear8Params& p, void* stream)
{
    constexpr int TM = 64 * WR, TN = 32 * FN;
    const long long items = (((long long)p.M + TM - 1) / TM) * ((p.N + TN - 1) / TN) * (SPLIT ? p.pieces : 1);
    if (items >= (1LL << 31) - 4096) return RAPID_ERR_SHAPE;
    const long long most = CUS * (4 / WR);
    hipLaunchKernelGGL((linear_wide_kernel<WR, FN, SPLIT, Linear8Params>), dim3((unsigned)(items < most ? items : most)), dim3(WR * 128), 0,
                       (hipStream_t)stream, p, (int)items);
    if constexpr (SPLIT) {
        const long long lanes = (long long)p.M * (p.pitch / 8);
        hipLaunchKernelGGL(linear8_join_kernel, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, (hipStream_t)stream, p);
    }
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

// Which tile, and how many pieces along K
enum Tile { T64x64, T128x128, T256x128, T256x160, T256x192, T256x256, TILES };
struct Plan {
    Tile tile;
    int pieces;
};

// What a product takes, in us, as rapid_linear.hip has it (steps of 128 inputs), fitted to 1200 products of 9 to 32768 rows, 16 to 9728 outputs
// and 64 to 9728 inputs timed in all tiles and 1 to 8 pieces, inputs changing from call to call, before the epilogue's roundings and the
// order of its scales were as they are now.  Of the kernels as they are, the plan found by it takes 1.012 times what the best one
// does in the geometric mean of 250 other products (1.19 at most).
struct TileCost {
    int rows, columns, slots;
    float alone, full, ends, odd, call, join, sum;
};
constexpr TileCost COST[TILES] = {
    {64, 64, 4, 0.324f, 1.047f, 1.30f, 2.06f, 3.42f, 2.32f, 1.90f}, {128, 128, 2, 0.502f, 1.091f, 3.28f, 3.19f, 2.31f, 1.87f, 1.93f},
    {256, 128, 1, 0.481f, 1.020f, 4.05f, 3.23f, 3.03f, 0.f, 0.f},   {256, 160, 1, 0.669f, 1.308f, 5.56f, 3.43f, 2.90f, 0.f, 0.f},
    {256, 192, 1, 0.654f, 1.299f, 6.30f, 4.78f, 2.19f, 0.f, 0.f},   {256, 256, 1, 0.820f, 1.645f, 8.02f, 5.66f, 2.57f, 0.f, 0.f}};

float cost_of(const TileCost& c, long long M, int N, int K, int pieces)
{
    const long long items = ((M + c.rows - 1) / c.rows) * ((N + c.columns - 1) / c.columns) * pieces, slots = CUS * c.slots;
    const int all = (K + STEP - 1) / STEP;
    const float steps = all > 2 ? (float)all / pieces : 2.f, load = (float)(items % slots) / CUS;
    const float ends = N % 8 != 0 && pieces == 1 ? c.ends + c.odd : c.ends;
    float t = c.call + (float)(items / slots) * (steps * c.full + ends);
    if (items % slots != 0) {
        const float crowd = c.slots == 1 ? load : load > 1.f ? (0.3f * load + 0.7f * ceilf(load) - 1.f) / (c.slots - 1) : 0.f;
        t += steps * (c.alone + (c.full - c.alone) * crowd) + ends;
    }
    return pieces > 1 ? t + c.join + c.sum * 1e-6f * (float)M * (float)N * pieces : t;
}

Plan plan_for(long long M, int N, int K, int most_pieces)
{
    Plan best = {T64x64, 1};
    float least = cost_of(COST[T64x64], M, N, K, 1);
    for (int t = 0; t < TILES; ++t) {
        // (a piece has three steps at least; larger tiles have work enough, or few steps; a lane number of the join has 32 bits)
        const int most = t <= T128x128 && M * N < (1LL << 31) ? most_pieces : 1;
        for (int pieces = 1; pieces <= most && (pieces == 1 || 3 * pieces * STEP <= K); ++pieces) {
            const float c = cost_of(COST[t], M, N, K, pieces);
            if (c < least) { least = c; best = {(Tile)t, pieces}; }
        }
    }
    return best;
}

constexpr int MOST_INPUTS = (1 << 17) - 16;            // 2^14 times as many fit 32 bits

}  // namespace

extern "C" {

size_t rapid_linear_int8_workspace_bytes(long long M, int N, int K)
{
    if (M <= 0 || M >= (1LL << 31) - 256 || N <= 0 || N > MAX_STRIDE || K <= 0 || K > MOST_INPUTS || K % 16 != 0 || by_dots(M, N, K)) return 0;
    const int pieces = plan_for(M, N, K, MOST_PIECES).pieces;
    return pieces > 1 ? (size_t)pieces * M * ((N + 7) / 8 * 8) * sizeof(int) : 0;
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
    p.g_sb = gate && (document ? documents : B) > 1 ? gate_stride : 0;
    if (p.g_sb < 0 || p.g_sb > (1LL << 40)) return RAPID_ERR_SHAPE;
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
    if (by_dots(M, N, K)) {
        if (M == 1) return launch_dot<1>(p, stream);
        if (M == 2) return launch_dot<2>(p, stream);
        return M <= 4 ? launch_dot<4>(p, stream) : launch_dot<8>(p, stream);
    }
    const Plan plan = plan_for(M, N, K, workspace ? MOST_PIECES : 1);
    p.pieces = plan.pieces;
    p.pitch = (N + 7) / 8 * 8;
    p.partial = (float*)workspace;
    p.even = even_rows(p);
    if (plan.pieces > 1) return plan.tile == T64x64 ? launch_wide<1, 2, true>(p, stream) : launch_wide<2, 4, true>(p, stream);
    switch (plan.tile) {
    case T64x64: return launch_wide<1, 2, false>(p, stream);
    case T128x128: return launch_wide<2, 4, false>(p, stream);
    case T256x128: return launch_wide<4, 4, false>(p, stream);
    case T256x160: return launch_wide<4, 5, false>(p, stream);
    case T256x192: return launch_wide<4, 6, false>(p, stream);
    default: return launch_wide<4, 8, false>(p, stream);
    }
}

}  // extern "C"
