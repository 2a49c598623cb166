// Linear layers of an MM-DiT layer for MI355X (gfx950): y = residual + gate * act(x w^T + bias).
// C ABI: include/rapid_layer.h.
//
// A handful of rows: linear_dot_kernel (bound by the bytes of w).  Everything else: linear_wide_kernel, tiles of matrix instructions,
// and where a product has few tiles and many inputs, linear_join_kernel behind it, which adds up pieces along K.  by_dots and
// plan_for at the end of the file choose.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "rapid_layer.h"
#include "rapid_wide.h"

namespace {

constexpr int STEP = 64;                               // inputs per step
constexpr int CUS = 256;
constexpr int MOST_PIECES = 8;                         // along K
static_assert(STEP == INPUTS<__bf16>, "");

// The sums of a product's pieces, in their order, and the epilogue: eight outputs a lane.
__global__ __launch_bounds__(256) void linear_join_kernel(LinearParams p)
{
    const unsigned per_row = (unsigned)p.pitch / 8, at = blockIdx.x * 256 + threadIdx.x, m = at / per_row;
    const int n = 8 * (int)(at - m * per_row);
    if (m >= (unsigned)p.M || n >= p.N) return;
    int b, r;
    sample_of(p, (int)m, b, r);
    bf16x8 bias = {}, gate = {}, residual = {};
    if (p.bias) bias = eight_of(p.bias, n, p.N, p.even);
    if (p.gate) gate = eight_of(p.gate + b * p.g_sb, n, p.N, p.even);
    if (p.residual) residual = eight_of(p.residual + b * p.r_sb + (long long)r * p.r_sn, n, p.N, p.even);
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (float)bias[i];
    const float* from = p.partial + (long long)m * p.pitch + n;
    f32x4 part[MOST_PIECES][2];                        // all of them on their way before the first is added
#pragma unroll
    for (int s = 0; s < MOST_PIECES; ++s)
        if (s < p.pieces) {
            part[s][0] = *(const f32x4*)(from + s * (long long)p.M * p.pitch);
            part[s][1] = *(const f32x4*)(from + s * (long long)p.M * p.pitch + 4);
        }
#pragma unroll
    for (int s = 0; s < MOST_PIECES; ++s)
        if (s < p.pieces)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] += part[s][i / 4][i % 4];
    store_eight(p.y + b * p.y_sb + (long long)r * p.y_sn, n, p.N, finished(p, z, gate, residual), p.even);
}

// ---------------------------------------------------------------------------
// A handful of rows (the conditioning's projections): MAX_M of x at most.  A wavefront takes OUT outputs of all rows and reads their
// rows of w end to end, 1 KB an access; two products an instruction, the lanes' sums are added at the end.  Bound by the bytes of w:
// 2 rows, 1536 -> 9216 (28 MB): 4.7 us = 6.0 TB/s where w is in the caches, 6.6 us = 4.3 TB/s where w changes
// from call to call; four outputs a wavefront and four wavefronts a workgroup, whose number then does not go evenly over the CUs:
// 4.9 and 7.2, and 9.2 instead of 5.3 us for 4 rows, 9728 -> 100.
// ---------------------------------------------------------------------------
constexpr int OUT = 2, DOT_WAVES = 2;

template <int MAX_M>
__global__ __launch_bounds__(DOT_WAVES * 64) void linear_dot_kernel(LinearParams p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = (blockIdx.x * DOT_WAVES + wave) * OUT;
    if (j0 >= p.N) return;
    const __bf16 *x[MAX_M], *w[OUT];
#pragma unroll
    for (int m = 0; m < MAX_M; ++m) {
        int b, r;
        sample_of(p, min(m, p.M - 1), b, r);
        x[m] = p.x + b * p.x_sb + (long long)r * p.x_sn;
    }
#pragma unroll
    for (int j = 0; j < OUT; ++j) w[j] = p.w + (long long)min(j0 + j, p.N - 1) * p.w_sn;
    float acc[OUT][MAX_M] = {};
    auto some = [&](int k, auto count) {               // count times 512 inputs from k on
        constexpr int COUNT = decltype(count)::value;
        u32x4 wv[COUNT][OUT], xv[COUNT][MAX_M];
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            const int at = k + 512 * c + 8 * lane;
            const u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < OUT; ++j) wv[c][j] = COUNT > 1 || at < p.K ? *(const u32x4*)(w[j] + at) : none;
#pragma unroll
            for (int m = 0; m < MAX_M; ++m) xv[c][m] = COUNT > 1 || at < p.K ? *(const u32x4*)(x[m] + at) : none;
        }
        __builtin_amdgcn_sched_barrier(0);             // all of them are on their way before the first product
#pragma unroll
        for (int c = 0; c < COUNT; ++c)
#pragma unroll
            for (int j = 0; j < OUT; ++j)
#pragma unroll
                for (int m = 0; m < MAX_M; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned a = wv[c][j][i], b = xv[c][m][i];
                        acc[j][m] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), acc[j][m], false);
                    }
    };
    constexpr int AHEAD = 3;
    int k = 0;
    for (; k + 512 * AHEAD <= p.K; k += 512 * AHEAD) some(k, std::integral_constant<int, AHEAD>());
    for (; k < p.K; k += 512) some(k, std::integral_constant<int, 1>());
    // lane j * MAX_M + m keeps the sum of output j of row m
    float mine = 0.f;
#pragma unroll
    for (int j = 0; j < OUT; ++j)
#pragma unroll
        for (int m = 0; m < MAX_M; ++m) {
            const float sum = sum_of_lanes(acc[j][m]);
            mine = lane == j * MAX_M + m ? sum : mine;
        }
    const int j = lane / MAX_M, m = lane - j * MAX_M, n = j0 + j;
    if (j >= OUT || m >= p.M || n >= p.N) return;
    int b, r;
    sample_of(p, m, b, r);
    if (p.bias) mine += (float)p.bias[n];
    mine = activated(mine, p.activation);
    if (p.gate) mine *= (float)p.gate[b * p.g_sb + n];
    if (p.residual) mine += (float)p.residual[b * p.r_sb + (long long)r * p.r_sn + n];
    p.y[b * p.y_sb + (long long)r * p.y_sn + n] = (__bf16)mine;
}

// Every wavefront reads all of x.  Five to eight rows, three sets of inputs in turn: 10.6 to 11.0 us here, 11.5 in tiles of matrix
// instructions at 1536 -> 9216, 8.9 to 9.2 and 11.5 at 6144 -> 1536, but 21 and 16.7 at 2432 -> 14592.  (Four: 7.7, 6.9 and 14.2 here.)
// Up to four always: include/rapid_layer.h says that the bits of their rows do not depend on how many there are.
bool by_dots(long long M, int N, int K) { return M <= 4 || (M <= 8 && (long long)N * K <= 1 << 24); }

// Rows of y, residual and gate that start at multiples of four bytes, or results too small for it to matter: 8192 rows, 1536 -> 4607 with
// gate and residual 148 us, and 129 in pieces; 2388 rows, 392 -> 2919 20.1 and 18.5; but 2009 rows, 280 -> 143 7.6 and 8.0.
bool even_rows(const LinearParams& p)
{
    const uintptr_t starts = (uintptr_t)p.y | (uintptr_t)p.residual | (uintptr_t)p.gate | 2 * (uintptr_t)(p.y_sb | p.y_sn | p.r_sb | p.r_sn | p.g_sb);
    return starts % 4 == 0 || (long long)p.M * p.N < 1 << 21;
}

template <int MAX_M>
int launch_dot(const LinearParams& p, void* stream)
{
    constexpr int EACH = OUT * DOT_WAVES;
    hipLaunchKernelGGL((linear_dot_kernel<MAX_M>), dim3((unsigned)((p.N + EACH - 1) / EACH)), dim3(DOT_WAVES * 64), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

template <int WR, int FN, bool SPLIT>
int launch_wide(const LinearParams& p, void* stream)
{
    constexpr int TM = 64 * WR, TN = 32 * FN;
    const long long items = (((long long)p.M + TM - 1) / TM) * ((p.N + TN - 1) / TN) * (SPLIT ? p.pieces : 1);
    if (items >= (1LL << 31) - 4096) return RAPID_ERR_SHAPE;
    const long long most = CUS * (4 / WR);
    hipLaunchKernelGGL((linear_wide_kernel<WR, FN, SPLIT, LinearParams>), dim3((unsigned)(items < most ? items : most)), dim3(WR * 128), 0,
                       (hipStream_t)stream, p, (int)items);
    if constexpr (SPLIT) {
        const long long lanes = (long long)p.M * (p.pitch / 8);
        hipLaunchKernelGGL(linear_join_kernel, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, (hipStream_t)stream, p);
    }
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

// ---------------------------------------------------------------------------
// Which tile, and how many pieces along K
// ---------------------------------------------------------------------------
enum Tile { T64x64, T128x128, T256x128, T256x160, T256x192, T256x256, TILES };
struct Plan {
    Tile tile;
    int pieces;
};

// What a product takes, in us.  Its items (tiles times pieces) go to 256 CUs with each slots of them at a time: full rounds, whose
// steps of 64 inputs take `full` each, and a last one whose steps take from `alone` (an item to a CU or less) to `full` (the fullest CU
// counts more than the mean); every round has `ends` (`odd` more where the width is no multiple of eight), every call `call`.
// Pieces are added up by a second kernel, which costs `join` and `sum` for every million numbers that it reads.  Fitted to 1050
// products of 9 to 32768 rows, 16 to 9728 outputs and 64 to 9728 inputs (odd sizes among them), timed in all tiles and 1 to 8
// pieces, inputs changing from call to call: the plan found by it takes 1.01 times what the best one does in the geometric mean.  So it
// does for 700 others of these ranges (1.4 times at most) and for 100 of up to 21504 outputs or inputs (1.15 at most), whose times in
// every form are in profiles/linear_tiles.txt.
struct TileCost {
    int rows, columns, slots;
    float alone, full, ends, odd, call, join, sum;
};
constexpr TileCost COST[TILES] = {
    {64, 64, 4, 0.397f, 0.787f, 1.62f, 1.28f, 2.40f, 2.16f, 1.85f}, {128, 128, 2, 0.507f, 0.936f, 3.39f, 2.15f, 1.79f, 2.72f, 1.24f},
    {256, 128, 1, 0.541f, 0.845f, 3.72f, 2.20f, 2.59f, 0.f, 0.f},   {256, 160, 1, 0.647f, 0.987f, 5.59f, 2.23f, 1.28f, 0.f, 0.f},
    {256, 192, 1, 0.792f, 1.212f, 5.21f, 2.97f, 1.88f, 0.f, 0.f},   {256, 256, 1, 0.996f, 1.537f, 6.63f, 3.56f, 1.80f, 0.f, 0.f}};

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

}  // namespace

extern "C" {

size_t rapid_linear_workspace_bytes(long long M, int N, int K)
{
    if (M <= 0 || M >= (1LL << 31) - 256 || N <= 0 || N > MAX_STRIDE || K <= 0 || K > MAX_STRIDE || K % 8 != 0 || by_dots(M, N, K)) return 0;
    const int pieces = plan_for(M, N, K, MOST_PIECES).pieces;
    return pieces > 1 ? (size_t)pieces * M * ((N + 7) / 8 * 8) * sizeof(float) : 0;
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
    if (B > 1 && (255 / n + 1) * p.x_sb + (long long)(n - 1) * p.x_sn + K > (1LL << 30)) return RAPID_ERR_SHAPE;
    if (y->ptr == x->ptr || y->ptr == w || y->ptr == bias || y->ptr == gate) return RAPID_ERR_ALIAS;
    if (residual && y->ptr == residual->ptr && (p.y_sb != p.r_sb || p.y_sn != p.r_sn)) return RAPID_ERR_ALIAS;
    const size_t need = workspace ? rapid_linear_workspace_bytes(M, N, K) : 0;
    if (workspace && (workspace_bytes < need || !aligned(workspace, 16))) return RAPID_ERR_WORKSPACE;
    p.x = (const __bf16*)x->ptr;
    p.w = (const __bf16*)w;
    p.bias = (const __bf16*)bias;
    p.gate = (const __bf16*)gate;
    p.residual = residual ? (const __bf16*)residual->ptr : nullptr;
    p.y = (__bf16*)y->ptr;
    p.w_sn = (int)w_stride;
    p.g_sb = gs;
    p.M = (int)M;
    p.n = n;
    p.N = N;
    p.K = K;
    p.activation = activation;
    if (B == 1) p.n = p.M;
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
