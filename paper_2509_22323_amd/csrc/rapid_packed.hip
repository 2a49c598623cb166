// Attention of documents packed into one joint sequence, for MI355X (gfx950).  C ABI: include/rapid_packed.h.
#include <hip/hip_runtime.h>
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "rapid_internal.h"
#include "rapid_packed.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f;

struct Side {                                          // of a segment
    const char *q, *k, *v;
    char* o;
    long long in_sb, in_sh, out_sb, out_sh;            // bytes
    int in_sn, out_sn;                                 // bytes
};
struct Known;
struct PackedParams {
    Side side[2];
    const int* document;
    const int* order;                                  // or null
    long long document_sb, order_sb;
    int n0, N, B, H;                                   // tokens of the first segment, of both
    int tiles0, tiles, groups0, groups1;               // tiles of the first segment, of both; groups of 128 queries of each
    Known* known;                                      // [B, tiles]
    int* sorted;                                       // [B, groups], most work first, or null
    int pieces;                                        // of what a group has to do
    float* partial;                                    // [B, H, groups, pieces]: what a piece comes to
    float scale;                                       // of a score, as exponent of 2
    float cap;                                         // as exponent of 2; 0: none
    float share;                                       // of the cap, of a score
    float small, series[5];                            // of a capped score: see series()
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

// tanh(u) / u as a polynomial in u^2, fitted to 1.0e-6 of it up to u = NEAR
constexpr float NEAR = 0.8f;
constexpr double TANH[5] = {0.999998994, -0.33325372, 0.132305656, -0.0491801422, 0.0121001386};

// A value such that nothing made from it is kept in registers over a loop.
template <class T>
__device__ __forceinline__ T here(T v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// The exponent of 2 that a product s = q k stands for: s scale, or cap tanh(u), u = s share.  Of two formulas of the latter, by |u| alone, so that a
// result does not depend on what else a tile holds: the polynomial, or cap - 2 cap / (1 + exp(2 u)), which is off by roundings of the cap.
__device__ __forceinline__ float beyond(float s, float cap, float share)
{
    return __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * share * (2.f * LOG2E))), cap);
}
// |s| <= p.small, the factors of all of it in the polynomial's
__device__ __forceinline__ float series(const PackedParams& p, float s)
{
    const float t = s * s;
    return __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(p.series[4], t, p.series[3]), t, p.series[2]), t, p.series[1]), t, p.series[0]);
}
// any s, where p.small is 0: those factors would not be numbers of fp32
__device__ __forceinline__ float out_of_proportion(float s, float scale, float cap, float share)
{
    const float u = s * share, t = u * u;
    float near = here((float)TANH[4]);
#pragma unroll
    for (int i = 3; i >= 0; --i) near = __builtin_fmaf(near, t, here((float)TANH[i]));
    return fabsf(u) <= NEAR ? s * scale * near : beyond(s, cap, share);
}
__device__ __forceinline__ float exponent(const PackedParams& p, float s)
{
    if (p.cap == 0.f) return s * p.scale;
    if (p.small == 0.f) return out_of_proportion(s, p.scale, p.cap, p.share);
    return fabsf(s) <= p.small ? s * series(p, s) : beyond(s, p.cap, p.share);
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
        const unsigned long long keys = __builtin_amdgcn_ballot_w64(seen);
        if (keys == 0ull) continue;
        const Side& from = p.side[j >= p.n0];
        const char* k = from.k + b * from.in_sb + h * from.in_sh + (long long)(j >= p.n0 ? j - p.n0 : j) * from.in_sn;
        float s = 0.f;
        for (int c = 0; c < D / 8; ++c) {
            const bf16x8 kv = *(const bf16x8*)(k + 16 * c), qv = *(const bf16x8*)(q + 16 * c);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)kv[i], (float)qv[i], s);
        }
        s = exponent(p, s);
        const float higher = fmaxf(m, most_of_lanes(seen ? s : -INFINITY));
        const float lower = m == higher ? 1.f : __builtin_amdgcn_exp2f(m - higher);
        m = higher;
        // (a score of -infinity is a weight of 0, also where there is no other yet)
        const float e = seen ? __builtin_amdgcn_exp2f(s - (m == -INFINITY ? 0.f : m)) : 0.f;
        l = l * lower + sum_of_lanes(e);
#pragma unroll
        for (int i = 0; i < EACH; ++i) acc[i] *= lower;
        if (l != l) break;                             // (so are all of the row's results)
        constexpr int AT_ONCE = 8;                     // whose values are on their way together
        for (int i = 0; i < 64; i += AT_ONCE) {
            if ((keys >> i & 0xffull) == 0ull) continue;
            float value[AT_ONCE][EACH];
#pragma unroll
            for (int c = 0; c < AT_ONCE; ++c) {
                const int key = min(first + i + c, p.N - 1);
                const Side& from = p.side[key >= p.n0];
                const __bf16* v = (const __bf16*)(from.v + b * from.in_sb + h * from.in_sh + (long long)(key >= p.n0 ? key - p.n0 : key) * from.in_sn) + EACH * lane;
#pragma unroll
                for (int j = 0; j < EACH; ++j) value[c][j] = (float)v[j];
            }
#pragma unroll
            for (int c = 0; c < AT_ONCE; ++c) {
                const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(e), i + c));
#pragma unroll
                for (int j = 0; j < EACH; ++j) acc[j] = __builtin_fmaf(by, (keys >> (i + c) & 1ull) != 0ull ? value[c][j] : 0.f, acc[j]);
            }
        }
    }
    __bf16* o = (__bf16*)(at.o + b * at.out_sb + h * at.out_sh + (long long)row * at.out_sn) + EACH * lane;
#pragma unroll
    for (int c = 0; c < EACH; ++c) o[c] = (__bf16)(own >= 0 ? acc[c] / l : 0.f);
}

// ---------------------------------------------------------------------------
// Tiles of 64 tokens, counted within each segment (the last one of a segment may be short).  What is known of a tile:
// ---------------------------------------------------------------------------
constexpr int TILE = 64, ROWS = 128;                   // keys of a tile; queries of a workgroup
constexpr int WAVES = ROWS / 32;

struct Known {
    int first, last;                                   // smallest (~ it: some token is of no document) and largest document; last < 0: none
    int early, late;                                   // smallest and largest order
};
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int smallest(const Known& k) { return k.first < 0 ? ~k.first : k.first; }

template <int CTRL>
__device__ __forceinline__ int moved(int v)
{
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
// f over the values of 8 and of 16 lanes, in each of them
template <class F>
__device__ __forceinline__ int over_8_lanes(int v, F f)
{
    v = f(v, moved<0xB1>(v));                          // lane ^ 1
    v = f(v, moved<0x4E>(v));                          // lane ^ 2
    return f(v, moved<0x141>(v));                      // 7 - lane of every 8
}
template <class F>
__device__ __forceinline__ int over_16_lanes(int v, F f)
{
    v = over_8_lanes(v, f);
    return f(v, moved<0x140>(v));                      // 15 - lane of every 16
}

// Of tiles `tile` .. `tile` + 3 of a sample (the last one again behind it), by a wavefront: lanes 16 i .. 16 i + 15 know of tile + i.
// (16 lanes a tile and four tokens a lane, not 64 lanes a tile: a quarter of the steps between lanes, which bind where a workgroup
// does this alone.)
__device__ __forceinline__ Known known_of(const PackedParams& p, int b, int tile, int lane)
{
    tile = min(tile + (lane >> 4), p.tiles - 1);
    const bool second = tile >= p.tiles0;
    const int row = (second ? tile - p.tiles0 : tile) * TILE + (lane & 15), n = second ? p.N - p.n0 : p.n0;
    const int* const document = p.document + b * p.document_sb + (second ? p.n0 : 0);
    const int* const order = p.order ? p.order + b * p.order_sb + (second ? p.n0 : 0) : nullptr;
    int d[4], o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = min(row + 16 * i, n - 1);
        d[i] = document[t];
        o[i] = order ? order[t] : 0;
    }
    Known k = {INT_MAX, -1, order ? INT_MAX : 0, order ? INT_MIN : 0};
    bool all = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool there = row + 16 * i < n && d[i] >= 0;
        all = all && there;
        if (!there) continue;
        k.first = min(k.first, d[i]);
        k.last = max(k.last, d[i]);
        k.early = min(k.early, o[i]);
        k.late = max(k.late, o[i]);
    }
    auto least = [](int a, int b) { return min(a, b); };
    auto most = [](int a, int b) { return max(a, b); };
    k.first = over_16_lanes(k.first, least);
    k.last = over_16_lanes(k.last, most);
    if (order) {
        k.early = over_16_lanes(k.early, least);
        k.late = over_16_lanes(k.late, most);
    }
    if ((__builtin_amdgcn_ballot_w64(!all) >> (lane & 48) & 0xffffull) != 0ull) k.first = ~k.first;
    return k;
}

enum { NONE, SOME, ALL };
// Whether queries of what is known as q see keys of k.
__device__ __forceinline__ int sees(const Known& q, const Known& k)
{
    const int qf = smallest(q), kf = smallest(k);
    if (q.last < 0 || k.last < 0 || kf > q.last || k.last < qf || k.early > q.late) return NONE;
    return k.first == k.last && qf == q.last && k.first == qf && k.late <= q.early ? ALL : SOME;
}

// What is known of the queries of group `group` (of the tiles in `known`).
__device__ __forceinline__ Known known_of_group(const PackedParams& p, const Known* known, int group)
{
    const bool second = group >= p.groups0;
    const int tile = second ? p.tiles0 + 2 * (group - p.groups0) : 2 * group;
    Known mine = known[tile];
    if (tile + 1 < (second ? p.tiles : p.tiles0)) {
        const Known k = known[tile + 1];
        mine.first = min(smallest(mine), smallest(k));
        mine.last = max(mine.last, k.last);
        mine.early = min(mine.early, k.early);
        mine.late = max(mine.late, k.late);
    }
    return mine;
}

// Tiles that every workgroup looks at itself, before its queries have come; a launch before it takes 3 us: 2 heads of 64, 256 tokens 9.5 us (12.6
// with the launch), 24 of 128, 512 23.8 (26.8), 1024 37.0 (40.1).  More would be a second round of loads in every workgroup.
constexpr int FEW = 16;

// What is known of all tiles, and the groups of a sample in the order of what they have to do, most first: workgroups go to the CUs in
// turn as these get free, so that what is left for last is short.  24 heads of 128, documents of 4608, 1101, 1357 and 376 tokens: 298 us, in the
// order of the sequence 314; where documents are alike it costs up to 3 %: 8200 tokens one by one 407 and 400 us.  Beyond PLANNED
// tiles, which LDS would not hold beside their groups, there are groups enough, and the last ones go first.  A workgroup a sample: 8 us.
constexpr int PLANNED = 1026;
__global__ __launch_bounds__(1024) void packed_plan_kernel(PackedParams p)
{
    __shared__ __align__(16) Known known[PLANNED];
    __shared__ __align__(16) int visits[(PLANNED / 2 + 1 + 3) / 4 * 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = p.groups0 + p.groups1, b = blockIdx.x;
    for (int first = 4 * wave; first < p.tiles; first += 64) {
        const Known k = known_of(p, b, first, lane);
        const int tile = first + (lane >> 4);
        if ((lane & 15) == 0 && tile < p.tiles) {
            known[tile] = k;
            p.known[(long long)b * p.tiles + tile] = k;
        }
    }
    if (tid < 4) visits[per / 4 * 4 + tid] = -1;       // (read in fours)
    __syncthreads();
    for (int first = 0; first < per; first += 128) {   // eight lanes a group
        const int group = min(first + tid / 8, per - 1);
        const Known mine = known_of_group(p, known, group);
        int count = 0;
        for (int tile = tid % 8; tile < p.tiles; tile += 8) count += sees(mine, known[tile]) != NONE;
        count = over_8_lanes(count, [](int a, int b) { return a + b; });
        if (tid % 8 == 0) visits[group] = count;       // (the last one by several, all of which have counted the same)
    }
    __syncthreads();
    for (int group = tid; group < per; group += 1024) {
        int before = 0;
        const int own = visits[group];
#pragma unroll 4
        for (int i = 0; i < per; i += 4) {
            const i32x4 others = *(const i32x4*)(visits + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) before += others[j] > own || (others[j] == own && i + j < group);
        }
        p.sorted[(long long)b * per + before] = group;
    }
}

// What is known of all tiles, four a wavefront.
__global__ __launch_bounds__(256) void packed_known_kernel(PackedParams p)
{
    const int lane = threadIdx.x & 63, first = 4 * (blockIdx.x * 4 + (threadIdx.x >> 6)), tile = first + (lane >> 4);
    const Known k = known_of(p, blockIdx.y, first, lane);
    if ((lane & 15) == 0 && tile < p.tiles) p.known[(long long)blockIdx.y * p.tiles + tile] = k;
}

// ---------------------------------------------------------------------------
// The kernel: a workgroup takes 128 queries of a head, a wavefront 32 of them, and goes over the tiles that one of them sees.
// S^T = K Q^T, one query a lane, and O^T += V^T P^T, v_mfma_f32_16x16x32_bf16; P goes from one product to the next in registers, and
// o = sum p v / sum p with p = 2^(x - m), x the exponents and m a reference that only moves when one is 2^8 above it, so that
// accumulators are rescaled a few times a row.  p is rounded to bf16 for the product, whose operands have as many bits as V has, and the sum is
// of the rounded values, so that no row's weights add up to another number than 1: outputs are 0.0020 to 0.0023 of their size off the exact ones in
// the mean square, of which their own rounding to bf16 is 0.0017.
// Tiles that every query sees whole take no mask at all; others compare the documents and orders that were copied beside their values.
//
// Two tiles of keys and two of values in LDS, copied past the registers a whole step ahead, one barrier a step; in a step the scores of the
// next tile and the sums of this one are matrix instructions, between which the vector work on the weights is dealt out by hand.
// Bound at D = 128 by the matrix pipe and the clock under it: 32 heads of 4096 tokens in 254 to 269 us from card to card (1.08 to 1.02 PFLOP/s), pipe and vector
// units busy half of the cycles each; without the barriers 2 % less time, without exponents 2.5 %.  At D = 64 by the vector instructions, which are the
// same for half the products: 161 to 170 us (0.85 to 0.81 PFLOP/s).  A cap is seven instructions a score more, where its polynomial serves: 322 to 341 us at
// D = 128, 234 to 240 at D = 64 (vector units 87 % busy).  Workgroups a CU: two of 230 registers at D = 128, three of 168 at 64.
// (52 to 64 scalars lie in lanes of vector registers, read back outside the loop but for a few.)
// 256 queries a workgroup at D = 128: 5 % less time for one document, 5 to 18 % more for documents of a few hundred tokens.  64 queries a
// wavefront at D = 64 (half the reads of LDS): 10 % more, with two wavefronts a SIMD for three.
// ---------------------------------------------------------------------------
typedef __attribute__((address_space(3))) char lds_char;

template <int D>
struct Lds {
    static constexpr int RB = D * 2, BYTES = TILE * RB, COPIES = BYTES / 1024 / WAVES, PER = 1024 / RB;     // PER: rows of a copy
    // 16-byte chunks of a row change places by row, so that the 16 rows (K) or 4 x 16 patches (V) that are read at a time lie in different banks
    static __device__ __forceinline__ int turn_k(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
    static __device__ __forceinline__ int turn_v(int row) { return D == 128 ? (row & 7) << 1 : (row >> 1 & 3) << 1; }
    // what PER j rows on change of a chunk's place in bytes, for rows PER j + 0 .. PER - 1 of 16
    static constexpr unsigned next_k(int j) { return 64u * j; }
    static constexpr unsigned next_v(int j) { return D == 128 ? 128u * (j & 1) : 0u; }
};

// 1 KB from 64 lanes' offsets into LDS; 5 wait states behind a vector instruction that wrote the descriptor, one behind the write of M0
template <bool FIRST>
__device__ __forceinline__ void copy_1k(const i32x4& buffer, unsigned off, unsigned dst)
{
    if constexpr (FIRST) asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(dst), "v"(off), "s"(buffer));
    else asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(dst), "v"(off), "s"(buffer));
}

// Everything that this wavefront has requested has arrived, then the barrier; nothing moves across.
__device__ __forceinline__ void arrive()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A tile that is visited: where it lies, and what else is asked of it.
struct Visit {
    unsigned low, high;                                // address of its keys: 48 bits; of `high` bit 31: not every query sees it whole; bit 30: second segment
    int bytes;                                         // from its first to the end of its last row
    int token;                                         // its first one in the joint sequence, and (rows - 1) << 24
};

// What a piece of a group leaves: [ROWS, D], and a number each for the rows
template <int D>
struct Part {
    static constexpr int SUM = ROWS * D, REFERENCE = SUM + ROWS, FLOATS = REFERENCE + ROWS;
};

template <int D, bool CAP>
__global__ __launch_bounds__(WAVES * 64, D == 64 ? 3 : 2) void packed_tiles_kernel(PackedParams p)
{
    typedef Lds<D> L;
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int LIST = 512;                          // tiles that are listed at a time
    __shared__ __align__(1024) char lds[4 * L::BYTES + 4 * TILE * 4];
    __shared__ __align__(16) Visit list[LIST];
    __shared__ int found[WAVES];
    __shared__ int mine_doc[ROWS], mine_turn[ROWS];    // of the queries
    __shared__ Known own_known[FEW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;

    // Which rows: 8 heads at a time, an XCD each, so that an L2 holds the keys and values of few of them; of these the groups with most to
    // do first; the heads that are left over are dealt out to all XCDs.
    const int per = p.groups0 + p.groups1, pairs = p.B * p.H, whole = pairs / 8, rest = pairs % 8;
    const int piece = blockIdx.x / 8 % p.pieces, xcd = blockIdx.x % 8, turn_in = blockIdx.x / 8 / p.pieces;
    int head, rank;
    if (turn_in < whole * per) {
        rank = turn_in / whole;
        head = xcd + 8 * (turn_in - rank * whole);
    } else {
        const int i = (turn_in - whole * per) * 8 + xcd;
        if (i >= rest * per) return;
        rank = i / rest;
        head = 8 * whole + i - rank * rest;
    }
    head = __builtin_amdgcn_readfirstlane(head);
    rank = __builtin_amdgcn_readfirstlane(rank);
    const int b = __builtin_amdgcn_readfirstlane(head / p.H), h = head - b * p.H;
    const int group = p.sorted ? p.sorted[(long long)b * per + rank] : per - 1 - rank;
    const bool second = group >= p.groups0;
    const Side& own = p.side[second];
    const int length = second ? p.N - p.n0 : p.n0, row0 = (second ? group - p.groups0 : group) * ROWS;
    const Known* const known = p.known + (long long)b * p.tiles;
    if (!p.known) {                                    // few tiles: every workgroup looks at them itself, which is faster than a launch before it
        static_assert(FEW == 4 * WAVES, "");
        const Known k = known_of(p, b, 4 * wave, lane);
        if (lane % 16 == 0) own_known[4 * wave + lane / 16] = k;
        __syncthreads();
    }
    const Known mine = p.known ? known_of_group(p, known, group) : known_of_group(p, own_known, group);

    // queries: lane (n, g) holds elements 32 t + 8 g .. + 7 of query 16 q + n
    const int q0 = row0 + 32 * wave;
    bf16x8 qf[2][KS];
    const long long at_in = b * own.in_sb + h * own.in_sh;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int row = min(q0 + 16 * q + n, length - 1);
        const char* from = own.q + at_in + (long long)row * own.in_sn + 16 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[q][k] = *(const bf16x8*)(from + 64 * k);
    }
    if (tid < ROWS) {
        const int t = min(row0 + tid, length - 1) + (second ? p.n0 : 0);
        mine_doc[tid] = p.document[b * p.document_sb + t];
        mine_turn[tid] = p.order ? p.order[b * p.order_sb + t] : 0;
    }

    // copies of a tile: this lane's rows and chunks
    const unsigned lds_at = (unsigned)(size_t)(lds_char*)lds;
    const unsigned crow = wave * L::COPIES * L::PER + lane / (64 / L::PER);
    const int cchunk = lane % (64 / L::PER);
    const unsigned ck = 16u * (cchunk ^ L::turn_k(crow)), cv = 16u * (cchunk ^ L::turn_v(crow));      // of the first copy; the others' differ by L::next_k, next_v
    const unsigned stride0 = p.side[0].in_sn, stride1 = p.side[1].in_sn;
    const long long delta0 = p.side[0].v - p.side[0].k, delta1 = p.side[1].v - p.side[1].k;
    const int* const documents = p.document + b * p.document_sb;
    const int* const orders = p.order ? p.order + b * p.order_sb : nullptr;
    auto copy = [&](const Visit& e, auto is_v, auto slot) {
        constexpr bool V = is_v.value;
        const bool s = (e.high >> 30 & 1) != 0;
        const unsigned sn = s ? stride1 : stride0;
        unsigned long long base = (unsigned long long)(e.high & 0xffffu) << 32 | e.low;
        if constexpr (V) base += (unsigned long long)(s ? delta1 : delta0);
        const i32x4 buffer = {(int)(unsigned)base, (int)((unsigned)(base >> 32) & 0xffffu), e.bytes, 0x00020000};
        const unsigned at = __umul24(crow, sn), chunk = here(V ? cv : ck);
#pragma unroll
        for (int j = 0; j < L::COPIES; ++j) {
            const unsigned off = at + (unsigned)(j * L::PER) * sn + (chunk ^ (V ? L::next_v(j) : L::next_k(j)));
            const unsigned dst = lds_at + slot.value * L::BYTES + (wave * L::COPIES + j) * 1024;
            if (j == 0) copy_1k<true>(buffer, off, dst);
            else copy_1k<false>(buffer, off, dst);
        }
        if constexpr (V) {                             // with the documents and orders of its tokens, 4 bytes a lane
            if ((int)e.high < 0 && wave < 2 && (wave == 0 || orders)) {
                const unsigned long long from = (unsigned long long)((wave == 0 ? documents : orders) + (e.token & 0xffffff));
                const i32x4 words = {__builtin_amdgcn_readfirstlane((int)(unsigned)from), __builtin_amdgcn_readfirstlane((int)((unsigned)(from >> 32) & 0xffffu)),
                                     __builtin_amdgcn_readfirstlane(4 * ((e.token >> 24) + 1)), 0x00020000};
                const unsigned dst = lds_at + 4 * L::BYTES + (2 * (slot.value - 2) + wave) * 4 * TILE, off = 4u * here(lane);
                asm volatile("s_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"{m0}"(dst), "v"(off), "s"(words));
            }
        }
    };

    // fragments in a tile
    unsigned kat[KS], vat[DT];
#pragma unroll
    for (int k = 0; k < KS; ++k) kat[k] = n * L::RB + (((4 * k + g) ^ L::turn_k(n)) << 4);
    const int vrow = 4 * g + (n >> 2);
#pragma unroll
    for (int d = 0; d < DT; ++d) vat[d] = vrow * L::RB + (((2 * d + ((n & 3) >> 1)) ^ L::turn_v(vrow)) << 4) + (n & 1) * 8;

    f32x4 acc[DT][2] = {};
    float sums[2] = {};                                // of this lane's weights
    float m[2] = {-1e30f, -1e30f};
    bool partly = false;
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
    typedef __attribute__((address_space(3))) const i32x4 lds_i32x4;
    typedef __attribute__((address_space(3))) i32x4 lds_i32x4_out;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const float scale = p.scale, cap = p.cap;

    auto scores = [&](auto slot, f32x4 (&s)[4][2]) {
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8 kf = *(lds_bf16x8*)((lds_char*)lds + slot.value * L::BYTES + kt * 16 * L::RB + kat[k]);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
                    s[kt][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[q][k], k == 0 ? none : s[kt][q], 0, 0, 0);
                }
            }
        }
    };
    auto mask = [&](const Visit& e, auto slot, f32x4 (&s)[4][2]) {
        const int own_lane = here(lane), n = own_lane & 15, g = own_lane >> 4;
        lds_char* const at = (lds_char*)lds + 4 * L::BYTES + 2 * slot.value * 4 * TILE + 16 * g;
        const int doc[2] = {mine_doc[32 * wave + n], mine_doc[32 * wave + 16 + n]}, turn[2] = {mine_turn[32 * wave + n], mine_turn[32 * wave + 16 + n]};
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const i32x4 d = *(lds_i32x4*)(at + 64 * kt);
            // Values of no document: zeros, before this wavefront reads them (others write the same), so that what padding holds costs nothing.
            if (__builtin_amdgcn_ballot_w64(min(min(d[0], d[1]), min(d[2], d[3])) < 0) != 0ull) {
                const int row = here(own_lane), none = here(0);
                lds_char* const to = (lds_char*)lds + (2 + slot.value) * L::BYTES + (16 * kt + 4 * (row >> 4)) * L::RB + 16 * (row & 15);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (d[r] < 0 && (row & 15) < D / 8) *(lds_i32x4_out*)(to + r * L::RB) = i32x4{none, none, none, none};
            }
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[kt][q][r] = d[r] == doc[q] ? s[kt][q][r] : -INFINITY;
        }
        if (orders) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                const i32x4 o = *(lds_i32x4*)(at + 4 * TILE + 64 * kt);
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[kt][q][r] = o[r] <= turn[q] ? s[kt][q][r] : -INFINITY;
            }
        }
        const int left = (e.token >> 24) + 1 - 4 * g;  // (rows that the tile does not have have come as zeros)
        if ((e.token >> 24) != TILE - 1) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[kt][q][r] = 16 * kt + r < left ? s[kt][q][r] : -INFINITY;
        }
    };
    auto each = [](auto a, auto b, auto&& f) {         // f with the numbers a .. b - 1 as constants
        auto go = [&](auto self, auto i) {
            if constexpr (i.value < b.value) {
                f(i);
                self(self, std::integral_constant<int, i.value + 1>());
            }
        };
        go(go, a);
    };
    auto largest = [&](const f32x4 (&s)[4][2], int q) {
        float v = s[0][q][0];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) v = fmaxf(v, s[kt][q][r]);
        return v;
    };
    float most[2];                                     // of this lane's scores of a tile
    constexpr std::integral_constant<int, 0> zero;
    constexpr std::integral_constant<int, 1> one;
    constexpr std::integral_constant<int, 2> two;
    constexpr std::integral_constant<int, 3> three;
    constexpr std::true_type values;
    constexpr std::false_type keys;
    // The weights of a tile whose scores are s, and what they add, beside the scores of the next one.  Items: one operand from LDS, requested
    // AHEAD items before, and the matrix instructions of both groups of queries; behind each a quarter or two of the work on a pair of weights.
    auto step = [&](const Visit& e, f32x4 (&s)[4][2], f32x4 (&next)[4][2], auto slot) {
        constexpr int T = slot.value;                  // K of this tile in slot T, V in slot 2 + T
        // (a bound on a capped tile's scores is at hand with the choice of its formula, so their maximum is looked for only where that is too large)
        bool look = true;
        if constexpr (CAP) {                           // (before the mask: what is hidden is not -cap)
            float size = 0.f;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int r = 0; r < 4; ++r) size = fmaxf(size, fabsf(s[kt][q][r]));
            const bool all_small = __builtin_amdgcn_ballot_w64(size > p.small) == 0ull;
            if (__builtin_expect(all_small, 1)) {
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[kt][q][r] *= series(p, s[kt][q][r]);
                size *= series(p, size);
            } else if (p.small != 0.f) {
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float x = s[kt][q][r];
                            s[kt][q][r] = fabsf(x) <= p.small ? x * series(p, x) : beyond(x, cap, p.share);
                        }
                size = cap;
            } else {
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[kt][q][r] = out_of_proportion(s[kt][q][r], scale, cap, p.share);
                size = cap;
            }
            look = __builtin_amdgcn_ballot_w64(size > fminf(m[0], m[1]) + 8.f) != 0ull;
        }
        if ((int)e.high < 0) {
            mask(e, slot, s);
            partly = true;
        }
        if ((int)e.high < 0 || (CAP && look)) {
#pragma unroll
            for (int q = 0; q < 2; ++q) most[q] = largest(s, q);
        }
        // a score far above the reference of its query: the reference moves up to the largest
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if constexpr (!CAP) most[q] *= scale;
        if (look && __builtin_amdgcn_ballot_w64(most[0] > m[0] + 8.f || most[1] > m[1] + 8.f) != 0ull) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float top = fmaxf(most[q], __shfl_xor(most[q], 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                top = fmaxf(top, m[q]);
                const float lower = __builtin_amdgcn_exp2f(m[q] - top);
                m[q] = top;
                sums[q] *= lower;
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d][q] *= lower;
            }
        }
        // Items 0 .. QK - 1: scores of the next tile (behind the last one: of what is there, which nobody looks at); QK .. : of 32 keys each,
        // what the weights add.  Pairs of weights 0 .. 7 of the first 32 keys, 8 .. 15 of the others, each before the items that take them.
        constexpr int QK = 4 * KS, PV = DT, ALL = QK + 2 * PV, AHEAD = D == 64 ? 1 : 3, EARLY = 40;
        bf16x8 f[AHEAD + 1];
        unsigned w[2][2][4];
        float x0, x1, e0, e1;
        auto request = [&](auto item) {
            constexpr int I = item.value;
            if constexpr (I < QK) {
                f[I % (AHEAD + 1)] = *(lds_bf16x8*)((lds_char*)lds + (1 - T) * L::BYTES + (I % 4) * 16 * L::RB + kat[I / 4]);
            } else {
                lds_char* v = (lds_char*)lds + (2 + T) * L::BYTES + ((I - QK) / PV) * 32 * L::RB + vat[(I - QK) % PV];
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)v), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v + 16 * L::RB));
                f[I % (AHEAD + 1)] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        // a quarter of the work on a pair: exponents, first and second weight, both as bf16
        auto quarter = [&](auto unit) {
            constexpr int P = unit.value / 4, part = unit.value % 4, half = P / 8, q = P % 8 / 4, i = P % 4;
            if constexpr (part == 0) {
                const float a = s[2 * half + i / 2][q][2 * (i % 2)], b = s[2 * half + i / 2][q][2 * (i % 2) + 1];
                x0 = CAP ? a - m[q] : __builtin_fmaf(a, scale, -m[q]);
                x1 = CAP ? b - m[q] : __builtin_fmaf(b, scale, -m[q]);
            } else if constexpr (part == 1) {
                e0 = __builtin_amdgcn_exp2f(x0);
            } else if constexpr (part == 2) {
                e1 = __builtin_amdgcn_exp2f(x1);
            } else {
                const bf16x2 both = {(__bf16)e0, (__bf16)e1};
                const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
                w[half][q][i] = __builtin_bit_cast(unsigned, both);
                sums[q] = __builtin_amdgcn_fdot2_f32_bf16(both, ones, sums[q], false);
            }
        };
        each(zero, std::integral_constant<int, AHEAD>(), request);
        each(zero, std::integral_constant<int, ALL>(), [&](auto item) {
            constexpr int I = item.value, half = I < QK + PV ? 0 : 1;
            if constexpr (I + AHEAD < ALL) request(std::integral_constant<int, I + AHEAD>());
            each(zero, two, [&](auto query) {
                constexpr int q = query.value, at = 2 * I + q;     // matrix instructions before this one
                if constexpr (I < QK) {
                    constexpr int kt = I % 4, k = I / 4;
                    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
                    next[kt][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[I % (AHEAD + 1)], qf[q][k], k == 0 ? none : next[kt][q], 0, 0, 0);
                } else {
                    constexpr int d = (I - QK) % PV;
                    const bf16x8 by = __builtin_bit_cast(bf16x8, w[half][q]);
                    acc[d][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[I % (AHEAD + 1)], by, acc[d][q], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                constexpr int M = 2 * QK, H = 2 * PV;
                constexpr int from = at < M ? at * EARLY / M : at < M + H ? EARLY + (at - M) * (64 - EARLY) / H : 64;
                constexpr int upto = at < M ? (at + 1) * EARLY / M : at < M + H ? EARLY + (at + 1 - M) * (64 - EARLY) / H : 64;
                each(std::integral_constant<int, from>(), std::integral_constant<int, upto>(), quarter);
                if constexpr (!CAP && I == ALL - 2) most[q] = largest(next, q);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };

    const int tiles = p.tiles;
    for (int from = 0; from < tiles; from += LIST) {
        // the tiles that someone here sees, in order
        const int upto = min(tiles - from, LIST);
        int count = 0;
        for (int i = 0; i < upto; i += WAVES * 64) {
            const int at = i + here(tid), tile = from + at, how = at < upto ? sees(mine, p.known ? known[tile] : own_known[tile % FEW]) : NONE;
            const unsigned long long some = __builtin_amdgcn_ballot_w64(how != NONE);
            __syncthreads();
            if (lane == 0) found[wave] = __popcll(some);
            __syncthreads();
            int before = count;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) before += found[w];
                count += found[w];
            }
            if (how != NONE) {
                const bool s = tile >= p.tiles0;
                const Side& of = p.side[s];
                const int row = (s ? tile - p.tiles0 : tile) * TILE, rows = min((s ? p.N - p.n0 : p.n0) - row, TILE);
                const unsigned long long at = (unsigned long long)(of.k + b * of.in_sb + h * of.in_sh + (long long)row * of.in_sn);
                list[before + __popcll(some & ((1ull << lane) - 1ull))] = Visit{
                    (unsigned)at, (unsigned)(at >> 32 & 0xffffu) | (how == SOME ? 1u << 31 : 0u) | (s ? 1u << 30 : 0u),
                    (rows - 1) * of.in_sn + L::RB, (s ? p.n0 : 0) + row | (rows - 1) << 24};
            }
        }
        __syncthreads();
        const int first = count * piece / p.pieces;
        count = __builtin_amdgcn_readfirstlane(count * (piece + 1) / p.pieces - first);
        if (count == 0) continue;
        auto visit = [&](int i) {
            const Visit e = list[first + i];
            return Visit{(unsigned)__builtin_amdgcn_readfirstlane(e.low), (unsigned)__builtin_amdgcn_readfirstlane(e.high),
                         __builtin_amdgcn_readfirstlane(e.bytes), __builtin_amdgcn_readfirstlane(e.token)};
        };
        // K: slots 0 and 1, V: slots 2 and 3
        f32x4 even[4][2], odd[4][2];
        Visit now = visit(0), then = count > 1 ? visit(1) : now;
        copy(now, keys, zero);
        copy(now, values, two);
        if (count > 1) copy(then, keys, one);
        arrive();
        // (zeros for queries of no document: what they hold is not to move the references of others)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (mine_doc[32 * wave + 16 * q + (here(lane) & 15)] < 0)
#pragma unroll
                for (int k = 0; k < KS; ++k) qf[q][k] = bf16x8{};
        scores(zero, even);
#pragma unroll
        for (int q = 0; q < 2; ++q) most[q] = largest(even, q);
        __syncthreads();
        for (int i = 0;; i += 2) {
            // K_{i+1} and V_i are there, and nobody reads K_i and V_{i-1} any more
            Visit later = then;
            if (i + 2 < count) {
                later = visit(i + 2);
                copy(later, keys, zero);
            }
            if (i + 1 < count) copy(then, values, three);
            step(now, even, odd, zero);
            if (i + 1 >= count) break;
            arrive();
            now = later;
            if (i + 3 < count) {
                later = visit(i + 3);
                copy(later, keys, one);
            }
            if (i + 2 < count) copy(now, values, two);
            step(then, odd, even, one);
            if (i + 2 >= count) break;
            arrive();
            then = later;
        }
        arrive();                                      // before the list and the slots serve the next tiles
    }

    const int end_lane = here(lane), end_n = end_lane & 15, end_g = end_lane >> 4;       // (not kept over the loop)
    float sum[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        sum[q] = sums[q] + __shfl_xor(sums[q], 16, 64);
        sum[q] += __shfl_xor(sum[q], 32, 64);
    }
    if (p.pieces > 1) {                                // this piece's part: sums of V under the weights, of the weights, and their reference
        typedef Part<D> P;
        float* const part = p.partial + (((long long)head * per + group) * p.pieces + piece) * P::FLOATS;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int row = 32 * wave + 16 * q + end_n;
#pragma unroll
            for (int d = 0; d < DT; ++d) *(f32x4*)(part + row * D + 16 * d + 4 * end_g) = acc[d][q];
            if (end_g == 0) {
                part[P::SUM + row] = sum[q];
                part[P::REFERENCE + row] = m[q];
            }
        }
        return;
    }

    // Results.  A weight of 0 times an infinity or NaN in a tile that not every query sees whole is NaN: such rows again, key by key.  So
    // are rows without a weight: no exponent of theirs is above the -1e30 that the references begin with.
    unsigned again = 0;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int row = q0 + 16 * q + end_n;
        const bool some = mine_doc[32 * wave + 16 * q + end_n] >= 0;
        const float inverse = 1.f / sum[q];
        float all = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) all = __builtin_fmaf(acc[d][q][r], 0.f, all);
        const unsigned long long bad = __builtin_amdgcn_ballot_w64((sum[q] == 0.f || (partly && all != 0.f)) && row < length && some);
        const unsigned rows = (unsigned)(bad | bad >> 16 | bad >> 32 | bad >> 48) & 0xffffu;
        again |= rows << (16 * q);
        if (row >= length || (rows >> end_n & 1) != 0) continue;
        char* o = own.o + b * own.out_sb + h * own.out_sh + (long long)row * own.out_sn + 8 * end_g;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            bf16x4 out;
#pragma unroll
            for (int r = 0; r < 4; ++r) out[r] = (__bf16)(some ? acc[d][q][r] * inverse : 0.f);
            *(bf16x4*)(o + 32 * d) = out;
        }
    }
    again = __builtin_amdgcn_readfirstlane(again);
    while (again != 0) {
        int sample = b;                                // (its addresses are not to be kept over the loop above)
        asm volatile("" : "+s"(sample));
        const int i = __builtin_ctz(again);
        again &= again - 1;
        row_by_keys<D>(p, sample, h, q0 + i + (second ? p.n0 : 0), end_lane);
    }
}

// The pieces of the groups' rows in their order: D / 4 lanes a row, four elements each.
template <int D>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedParams p)
{
    typedef Part<D> P;
    constexpr int LANES = D / 4, EACH = 256 / LANES;
    const int per = p.groups0 + p.groups1, lane = threadIdx.x % LANES, parts = ROWS / EACH;
    const int item = blockIdx.x / parts, in = (int)(blockIdx.x % parts) * EACH + threadIdx.x / LANES;
    const int head = item / per, group = item - head * per, b = head / p.H, h = head - b * p.H;
    const bool second = group >= p.groups0;
    const int row = (second ? group - p.groups0 : group) * ROWS + in, length = second ? p.N - p.n0 : p.n0, t = min(row, length - 1) + (second ? p.n0 : 0);
    const bool some = p.document[b * p.document_sb + t] >= 0;
    const float* const part = p.partial + (long long)item * p.pieces * P::FLOATS;
    float top = -1e30f;
    for (int i = 0; i < p.pieces; ++i) top = fmaxf(top, part[i * P::FLOATS + P::REFERENCE + in]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (int i = 0; i < p.pieces; ++i) {
        const float* const from = part + i * P::FLOATS;
        const float by = __builtin_amdgcn_exp2f(from[P::REFERENCE + in] - top);
        acc += by * *(const f32x4*)(from + in * D + 4 * lane);
        sum += by * from[P::SUM + in];
    }
    const float inverse = 1.f / sum;
    float all = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) all = __builtin_fmaf(acc[r], 0.f, all);
    // (rows that are not finite or have no weight again, key by key, as above)
    unsigned long long bad = __builtin_amdgcn_ballot_w64((all != 0.f || sum == 0.f) && row < length && some);
    const int first = threadIdx.x / 64 * (64 / LANES), own = threadIdx.x % 64 / LANES;
    const unsigned long long mine = (LANES == 32 ? 0xffffffffull : 0xffffull) << (own * LANES);
    if (row < length && (bad & mine) == 0ull) {
        const Side& to = p.side[second];
        bf16x4 out;
#pragma unroll
        for (int r = 0; r < 4; ++r) out[r] = (__bf16)(some ? acc[r] * inverse : 0.f);
        *(bf16x4*)(to.o + b * to.out_sb + h * to.out_sh + (long long)row * to.out_sn + 8 * lane) = out;
    }
    while (bad != 0ull) {
        const int i = __builtin_ctzll(bad) / LANES;    // of the wavefront's rows
        bad &= ~((LANES == 32 ? 0xffffffffull : 0xffffull) << (i * LANES));
        const int row_again = (second ? group - p.groups0 : group) * ROWS + (int)(blockIdx.x % parts) * EACH + first + i;
        row_by_keys<D>(p, b, h, row_again + (second ? p.n0 : 0), threadIdx.x % 64);
    }
}

// Into how many pieces the tiles of every group are cut where the groups do not fill the card (a tile of a workgroup that has a CU to itself takes
// 1.3 us, most of it waiting): as many as make 512 workgroups, of four tiles at least, or 768 of twelve, of groups that see all of the sequence
// (the host does not know the documents).  us, whole / cut, one document, one head of
// 64 1000 tokens 26.9 / 16.2, 8000 172.8 / 43.4; five 4000 92.2 / 42.6, 8000 178.8 / 110.3; two of 128 1000 34.3 / 20.2, 4000 113.2 / 40.9 (into twelve
// 48.5); eight of 128 2000 63.6 / 41.8 (768 workgroups of five tiles 47.5), 4000 116.0 / 76.0 (512 of 31 tiles 82.8).  Groups of short
// documents see few tiles, most of their pieces none, and the parts and the join cost 4 to 25 us more than they save: documents of
// 128 tokens, 1000 tokens in all, two heads of 64 8.5 / 12.5, of 128 10.7 / 15.4; 8000 16.1 / 30.9, 18.7 / 43.5; documents of 1024 tokens 28.6 / 33.7
// and 36.1 / 50.7 there, but 21.3 / 15.6 and 28.2 / 19.6 of 1000 in all.  (Pieces of four tiles that the
// group sees, the others not written and not joined, on another card: 22 to 39 us for documents of 128 tokens among 4608 and 8000, but 12.5 became
// 13.4 and 15.4 15.8, and one document takes 3 to 8 % more.)
int pieces_for(long long groups, long long tiles)
{
    constexpr long long MOST = 8;
    auto least = [](long long a, long long b) { return a < b ? a : b; };
    const long long some = least(512 / groups, tiles / 4), more = least(768 / groups, tiles / 12), pieces = least(some > more ? some : more, MOST);
    return pieces < 2 ? 1 : (int)pieces;
}

// The workspace: what is known of the tiles, the groups in order, the pieces
struct Space {
    size_t sorted, partial, bytes;
};
Space space_of(int B, int H, long long tiles, long long groups, int D, int pieces)
{
    Space s;
    s.sorted = (size_t)B * tiles * sizeof(Known);
    s.partial = s.sorted + ((size_t)B * groups * sizeof(int) + 15) / 16 * 16;
    s.bytes = s.partial + (pieces > 1 ? (size_t)B * H * groups * pieces * sizeof(float) * (D == 64 ? Part<64>::FLOATS : Part<128>::FLOATS) : 0);
    return s;
}

// (a launch has less than 2^32 lanes)
inline bool too_large(int B, int H, long long N) { return (long long)B * H * ((N + ROWS - 1) / ROWS + 1) >= (1LL << 24) - 16; }

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

extern "C" {

size_t rapid_attn_packed_workspace_bytes(int B, int H, int N, int D)
{
    if (B <= 0 || H <= 0 || N <= 0 || N > (1 << 22) || (long long)B * H > 524287 || too_large(B, H, N) || (D != 64 && D != 128)) return 0;
    const long long tiles = (N + TILE - 1) / TILE + 1, groups = (N + ROWS - 1) / ROWS + 1;         // (one more where there are two segments)
    const Space s = space_of(B, H, tiles, groups, D, pieces_for((long long)B * H * (groups - 1), tiles));
    const Space whole = space_of(B, H, tiles, groups, D, 1);
    return s.bytes > whole.bytes ? s.bytes : whole.bytes;
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
            if (s[0] < 0 || s[0] > (1LL << 40) || s[1] < 0 || s[1] > (1LL << 40) || s[2] < D || s[2] >= (1 << 23)) return RAPID_ERR_SHAPE;
            if ((s[0] | s[1] | s[2]) % 8 != 0) return RAPID_ERR_ALIGN;
        }
        if (!aligned(g.q, 16) || !aligned(g.k, 16) || !aligned(g.v, 16) || !aligned(g.o, 16)) return RAPID_ERR_ALIGN;
        p.side[i] = {(const char*)g.q, (const char*)g.k, (const char*)g.v, (char*)g.o, 2 * in[0], 2 * in[1], 2 * out[0], 2 * out[1], (int)(2 * in[2]), (int)(2 * out[2])};
    }
    if (N > (1 << 22) || too_large(B, H, N)) return RAPID_ERR_SHAPE;
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
    // (numbers of fp32, whatever cap and scale: a product of 0 has the exponent 0; a cap that is cut is cut for its share of a score, too)
    scale = fminf(scale, FLT_MAX / LOG2E);
    cap = fminf(cap, FLT_MAX / 4 / LOG2E);
    p.scale = fminf(scale * LOG2E, FLT_MAX);
    p.cap = cap * LOG2E;
    p.share = cap > 0.f ? fminf(scale / cap, FLT_MAX) : 0.f;
    // The series' factors, cap u^(2 i + 1), are numbers of fp32 for all but caps and scales out of proportion to each other or to 1.
    const double u = p.share;
    if (u > 0x1p-12 && u < 0x1p12) {
        p.small = (float)(NEAR / u);
        for (int i = 0; i < 5; ++i) {
            p.series[i] = (float)(TANH[i] * p.cap * pow(u, 2 * i + 1));
            if (isinf(p.series[i])) p.small = 0.f;
        }
    }
    const int n1 = p.N - p.n0;
    p.tiles0 = (p.n0 + TILE - 1) / TILE;
    p.tiles = p.tiles0 + (n1 + TILE - 1) / TILE;
    p.groups0 = (p.n0 + ROWS - 1) / ROWS;
    p.groups1 = (n1 + ROWS - 1) / ROWS;
    const int per = p.groups0 + p.groups1, pairs = B * H;
    p.pieces = pieces_for((long long)pairs * per, p.tiles);
    const Space space = space_of(B, H, p.tiles, per, D, p.pieces);
    p.partial = (float*)((char*)workspace + space.partial);
    p.known = p.tiles <= FEW ? nullptr : (Known*)workspace;
    if (!p.known) {
    } else if (p.tiles <= PLANNED) {
        p.sorted = (int*)((char*)workspace + space.sorted);
        hipLaunchKernelGGL(packed_plan_kernel, dim3((unsigned)B), dim3(1024), 0, (hipStream_t)stream, p);
    } else {
        hipLaunchKernelGGL(packed_known_kernel, dim3((unsigned)((p.tiles + 15) / 16), (unsigned)B), dim3(256), 0, (hipStream_t)stream, p);
    }
    const dim3 grid(8u * (unsigned)(pairs / 8 * per + (pairs % 8 * per + 7) / 8) * (unsigned)p.pieces);
    auto kernel = D == 64 ? cap > 0.f ? packed_tiles_kernel<64, true> : packed_tiles_kernel<64, false>
                          : cap > 0.f ? packed_tiles_kernel<128, true> : packed_tiles_kernel<128, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(WAVES * 64), 0, (hipStream_t)stream, p);
    if (p.pieces > 1) {
        const int lanes = D / 4;
        hipLaunchKernelGGL(D == 64 ? packed_join_kernel<64> : packed_join_kernel<128>, dim3((unsigned)(pairs * per) * (unsigned)(ROWS * lanes / 256)),
                           dim3(256), 0, (hipStream_t)stream, p);
    }
    return hipGetLastError() == hipSuccess ? RAPID_OK : RAPID_ERR_DEVICE;
}

}  // extern "C"
