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

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f;

template <int CTRL>
__device__ __forceinline__ float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// The sum over the wavefront, in every lane.
__device__ __forceinline__ float sum_of_lanes(float v)
{
    v += moved<0xB1>(v);                               // lane ^ 1
    v += moved<0x4E>(v);                               // lane ^ 2
    v += moved<0x141>(v);                              // 7 - lane of every 8
    v += moved<0x140>(v);                              // 15 - lane of every 16
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

struct LinearParams {
    const __bf16* x;
    const __bf16* w;
    const __bf16* bias;
    const __bf16* gate;
    const __bf16* residual;
    __bf16* y;
    long long x_sb, y_sb, r_sb, g_sb;
    int x_sn, y_sn, r_sn, w_sn;
    int M, n, N, K;          // M rows in samples of n (n = M where samples make no difference)
    int activation;
    int pieces, pitch;       // a product in pieces along K: how many, and floats from row to row of their sums
    float* partial;          // [pieces, M, pitch]
    bool even;               // 16 bytes an access in the epilogue, see even_rows
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
    constexpr float C = 1.5957691216057308f * LOG2E;
    const float e = activation == RAPID_ACT_SILU ? -LOG2E * z : z * __builtin_fmaf(z * z, -0.044715f * C, -C);
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(e));
}

// What the epilogue adds and multiplies, and writes, eight outputs at a time.  Rows of odd widths start anywhere; an access of 16 bytes is
// as fast at any multiple of four, but takes twice as long and more at odd numbers of elements (75 MB written by 8192 rows of 4608: 32 us
// and 55), where it is made in pieces instead: the first element, three pairs and the last one (43 us).
typedef bf16x8 bf16x8_anywhere __attribute__((aligned(2)));
typedef bf16x4 bf16x4_anywhere __attribute__((aligned(2)));
typedef unsigned u32_alias __attribute__((may_alias));
typedef unsigned short u16_alias __attribute__((may_alias));

__device__ __forceinline__ bool odd(const __bf16* at, bool even) { return !even && ((uintptr_t)at & 2) != 0; }

// Eight elements as they were loaded: the four pairs, or the three inner ones, the first and the last element.
struct Loaded {
    unsigned d[5];
};
__device__ __forceinline__ Loaded loaded(const __bf16* at, bool even)
{
    Loaded v;
    if (odd(at, even)) {
        const u32_alias* inner = (const u32_alias*)(at + 1);
        v.d[0] = inner[0];
        v.d[1] = inner[1];
        v.d[2] = inner[2];
        v.d[3] = *(const u16_alias*)at;
        v.d[4] = *(const u16_alias*)(at + 7);
    } else {
        const u32x4 pairs = __builtin_bit_cast(u32x4, (bf16x8)*(const bf16x8_anywhere*)at);
        v.d[0] = pairs[0];
        v.d[1] = pairs[1];
        v.d[2] = pairs[2];
        v.d[3] = pairs[3];
        v.d[4] = 0;
    }
    return v;
}
__device__ __forceinline__ bf16x8 eight(const Loaded& v, bool odd)
{
    const unsigned d0 = odd ? v.d[0] << 16 | v.d[3] : v.d[0], d1 = odd ? __builtin_amdgcn_alignbit(v.d[1], v.d[0], 16) : v.d[1];
    const unsigned d2 = odd ? __builtin_amdgcn_alignbit(v.d[2], v.d[1], 16) : v.d[2], d3 = odd ? v.d[4] << 16 | v.d[2] >> 16 : v.d[3];
    return __builtin_bit_cast(bf16x8, (u32x4){d0, d1, d2, d3});
}
__device__ __forceinline__ void store(__bf16* at, bf16x8 v, bool even)
{
    if (odd(at, even)) {
        const u32x4 d = __builtin_bit_cast(u32x4, v);
        const unsigned d0 = d[0], d1 = d[1], d2 = d[2], d3 = d[3];
        u32_alias* inner = (u32_alias*)(at + 1);
        inner[0] = __builtin_amdgcn_alignbit(d1, d0, 16);
        inner[1] = __builtin_amdgcn_alignbit(d2, d1, 16);
        inner[2] = __builtin_amdgcn_alignbit(d3, d2, 16);
        *(u16_alias*)at = (unsigned short)d0;
        *(u16_alias*)(at + 7) = (unsigned short)(d3 >> 16);
    } else {
        *(bf16x8_anywhere*)at = v;
    }
}

// Outputs j .. j + 7 of a row, or as many as there are (what the others hold is not used)
__device__ __forceinline__ Loaded loaded(const __bf16* at, int j, int N, bool even)
{
    if (j + 8 <= N) return loaded(at + j, even);
    unsigned e[8] = {};
#pragma unroll
    for (int i = 0; i < 7; ++i) e[i] = ((const u16_alias*)at)[min(j + i, N - 1)];
    Loaded v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.d[i] = e[2 * i] | e[2 * i + 1] << 16;
    v.d[4] = 0;
    return v;
}
__device__ __forceinline__ bf16x8 eight(const Loaded& v, const __bf16* at, int j, int N, bool even)
{
    return eight(v, odd(at + j, even) && j + 8 <= N);
}
__device__ __forceinline__ bf16x8 eight_of(const __bf16* at, int j, int N, bool even) { return eight(loaded(at, j, N, even), at, j, N, even); }
__device__ __forceinline__ void store_eight(__bf16* at, int j, int N, bf16x8 v, bool even)
{
    if (j + 8 <= N) { store(at + j, v, even); return; }
    const u32x4 d = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const unsigned two = d[i / 2];
        if (j + i < N) ((u16_alias*)at)[j + i] = (unsigned short)(i % 2 ? two >> 16 : two);
    }
}

// residual + gate * act(sum), everything in fp32, rounded once.  (What is not there is skipped by scalar branches.)
__device__ __forceinline__ bf16x8 finished(const LinearParams& p, float (&z)[8], bf16x8 gate, bf16x8 residual)
{
    if (p.activation != RAPID_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = activated(z[i], p.activation);
    }
    if (p.gate) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= (float)gate[i];
    }
    if (p.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += (float)residual[i];
    }
    bf16x8 out;
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = (__bf16)z[i];
    return out;
}

// ---------------------------------------------------------------------------
// Tiles: 64*WR x 32*FN outputs per workgroup of 2*WR wavefronts (WR along the rows of x, two along those of w; a wavefront has
// 64 x 16*FN), 64 inputs per step.  The operands change places, A = rows of w and B = rows of x, so that a lane ends with four outputs of a
// row side by side.  Copies go from memory into LDS past the registers, two or three steps ahead, one barrier a step; workgroups
// stay and go on to their next item, whose first steps are on their way before the results of the last one are written.
//
// Bound by the matrix pipe and the clock it leaves: 8192 rows, 9728 -> 2432 (388 GFLOP, tile 256 x 160) takes 291 to 320 us from card to
// card (1.33 to 1.21 PFLOP/s), the pipe busy 70 to 72 % of the cycles; on the card where it takes 291 the same loop takes 264 without
// copies, 250 without reads of LDS, 234 without either, 285 without the barrier.
// 8192 rows, 1536 -> 4608 (116 GFLOP, 256 x 192): 98 to 104 us, of which the ends of tiles are a sixth.  Measured and not taken: other
// orders of tiles (GROUP 2, 6, 8, 16), weights past the caches, touching the next steps in the L2 first, 128 x 64 outputs a wavefront
// with four wavefronts, all copies in a step's first half, priorities of waves, five steps in LDS for the small tiles: none faster over
// products of 64 to 8192 rows, most 1 to 20 % slower.
// ---------------------------------------------------------------------------
constexpr int STEP = 64;                               // inputs per step: 128 bytes of a row
constexpr int ROW = STEP * 2;
constexpr int CUS = 256;
constexpr int MOST_PIECES = 8;                         // along K
constexpr unsigned NOWHERE = 0xC0000000u;              // an offset outside any buffer below
constexpr unsigned BUFFER = 0x81000000u;               // bytes that a tile's rows may span, and the inputs of a row

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

// 1 KB from 64 lanes' addresses into LDS: lane i's 16 bytes go to dst + 1024 C + 16 i.  (The instruction's offset counts on both
// sides: LESS is taken off the lanes' offsets.)  Assembly, so that only the waits below order it; a wait state between the scalar
// write of M0 and the copy.
constexpr unsigned LESS = 3 * 1024;
template <int C>
__device__ __forceinline__ void copy_1k(const i32x4& buffer, unsigned off, int at, unsigned dst)
{
    static_assert(C >= 0 && C < 4, "an offset of 12 bits");
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen offset:%4 lds" ::"{m0}"(dst), "v"(off), "s"(buffer), "s"(at), "i"(1024 * C));
}
__device__ __forceinline__ i32x4 buffer_at(const void* p)
{
    const unsigned long long base = (unsigned long long)p - LESS;
    return i32x4{(int)(unsigned)base, (int)((unsigned)(base >> 32) & 0xffffu), (int)BUFFER, 0x00020000};
}

// s_waitcnt vmcnt(VM) lgkmcnt(0), then the barrier; nothing moves across.
template <int VM>
__device__ __forceinline__ void arrive()
{
    static_assert(VM >= 0 && VM < 64, "vmcnt is a 6-bit counter");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0070 | (VM & 15) | ((VM >> 4) << 14));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Workgroups go to the XCDs in turn; every XCD gets a run of consecutive items.
__device__ __forceinline__ int turn_of(int id, int items)
{
    constexpr int XCDS = 8;
    const int x = id % XCDS, each = items / XCDS, more = items % XCDS;
    return x * each + min(x, more) + id / XCDS;
}
// Consecutive tiles: GROUP of them along the rows of x, then along the rows of w, so that what an L2 holds is used by many.
__device__ __forceinline__ void tile_of(int t, int mt, int nt, int& m, int& n)
{
    constexpr int GROUP = 4;
    const int run = t / (GROUP * nt), in = t - run * GROUP * nt, rows = min(GROUP, mt - run * GROUP);
    n = in / rows;
    m = run * GROUP + in - n * rows;
}

// A pointer into the GPU's memory (and not to LDS, which nothing says of one that is read from an argument block)
template <typename T>
__device__ __forceinline__ T* in_memory(T* p)
{
    return (T*)(__attribute__((address_space(1))) T*)(uintptr_t)p;
}

template <int WR, int FN, bool SPLIT>
__global__ __launch_bounds__(WR * 128, 2) void linear_wide_kernel(LinearParams p, int items)
{
    constexpr int FM = 4, TM = 64 * WR, TN = 32 * FN, WAVES = 2 * WR, PER_CU = 4 / WR;
    constexpr int XB = TM * ROW, WB = TN * ROW;                       // bytes of a step
    // Steps in LDS: three of both operands where they fit, else of the one that comes from further away: x where tiles are large
    // (many rows; all of them use w at the same time), w where they are small.
    constexpr bool BOTH = 3 * (XB + WB) <= 160 * 1024 / PER_CU;
    constexpr int XS = BOTH || WR == 4 ? 3 : 2, WS = BOTH || WR < 4 ? 3 : 2, MOST = 3;
    static_assert(XS * XB + WS * WB <= 160 * 1024 / PER_CU, "");
    constexpr int XC = TM / 8 / WAVES, WC = TN / 8 / WAVES, WREST = TN / 8 % WAVES;    // copies of a wavefront: of x; of w, and one more for some
    constexpr int WALL = WC + (WREST ? 1 : 0);
    // The copies are spread over the two halves of a step (a CU's memory pipeline takes 16 cycles for each): those of the deeper
    // buffer, for two steps on, go with the first half, the other operand's with the second.
    constexpr bool X_FIRST = XS == 3;
    constexpr int FIRST = X_FIRST ? XC : WALL, SECOND = X_FIRST ? WALL : XC;
    constexpr int XA = X_FIRST ? 2 : XS, WA = X_FIRST ? WS : 2;       // steps ahead at which x and w are copied
    constexpr int LATE = BOTH ? XC + WC : X_FIRST ? XC : WC;          // copies that may be on their way yet when a step begins
    __shared__ __align__(1024) char lds[XS * XB + WS * WB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool one = p.n == p.M;
    const int wfirst = wave * WC + min(wave, WREST);                  // copies of w: WC + 1 of the first WREST wavefronts
    const int mt = (p.M + TM - 1) / TM, nt = (p.N + TN - 1) / TN, all_steps = (p.K + STEP - 1) / STEP;

    // Where the tile's copies come from.  Its first sample is the base of its x rows (its first row where there is one sample).
    int m0, j0, b0, piece = 0, first = 0, steps = max(all_steps, MOST);
    // Rows lie a multiple of many memory channels apart, so the same step of all of them lies in few channels: every XCD begins
    // at another step and comes round to those before it (its workgroups stay together, they share what its L2 holds).
    const int turn = !SPLIT && all_steps >= 8 && p.K % STEP == 0 ? (int)(blockIdx.x % 8) * all_steps / 8 : 0;
    const bool ragged = p.K % STEP != 0 || all_steps < MOST;
    i32x4 xbuffer, wbuffer;
    int xk, wk;                                        // bytes of a row before the step that is copied next
    unsigned xoff[XC], woff[WALL];
    auto locate = [&](int id) {
        int mi, ni, t = turn_of(id, items);
        if constexpr (SPLIT) {
            piece = __builtin_amdgcn_readfirstlane(t / (mt * nt));
            t -= piece * mt * nt;
            first = __builtin_amdgcn_readfirstlane(piece * all_steps / p.pieces);
            steps = max(__builtin_amdgcn_readfirstlane((piece + 1) * all_steps / p.pieces) - first, MOST);
        }
        tile_of(t, mt, nt, mi, ni);
        m0 = __builtin_amdgcn_readfirstlane(mi) * TM;
        j0 = __builtin_amdgcn_readfirstlane(ni) * TN;
    };
    // The arguments read again, and the lane's number, such that nothing made from them is kept in registers over the loops (scalar
    // ones that do not fit go to lanes of vector registers, and back in every step).
    auto arguments = [] {
        auto at = __builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(at));
        struct Words {
            unsigned long long word[sizeof(LinearParams) / 8];
        } words;
#pragma unroll
        for (unsigned i = 0; i < sizeof(LinearParams) / 8; ++i) words.word[i] = ((const __attribute__((address_space(4))) unsigned long long*)at)[i];
        LinearParams p = __builtin_bit_cast(LinearParams, words);
        p.bias = in_memory(p.bias);
        p.gate = in_memory(p.gate);
        p.residual = in_memory(p.residual);
        p.y = in_memory(p.y);
        p.partial = in_memory(p.partial);
        return p;
    };
    auto lane_here = [&] {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    // A row's 16-byte chunk c lies at c ^ (row / 2 % 8), so that the 16 rows that are read at a time are in different banks: the
    // chunk that a lane fetches in the copy of rows 8 i .. 8 i + 7.
    auto chunk_of = [](int lane, int i) { return (lane & 7) ^ ((i & 1) << 2 | lane >> 4); };
    auto sources_x = [&] {
        int r0;
        const int lane = lane_here();
        const LinearParams p = arguments();
        sample_of(p, m0, b0, r0);
        b0 = __builtin_amdgcn_readfirstlane(b0);
        r0 = __builtin_amdgcn_readfirstlane(r0);
        xbuffer = buffer_at(p.x + b0 * p.x_sb + (one ? (long long)r0 * p.x_sn : 0));
        xk = (first + turn) * ROW;
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            int b, r;
            sample_of(p, min(m0 + (wave * XC + i) * 8 + (lane >> 3), p.M - 1), b, r);
            xoff[i] = (unsigned)(b - b0) * (unsigned)(p.x_sb * 2) + (unsigned)(one ? r - r0 : r) * (unsigned)(p.x_sn * 2) + chunk_of(lane, wave * XC + i) * 16u + (LESS - 1024u * i);
        }
    };
    auto sources_w = [&] {
        const int lane = lane_here();
        const LinearParams p = arguments();
        wbuffer = buffer_at(p.w + (long long)j0 * p.w_sn);
        wk = (first + turn) * ROW;
#pragma unroll
        for (int i = 0; i < WALL; ++i)
            woff[i] = (unsigned)min((wfirst + i) * 8 + (lane >> 3), p.N - 1 - j0) * (unsigned)(p.w_sn * 2) + chunk_of(lane, wfirst + i) * 16u + (LESS - 1024u * i);
    };
    auto mask = [&](int k, int i, auto& off) {         // zeros for what lies behind the rows' ends (i: the first copy)
        const int left = 2 * p.K - k;
        if (left >= ROW) return;
        const int lane = lane_here();
        for (unsigned& o : off)
            if (chunk_of(lane, i++) * 16 >= left) o = NOWHERE;
    };
    static_assert(XC <= 4 && WALL <= 4, "");
    const unsigned lds_at = (unsigned)(size_t)(lds_char*)lds, xdst = lds_at + wave * XC * 1024, wdst = lds_at + XS * XB + wfirst * 1024;
    auto copy_x = [&](int slot, auto c) { copy_1k<c.value>(xbuffer, xoff[c.value], xk, xdst + slot); };
    auto copy_w = [&](int slot, auto c) {
        if (c.value < WC || wave < WREST) copy_1k<c.value>(wbuffer, woff[c.value], wk, wdst + slot);
    };
    auto on = [&](int& k) {                            // round to the item's first step behind its last
        k += ROW;
        k = k == (first + steps) * ROW ? first * ROW : k;
    };

    // Fragments: lane (i, g) of 16 x 4 has row i's inputs 8 g .. 8 g + 7 of 32; the second half of a step is 64 bytes on.
    const int wm = wave >> 1, wn = wave & 1;
    const unsigned in_row = (unsigned)((lane & 15) * ROW + (((lane >> 4) ^ (lane >> 1 & 7)) << 4));
    const unsigned xat = in_row + wm * (16 * FM * ROW), wat = in_row + XS * XB + wn * (16 * FN * ROW);
    bf16x8 xf[2][FM], wf[2][FN];
    auto fetch_one = [&](int xslot, int wslot, int half, int r, bf16x8 (&x)[FM], bf16x8 (&w)[FN]) {
        if (r < FM) x[r] = *(lds_bf16x8*)((lds_char*)lds + xslot + (xat ^ (half * 64)) + r * 16 * ROW);
        else w[r - FM] = *(lds_bf16x8*)((lds_char*)lds + wslot + (wat ^ (half * 64)) + (r - FM) * 16 * ROW);
    };
    f32x4 acc[FN][FM];
    // Calls f with the numbers A .. B - 1 as constants.
    auto each = [](auto a, auto b, auto&& f) {
        auto go = [&](auto self, auto i) {
            if constexpr (i.value < b.value) {
                f(i);
                self(self, std::integral_constant<int, i.value + 1>());
            }
        };
        go(go, a);
    };
    // Half a step: FN blocks of FM MFMAs, each behind its share of the reads for the next half and of the copies for a step
    // to come.
    auto half_step = [&](const bf16x8 (&x)[FM], const bf16x8 (&w)[FN], auto&& read, auto copies, auto&& put) {
        constexpr int READS = FM + FN, READING = FN > 2 ? FN - 2 : 1, COPIES = copies.value;    // the last blocks' MFMAs cover the last reads
        each(std::integral_constant<int, 0>(), std::integral_constant<int, FN>(), [&](auto block) {
            constexpr int i = block.value;
#pragma unroll
            for (int r = i * READS / READING; r < (i + 1) * READS / READING && r < READS; ++r) read(r);
            each(std::integral_constant<int, i * COPIES / FN>(), std::integral_constant<int, (i + 1) * COPIES / FN>(), put);
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[i], x[j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // A lane's sums begin with the bias of its four columns of each fragment.
    bf16x4 bias[FN] = {};
    auto load_bias = [&] {
        const int n = j0 + wn * 16 * FN + 4 * (lane_here() >> 4);
        const LinearParams p = arguments();
        if (SPLIT || p.bias == nullptr) return;
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            if (j0 + TN <= p.N) {
                bias[i] = *(const bf16x4_anywhere*)(p.bias + n + 16 * i);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) bias[i][q] = p.bias[min(n + 16 * i + q, p.N - 1)];
            }
        }
    };

    int id = blockIdx.x;
    locate(id);
    load_bias();
    sources_x();
    sources_w();
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        if (i < XA) {
            if (ragged) mask(xk, wave * XC, xoff);
            each(std::integral_constant<int, 0>(), std::integral_constant<int, XC>(), [&](auto c) { copy_x(i * XB, c); });
            on(xk);
        }
        if (i < WA) {
            if (ragged) mask(wk, wfirst, woff);
            each(std::integral_constant<int, 0>(), std::integral_constant<int, WALL>(), [&](auto c) { copy_w(i * WB, c); });
            on(wk);
        }
    }
    arrive<XC + WC + (BOTH ? WC : 0)>();               // (all but the steps behind the first)
    bool stored = false;
    for (int xslot = 0, wslot = 0;;) {
#pragma unroll
        for (int r = 0; r < FM + FN; ++r) fetch_one(xslot, wslot, 0, r, xf[0], wf[0]);
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i][j][q] = (float)bias[i][q];
        const int mw = m0 + wm * 16 * FM, nw = j0 + wn * 16 * FN, first_sample = b0, own_piece = piece, tile_first = m0, tile_right = j0 + TN;
        const bool more = id + (int)gridDim.x < items;
        const int length = steps;
        // A step's buffer is free once its second half is in registers; behind the last steps follow the first ones of this
        // workgroup's next item, or nothing (a buffer without bytes).
        for (int left = steps; left > 0; --left) {
            if (left <= MOST) {
                if (left == (XA > WA ? XA : WA) && more) {
                    id += gridDim.x;
                    locate(id);
                }
                if (left == XA) {
                    if (more) sources_x();
                    else xbuffer[2] = 0;
                }
                if (left == WA) {
                    if (more) sources_w();
                    else wbuffer[2] = 0;
                }
            }
            if (ragged) {
                mask(xk, wave * XC, xoff);
                mask(wk, wfirst, woff);
            }
            const int before = X_FIRST ? (xslot == 0 ? (XS - 1) * XB : xslot - XB) : (wslot == 0 ? (WS - 1) * WB : wslot - WB);
            half_step(xf[0], wf[0], [&](int r) { fetch_one(xslot, wslot, 1, r, xf[1], wf[1]); }, std::integral_constant<int, FIRST>(), [&](auto c) {
                if constexpr (X_FIRST) copy_x(before, c);
                else copy_w(before, c);
            });
            // Everyone has read this step, and the next one has arrived.  (Behind an item's results everything is awaited: stores
            // are counted too.)
            if (left < length || !stored) arrive<LATE>();
            else arrive<0>();
            const int xfree = xslot, wfree = wslot;
            xslot = xslot == (XS - 1) * XB ? 0 : xslot + XB;
            wslot = wslot == (WS - 1) * WB ? 0 : wslot + WB;
            half_step(xf[1], wf[1], [&](int r) { fetch_one(xslot, wslot, 0, r, xf[0], wf[0]); }, std::integral_constant<int, SECOND>(), [&](auto c) {
                if constexpr (X_FIRST) copy_w(wfree, c);
                else copy_x(xfree, c);
            });
            asm volatile("" ::: "memory");
            on(xk);
            on(wk);
        }

        const int lane = lane_here();
        const LinearParams p = arguments();
        if constexpr (SPLIT) {                         // this piece's sums, as they are
            const int n = nw + 4 * (lane >> 4);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int m = mw + 16 * j + (lane & 15);
                float* at = p.partial + ((long long)own_piece * p.M + m) * p.pitch + n;
#pragma unroll
                for (int i = 0; i < FN; ++i)
                    if (m < p.M && n + 16 * i < p.pitch) *(f32x4*)(at + 16 * i) = acc[i][j];
            }
        } else {
        // Pairs of fragments trade rows of lanes, so that a lane has eight consecutive outputs of a row: of (a, b) the lanes of
        // rows 0, 2 get a's 0..7 and 8..15, those of rows 1, 3 b's.  Fragments side by side; of an odd number the last ones in
        // pairs below each other.
        const bool one_sample = one || min(tile_first + TM, p.M) <= (first_sample + 1) * p.n;
        const int g = lane >> 4;
        constexpr int SIDE = FN / 2, UNITS = FM * SIDE, ALL = UNITS + (FN % 2) * FM / 2;
        auto row = [&](int u) { return mw + 16 * (u < UNITS ? u / SIDE : 2 * (u - UNITS) + (g & 1)) + (lane & 15); };
        auto column = [&](int u) { return nw + (u < UNITS ? 32 * (u % SIDE) + (g & 1) * 16 : 16 * (FN - 1)) + (g >> 1) * 8; };
        // Whole: eight outputs or none wherever a lane writes.  Even: 16 bytes an access.
        // Single: one sample.  Bare: neither activation, gate nor residual.  Most tiles need the first two forms alone, which are
        // short (one form for all cases, 7000 instructions long: 7 us a tile of 256 x 192).
        auto results = [&](auto whole, auto even, auto single, auto bare) {
            constexpr bool WHOLE = whole.value, EVEN = even.value, SINGLE = single.value, BARE = bare.value;
            auto of = [&](int m, const __bf16* t, long long sb, int sn) {   // row m of a tensor
                int b = first_sample, r = m - first_sample * p.n;
                if (!SINGLE && !one_sample) sample_of(p, m, b, r);
                return t + b * sb + (long long)r * sn;
            };
            typedef std::conditional_t<EVEN, bf16x8, Loaded> Eight;
            auto load = [&](const __bf16* at, int n) {
                if constexpr (EVEN) return (bf16x8)*(const bf16x8_anywhere*)(at + n);
                else if constexpr (WHOLE) return loaded(at + n, false);
                else return loaded(at, n, p.N, p.even);
            };
            auto value = [&](const Eight& v, const __bf16* at, int n) {
                if constexpr (EVEN) return v;
                else if constexpr (WHOLE) return eight(v, odd(at, false));
                else return eight(v, at, n, p.N, p.even);
            };
            // residuals on their way, and gates where a tile has several (as many as there are registers for)
            constexpr int MOST_AHEAD = EVEN ? FN == 8 ? 4 : 6 : FN == 8 ? 1 : 3, AHEAD = ALL < MOST_AHEAD ? ALL : MOST_AHEAD;
            bf16x8 gate[SIDE + 1] = {};
            Eight residuals[AHEAD] = {}, gates[SINGLE ? 1 : AHEAD] = {};
            auto load_ahead = [&](int u) {
                const int m = row(u), n = column(u);
                if (m >= p.M || n >= p.N) return;
                if (p.residual) residuals[u % AHEAD] = load(of(m, p.residual, p.r_sb, p.r_sn), n);
                if (!SINGLE && p.gate && !one_sample) gates[u % AHEAD] = load(of(m, p.gate, p.g_sb, 0), n);
            };
            if constexpr (!BARE) {
                if (p.gate && one_sample) {
#pragma unroll
                    for (int c = 0; c < SIDE + FN % 2; ++c) {
                        const int n = column(c < SIDE ? c : UNITS);
                        if (n < p.N) gate[c] = eight_of(p.gate + first_sample * p.g_sb, n, p.N, p.even);
                    }
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) load_ahead(u);
            }
#pragma unroll
            for (int u = 0; u < ALL; ++u) {
                const int i = u < UNITS ? 2 * (u % SIDE) : FN - 1, j = u < UNITS ? u / SIDE : 2 * (u - UNITS);
                const f32x4 a = acc[i][j], b = u < UNITS ? acc[i + 1][j] : acc[i][j + 1];
                float z[8];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[q]), __float_as_uint(b[q]), false, false);
                    z[q] = __uint_as_float(both[0]);
                    z[4 + q] = __uint_as_float(both[1]);
                }
                const int m = row(u), n = column(u);
                bf16x8 out;
                if constexpr (BARE) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) out[q] = (__bf16)z[q];
                } else {
                    bf16x8 by = gate[u < UNITS ? u % SIDE : SIDE];
                    bf16x8 residual = {};
                    if (p.residual) residual = value(residuals[u % AHEAD], of(m, p.residual, p.r_sb, p.r_sn), n);
                    if (!SINGLE && p.gate && !one_sample) by = value(gates[u % AHEAD], of(m, p.gate, p.g_sb, 0), n);
                    out = finished(p, z, by, residual);
                    if (u + AHEAD < ALL) load_ahead(u + AHEAD);
                }
                if (u == ALL / 2 && more) load_bias();     // (half of the sums' registers are free)
                if (m < p.M && n < p.N) {
                    __bf16* y = (__bf16*)of(m, p.y, p.y_sb, p.y_sn);
                    if constexpr (EVEN) *(bf16x8_anywhere*)(y + n) = out;
                    else if constexpr (WHOLE) store(y + n, out, false);
                    else store_eight(y, n, p.N, out, p.even);
                }
            }
        };
        constexpr std::true_type yes;
        constexpr std::false_type no;
        const bool cut = p.N % 8 != 0 && tile_right > p.N, bare_call = p.activation == RAPID_ACT_NONE && !p.gate && !p.residual;
        if (__builtin_expect(p.even && one_sample && !cut, 1)) {
            if (bare_call) results(yes, yes, yes, yes);
            else results(yes, yes, yes, no);
        } else if (cut || !(one_sample || p.even)) results(no, no, no, no);
        else if (one_sample) results(yes, no, yes, no);
        else results(yes, yes, no, no);
        }
        if (!more) break;
        stored = true;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last copies, of nothing, write zeros: not into another workgroup's LDS
}

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
    hipLaunchKernelGGL((linear_wide_kernel<WR, FN, SPLIT>), dim3((unsigned)(items < most ? items : most)), dim3(WR * 128), 0,
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

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr long long MAX_STRIDE = 1LL << 22;            // elements, of a row

// Strides of dimensions of size 1 replaced by what changes no address; false: out of range.
bool rows_ok(const rapid_rows& a, int B, int n, int width, bool written, long long& sb, int& row_stride)
{
    const long long sn = n == 1 ? width : a.stride_n;
    sb = B == 1 ? 0 : a.stride_b;
    row_stride = (int)sn;
    if (sn < 0 || sn > MAX_STRIDE || sb < 0 || sb > (1LL << 40)) return false;
    if (!written) return true;
    // apart: rows behind each other and samples behind each other, or samples within the rows' distance (sb <= sn <= 2^22 there:
    // of larger ones a product by B could leave 64 bits)
    if (n > 1 && B > 1) return (sn >= width && sb >= (n - 1) * sn + width) || (sb >= width && sb <= sn && sn >= (B - 1) * sb + width);
    return n > 1 ? sn >= width : B == 1 || sb >= width;
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
