// Products of rows in tiles of matrix instructions, y = residual + gate * act(x w^T + bias): of bf16 (rapid_linear.hip) and of 8-bit integers
// with scales (rapid_linear8.hip).
#ifndef RAPID_WIDE_H
#define RAPID_WIDE_H

#include "rapid_tiles.h"

namespace {

// A product of rows of T
template <class T>
struct ProductParams {
    typedef T Type;
    const T* x;
    const T* w;
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
typedef ProductParams<__bf16> LinearParams;
struct Linear8Params : ProductParams<signed char> {
    const float* x_scale;    // [M]
    const float* w_scale;    // [N]
    const int* document;     // [M], or null: the rows of the gate
    int documents;
};

// The sample and row of row m.
template <class P>
__device__ __forceinline__ void sample_of(const P& p, int m, int& b, int& r)
{
    if (p.n == p.M) { b = 0; r = m; return; }
    b = (int)((unsigned)m / (unsigned)p.n);
    r = m - b * p.n;
}

// Products of whole numbers: the sum is exact, and behind it every rounding is written down here, so that no kernel's compiler joins a
// multiplication and an addition that another's leaves apart: the same row gives the same bits in all of them.
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale, float bias) { return __builtin_fmaf((float)sum * x_scale, w_scale, bias); }
__device__ __forceinline__ float ended(float z, float gate, float residual) { return __builtin_fmaf(z, gate, residual); }

// residual + gate * act(sum), everything in fp32, rounded once.  (What is not there is skipped by scalar branches.)
template <class P>
__device__ __forceinline__ bf16x8 finished(const P& p, float (&z)[8], bf16x8 gate, bf16x8 residual)
{
    if (p.activation != RAPID_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = activated(z[i], p.activation);
    }
    if constexpr (std::is_same_v<P, Linear8Params>) {
        bf16x8 out;
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (__bf16)ended(z[i], p.gate ? (float)gate[i] : 1.f, p.residual ? (float)residual[i] : 0.f);
        return out;
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
// The ends of tiles keep lane masks of all their units at once, of which some go to lanes of vector registers and back: 8 to 31 scalars in bf16
// (435 v_readlane among 14416 instructions at 128 x 128), 18 to 113 in 8 bits, but 596 at 128 x 128, with 7160 v_readlane among 23139
// instructions: tiles that end slower than they could.
// Of 8-bit integers, 128 inputs a step, the same copies feed twice the products: 8192 x 8192 x 8192 405 us (2.72 P/s; the matrix library's
// plain product 450), 9728 -> 2432 with gate and residual 195 to 203 us, pipe busy 57 %, 1536 -> 4608 60 to 66, 47 %: twelve steps a tile, then
// scales, bias and 75 MB of results.
// ---------------------------------------------------------------------------
constexpr int ROW = 128;                               // bytes of a row per step
template <class T>
constexpr int INPUTS = ROW / (int)sizeof(T);           // of a step

template <int WR, int FN, bool SPLIT, class P>
__global__ __launch_bounds__(WR * 128, 2) void linear_wide_kernel(P p, int items)
{
    typedef typename P::Type T;
    constexpr bool WHOLES = std::is_same_v<T, signed char>;           // products of whole numbers: sums in 32 bits, scales behind them
    constexpr int SIZE = sizeof(T), STEP = INPUTS<T>;
    typedef std::conditional_t<WHOLES, i32x4, bf16x8> Operand;
    typedef std::conditional_t<WHOLES, i32x4, f32x4> Sum;
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
            unsigned long long word[sizeof(P) / 8];
        } words;
#pragma unroll
        for (unsigned i = 0; i < sizeof(P) / 8; ++i) words.word[i] = ((const __attribute__((address_space(4))) unsigned long long*)at)[i];
        P p = __builtin_bit_cast(P, words);
        p.bias = in_memory(p.bias);
        p.gate = in_memory(p.gate);
        p.residual = in_memory(p.residual);
        p.y = in_memory(p.y);
        p.partial = in_memory(p.partial);
        if constexpr (WHOLES) {
            p.x_scale = in_memory(p.x_scale);
            p.w_scale = in_memory(p.w_scale);
            p.document = in_memory(p.document);
        }
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
        const P p = arguments();
        sample_of(p, m0, b0, r0);
        b0 = __builtin_amdgcn_readfirstlane(b0);
        r0 = __builtin_amdgcn_readfirstlane(r0);
        xbuffer = buffer_at(p.x + b0 * p.x_sb + (one ? (long long)r0 * p.x_sn : 0));
        xk = (first + turn) * ROW;
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            int b, r;
            sample_of(p, min(m0 + (wave * XC + i) * 8 + (lane >> 3), p.M - 1), b, r);
            xoff[i] = (unsigned)(b - b0) * (unsigned)(p.x_sb * SIZE) + (unsigned)(one ? r - r0 : r) * (unsigned)(p.x_sn * SIZE) + chunk_of(lane, wave * XC + i) * 16u + (LESS - 1024u * i);
        }
    };
    auto sources_w = [&] {
        const int lane = lane_here();
        const P p = arguments();
        wbuffer = buffer_at(p.w + (long long)j0 * p.w_sn);
        wk = (first + turn) * ROW;
#pragma unroll
        for (int i = 0; i < WALL; ++i)
            woff[i] = (unsigned)min((wfirst + i) * 8 + (lane >> 3), p.N - 1 - j0) * (unsigned)(p.w_sn * SIZE) + chunk_of(lane, wfirst + i) * 16u + (LESS - 1024u * i);
    };
    auto mask = [&](int k, int i, auto& off) {         // zeros for what lies behind the rows' ends (i: the first copy)
        const int left = SIZE * p.K - k;
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
    Operand xf[2][FM], wf[2][FN];
    auto fetch_one = [&](int xslot, int wslot, int half, int r, Operand (&x)[FM], Operand (&w)[FN]) {
        typedef __attribute__((address_space(3))) const Operand lds_operand;
        if (r < FM) x[r] = *(lds_operand*)((lds_char*)lds + xslot + (xat ^ (half * 64)) + r * 16 * ROW);
        else w[r - FM] = *(lds_operand*)((lds_char*)lds + wslot + (wat ^ (half * 64)) + (r - FM) * 16 * ROW);
    };
    Sum acc[FN][FM];
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
    auto half_step = [&](const Operand (&x)[FM], const Operand (&w)[FN], auto&& read, auto copies, auto&& put) {
        constexpr int READS = FM + FN, READING = FN > 2 ? FN - 2 : 1, COPIES = copies.value;    // the last blocks' MFMAs cover the last reads
        each(std::integral_constant<int, 0>(), std::integral_constant<int, FN>(), [&](auto block) {
            constexpr int i = block.value;
#pragma unroll
            for (int r = i * READS / READING; r < (i + 1) * READS / READING && r < READS; ++r) read(r);
            each(std::integral_constant<int, i * COPIES / FN>(), std::integral_constant<int, (i + 1) * COPIES / FN>(), put);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                if constexpr (WHOLES) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
                else acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[i], x[j], acc[i][j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // A lane's sums begin with the bias of its four columns of each fragment (of whole numbers with nothing).
    bf16x4 bias[FN] = {};
    auto load_bias = [&] {
        const int n = j0 + wn * 16 * FN + 4 * (lane_here() >> 4);
        const P p = arguments();
        if (WHOLES || SPLIT || p.bias == nullptr) return;
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
                for (int q = 0; q < 4; ++q) acc[i][j][q] = WHOLES ? 0 : (float)bias[i][q];
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
        const P p = arguments();
        if constexpr (SPLIT) {                         // this piece's sums, as they are
            const int n = nw + 4 * (lane >> 4);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int m = mw + 16 * j + (lane & 15);
                float* at = p.partial + ((long long)own_piece * p.M + m) * p.pitch + n;
#pragma unroll
                for (int i = 0; i < FN; ++i)
                    if (m < p.M && n + 16 * i < p.pitch) *(Sum*)(at + 16 * i) = acc[i][j];
            }
        } else {
        // Pairs of fragments trade rows of lanes, so that a lane has eight consecutive outputs of a row: of (a, b) the lanes of
        // rows 0, 2 get a's 0..7 and 8..15, those of rows 1, 3 b's.  Fragments side by side; of an odd number the last ones in
        // pairs below each other.
        bool one_sample = one || min(tile_first + TM, p.M) <= (first_sample + 1) * p.n;
        if constexpr (WHOLES) one_sample = one_sample && !p.document;
        const int g = lane >> 4;
        constexpr int SIDE = FN / 2, UNITS = FM * SIDE, ALL = UNITS + (FN % 2) * FM / 2;
        // (Of whole numbers column by column, as their scales are read; else row by row.)
        auto down = [](int u) { return WHOLES ? u % FM : u / SIDE; };
        auto across = [](int u) { return WHOLES ? u / FM : u % SIDE; };
        auto row = [&](int u) { return mw + 16 * (u < UNITS ? down(u) : 2 * (u - UNITS) + (g & 1)) + (lane & 15); };
        auto column = [&](int u) { return nw + (u < UNITS ? 32 * across(u) + (g & 1) * 16 : 16 * (FN - 1)) + (g >> 1) * 8; };
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
            constexpr int MOST_AHEAD = EVEN ? FN == 8 ? (WHOLES ? 2 : 4) : 6 : FN == 8 ? 1 : 3, AHEAD = ALL < MOST_AHEAD ? ALL : MOST_AHEAD;
            bf16x8 gate[SIDE + 1] = {};
            Eight residuals[AHEAD] = {}, gates[SINGLE ? 1 : AHEAD] = {};
            // of whole numbers: the scales and documents of this lane's rows, and the scales and bias of a column of units, the next one under
            // way where there are registers for it
            constexpr int HELD = FN == 8 ? 1 : 2;
            constexpr int MINE = WHOLES ? FM + FN % 2 * FM / 2 : 1;
            float x_scale[MINE] = {};
            int document[MINE] = {};
            f32x4 w_scale[HELD][2] = {};
            bf16x8 added[HELD] = {};
            auto of_row = [](int u) { return u < UNITS ? u % FM : FM + u - UNITS; };
            auto load_column = [&](const auto& p, int c) {
                const int n = column(c < SIDE ? c * FM : UNITS);
                if (n >= p.N) return;
                if (WHOLE || n + 8 <= p.N) {
                    typedef f32x4 f32x4_anywhere __attribute__((aligned(4)));
                    w_scale[c % HELD][0] = *(const f32x4_anywhere*)(p.w_scale + n);
                    w_scale[c % HELD][1] = *(const f32x4_anywhere*)(p.w_scale + n + 4);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q) w_scale[c % HELD][q / 4][q % 4] = p.w_scale[min(n + q, p.N - 1)];
                }
                if (p.bias) added[c % HELD] = eight_of(p.bias, n, p.N, p.even);
            };
            if constexpr (WHOLES) {
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    const int m = min(row(i < FM ? i : UNITS + i - FM), p.M - 1);
                    x_scale[i] = p.x_scale[m];
                    if (!SINGLE && p.document) document[i] = p.document[m];
                }
                load_column(p, 0);
            }
            // where the gate of row m begins, and whether the row is written
            [[maybe_unused]] auto gate_of = [&](const auto& p, int u, int m) {
                if constexpr (WHOLES && !SINGLE) {
                    if (p.document) {
                        const int d = document[of_row(u)];
                        return p.gate + ((unsigned)d < (unsigned)p.documents ? d : 0) * p.g_sb;
                    }
                }
                return of(m, p.gate, p.g_sb, 0);
            };
            [[maybe_unused]] auto written = [&](const auto& p, int u) {
                if constexpr (WHOLES && !SINGLE) return !p.document || (unsigned)document[of_row(u)] < (unsigned)p.documents;
                else return true;
            };
            auto load_ahead = [&](int u) {
                const int m = row(u), n = column(u);
                if (m >= p.M || n >= p.N) return;
                if (p.residual) residuals[u % AHEAD] = load(of(m, p.residual, p.r_sb, p.r_sn), n);
                if constexpr (WHOLES) {
                    if (!SINGLE && p.gate && !one_sample) gates[u % AHEAD] = load(gate_of(p, u, m), n);
                } else if (!SINGLE && p.gate && !one_sample) gates[u % AHEAD] = load(of(m, p.gate, p.g_sb, 0), n);
            };
            if constexpr (!BARE) {
                if (p.gate && one_sample) {
#pragma unroll
                    for (int c = 0; c < SIDE + FN % 2; ++c) {
                        const int n = column(c < SIDE ? (WHOLES ? c * FM : c) : UNITS);
                        if (n < p.N) gate[c] = eight_of(p.gate + first_sample * p.g_sb, n, p.N, p.even);
                    }
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) load_ahead(u);
            }
#pragma unroll
            for (int u = 0; u < ALL; ++u) {
                const int i = u < UNITS ? 2 * across(u) : FN - 1, j = u < UNITS ? down(u) : 2 * (u - UNITS);
                const Sum a = acc[i][j], b = u < UNITS ? acc[i + 1][j] : acc[i][j + 1];
                float z[8];
                if constexpr (WHOLES) {
                    const float by = x_scale[of_row(u)];
                    const int c = u < UNITS ? across(u) : SIDE;
                    if (HELD == 2 && u % FM == 0 && u < UNITS && c + 1 < SIDE + FN % 2) load_column(p, c + 1);
                    if (HELD == 1 && u % FM == 0 && c > 0) load_column(p, c);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        auto both = __builtin_amdgcn_permlane16_swap(a[q], b[q], false, false);
                        z[q] = scaled((int)both[0], by, w_scale[c % HELD][0][q], p.bias ? (float)added[c % HELD][q] : 0.f);
                        z[4 + q] = scaled((int)both[1], by, w_scale[c % HELD][1][q], p.bias ? (float)added[c % HELD][4 + q] : 0.f);
                    }
                } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[q]), __float_as_uint(b[q]), false, false);
                    z[q] = __uint_as_float(both[0]);
                    z[4 + q] = __uint_as_float(both[1]);
                }
                }
                const int m = row(u), n = column(u);
                bf16x8 out;
                if constexpr (BARE) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) out[q] = (__bf16)z[q];
                } else {
                    bf16x8 by = gate[u < UNITS ? across(u) : SIDE];
                    bf16x8 residual = {};
                    if (p.residual) residual = value(residuals[u % AHEAD], of(m, p.residual, p.r_sb, p.r_sn), n);
                    if constexpr (WHOLES) {
                        if (!SINGLE && p.gate && !one_sample) by = value(gates[u % AHEAD], gate_of(p, u, m), n);
                    } else if (!SINGLE && p.gate && !one_sample) by = value(gates[u % AHEAD], of(m, p.gate, p.g_sb, 0), n);
                    out = finished(p, z, by, residual);
                    if (u + AHEAD < ALL) load_ahead(u + AHEAD);
                }
                if (u == ALL / 2 && more) load_bias();     // (half of the sums' registers are free)
                if constexpr (WHOLES)
                    if (!written(p, u)) continue;
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

}  // namespace
#endif
