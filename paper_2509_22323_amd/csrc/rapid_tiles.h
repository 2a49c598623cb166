// What the products of linear layers in bf16 (rapid_linear.hip) and in 8-bit integers (rapid_linear8.hip) have in common: accesses of
// eight outputs at any address, activations, copies from memory into LDS, the order of tiles, and the checks of rows.
#ifndef RAPID_TILES_H
#define RAPID_TILES_H

#include <hip/hip_runtime.h>
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

constexpr unsigned NOWHERE = 0xC0000000u;              // an offset outside any buffer below
constexpr unsigned BUFFER = 0x81000000u;               // bytes that a tile's rows may span, and the inputs of a row

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

// 1 KB from 64 lanes' addresses into LDS: lane i's 16 bytes go to dst + 1024 C + 16 i.  (The instruction's offset counts on both
// sides: LESS is taken off the lanes' offsets.)  Assembly, so that only the waits below order it; a wait state between the scalar
// write of M0 and the copy.  It would take five behind a vector instruction that writes the descriptor or the offset, as one that reads a
// scalar back from a lane does: the compiler has none there, which tests/test_wait_states.py looks at before anything runs.
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

// ---- host
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr long long MAX_STRIDE = 1LL << 22;            // elements, of a row

// Strides of dimensions of size 1 replaced by what changes no address; false: out of range.
inline bool rows_ok(const rapid_rows& a, int B, int n, int width, bool written, long long& sb, int& row_stride)
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
#endif
