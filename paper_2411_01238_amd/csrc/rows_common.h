// Device-side building blocks of the row kernels (element dropout, layer norm): eight consecutive elements of a row in any type,
// the counter-based mask, sums over a wavefront.
#ifndef SDROP_ROWS_COMMON_H
#define SDROP_ROWS_COMMON_H
#include "sdrop_internal.h"

namespace sdrop {
namespace {

// Eight consecutive elements.  The type promises the alignment of one element only: rows of an odd length, and columns of a
// wider matrix, begin anywhere.  The loads are 16 bytes wide all the same, the memory pipeline takes any address.
template <class T> struct Oct { typedef __attribute__((__vector_size__(8 * sizeof(T)), __aligned__(sizeof(T)))) T type; };

// n (1 .. 8) elements at p, the others 0.  TAIL = false: n is 8.
template <class T, bool TAIL> __device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if (!TAIL || n >= 8) {
        const typename Oct<T>::type x = *reinterpret_cast<const typename Oct<T>::type *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? static_cast<float>(p[i]) : 0.f;
    }
}

// v, rounded to nearest even, to n elements at p; v holds the rounded values afterwards
template <class T, bool TAIL> __device__ __forceinline__ void store8(T *p, int n, float (&v)[8])
{
    typename Oct<T>::type x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = static_cast<T>(v[i]);
        v[i] = static_cast<float>(x[i]);
    }
    if (!TAIL || n >= 8) {
        *reinterpret_cast<typename Oct<T>::type *>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = x[i];
    }
}

// The dropout's mask.  One Philox4x32-10 call (Salmon et al., SC'11) serves eight consecutive elements of a row, 16 bits each:
// a 32-bit draw per element would be two calls, and twenty 64-bit multiplies for 8 elements take as long as moving them.  The
// rate is therefore a multiple of 2^-16, and the scale is derived from that multiple: the expected value is exact.
// Counter: the number of the 8-element chunk over all rows (rows padded to whole chunks) and the generator's stream; key: the
// seed.  The top bit of the 64-bit chunk number is set: the block mask of the same seed and stream uses counters without it.
struct ElementMask {
    uint32_t key0, key1, ctr2, ctr3;
    uint32_t threshold;         // keep where the 16 bits are >= this; 0: nothing is drawn; 65536: nothing is kept
    float scale;                // 65536 / (65536 - threshold), 0 where nothing is kept
};

inline ElementMask element_mask(double p, uint64_t seed, uint64_t rng_stream)
{
    ElementMask m;
    m.key0 = (uint32_t)seed;
    m.key1 = (uint32_t)(seed >> 32);
    m.ctr2 = (uint32_t)rng_stream;
    m.ctr3 = (uint32_t)(rng_stream >> 32);
    const double t = p * 65536.0 + 0.5;
    m.threshold = p >= 1.0 ? 65536u : t >= 65535.0 ? 65535u : (uint32_t)t;
    m.scale = m.threshold >= 65536u ? 0.f : (float)(65536.0 / (65536.0 - (double)m.threshold));
    return m;
}

// factor[i] = scale or 0 for the elements of chunk `chunk`
__device__ __forceinline__ void mask8(const ElementMask &m, uint64_t chunk, float (&factor)[8])
{
    constexpr uint64_t MUL0 = 0xD2511F53u, MUL1 = 0xCD9E8D57u;
    uint32_t c0 = (uint32_t)chunk, c1 = (uint32_t)(chunk >> 32) | 0x80000000u, c2 = m.ctr2, c3 = m.ctr3, k0 = m.key0, k1 = m.key1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = MUL0 * (uint64_t)c0, p1 = MUL1 * (uint64_t)c2;
        const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0, n2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c0 = n0; c1 = (uint32_t)p1; c2 = n2; c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
        factor[i] = u >= m.threshold ? m.scale : 0.f;
    }
}

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// Sum over the 64 lanes, in every lane, in an order of its own that does not change: pairs, quads, eights and sixteens by
// lane permutations of the vector unit, then rows of 16 and halves by the swap instructions (no trip through LDS).
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp<0xB1>(v);          // lane ^ 1
    v += dpp<0x4E>(v);          // lane ^ 2
    v += dpp<0x141>(v);         // mirrored within 8
    v += dpp<0x140>(v);         // mirrored within 16
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)a[0]) + __builtin_bit_cast(float, (unsigned)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return __builtin_bit_cast(float, (unsigned)b[0]) + __builtin_bit_cast(float, (unsigned)b[1]);
}

}  // namespace

// What the row entry points share on the host.
inline size_t type_size(int dtype) { return dtype == SDROP_F32 ? 4 : 2; }
inline bool type_ok(int dtype) { return dtype == SDROP_F16 || dtype == SDROP_BF16 || dtype == SDROP_F32; }
// (a null pointer is aligned; leading dimension 0: contiguous)
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline bool row_ld_ok(int64_t ld, int64_t N) { return ld == 0 || (ld >= N && ld <= (int64_t(1) << 24)); }
inline bool rows_shape_ok(int64_t M, int64_t N) { return M >= 1 && N >= 1 && M <= (int64_t(1) << 30) && N <= (int64_t(1) << 24); }

}  // namespace sdrop
#endif
