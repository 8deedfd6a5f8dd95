// What the attention kernels share: the problem's description, sequences and their bounds, tiles of keys or queries in LDS.
//
//     S = c Q K^T,  P = softmax over the keys a query may see,  O = P V
//
// Queries of the heads that share a key / value head are rows of one problem: row r of (sequence, key head) is token r / G,
// head r % G of the group of G.  A tile of rows then reads each key once for the whole group.
#ifndef SDROP_ATTN_COMMON_H
#define SDROP_ATTN_COMMON_H
#include "gemm_device_common.h"

namespace sdrop {

struct AttnParams {
    const char *q, *k, *v, *o, *dout;       // o, dout: backward
    const char *rest;                       // backward: what o's rounding took, or null
    char *out, *out_rest, *dq, *dk, *dv;    // out_rest may be null
    float *lse, *delta;
    float *part_o, *part_lse;               // forward over parts of the keys: [splits][B * Hkv][max_rows][D] and [..] of them
    // bytes between sequences (dense), tokens and heads
    int64_t q_b, q_t, q_h, k_b, k_t, k_h, v_b, v_t, v_h, o_b, o_t, o_h, do_b, do_t, do_h;
    int64_t dq_b, dq_t, dq_h, dk_b, dk_t, dk_h, dv_b, dv_t, dv_h;
    const int32_t *cu_q, *cu_k, *k_len;
    int64_t total_q, total_k;
    int32_t B, max_q, max_k, Hq, Hkv, G, D, causal;
    int32_t max_rows;                       // max_q * G
    int32_t tiles, splits;                  // row tiles of the longest sequence; parts of the keys
    uint32_t g_mul;                         // r / G = (mulhi(r, g_mul) + r) >> g_shift
    int32_t g_shift;
    int32_t steady;                         // backward: 16 rows are whole tokens (G divides 16), 32 rows lie within 31 bits of bytes
    float scale, c;                         // c = scale * log2(e)
    int *status;
};

// The backward pass subtracts row sums of dO O from dP, and where few keys carry a row the two nearly cancel: there O has to be better than
// its type.  What O's own rounding took is kept for the backward pass (o_rest, every row).  What P's rounding took matters where one
// key has a good part of its row; over many small parts it averages out.  A lane whose largest P of a tile is more than this share of its
// sum before it (over half of the row's keys, so usually a fourth of the row's) has the tile's product once more with what the rounding took.
// Norm of dQ's error over that of rounding dQ alone, bf16, 1024 tokens, causal, heads of 128, scores of deviation 1 / 3 / 10: 1.39 / 1.45 /
// 1.47, and with half this share the same; without both, for rows of more than 128 keys: 1.39 / 1.75 / 2.93.  With scores of deviation 1 a
// fifth of the tiles has that product at 1024 keys, one in twenty at 4096; most have it at deviation 3.
constexpr float kLargeShare = 0.5f;

namespace {

// One sequence of the call: where its tokens begin (rows of a packed array; 0 in dense ones) and how many there are.
struct Sequence {
    int64_t q0, k0;
    int Lq, Lk;
    bool ok;
};

// Lengths and offsets are device data: what does not fit the call is left out (nothing of that sequence is read or written) and
// recorded in the status word.
__device__ __forceinline__ Sequence sequence_of(const AttnParams &P, int b)
{
    Sequence s;
    s.q0 = s.k0 = 0;
    s.Lq = P.max_q;
    s.Lk = P.max_k;
    s.ok = true;
    if (P.cu_q) {
        const int a = uni(P.cu_q[b]), e = uni(P.cu_q[b + 1]);
        s.q0 = a;
        s.Lq = e - a;
        s.ok = a >= 0 && e >= a && e <= P.total_q && s.Lq <= P.max_q;
    }
    if (P.cu_k) {
        const int a = uni(P.cu_k[b]), e = uni(P.cu_k[b + 1]);
        s.k0 = a;
        s.Lk = e - a;
        s.ok = s.ok && a >= 0 && e >= a && e <= P.total_k && s.Lk <= P.max_k;
    } else if (P.k_len) {
        s.Lk = uni(P.k_len[b]);
        s.ok = s.ok && s.Lk >= 0 && s.Lk <= P.max_k;
    }
    if (!s.ok && P.status && threadIdx.x == 0) atomicOr(P.status, SDROP_STATUS_BAD_LENGTHS);
    return s;
}

__device__ __forceinline__ int token_of(const AttnParams &P, int r)
{
    return (int)((__umulhi((uint32_t)r, P.g_mul) + (uint32_t)r) >> P.g_shift);
}

// The lane's number from nothing: what is worked out of threadIdx.x the compiler would keep in registers over a loop instead.
__device__ __forceinline__ int lane_again()
{
    int ones = -1;
    asm volatile("" : "+s"(ones));
    return __builtin_amdgcn_mbcnt_hi(ones, __builtin_amdgcn_mbcnt_lo(ones, 0));
}

// Workgroup id -> (sequence and key head, unit).  Consecutive workgroups go to the eight XCDs in turn.
// Where all units cost the same: eight heads at a time, one for each XCD, so that the workgroups that read the same keys share
// an L2.  Where they do not (a causal mask, sequences of different lengths): the first unit of every head, then the second, the
// costly units being the first ones.  A head's units one after the other would start the last heads' costly ones
// late (forward, 2 x 4096 tokens, 16 heads of 128, causal: 247 us against 190).
__device__ __forceinline__ void place(const AttnParams &P, int units, int &bh, int &unit)
{
    const int n = P.B * P.Hkv, id = blockIdx.x;
    if (P.causal || P.cu_q || P.cu_k || P.k_len) {
        unit = uni(id / n);
        bh = uni(id - unit * n);
    } else {
        const int g = id / (8 * units), rem = id - g * 8 * units;
        const int here = n - 8 * g < 8 ? n - 8 * g : 8;
        bh = uni(8 * g + rem % here);
        unit = uni(rem / here);
    }
}

// ---- tiles in LDS: [rows][HD] of 16-bit values ----
//
// One load instruction of a wavefront fills 1 KiB, 4 rows of 128 values or 8 of 64; such groups lie 1040 bytes apart.  In a group 16-byte
// chunk c of row r lies in slot c ^ swz_a(r).  Operands are read along the rows (ds_read_b128: one chunk, 16 rows at a time: 0 .. 3, 12 .. 15
// and 20 .. 27, then those between) and across them (ds_read_b64_tr_b16: 4 consecutive rows x 64 bytes): the XOR keeps four rows apart and
// the 16 bytes between groups the fours, so that either read is spread over all banks (no conflicts, counted; rows of 64 values told apart
// by their third bit too collided with the fours behind, a third of LDS's cycles: 2 x 4096, 16 heads, no mask, forward 173 -> 166 us).
// An XOR of all 16 rows' bits would do the same without the gap, but leave twice as many lane addresses to be made or kept.
template <int HD> constexpr int tile_bytes(int rows) { return rows * HD / 512 * 1040; }
template <int HD> __device__ __forceinline__ constexpr int swz_a(int r)
{
    return HD >= 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
}
// byte offset of row r (without its chunk)
template <int HD> __device__ __forceinline__ constexpr int row_at(int r)
{
    constexpr int G = 512 / HD;
    return r / G * 1040 + r % G * 2 * HD;
}

// Loads a tile of ROWS rows with NW wavefronts, HBM -> LDS without registers: one instruction fills 1 KiB, lane l its bytes
// 16 l ..; the lane fetches the chunk whose slot that is.
template <int HD, int ROWS, int NW> struct TileLoad {
    static constexpr int ROW_BYTES = 2 * HD, RPI = 1024 / ROW_BYTES, PASSES = ROWS / (RPI * NW);
    static_assert(ROWS % (RPI * NW) == 0, "whole passes");
    uint32_t voff;
    int row, chunk, wave;
    __device__ __forceinline__ void init(int64_t stride, int w)
    {
        const int lane = threadIdx.x & 63;
        wave = w;
        row = RPI * w + (lane * 16) / ROW_BYTES;
        chunk = ((lane * 16) % ROW_BYTES >> 4) ^ swz_a<HD>(row);
        voff = (uint32_t)row * (uint32_t)stride + (chunk << 4);
    }
    // rows: how many of the tile exist; nch: 16-byte chunks of a row that do.  What does not is 0 in LDS.
    __device__ __forceinline__ void issue(const char *base, int64_t stride, char *lds, int rows, int nch) const
    {
        if (rows >= ROWS && nch == HD / 8) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i, base += RPI * NW * stride) dma16(base, voff, lds + (wave + NW * i) * 1040);
        } else {
            // (made here: four registers that would be kept for the whole loop)
            uint4 zero = make_uint4(0, 0, 0, 0);
            asm volatile("" : "+v"(zero.x), "+v"(zero.y), "+v"(zero.z), "+v"(zero.w));
#pragma unroll
            for (int i = 0; i < PASSES; ++i, base += RPI * NW * stride) {
                char *const dst = lds + (wave + NW * i) * 1040;
                if (row + RPI * NW * i < rows && chunk < nch) dma16(base, voff, dst);
                else *reinterpret_cast<uint4 *>(dst + lane_again() * 16) = zero;
            }
        }
    }
};

// The same for a lane's own 64-bit address (see dma16).
__device__ __forceinline__ void dma16_at(const char *src, const char *lds)
{
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)lds;
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(lds_base));
}

// What this wavefront has requested has landed, and so has everyone else's; nothing is moved across.  (The wait as a builtin: the
// compiler then knows that its own loads have landed too.  It would otherwise wait for them again at their first use in a loop,
// by a count that takes in the loads into LDS that it does not know of.)
__device__ __forceinline__ void landed()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// (Lane addresses are a base and an XOR with what the compiler knows.  Kept for a whole loop they would be eight registers a tile:
// fresh() hides the base's origin, so that they are made again where they are used.)
// Operand of 32 rows of a tile, reduction along them (16 columns from 16 kk): lane l has row base + l % 32, columns 16 kk + 8 (l / 32) ..
// `offset`: bytes from the operand's own tile, a constant.
template <int HD, class T> struct RowOperand {
    const char *at;
    int f;
    __device__ __forceinline__ RowOperand(const char *lds)
    {
        const int l = threadIdx.x & 63;
        at = lds + row_at<HD>(l & 31);
        f = (swz_a<HD>(l & 31) ^ (l >> 5)) << 4;
    }
    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(f)); }
    __device__ __forceinline__ typename In<T>::vec get(int offset, int kk) const
    {
        // (of the bits that the XOR leaves alone the address is a sum)
        constexpr int PLAIN = 32;
        return *reinterpret_cast<const typename In<T>::vec *>(at + (f ^ ((kk << 5) & ~PLAIN)) + ((kk << 5) & PLAIN) + offset);
    }
};

// Operand of 32 columns of a tile, reduction across its rows (16 rows from 16 ks).  Lane l has column base + l % 32; its eight values
// are rows 16 ks + 4 (l / 32) + {0 .. 3, 8 .. 11}: the order in which a 32 x 32 result lies in a lane's registers, so that such a
// result is the other operand as it is.
template <int HD, class T> struct ColOperand {
    const char *at;
    int f;
    __device__ __forceinline__ ColOperand(const char *lds)
    {
        const int l = threadIdx.x & 63, r = 4 * (l >> 5) + ((l & 15) >> 2), chunk = 2 * ((l >> 4) & 1) + ((l & 3) >> 1);
        at = lds + row_at<HD>(r) + ((l & 1) << 3);
        f = (chunk ^ swz_a<HD>(r)) << 4;
    }
    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(f)); }
    __device__ __forceinline__ typename In<T>::vec get(int offset, int db, int ks) const
    {
        static_assert(swz_a<HD>(8) == swz_a<HD>(0) && swz_a<HD>(16) == swz_a<HD>(0), "the same for every eight rows");
        const char *const p = at + (f ^ (db << 6)) + row_at<HD>(16) * ks + offset;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + row_at<HD>(8)));
        return __builtin_bit_cast(typename In<T>::vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Eight values of a 32 x 32 result (registers 8 part .. 8 part + 7) rounded to the operands' type.
template <class T> __device__ __forceinline__ typename In<T>::vec narrow8(const f32x16 &v, int part)
{
    typedef __attribute__((__vector_size__(8 * sizeof(typename In<T>::out16)))) typename In<T>::out16 e8;
    e8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = static_cast<typename In<T>::out16>(v[8 * part + i]);
    return __builtin_bit_cast(typename In<T>::vec, o);
}

// What that rounding took, rounded in turn, under a mask of bits.
template <class T> __device__ __forceinline__ typename In<T>::vec narrow8_rest(const f32x16 &v, int part, uint32_t mask)
{
    typedef __attribute__((__vector_size__(8 * sizeof(typename In<T>::out16)))) typename In<T>::out16 e8;
    e8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        o[i] = static_cast<typename In<T>::out16>(v[8 * part + i] - static_cast<float>(static_cast<typename In<T>::out16>(v[8 * part + i])));
    const uint4 w = __builtin_bit_cast(uint4, o);
    return __builtin_bit_cast(typename In<T>::vec, make_uint4(w.x & mask, w.y & mask, w.z & mask, w.w & mask));
}

__device__ __forceinline__ f32x16 zero16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

// The other half of the wavefront's value (lane ^ 32).
template <class F> __device__ __forceinline__ float join_halves(float v, F &&f)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return f(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
}

// 32 consecutive columns of one row per lane pair (l, l ^ 32), from a 32 x 32 result whose column is the row (lane l % 32) and whose
// rows are the columns: rounded, 16 bytes per store.  n: columns that exist (a multiple of 8).  rest: null, or where what the
// rounding took goes, rounded in turn.
template <class T> __device__ __forceinline__ void store_row32(char *p, const f32x16 &v, float mul, int n, bool live, char *rest = nullptr)
{
    using E = typename In<T>::out16;
    typedef __attribute__((__vector_size__(4 * sizeof(E)))) E e4;
    const int h = lane_again() >> 5;
    auto put = [&](char *to, e4 a, e4 b, int g) __attribute__((always_inline)) {
        const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
        const auto s = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false), t = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
        // the lower lane has columns 16 g .. 16 g + 7, the upper one the next eight
        const int col = 16 * g + 8 * h;
        if (live && col < n) *reinterpret_cast<uint4 *>(to + 2 * col) = make_uint4(s[0], t[0], s[1], t[1]);
    };
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        e4 a, b;                    // columns 16 g + 4 h .. and 16 g + 8 + 4 h ..
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = static_cast<E>(v[8 * g + i] * mul);
            b[i] = static_cast<E>(v[8 * g + 4 + i] * mul);
        }
        put(p, a, b, g);
        if (rest) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = static_cast<E>(v[8 * g + i] * mul - static_cast<float>(a[i]));
                b[i] = static_cast<E>(v[8 * g + 4 + i] * mul - static_cast<float>(b[i]));
            }
            put(rest, a, b, g);
        }
    }
}

}  // namespace

inline bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Checks a call and fills the parameters both directions share (SDROP_OK or an error).
int attn_params(const sdrop_attn_t *a, bool backward, AttnParams &P);

}  // namespace sdrop
#endif
