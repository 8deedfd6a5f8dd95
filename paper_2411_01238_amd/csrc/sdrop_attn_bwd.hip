// Attention, backward: the gradients of q, k and v from that of O.
//
//     P = exp(S - lse),  dP = dO V^T,  delta = row sums of dO O,  dS = P (dP - delta)
//     dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO
//
// Scores are computed again from q, k and the forward pass's lse; nothing of their size is stored.  Two launches: dQ, a workgroup per
// tile of rows that walks the keys (it has dO and O of its rows at hand and leaves lse and delta for the other), then dK and dV, a
// workgroup per tile of keys that walks the rows of all query heads that share them.  Each gradient is summed in registers in
// a fixed order: no atomics, results repeat bit for bit, at the price of computing S and dP twice (7 products instead of 5).
// Many sequences of up to 256 keys: one launch, a workgroup per sequence and key head, 5 products.
#include "attn_common.h"
#include <math.h>

namespace sdrop {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Statistics of the rows, as dK and dV's accumulators begin: -lse / scale, so that exp2(c S) is P, and -delta, so that dP - delta comes out of
// the matrix cores.  fp16's P is held as 256 P: over thousands of keys P itself would fall among its smallest numbers, whose steps are
// coarse.  The factor is part of the first and is taken out again.
template <class T> constexpr float kPShift = 0.f;
template <> constexpr float kPShift<F16> = 8.f;
template <class T> constexpr float kPScale = 1.f;
template <> constexpr float kPScale<F16> = 1.f / 256.f;
// fp16's dS is P times a gradient, smaller still, and may be large too: it is rounded times a power of two that brings it near the top of
// fp16's numbers, taken out where the sums are written.  dQ: one per row, from the size of its dO (|dP - delta| is about |dO| |v| at most); dK:
// one per key, from the largest so far; either is made smaller, and the sums with it, where a value would pass kMost.  Errors of dQ
// over those of rounding dQ alone, 2048 keys, heads of 64, dO of deviation 1 / 10^-2 / 10^-3: 1.43 / 1.82 / 5.75 without, 1.43 / 1.43 /
// 1.10 with them (4 x 4096 tokens, 16 heads of 64, 4 of keys, causal 561 -> 582 us, 64 x 256 73 -> 82).
template <class T> constexpr bool kScaled = false;
template <> constexpr bool kScaled<F16> = true;
constexpr float kMost = 32768.f;

// floor(log2 v) of a positive number; 128 of an infinity or NaN, -127 of 0
__device__ __forceinline__ int exponent_of(float v) { return (int)((__builtin_bit_cast(uint32_t, v) >> 23) & 255) - 127; }
__device__ __forceinline__ float largest_of(const f32x16 &v)
{
    float mx = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, fabsf(v[e]));
    return join_halves(mx, [](float a, float b) { return fmaxf(a, b); });
}

// Two arrays, and where the rows of (sequence b, key head hkv) begin in each: on 16 bytes, sequences and heads apart.  A tile of 64 rows
// is read whole, so each is that much longer than its last row.
__host__ __device__ __forceinline__ int64_t stats_rows(const AttnParams &P)
{
    return P.cu_q ? P.Hkv * ((P.total_q * P.G + 4 * P.B + 3) & ~int64_t(3)) : (int64_t)P.B * P.Hkv * ((P.max_rows + 3) & ~3);
}
__device__ __forceinline__ int64_t stats_at(const AttnParams &P, const Sequence &s, int b, int hkv)
{
    return P.cu_q ? hkv * ((P.total_q * P.G + 4 * P.B + 3) & ~int64_t(3)) + ((s.q0 * P.G + 4 * b) & ~int64_t(3))
                  : ((int64_t)b * P.Hkv + hkv) * ((P.max_rows + 3) & ~3);
}

template <class T> __device__ __forceinline__ float dot8(uint4 a, uint4 b, float sum)
{
    typedef __attribute__((__vector_size__(8 * sizeof(typename In<T>::out16)))) typename In<T>::out16 e8;
    const e8 x = __builtin_bit_cast(e8, a), y = __builtin_bit_cast(e8, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += static_cast<float>(x[i]) * static_cast<float>(y[i]);
    return sum;
}

template <int CTRL> __device__ __forceinline__ float lane_sum(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// The largest of 32 lanes' values, l % 32, in all of them.
__device__ __forceinline__ float largest_of_32(float v)
{
    v = fmaxf(v, lane_sum<0xB1>(v));
    v = fmaxf(v, lane_sum<0x4E>(v));
    v = fmaxf(v, lane_sum<0x141>(v));
    v = fmaxf(v, lane_sum<0x140>(v));
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
}

// dQ.  As in the forward pass a lane holds keys of one query: S^T = K Q^T, dP^T = V dO^T, dQ^T = K^T dS^T; lse and delta are one number
// per lane each.
// QW wavefronts own rows of their own; the 4 / QW wavefronts of the same rows take a tile's blocks of 32 keys in turn and are joined at
// the end.  Heads of 64 leave room for four wavefronts per SIMD, whose products run beside each other's exponentials (24 sequences of 64
// to 2000 tokens, 16 heads, 4 of keys, causal, the whole backward pass: 394 -> 377 us).
template <class T, int HD, int QW>
__global__ __launch_bounds__(256, HD <= 64 ? 4 : 2) void attn_dq_kernel(AttnParams P)
{
    constexpr int TKV = 64, TILE = tile_bytes<HD>(TKV), DB = HD / 32, KW = 4 / QW, ROWS = 32 * QW;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TILE];
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), h = lane >> 5, wq = wave % QW, wk = wave / QW;
    int bh, unit;
    place(P, P.tiles, bh, unit);
    const int b = bh / P.Hkv, hkv = bh - b * P.Hkv, tile = P.tiles - 1 - unit;
    const Sequence s = sequence_of(P, b);
    if (!s.ok) return;
    const int rows = s.Lq * P.G, R0 = tile * ROWS;
    if (R0 >= rows) return;
    const int off = s.Lk - s.Lq, r_last = min(R0 + ROWS, rows) - 1;
    const int k_end = P.causal ? min(s.Lk, token_of(P, r_last) + off + 1) : s.Lk;
    const int n_tiles = k_end > 0 ? (k_end + TKV - 1) / TKV : 0;

    const int w0 = R0 + 32 * wq, r = w0 + (lane & 31);
    const bool live = r < rows;
    const int i = token_of(P, min(r, rows - 1)), head = hkv * P.G + (min(r, rows - 1) - i * P.G);
    const int lim = !live ? -1 : P.causal ? min(s.Lk - 1, i + off) : s.Lk - 1;
    const bool any = w0 < rows;
    const int w_first = any ? uni(token_of(P, w0)) + off : 0, w_last = any ? uni(token_of(P, min(w0 + 31, rows - 1))) + off : -1;

    typename In<T>::vec qf[HD / 16], gf[HD / 16];
    float delta = 0.f, size = 0.f;
    {
        const char *const qp = P.q + (P.cu_q ? 0 : b * P.q_b) + (s.q0 + i) * P.q_t + head * P.q_h;
        const char *const gp = P.dout + (P.cu_q ? 0 : b * P.do_b) + (s.q0 + i) * P.do_t + head * P.do_h;
        const int64_t at = (P.cu_q ? 0 : b * P.o_b) + (s.q0 + i) * P.o_t + head * P.o_h;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
            const int col = 16 * kk + 8 * h;
            uint4 x = make_uint4(0, 0, 0, 0), g = x, o = x, rest = x;
            if (live && col < P.D) {
                x = *reinterpret_cast<const uint4 *>(qp + 2 * col);
                g = *reinterpret_cast<const uint4 *>(gp + 2 * col);
                o = *reinterpret_cast<const uint4 *>(P.o + at + 2 * col);
                if (P.rest) rest = *reinterpret_cast<const uint4 *>(P.rest + at + 2 * col);
            }
            qf[kk] = __builtin_bit_cast(typename In<T>::vec, x);
            gf[kk] = __builtin_bit_cast(typename In<T>::vec, g);
            delta = dot8<T>(g, rest, dot8<T>(g, o, delta));
            if constexpr (kScaled<T>) size = dot8<T>(g, g, size);
        }
    }
    delta = join_halves(delta, [](float a, float c) { return a + c; });
    // (a row that saw no key: +inf makes every P of it 0)
    float lse2 = INFINITY;
    if (live) {
        const float x = P.lse[P.cu_q ? head * P.total_q + s.q0 + i : ((int64_t)b * P.Hq + head) * P.max_q + i];
        if (x != -INFINITY) lse2 = x * kLog2e;
        if (h == 0 && wk == 0) {
            float *const st = P.delta + stats_at(P, s, b, hkv) + r;
            st[0] = (kPShift<T> - lse2) / P.c;
            st[stats_rows(P) + 64] = -delta;
        }
    }
    // (the power of two is part of P's exponent)
    int up = 0;
    if constexpr (kScaled<T>) {
        up = 10 - ((exponent_of(join_halves(size, [](float a, float c) { return a + c; })) + 1) >> 1);
        up = max(-40, min(up, 40));
        lse2 -= (float)up;
    }

    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();
    // dP's accumulators begin at -delta; heads of 64 have no registers to keep that in, and subtract it
    constexpr bool BEGIN = HD > 64;
    f32x16 dp0 = zero16();
    if constexpr (BEGIN) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            dp0[e] = -delta;
            asm volatile("" : "+v"(dp0[e]));
        }
    }
    const char *kb = P.k + (P.cu_k ? 0 : b * P.k_b) + s.k0 * P.k_t + hkv * P.k_h;
    const char *vb = P.v + (P.cu_k ? 0 : b * P.v_b) + s.k0 * P.v_t + hkv * P.v_h;
    const int nch = P.D / 8;
    TileLoad<HD, TKV, 4> lk, lv;
    lk.init(P.k_t, wave);
    lv.init(P.v_t, wave);
    auto request = [&](int t, int buf) __attribute__((always_inline)) {
        const int left = s.Lk - t * TKV;
        lk.issue(kb, P.k_t, lds + buf * 2 * TILE, left, nch);
        lv.issue(vb, P.v_t, lds + buf * 2 * TILE + TILE, left, nch);
        kb += TKV * P.k_t;
        vb += TKV * P.v_t;
    };
    if (n_tiles > 0) request(0, 0);
    for (int t = 0; t < n_tiles; ++t) {
        const int buf = t & 1;
        landed();
        if (t + 1 < n_tiles) request(t + 1, buf ^ 1);
        const int kv0 = t * TKV;
        if (P.causal && kv0 > w_last) continue;
        const char *const kt = lds + buf * 2 * TILE, *const vt = kt + TILE;
        const bool masked = kv0 + TKV > s.Lk || (P.causal && kv0 + TKV - 1 > w_first);
        auto block = [&](int mb) __attribute__((always_inline)) {
            const RowOperand<HD, T> ka(kt + mb * row_at<HD>(32)), va(vt + mb * row_at<HD>(32));
            const ColOperand<HD, T> kc(kt + mb * row_at<HD>(32));
            f32x16 sc = zero16(), dp = dp0;
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) sc = In<T>::mfma(ka.get(0, kk), qf[kk], sc);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) dp = In<T>::mfma(va.get(0, kk), gf[kk], dp);
            if (masked) {
                const int last = lim - kv0 - 32 * mb - 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e >> 2) + (e & 3) > last) sc[e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = __builtin_amdgcn_exp2f(sc[e] * P.c - lse2) * (BEGIN ? dp[e] : dp[e] - delta);
            if constexpr (kScaled<T>) {
                const float mx = largest_of(sc);
                if (__any(mx > kMost)) {
                    const int down = mx > kMost ? exponent_of(mx) - 10 : 0;
                    const float f = ldexpf(1.f, -down);
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[e] *= f;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[d][e] *= f;
                    up -= down;
                    lse2 += (float)down;
                }
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const typename In<T>::vec ds = narrow8<T>(sc, ks);
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] = In<T>::mfma(kc.get(0, d, ks), ds, acc[d]);
            }
        };
        // (one block of 32 keys after the other: the registers of two do not fit beside Q, dO and dQ)
        if constexpr (KW == 2) {
            block(wk);
        } else {
#pragma unroll 1
            for (int mb = 0; mb < 2; ++mb) block(mb);
        }
    }
    if constexpr (kScaled<T>) {
        const float f = ldexpf(1.f, -up);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[d][e] *= f;
    }
    if constexpr (KW == 2) {
        float *const joined = reinterpret_cast<float *>(lds) + wq * DB * 16 * 64 + lane;
        static_assert(QW * DB * 16 * 64 * 4 <= 4 * TILE, "room for the accumulators of half of the wavefronts");
        landed();
        if (wk == 1) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) joined[(d * 16 + e) * 64] = acc[d][e];
        }
        __syncthreads();
        if (wk == 1) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[d][e] += joined[(d * 16 + e) * 64];
    }
    char *const dst = P.dq + (P.cu_q ? 0 : b * P.dq_b) + (s.q0 + i) * P.dq_t + head * P.dq_h;
#pragma unroll
    for (int d = 0; d < DB; ++d) store_row32<T>(dst + 64 * d, acc[d], P.scale, P.D - 32 * d, live);
}

// dK and dV.  A wavefront owns 32 keys; a lane holds rows (queries) of one key: S = Q K^T, dP = dO V^T, dV^T = dO^T P, dK^T = Q^T dS.
// KW wavefronts own keys of their own; the 4 / KW wavefronts of the same keys take a tile's blocks of 32 rows in turn and are joined at
// the end.
template <class T, int HD, int KW>
__global__ __launch_bounds__(256, HD <= 64 ? 3 : 2) void attn_dkv_kernel(AttnParams P)
{
    constexpr int TQ = 64, TILE = tile_bytes<HD>(TQ), DB = HD / 32, RW = 4 / KW, KEYS = 32 * KW;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TILE + 2 * TQ * 8];
    float *const st = reinterpret_cast<float *>(lds + 4 * TILE);       // [2][2][TQ]
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), h = lane >> 5;
    int bh, unit;
    place(P, P.tiles, bh, unit);
    const int b = bh / P.Hkv, hkv = bh - b * P.Hkv, K0 = unit * KEYS, wk = wave % KW, wr = wave / KW;
    const Sequence s = sequence_of(P, b);
    if (!s.ok) return;
    // rows of dK and dV that this call writes; behind a dense sequence's last key they are 0
    const int out_rows = P.cu_k ? s.Lk : P.max_k;
    if (K0 >= out_rows) return;
    const int rows = K0 < s.Lk ? s.Lq * P.G : 0, off = s.Lk - s.Lq;
    // causal: the first row that sees a key of this tile
    const int r_first = P.causal ? min(max(K0 - off, 0), s.Lq) * P.G : 0;
    const int t0 = r_first / TQ, t1 = (rows + TQ - 1) / TQ;

    const int w0 = K0 + 32 * wk, key = w0 + (lane & 31);
    const bool live = key < s.Lk;
    const int first_row = (int)max((int64_t)-1, min((int64_t)(key - off) * P.G, (int64_t)INT_MAX));      // causal: of those that see the key
    typename In<T>::vec kf[HD / 16], vf[HD / 16];
    {
        const int64_t at = s.k0 + min(key, max(s.Lk - 1, 0));
        const char *const kp = P.k + (P.cu_k ? 0 : b * P.k_b) + at * P.k_t + hkv * P.k_h;
        const char *const vp = P.v + (P.cu_k ? 0 : b * P.v_b) + at * P.v_t + hkv * P.v_h;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
            const int col = 16 * kk + 8 * h;
            uint4 x = make_uint4(0, 0, 0, 0), y = x;
            if (live && col < P.D) {
                x = *reinterpret_cast<const uint4 *>(kp + 2 * col);
                y = *reinterpret_cast<const uint4 *>(vp + 2 * col);
            }
            kf[kk] = __builtin_bit_cast(typename In<T>::vec, x);
            vf[kk] = __builtin_bit_cast(typename In<T>::vec, y);
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zero16();
    float up = kScaled<T> ? 0x1p32f : 1.f;          // what dS / kPScale is multiplied with

    const char *const qb = P.q + (P.cu_q ? 0 : b * P.q_b) + s.q0 * P.q_t + (int64_t)hkv * P.G * P.q_h;
    const char *const gb = P.dout + (P.cu_q ? 0 : b * P.do_b) + s.q0 * P.do_t + (int64_t)hkv * P.G * P.do_h;
    const char *const stats = reinterpret_cast<const char *>(P.delta + stats_at(P, s, b, hkv));
    const int64_t second = (stats_rows(P) + 64) * 4;
    const int nch = P.D / 8;
    // rows of a tile are tokens and heads of the group in turn: each lane works out where its rows lie
    constexpr int ROW_BYTES = 2 * HD, RPI = 1024 / ROW_BYTES, PASSES = TQ / (RPI * 4);
    // offsets of a lane's part of a tile (see request)
    auto offsets = [&](int ln, int &lrow, int &chunk, uint32_t &qo, uint32_t &go) __attribute__((always_inline)) {
        lrow = RPI * wave + (ln * 16) / ROW_BYTES;
        chunk = ((ln * 16) % ROW_BYTES >> 4) ^ swz_a<HD>(lrow);
        const uint32_t tok = lrow >> P.g_shift, g = lrow & (P.G - 1);
        qo = tok * (uint32_t)P.q_t + g * (uint32_t)P.q_h + chunk * 16;
        go = tok * (uint32_t)P.do_t + g * (uint32_t)P.do_h + chunk * 16;
    };
    int lrow0, chunk0;
    uint32_t qo0, go0;
    offsets(lane, lrow0, chunk0, qo0, go0);
    auto request = [&](int t, int buf) __attribute__((always_inline)) {
        int ln = lane, lrow = lrow0, chunk = chunk0;
        uint32_t qo = qo0, go = go0;
        if constexpr (HD > 64) {
            // (made anew for every tile: kept over the loop they are registers that the accumulators need)
            asm volatile("" : "+v"(ln));
            offsets(ln, lrow, chunk, qo, go);
        }
        char *const dst = lds + buf * 2 * TILE;
        if (P.steady && (t + 1) * TQ <= rows && nch == HD / 8) {
            // every pass has the same heads of the group, tokens further on: 32-bit offsets from addresses that the lanes share
            const int t_tok = t * TQ >> P.g_shift, step = RPI * 4 >> P.g_shift;
            const char *q_at = qb + t_tok * P.q_t, *g_at = gb + t_tok * P.do_t;
#pragma unroll
            for (int p = 0; p < PASSES; ++p, q_at += step * P.q_t, g_at += step * P.do_t) {
                char *const at = dst + (wave + 4 * p) * 1040;
                dma16(q_at, qo, at);
                dma16(g_at, go, at + TILE);
            }
        } else {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int rr = t * TQ + lrow + RPI * 4 * p;
                char *const at = dst + (wave + 4 * p) * 1040;
                if (rr < rows && chunk < nch) {
                    const int tok = token_of(P, rr), g = rr - tok * P.G;
                    dma16_at(qb + tok * P.q_t + g * P.q_h + chunk * 16, at);
                    dma16_at(gb + tok * P.do_t + g * P.do_h + chunk * 16, at + TILE);
                } else {
                    *reinterpret_cast<uint4 *>(at + ln * 16) = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4 *>(at + TILE + ln * 16) = make_uint4(0, 0, 0, 0);
                }
            }
        }
        if (threadIdx.x < TQ / 2) dma16_at(stats + (int64_t)t * TQ * 4 + (ln & 15) * 16 + (ln < 16 ? 0 : second), lds + 4 * TILE + buf * TQ * 8);
    };
    if (t0 < t1) request(t0, 0);
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        landed();
        if (t + 1 < t1) request(t + 1, buf ^ 1);
        auto block = [&](int mb) __attribute__((always_inline)) {
            const int rb = t * TQ + 32 * mb;
            if (rb >= rows) return;
            const int see_first = P.causal ? uni(token_of(P, rb)) + off : s.Lk, see_last = P.causal ? uni(token_of(P, min(rb + 31, rows - 1))) + off : s.Lk;
            if (see_last < w0) return;            // none of these rows sees a key of this wavefront
            RowOperand<HD, T> ra(lds + buf * 2 * TILE + mb * row_at<HD>(32));
            ColOperand<HD, T> ca(lds + buf * 2 * TILE + mb * row_at<HD>(32));
            ra.fresh();
            ca.fresh();
            // (a wavefront at its matrix instructions goes before the one beside it at its exponentials: 2 x 4096, 16 heads of 128, causal
            // 350 -> 332 us)
            __builtin_amdgcn_s_setprio(1);
            f32x16 sc, dp;
            const float *const stb = st + buf * 2 * TQ + 32 * mb + 4 * h;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32q a4 = *reinterpret_cast<const f32q *>(stb + 8 * g), b4 = *reinterpret_cast<const f32q *>(stb + TQ + 8 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) { sc[4 * g + e] = a4[e]; dp[4 * g + e] = b4[e]; }
            }
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) sc = In<T>::mfma(ra.get(0, kk), kf[kk], sc);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) dp = In<T>::mfma(ra.get(TILE, kk), vf[kk], dp);
            // the operands are read two ahead of the matrix instructions (three would not leave the accumulators their registers)
            __builtin_amdgcn_sched_group_barrier(0x100, 8 + 2, 0);
#pragma unroll
            for (int i = 0; i < HD / 8 - 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[e] = __builtin_amdgcn_exp2f(sc[e] * P.c);
                dp[e] *= sc[e];
            }
            // rows that do not see the key, and rows that do not exist (whose statistics are another's, or none)
            if ((P.causal && see_first < w0 + 31) || rb + 32 > rows) {
                const int from = (P.causal ? first_row : 0) - rb - 4 * h, to = rows - rb - 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int at = 8 * (e >> 2) + (e & 3);
                    if (at < from || at >= to) sc[e] = dp[e] = 0.f;
                }
            }
            if constexpr (kScaled<T>) {
                const float mx = largest_of(dp);
                if (__any(mx * up > kMost)) {
                    const float next = mx * up > kMost ? ldexpf(1.f, 11 - exponent_of(mx)) : up, f = next / up;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) dk[d][e] *= f;
                    up = next;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[e] *= up;
            }
            __builtin_amdgcn_sched_barrier(0);
            typename In<T>::vec pn[2], dn[2];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) { pn[ks] = narrow8<T>(sc, ks); dn[ks] = narrow8<T>(dp, ks); }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const typename In<T>::vec p = pn[ks], ds = dn[ks];
#pragma unroll
                for (int d = 0; d < DB; ++d) dv[d] = In<T>::mfma(ca.get(TILE, d, ks), p, dv[d]);
#pragma unroll
                for (int d = 0; d < DB; ++d) dk[d] = In<T>::mfma(ca.get(0, d, ks), ds, dk[d]);
            }
            // two operands ahead
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < 4 * DB - 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
        };
        if constexpr (RW == 2) {
            block(wr);
        } else {
            // (one block of 32 rows after the other: the registers of two do not fit beside K, V, dK and dV)
#pragma unroll 1
            for (int mb = 0; mb < 2; ++mb) block(mb);
        }
    }
    if constexpr (kScaled<T>) {
        const float f = kPScale<T> / up;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) dk[d][e] *= f;
    }
    if constexpr (RW == 2) {
        static_assert(2 * KW * DB * 16 * 64 * 4 <= 4 * TILE, "room for the accumulators of half of the wavefronts");
        int ln = lane;
        asm volatile("" : "+v"(ln));
        float *const joined = reinterpret_cast<float *>(lds) + wk * 2 * DB * 16 * 64 + ln;
        landed();
        if (wr == 1) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    joined[(d * 16 + e) * 64] = dk[d][e];
                    joined[((DB + d) * 16 + e) * 64] = dv[d][e];
                }
        }
        __syncthreads();
        if (wr == 1) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                dk[d][e] += joined[(d * 16 + e) * 64];
                dv[d][e] += joined[((DB + d) * 16 + e) * 64];
            }
    }
    // (made again, as in request)
    int mine = lane & 31;
    asm volatile("" : "+v"(mine));
    mine += w0;
    if (mine >= s.Lk) {
#pragma unroll
        for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zero16();
    }
    const bool write = mine < out_rows;
    char *const dkp = P.dk + (P.cu_k ? 0 : b * P.dk_b) + (s.k0 + mine) * P.dk_t + hkv * P.dk_h;
    char *const dvp = P.dv + (P.cu_k ? 0 : b * P.dv_b) + (s.k0 + mine) * P.dv_t + hkv * P.dv_h;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_row32<T>(dkp + 64 * d, dk[d], P.scale, P.D - 32 * d, write);
        store_row32<T>(dvp + 64 * d, dv[d], kPScale<T>, P.D - 32 * d, write);
    }
}

// All three gradients of sequences that one workgroup takes whole: W wavefronts own 32 keys each and walk the rows in tiles of 32, as for
// dK and dV; their dS also goes to LDS, where the wavefronts whose turn it is multiply it with K into dQ during the next tile.  Five
// products instead of seven, and one pass over memory (64 x 256 tokens, 8 heads of 128: 302 MB in 87 us, 3.5 TB/s; what bounds it is that the
// two wavefronts of a SIMD meet at every tile, for LDS holds one workgroup per CU).
template <class T, int HD, int W>
__global__ __launch_bounds__(64 * W, 2) void attn_bwd_short_kernel(AttnParams P)
{
    constexpr int TQ = 32, KEYS = 32 * W, DB = HD / 32, QT = tile_bytes<HD>(TQ), KT = tile_bytes<HD>(KEYS), ST = tile_bytes<64>(KEYS), TURNS = W / DB;
    static_assert(W % DB == 0, "whole turns");
    // K; dS [keys][32 rows of an even tile, 32 of an odd one]; two tiles of Q and dO; two of the rows' statistics
    __shared__ __attribute__((aligned(1024))) char lds[KT + ST + 4 * QT + 4 * TQ * 4 + (kScaled<T> ? 2 * TQ + W : 0) * 4];
    char *const k_lds = lds, *const s_lds = lds + KT, *const q_lds = s_lds + ST;
    float *const st = reinterpret_cast<float *>(q_lds + 4 * QT);       // [2][2][TQ]
    float *const dO2 = st + 4 * TQ, *const v2 = dO2 + 2 * TQ;           // (scaled dS) |dO|^2 of the rows [2][TQ]; the largest |v|^2 of each wavefront
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), h = lane >> 5;
    const int bh = uni(blockIdx.x), b = bh / P.Hkv, hkv = bh - b * P.Hkv;
    const Sequence s = sequence_of(P, b);
    if (!s.ok) return;
    const int out_rows = P.cu_k ? s.Lk : P.max_k, rows = s.Lq * P.G, off = s.Lk - s.Lq, n = (rows + TQ - 1) / TQ, nch = P.D / 8;
    const int w0 = 32 * wave, key = w0 + (lane & 31);
    const int first_row = (int)max((int64_t)-1, min((int64_t)(key - off) * P.G, (int64_t)INT_MAX));      // causal: of those that see the key
    auto see_last = [&](int t) __attribute__((always_inline)) { return P.causal ? uni(token_of(P, min(t * TQ + TQ, rows) - 1)) + off : s.Lk - 1; };

    {
        TileLoad<HD, KEYS, W> lk;
        lk.init(P.k_t, wave);
        lk.issue(P.k + (P.cu_k ? 0 : b * P.k_b) + s.k0 * P.k_t + hkv * P.k_h, P.k_t, k_lds, s.Lk, nch);
    }
    typename In<T>::vec vf[HD / 16];
    {
        const int64_t at = s.k0 + min(key, max(s.Lk - 1, 0));
        const char *const vp = P.v + (P.cu_k ? 0 : b * P.v_b) + at * P.v_t + hkv * P.v_h;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
            const int col = 16 * kk + 8 * h;
            uint4 y = make_uint4(0, 0, 0, 0);
            if (key < s.Lk && col < P.D) y = *reinterpret_cast<const uint4 *>(vp + 2 * col);
            vf[kk] = __builtin_bit_cast(typename In<T>::vec, y);
        }
    }
    if constexpr (kScaled<T>) {
        float size = 0.f;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) size = dot8<T>(__builtin_bit_cast(uint4, vf[kk]), __builtin_bit_cast(uint4, vf[kk]), size);
        size = join_halves(size, [](float a, float c) { return a + c; });
        size = largest_of_32(size < INFINITY ? size : 0.f);
        if (lane == 0) v2[wave] = size;
    }
    const char *const qb = P.q + (P.cu_q ? 0 : b * P.q_b) + s.q0 * P.q_t + (int64_t)hkv * P.G * P.q_h;
    const char *const gb = P.dout + (P.cu_q ? 0 : b * P.do_b) + s.q0 * P.do_t + (int64_t)hkv * P.G * P.do_h;

    // Q and dO of a tile: pieces of 1 KiB, shared out to the wavefronts
    constexpr int ROW_BYTES = 2 * HD, RPI = 1024 / ROW_BYTES, PIECES = TQ / RPI;
    static_assert(2 * PIECES % W == 0, "every wavefront has as many");
    auto request = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < 2 * PIECES / W; ++p) {
            const int piece = wave + W * p, which = piece / PIECES, i = piece % PIECES, ln = lane_again();
            const int lrow = RPI * i + (ln * 16) / ROW_BYTES, chunk = ((ln * 16) % ROW_BYTES >> 4) ^ swz_a<HD>(lrow);
            const char *const base = which ? gb : qb;
            const int64_t xt = which ? P.do_t : P.q_t, xh = which ? P.do_h : P.q_h;
            char *const at = q_lds + (2 * buf + which) * QT + i * 1040;
            if (P.steady && (t + 1) * TQ <= rows && nch == HD / 8) {
                const uint32_t tok = lrow >> P.g_shift, g = lrow & (P.G - 1);
                dma16(base + (t * TQ >> P.g_shift) * xt, tok * (uint32_t)xt + g * (uint32_t)xh + chunk * 16, at);
            } else {
                const int rr = t * TQ + lrow;
                if (rr < rows && chunk < nch) {
                    const int tok = token_of(P, rr), g = rr - tok * P.G;
                    dma16_at(base + tok * xt + g * xh + chunk * 16, at);
                } else {
                    *reinterpret_cast<uint4 *>(at + ln * 16) = make_uint4(0, 0, 0, 0);
                }
            }
        }
    };

    // The rows' statistics: 16 bytes of a row per thread, asked for before and added up behind the work on the tile before
    constexpr int CH = HD / 8;
    const bool adds = threadIdx.x < TQ * CH && (int)threadIdx.x % CH < nch;
    uint4 xg, xo, xr;
    float xl;
    const char *g_at, *o_at;
    const float *l_at;
    auto find = [&](int t) __attribute__((always_inline)) {
        const int r = min(t * TQ + (int)threadIdx.x / CH, rows - 1), i = token_of(P, r), g = r - i * P.G, head = hkv * P.G + g, chunk = threadIdx.x % CH;
        g_at = gb + i * P.do_t + g * P.do_h + chunk * 16;
        o_at = P.o + (P.cu_q ? 0 : b * P.o_b) + (s.q0 + i) * P.o_t + head * P.o_h + chunk * 16;
        l_at = P.lse + (P.cu_q ? head * P.total_q + s.q0 + i : ((int64_t)b * P.Hq + head) * P.max_q + i);
    };
    auto fetch = [&](int t) __attribute__((always_inline)) {
        const int r = t * TQ + (int)threadIdx.x / CH;
        xg = xo = xr = make_uint4(0, 0, 0, 0);
        xl = -INFINITY;
        if (t == 0 || !P.steady) {
            find(t);
        } else {
            // (whole tokens further on, the same head)
            const int step = TQ >> P.g_shift;
            g_at += step * P.do_t;
            o_at += step * P.o_t;
            l_at += step;
        }
        if (adds && r < rows) {
            xg = *reinterpret_cast<const uint4 *>(g_at);
            xo = *reinterpret_cast<const uint4 *>(o_at);
            if (P.rest) xr = *reinterpret_cast<const uint4 *>(o_at + (P.rest - P.o));
            xl = *l_at;
        }
    };
    auto statistics = [&](int buf) __attribute__((always_inline)) {
        float delta = dot8<T>(xg, xr, dot8<T>(xg, xo, 0.f));
        delta += lane_sum<0xB1>(delta);
        delta += lane_sum<0x4E>(delta);
        delta += lane_sum<0x141>(delta);
        if constexpr (CH == 16) delta += lane_sum<0x140>(delta);
        if (threadIdx.x < TQ * CH && threadIdx.x % CH == 0) {
            float *const at = st + buf * 2 * TQ + threadIdx.x / CH;
            // (a row that saw no key, or that does not exist: P = 0)
            at[0] = xl == -INFINITY ? -INFINITY : (kPShift<T> - xl * kLog2e) / P.c;
            at[TQ] = -delta;
        }
        if constexpr (kScaled<T>) {
            float size = dot8<T>(xg, xg, 0.f);
            size += lane_sum<0xB1>(size);
            size += lane_sum<0x4E>(size);
            size += lane_sum<0x141>(size);
            if constexpr (CH == 16) size += lane_sum<0x140>(size);
            if (threadIdx.x < TQ * CH && threadIdx.x % CH == 0) dO2[buf * TQ + threadIdx.x / CH] = size < INFINITY ? size : 0.f;
        }
    };

    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zero16();

    // One power of two for all of a tile's dS, 2^up: |dP - delta| is at most 2 |dO| |v| (O is a mean of v), so that with the largest |dO| of the
    // tile and the largest |v| of the sequence dS stays below 2^14.  (Rows and keys that are not finite have results that are not, whatever
    // the factor; others do not go by them.)  It follows the tiles up in steps of 2^4, down at once.
    int up = 0;
    float most_v2 = 0.f;
    auto scale_of = [&](int t) __attribute__((always_inline)) {
        if (t == 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) most_v2 = fmaxf(most_v2, v2[w]);
        }
        const float both = largest_of_32(dO2[(t & 1) * TQ + (lane_again() & 31)]) * most_v2;
        const int next = max(-60, min(13 - ((uni(exponent_of(both)) + 2) >> 1), 40));
        if (t > 0 && next >= up && next <= up + 4) return;
        const float f = ldexpf(1.f, next - up);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) dk[d][e] *= f;
        up = next;
    };
    auto rows_and_keys = [&](int t) __attribute__((always_inline)) {
        const int buf = t & 1, rb = t * TQ;
        const int see_first = P.causal ? uni(token_of(P, rb)) + off : s.Lk;
        if constexpr (kScaled<T>) scale_of(t);
        if (see_last(t) < w0 || w0 >= s.Lk) return;
        const RowOperand<HD, T> ra(q_lds + buf * 2 * QT), ka(k_lds + row_at<HD>(32) * wave);
        const ColOperand<HD, T> ca(q_lds + buf * 2 * QT);
        f32x16 sc, dp;
        const float *const stb = st + buf * 2 * TQ + 4 * h;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32q a4 = *reinterpret_cast<const f32q *>(stb + 8 * g), b4 = *reinterpret_cast<const f32q *>(stb + TQ + 8 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) { sc[4 * g + e] = a4[e]; dp[4 * g + e] = b4[e]; }
        }
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) sc = In<T>::mfma(ra.get(0, kk), ka.get(0, kk), sc);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) dp = In<T>::mfma(ra.get(QT, kk), vf[kk], dp);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            sc[e] = __builtin_amdgcn_exp2f(sc[e] * P.c);
            dp[e] *= kScaled<T> ? sc[e] * ldexpf(kPScale<T>, up) : sc[e];
        }
        // rows that do not see the key, and keys that do not exist
        if ((P.causal && see_first < w0 + 31) || w0 + 32 > s.Lk) {
            const int from = key >= s.Lk ? TQ : P.causal ? first_row - rb - 4 * h : 0;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (8 * (e >> 2) + (e & 3) < from) sc[e] = dp[e] = 0.f;
        }
        typename In<T>::vec pn[2], dn[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) { pn[ks] = narrow8<T>(sc, ks); dn[ks] = narrow8<T>(dp, ks); }
        char *const to = s_lds + row_at<64>(32) * wave + row_at<64>(lane & 31) + 8 * h;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const uint4 x = __builtin_bit_cast(uint4, dn[ks]);
            *reinterpret_cast<uint2 *>(to + (((4 * buf + 2 * ks) ^ swz_a<64>(lane & 31)) << 4)) = make_uint2(x.x, x.y);
            *reinterpret_cast<uint2 *>(to + (((4 * buf + 2 * ks + 1) ^ swz_a<64>(lane & 31)) << 4)) = make_uint2(x.z, x.w);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int d = 0; d < DB; ++d) dv[d] = In<T>::mfma(ca.get(QT, d, ks), pn[ks], dv[d]);
#pragma unroll
            for (int d = 0; d < DB; ++d) dk[d] = In<T>::mfma(ca.get(0, d, ks), dn[ks], dk[d]);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 4 * DB - 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // dQ^T = K^T dS^T of a tile whose turn is this wavefront's, 32 columns
    auto queries = [&](int t) __attribute__((always_inline)) {
        if (wave / DB != t % TURNS) return;
        const int d = wave % DB, steps = (min(s.Lk, see_last(t) + 1) + 15) / 16;
        const ColOperand<HD, T> kc(k_lds);
        const ColOperand<64, T> sa(s_lds);
        f32x16 acc = zero16();
        int ks = 0;
        for (; ks + 4 <= steps; ks += 4) {
#pragma unroll
            for (int u = 0; u < 4; ++u) acc = In<T>::mfma(kc.get(0, d, ks + u), sa.get(0, t & 1, ks + u), acc);
        }
        for (; ks < steps; ++ks) acc = In<T>::mfma(kc.get(0, d, ks), sa.get(0, t & 1, ks), acc);
        if constexpr (kScaled<T>) {
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = ldexpf(acc[e], -up);
        }
        const int r = t * TQ + (lane_again() & 31), i = token_of(P, min(r, rows - 1)), head = hkv * P.G + (min(r, rows - 1) - i * P.G);
        char *const dst = P.dq + (P.cu_q ? 0 : b * P.dq_b) + (s.q0 + i) * P.dq_t + head * P.dq_h;
        store_row32<T>(dst + 64 * d, acc, P.scale, P.D - 32 * d, r < rows);
    };

    if (n > 0) {
        request(0, 0);
        fetch(0);
        statistics(0);
    }
    for (int t = 0; t < n; ++t) {
        landed();
        if (t + 1 < n) {
            request(t + 1, (t + 1) & 1);
            fetch(t + 1);
        }
        if (t > 0) queries(t - 1);
        rows_and_keys(t);
        if (t + 1 < n) statistics((t + 1) & 1);
    }
    landed();
    if (n > 0) queries(n - 1);

    if constexpr (kScaled<T>) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) dk[d][e] = ldexpf(dk[d][e], -up);
    }
    const int mine = w0 + (lane_again() & 31);
    if (mine >= s.Lk) {
#pragma unroll
        for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zero16();
    }
    const bool write = mine < out_rows;
    char *const dkp = P.dk + (P.cu_k ? 0 : b * P.dk_b) + (s.k0 + mine) * P.dk_t + hkv * P.dk_h;
    char *const dvp = P.dv + (P.cu_k ? 0 : b * P.dv_b) + (s.k0 + mine) * P.dv_t + hkv * P.dv_h;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_row32<T>(dkp + 64 * d, dk[d], P.scale, P.D - 32 * d, write);
        store_row32<T>(dvp + 64 * d, dv[d], kPScale<T>, P.D - 32 * d, write);
    }
}

// dK and dV on tiles of 64 keys, two wavefronts sharing out the rows of the same keys, instead of 128: where the larger tiles leave the
// chip half empty, or where they are all at work at once and the longest of them (the first keys under a causal mask, the longest of
// packed sequences) is what the call waits for.  Small tiles read each row twice as often.  us of the backward pass, 128 -> 64: 4096 tokens,
// 8 heads of 128, no mask 250 -> 239, causal 207 -> 168; 2 x 2048, 16 heads of 64, causal 93 -> 82; 40 packed sequences of up to 1024 tokens,
// 16 heads of 64, 4 of keys 243 -> 230; but 2 x 4096, 16 heads of 128, causal 471 -> 482; 4 x 1024 93 -> 94; 100 packed sequences of up to
// 2048 tokens, 16 heads of 64, 4 of keys 1407 -> 1494.
bool few_key_tiles(const AttnParams &P)
{
    const int64_t keys = P.cu_k ? P.total_k : (int64_t)P.B * P.max_k, tiles = keys / 128 * P.Hkv, cus = cu_count();
    if (P.max_k < (P.cu_k ? 512 : 1024)) return false;
    if (P.cu_k) return tiles <= (P.D <= 64 ? 4 : 2) * cus;
    return tiles <= (P.causal && P.max_k >= 2048 ? 2 : 1) * cus;
}

// dQ on 64 rows a workgroup, two wavefronts sharing out the keys of the same rows, instead of 128.  us, 128 -> 64: 2048 tokens, 8
// heads of 128, no mask 65 -> 44, causal 62 -> 40; 4096 tokens, causal 121 -> 86; but 2 x 4096, 16 heads of 128 257 -> 282, 32 x 128, 8
// heads of 128 18.5 -> 20.0.  16 heads of 64 (the whole backward pass): 2 x 2048, causal 100 -> 93, 8192 tokens, causal 531 -> 522; but
// 2 x 4096, no mask 521 -> 530, 4 x 4096, 4 key heads, causal 587 -> 600.
bool few_rows(const AttnParams &P)
{
    const int64_t full = (int64_t)P.B * P.Hkv * ((P.max_rows + 127) / 128), cus = cu_count();
    return (P.max_k >= 512 && full <= cus) || (P.D <= 64 && P.causal && P.max_k >= 2048 && full <= 4 * cus);
}

// One workgroup per sequence and key head, all three gradients in one pass over memory, instead of dQ and then dK and dV: up to 256 keys (what
// LDS holds), with heads enough for a quarter of the CUs.  It walks all rows of its key head (queries x query heads of it), which dQ's launch
// spreads over the chip: with more than 256 of them, heads enough for half of the CUs, or for three quarters where heads are small and dQ is
// quick.  us, two launches -> one: 64 x 256 tokens, 8 heads of 128, no mask 120 -> 87, causal 106 -> 75; 32 x 128, causal 32 -> 20.5; 128 x 197,
// 12 heads of 64 159 -> 136; 64 x 128, no mask 49 -> 31; but 4 x 256, 8 heads of 128 30 -> 33.  Many rows: 16 x 1024 queries over 128 keys,
// 32 heads of 128, 8 of keys, causal 398 -> 219; 24 x 512 over 256, 64 heads of 64, 8 of keys, causal 315 -> 198; but 8 x 2048 over 256, 8
// heads of 128 138 -> 200; 8 x 256, 32 heads of 128, 8 of keys, no mask 94 -> 105 (causal 95 -> 88); 8 x 1024 over 256, 64 heads of 128, 8
// of keys 504 -> 766; 64 x 512 over 128, 32 heads of 64, 1 of keys, causal 337 -> 779.
bool whole_sequences(const AttnParams &P)
{
    const int64_t heads = (int64_t)P.B * P.Hkv, quarters = P.max_rows <= 256 ? 1 : P.D > 64 ? 2 : 3;
    return P.max_k <= 256 && 4 * heads >= quarters * cu_count() && heads <= (1 << 22);
}

template <class T, int HD> int launch_bwd(AttnParams P, hipStream_t st)
{
    if (whole_sequences(P)) {
        const dim3 grid((unsigned)((int64_t)P.B * P.Hkv));
        if (HD <= 64 && P.max_k <= 128) hipLaunchKernelGGL((attn_bwd_short_kernel<T, 64, 4>), grid, dim3(256), 0, st, P);
        else hipLaunchKernelGGL((attn_bwd_short_kernel<T, HD, 8>), grid, dim3(512), 0, st, P);
        return hip_status(hipGetLastError());
    }
    const int rows = few_rows(P) ? 64 : 128;
    P.tiles = (P.max_rows + rows - 1) / rows;
    const dim3 row_grid((unsigned)((int64_t)P.B * P.Hkv * P.tiles));
    if (rows == 64) hipLaunchKernelGGL((attn_dq_kernel<T, HD, 2>), row_grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL((attn_dq_kernel<T, HD, 4>), row_grid, dim3(256), 0, st, P);
    const int rc = hip_status(hipGetLastError());
    if (rc != SDROP_OK) return rc;
    const bool few = few_key_tiles(P);
    const int keys = few ? 64 : 128;
    P.tiles = (P.max_k + keys - 1) / keys;
    const dim3 grid((unsigned)((int64_t)P.B * P.Hkv * P.tiles));
    if (few) hipLaunchKernelGGL((attn_dkv_kernel<T, HD, 2>), grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL((attn_dkv_kernel<T, HD, 4>), grid, dim3(256), 0, st, P);
    return hip_status(hipGetLastError());
}

size_t stats_bytes(const AttnParams &P) { return (size_t)(stats_rows(P) + 64) * 2 * sizeof(float); }

}  // namespace
}  // namespace sdrop

using namespace sdrop;

extern "C" {

size_t sdrop_attn_bwd_workspace_bytes(const sdrop_attn_t *a)
{
    AttnParams P;
    return attn_params(a, true, P) == SDROP_OK ? stats_bytes(P) : 0;
}

int sdrop_attn_bwd(const void *dO, const void *q, const void *k, const void *v, const void *o, const void *o_rest, const float *lse,
                   void *dq, void *dk, void *dv, const sdrop_attn_t *a, void *ws, size_t ws_bytes, void *stream)
{
    if (!dO || !q || !k || !v || !o || !lse || !dq || !dk || !dv) return SDROP_EINVAL;
    AttnParams P;
    const int rc = attn_params(a, true, P);
    if (rc != SDROP_OK) return rc;
    if (!aligned16(dO) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(o_rest) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || reinterpret_cast<uintptr_t>(lse) % 4) return SDROP_EALIGN;
    if (!ws || ws_bytes < stats_bytes(P) || !aligned16(ws)) return SDROP_EWORKSPACE;
    const int64_t most = (int64_t(1) << 24) - 1, heads = (int64_t)P.B * P.Hkv;      // (a launch counts its threads in 32 bits)
    if (heads * (((int64_t)P.max_rows + 63) / 64) > most || heads * (((int64_t)P.max_k + 63) / 64) > most) return SDROP_ESHAPE;
    P.dout = static_cast<const char *>(dO);
    P.q = static_cast<const char *>(q);
    P.k = static_cast<const char *>(k);
    P.v = static_cast<const char *>(v);
    P.o = static_cast<const char *>(o);
    P.rest = static_cast<const char *>(o_rest);
    P.lse = const_cast<float *>(lse);
    P.dq = static_cast<char *>(dq);
    P.dk = static_cast<char *>(dk);
    P.dv = static_cast<char *>(dv);
    P.delta = static_cast<float *>(ws);
    auto narrow = [&](int64_t t, int64_t h) { return (P.G - 1) * h + 32 / P.G * t < (int64_t(1) << 31); };
    P.steady = 16 % P.G == 0 && narrow(P.q_t, P.q_h) && narrow(P.do_t, P.do_h);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->dtype == SDROP_F16) return P.D <= 64 ? launch_bwd<F16, 64>(P, st) : launch_bwd<F16, 128>(P, st);
    return P.D <= 64 ? launch_bwd<BF16, 64>(P, st) : launch_bwd<BF16, 128>(P, st);
}

}  // extern "C"
