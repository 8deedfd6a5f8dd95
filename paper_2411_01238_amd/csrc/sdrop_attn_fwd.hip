// Attention, forward: one pass over the keys with a running maximum and sum.
//
// A wavefront owns 32 rows (see attn_common.h) and computes S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 matrix instructions: a lane
// then holds keys of ONE query (column l % 32), so that maximum, sum and the rescaling of O need no exchange but with lane
// l ^ 32, and P^T is the second product's operand in the registers it was computed in (ColOperand reads V across its rows in
// the same order).  K and V tiles go from memory to LDS without registers, one tile ahead.
#include "attn_common.h"
#include <math.h>

namespace sdrop {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// QW: wavefronts of the workgroup that own rows of their own (32 each); KW (1 or 2) wavefronts of the same rows take the keys of a tile in
// turn and are joined at the end.  MB: blocks of 32 keys per wavefront and tile.  STAGES: tiles that LDS holds.
// Heads of 64 are bound by the exponentials: four wavefronts per SIMD, so that products run beside them (2 x 4096, 16 heads, no mask 171 ->
// 158 us; 24 sequences of 64 to 2000 tokens, 16 heads, 4 of keys, causal 121 -> 104).  That leaves 128 registers, hence operands that
// are read two ahead of the matrix instructions and no more.
template <class T, int HD, int QW, int KW, int MB, int STAGES>
__global__ __launch_bounds__(64 * QW * KW, QW * KW == 4 ? (HD <= 64 ? 4 : 2) : 1) void attn_fwd_kernel(AttnParams P)
{
    constexpr int TKV = 32 * MB * KW, TILE = tile_bytes<HD>(TKV), DB = HD / 32;
    __shared__ __attribute__((aligned(1024))) char lds[STAGES * 2 * TILE];
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), wq = wave % QW, wk = wave / QW, h = lane >> 5;

    int bh, unit;
    place(P, P.tiles * P.splits, bh, unit);
    const int b = bh / P.Hkv, hkv = bh - b * P.Hkv;
    const int tile = P.tiles - 1 - unit / P.splits, split = unit % P.splits;        // (under a causal mask the last rows have most to do)
    const Sequence s = sequence_of(P, b);
    if (!s.ok) return;
    const int rows = s.Lq * P.G, R0 = tile * 32 * QW;
    if (R0 >= rows) return;
    const int off = s.Lk - s.Lq;                    // causal: token i sees keys up to i + off
    const int r_last = min(R0 + 32 * QW, rows) - 1;
    const int k_end = P.causal ? min(s.Lk, token_of(P, r_last) + off + 1) : s.Lk;
    // this workgroup's part of the key tiles
    const int n_tiles = k_end > 0 ? (k_end + TKV - 1) / TKV : 0, per = (n_tiles + P.splits - 1) / P.splits;
    const int t0 = min(split * per, n_tiles), t1 = min(t0 + per, n_tiles);

    // this lane's row, and this wavefront's first and last
    const int r = R0 + 32 * wq + (lane & 31), w0 = R0 + 32 * wq;
    const bool live = r < rows;
    const int i = token_of(P, min(r, rows - 1)), head = hkv * P.G + (min(r, rows - 1) - i * P.G);
    const int lim = !live ? -1 : P.causal ? min(s.Lk - 1, i + off) : s.Lk - 1;      // last key this row sees
    const bool any = w0 < rows;
    const int w_first = any ? uni(token_of(P, w0)) + off : 0, w_last = any ? uni(token_of(P, min(w0 + 31, rows - 1))) + off : -1;

    typename In<T>::vec qf[HD / 16];
    auto load_q = [&]() __attribute__((always_inline)) {
        const char *const qp = P.q + (P.cu_q ? 0 : b * P.q_b) + (s.q0 + i) * P.q_t + head * P.q_h;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
            const int col = 16 * kk + 8 * h;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (live && col < P.D) x = *reinterpret_cast<const uint4 *>(qp + 2 * col);
            qf[kk] = __builtin_bit_cast(typename In<T>::vec, x);
        }
    };

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zero16();
    float m = -INFINITY, l = 0.f;           // running maximum (of S before the scale) and this lane's part of the sum
    const float rc = __builtin_amdgcn_rcpf(P.c);
    float large_from = -INFINITY;           // scores above this have a large share (kLargeShare), or are 2^8 beyond the maximum

    // 32 * MB keys from kv0 on, whose K and V lie at kt and vt
    auto compute_keys = [&](int kv0, const char *kt, const char *vt) __attribute__((always_inline)) {
        f32x16 sc[MB];
        const RowOperand<HD, T> ka(kt);
        // (a wavefront at its matrix instructions goes before the one beside it at its exponentials: 8192 tokens, 16 heads of 128, causal
        // 305 -> 275 us)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            sc[mb] = zero16();
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) sc[mb] = In<T>::mfma(ka.get(row_at<HD>(32) * mb, kk), qf[kk], sc[mb]);
        }
        if constexpr (HD <= 64 && MB == 2) {
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
            for (int i = 0; i < MB * HD / 16 - 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (kv0 + 32 * MB > s.Lk || (P.causal && kv0 + 32 * MB - 1 > w_first)) {
            const int last = lim - kv0 - 4 * h;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * mb + 8 * (e >> 2) + (e & 3) > last) sc[mb][e] = -INFINITY;
        }
        float mx = sc[0][0];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[mb][e]);
        mx = join_halves(mx, [](float a, float b2) { return fmaxf(a, b2); });
        const bool large = mx > large_from;
        const uint64_t any_large = __ballot(large);
        // O and the sum are rescaled only when a maximum has grown by more than 2^8 in P: until then P stays below 256
        if (any_large && __any(mx > m && (mx - m) * P.c > 8.f)) {
            const float mn = fmaxf(m, mx);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * P.c);
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= f;
            m = mn;
        }
        const float mc = m == -INFINITY ? 0.f : m * P.c;       // (a row that has seen no key yet: P = 0)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[mb][e] = __builtin_amdgcn_exp2f(sc[mb][e] * P.c - mc);
                l += sc[mb][e];
            }
        // (few rows wait for the memory: every tile has the product with what P's rounding took beside it)
        if constexpr (QW > 1) large_from = m + fminf(__builtin_amdgcn_logf(kLargeShare * l), 8.f) * rc;
        const ColOperand<HD, T> va(vt);
        if constexpr (HD <= 64 && MB == 2) __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < 2 * MB; ++ks) {
            const typename In<T>::vec p = narrow8<T>(sc[ks >> 1], ks & 1);
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] = In<T>::mfma(va.get(0, d, ks), p, o[d]);
        }
        if constexpr (HD <= 64 && MB == 2) {
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < 2 * MB * DB - 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (any_large) {
            // (nothing is added to other rows: a row's result does not depend on those beside it)
            const uint32_t mask = large ? ~0u : 0u;
#pragma unroll
            for (int ks = 0; ks < 2 * MB; ++ks) {
                const typename In<T>::vec p = narrow8_rest<T>(sc[ks >> 1], ks & 1, mask);
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] = In<T>::mfma(va.get(0, d, ks), p, o[d]);
            }
        }
    };

    const int kv_first = t0 * TKV, nch = P.D / 8;
    if constexpr (QW > 1) {
        const char *kb = P.k + (P.cu_k ? 0 : b * P.k_b) + (s.k0 + kv_first) * P.k_t + hkv * P.k_h;
        const char *vb = P.v + (P.cu_k ? 0 : b * P.v_b) + (s.k0 + kv_first) * P.v_t + hkv * P.v_h;
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
        load_q();
        if (t0 < t1) request(t0, 0);
        for (int t = t0; t < t1; ++t) {
            const int buf = (t - t0) & 1;
            landed();
            if (t + 1 < t1) request(t + 1, buf ^ 1);
            const int kv0 = t * TKV + 32 * MB * wk;
            if ((KW > 1 && kv0 >= s.Lk) || (P.causal && kv0 > w_last)) continue;        // (nothing for these rows)
            const char *const kt = lds + buf * 2 * TILE + wk * row_at<HD>(32 * MB);
            compute_keys(kv0, kt, kt + TILE);
        }
    } else {
        // A wavefront streams its own keys through its own part of LDS, STAGES blocks of 32 ahead and without barriers: few rows
        // are bound by the memory, which wants as much under way as there is room for.
        constexpr int BLOCK = tile_bytes<HD>(32), LOADS = 2 * 32 * HD / 512;
        static_assert(MB == 1 && LOADS * (STAGES - 1) < 64, "blocks of 32 keys; what is under way is counted in six bits");
        char *const mine = lds + wave * STAGES * 2 * BLOCK;
        const char *kb = P.k + (P.cu_k ? 0 : b * P.k_b) + (s.k0 + kv_first + 32 * wk) * P.k_t + hkv * P.k_h;
        const char *vb = P.v + (P.cu_k ? 0 : b * P.v_b) + (s.k0 + kv_first + 32 * wk) * P.v_t + hkv * P.v_h;
        TileLoad<HD, 32, 1> lk, lv;
        lk.init(P.k_t, 0);
        lv.init(P.v_t, 0);
        const int end = min(k_end, t1 * TKV);
        auto request = [&](int kv0, int stage) __attribute__((always_inline)) {
            if (kv0 < end) {
                lk.issue(kb, P.k_t, mine + stage * 2 * BLOCK, s.Lk - kv0, nch);
                lv.issue(vb, P.v_t, mine + stage * 2 * BLOCK + BLOCK, s.Lk - kv0, nch);
            }
            kb += TKV * P.k_t;
            vb += TKV * P.v_t;
        };
        int kv0 = kv_first + 32 * wk;
#pragma unroll 1
        for (int i2 = 0; i2 < STAGES; ++i2) request(kv0 + i2 * TKV, i2);
        load_q();
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
        for (int stage = 0; kv0 < end; kv0 += TKV) {
            // the blocks behind this one may still be under way: all of their loads if the last of them is whole
            const int far = kv0 + (STAGES - 1) * TKV;
            asm volatile("" ::: "memory");
            if (far < end && far + 32 <= s.Lk) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(LOADS * (STAGES - 1)));
            else __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            const char *const kt = mine + stage * 2 * BLOCK;
            compute_keys(kv0, kt, kt + BLOCK);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            request(kv0 + STAGES * TKV, stage);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
    }
    l = join_halves(l, [](float a, float b2) { return a + b2; });

    // the two wavefronts of the same rows, scaled to their common maximum; the first one goes on
    if constexpr (KW == 2) {
        float *const ml = reinterpret_cast<float *>(lds) + wq * (2 + DB * 16) * 64 + lane, *const ob = ml + 128;
        static_assert(QW * (2 + DB * 16) * 64 * 4 <= STAGES * 2 * TILE, "room for half of the wavefronts");
        landed();
        if (wk == 1) {
            ml[0] = m;
            ml[64] = l;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) ob[(d * 16 + e) * 64] = o[d][e];
        }
        __syncthreads();
        if (wk == 1) return;
        const float m1 = ml[0], mn = fmaxf(m, m1), ref = mn == -INFINITY ? 0.f : mn;
        const float f0 = __builtin_amdgcn_exp2f((m - ref) * P.c), f1 = __builtin_amdgcn_exp2f((m1 - ref) * P.c);
        l = l * f0 + ml[64] * f1;
        m = mn;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = o[d][e] * f0 + ob[(d * 16 + e) * 64] * f1;
    }
    // (this lane's row once more: kept over the loop it would be registers that the fourth wavefront of a SIMD does not leave)
    const int ln = lane_again(), r_out = R0 + 32 * wq + (ln & 31), h_out = ln >> 5;
    const int r_in = min(r_out, rows - 1), i_out = token_of(P, r_in), head_out = hkv * P.G + (r_in - i_out * P.G);
    const bool live_out = r_out < rows;
    const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;         // (no key seen: 0; NaN stays NaN)
    const float lse = l > 0.f || l != l ? (m * P.c + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    if (P.splits > 1) {
        const int64_t row = ((int64_t)split * P.B * P.Hkv + bh) * P.max_rows + r_out;
        if (live_out && h_out == 0) P.part_lse[row] = lse;
        float *const dst = P.part_o + row * P.D;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * d + 8 * g + 4 * h_out;
                const f32q x = {o[d][4 * g] * inv, o[d][4 * g + 1] * inv, o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv};
                if (live_out && col < P.D) *reinterpret_cast<f32q *>(dst + col) = x;
            }
        }
        return;
    }
    if (P.lse && live_out && h_out == 0) P.lse[P.cu_q ? head_out * P.total_q + s.q0 + i_out : ((int64_t)b * P.Hq + head_out) * P.max_q + i_out] = lse;
    const int64_t at = (P.cu_q ? 0 : b * P.o_b) + (s.q0 + i_out) * P.o_t + head_out * P.o_h;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_row32<T>(P.out + at + 64 * d, o[d], inv, P.D - 32 * d, live_out, P.out_rest ? P.out_rest + at + 64 * d : nullptr);
    }
}

// Joins the parts of the keys: a wavefront per row, O = sum of exp(lse_s - lse) O_s in the parts' order.
template <class T>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnParams P)
{
    using E = typename In<T>::out16;
    typedef __attribute__((__vector_size__(2 * sizeof(E)))) E e2;
    const int lane = threadIdx.x & 63;
    const int64_t n = (int64_t)P.B * P.Hkv * P.max_rows;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < n; w += (int64_t)gridDim.x * 4) {
        const int bh = (int)(w / P.max_rows), r = (int)(w - (int64_t)bh * P.max_rows), b = bh / P.Hkv;
        const Sequence s = sequence_of(P, uni(b));
        if (!s.ok || r >= s.Lq * P.G) continue;
        const int i = token_of(P, r), head = (bh - b * P.Hkv) * P.G + r - i * P.G;
        // a lane has the weights of parts lane and lane + 64; the parts' O are asked for eight at a time
        float x[2], mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int p = lane + 64 * u;
            x[u] = p < P.splits ? P.part_lse[(int64_t)p * n + w] : -INFINITY;
            mx = fmaxf(mx, x[u]);
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 64));
        const float ref = mx == -INFINITY ? 0.f : mx;
        float sum = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            x[u] = __builtin_amdgcn_exp2f((x[u] - ref) * kLog2e);
            sum += x[u];
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
        const float *const src = P.part_o + w * P.D + 2 * lane;
        for (int p0 = 0; p0 < P.splits; p0 += 8) {
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                v[u] = make_float2(0.f, 0.f);
                if (p0 + u < P.splits && 2 * lane < P.D) v[u] = *reinterpret_cast<const float2 *>(src + (int64_t)(p0 + u) * n * P.D);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int p = p0 + u;
                const float f = __shfl(p < 64 ? x[0] : x[1], p & 63, 64);
                a0 += f * v[u].x;
                a1 += f * v[u].y;
            }
        }
        const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
        if (2 * lane < P.D) {
            const e2 x = {static_cast<E>(a0 * inv), static_cast<E>(a1 * inv)};
            const int64_t at = (P.cu_q ? 0 : b * P.o_b) + (s.q0 + i) * P.o_t + head * P.o_h + 4 * lane;
            *reinterpret_cast<e2 *>(P.out + at) = x;
            if (P.out_rest) {
                const e2 y = {static_cast<E>(a0 * inv - static_cast<float>(x[0])), static_cast<E>(a1 * inv - static_cast<float>(x[1]))};
                *reinterpret_cast<e2 *>(P.out_rest + at) = y;
            }
        }
        if (P.lse && lane == 0)
            P.lse[P.cu_q ? head * P.total_q + s.q0 + i : ((int64_t)b * P.Hq + head) * P.max_q + i] = sum > 0.f || sum != sum ? ref + __builtin_amdgcn_logf(sum) * kLn2 : -INFINITY;
    }
}

// How the forward pass is laid out: rows per workgroup (32: all of its wavefronts share out the keys of the same rows), row tiles and
// parts of the keys.
struct FwdPlan { int rows; int64_t tiles, splits; };

template <class T, int HD> int launch_fwd(AttnParams P, const FwdPlan &p, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)P.B * P.Hkv * P.tiles * P.splits));
    if (p.rows == 32) hipLaunchKernelGGL((attn_fwd_kernel<T, HD, 1, 2, 1, HD <= 64 ? 4 : 2>), grid, dim3(128), 0, st, P);
    else if (p.rows == 64) hipLaunchKernelGGL((attn_fwd_kernel<T, HD, 2, 2, 1, 2>), grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL((attn_fwd_kernel<T, HD, 4, 1, 2, 2>), grid, dim3(256), 0, st, P);
    const int rc = hip_status(hipGetLastError());
    if (rc != SDROP_OK || P.splits == 1) return rc;
    const int64_t groups = ((int64_t)P.B * P.Hkv * P.max_rows + 3) / 4;
    hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)(groups < 65536 ? groups : 65536)), dim3(256), 0, st, P);
    return hip_status(hipGetLastError());
}

// 64 rows a workgroup, two wavefronts sharing out the keys of the same rows, where 128 would leave CUs without work, or with one
// workgroup each and keys enough to share.  us, 128 (in parts of the keys and joined, where that was the faster) -> 64: 2048 tokens,
// 8 heads of 128, no mask 41 -> 34, causal 34 -> 32; 4096 tokens, causal 76 -> 67; 2 x 2048, 16 heads of 64, causal 38 -> 32; but
// 2 x 2048, 16 heads of 128, causal 55 -> 58; 32 x 128, 8 heads of 128, causal 12.1 -> 13.4.
// Parts of the keys cost a pass over what they leave (12 us for 2048 rows of 8 heads): for few rows they fill the chip twice (16384
// keys of 16 sequences, 8 heads of 128: 4 parts 144 us, 16 parts 145), for more rows once.
FwdPlan fwd_plan(const AttnParams &P)
{
    FwdPlan p;
    const int64_t heads = (int64_t)P.B * P.Hkv, cus = cu_count(), full = heads * ((P.max_rows + 127) / 128);
    const bool share = (full <= cus && P.max_k >= 512) || (P.D <= 64 && full <= 2 * cus && P.max_k >= 2048);
    p.rows = P.max_rows <= 32 ? 32 : share ? 64 : 128;
    p.tiles = (P.max_rows + p.rows - 1) / p.rows;
    const int64_t groups = heads * p.tiles, key_tiles = (P.max_k + 63) / 64, want = (p.rows == 32 ? 2 : 1) * cus;
    p.splits = 1;
    if (groups < want) {
        p.splits = (want + groups - 1) / groups;
        const int64_t most = key_tiles / 4;             // at least four tiles of keys each
        if (p.splits > most) p.splits = most < 1 ? 1 : most;
        if (p.splits > 128) p.splits = 128;
    }
    return p;
}

size_t part_bytes(const AttnParams &P, const FwdPlan &p)
{
    return p.splits == 1 ? 0 : (size_t)p.splits * P.B * P.Hkv * P.max_rows * (P.D + 4) * sizeof(float);
}

bool stride_ok(int64_t s, int64_t most) { return s >= 0 && s <= most && s % 8 == 0; }

}  // namespace

int attn_params(const sdrop_attn_t *a, bool backward, AttnParams &P)
{
    if (!a || !(a->scale > 0.0 && a->scale < INFINITY) || (a->causal != 0 && a->causal != 1)) return SDROP_EINVAL;
    if (a->k_len && a->cu_k) return SDROP_EINVAL;
    if (a->dtype != SDROP_F16 && a->dtype != SDROP_BF16) return SDROP_EDTYPE;
    const int64_t lim = int64_t(1) << 30;
    if (a->B < 1 || a->max_q < 1 || a->max_k < 1 || a->Hq < 1 || a->Hkv < 1 || a->Hq % a->Hkv || a->D < 8 || a->D > 128 || a->D % 8) return SDROP_ESHAPE;
    if (a->B > (1 << 20) || a->max_q > lim || a->max_k > lim || a->Hq > 65536 || a->max_q * a->Hq > lim || a->B * a->Hq > (int64_t(1) << 24)) return SDROP_ESHAPE;
    if ((a->cu_q && (a->total_q < 1 || a->total_q > lim)) || (a->cu_k && (a->total_k < 1 || a->total_k > lim))) return SDROP_ESHAPE;
    const int64_t token = int64_t(1) << 24, wide = int64_t(1) << 50;
    const int64_t strides[8][3] = {{a->q_b, a->q_t, a->q_h}, {a->k_b, a->k_t, a->k_h}, {a->v_b, a->v_t, a->v_h}, {a->o_b, a->o_t, a->o_h},
                                   {a->do_b, a->do_t, a->do_h}, {a->dq_b, a->dq_t, a->dq_h}, {a->dk_b, a->dk_t, a->dk_h}, {a->dv_b, a->dv_t, a->dv_h}};
    for (int i = 0; i < (backward ? 8 : 4); ++i) {
        if (!stride_ok(strides[i][0], wide) || !stride_ok(strides[i][1], token) || !stride_ok(strides[i][2], wide)) return SDROP_ESHAPE;
        // an output's elements have places of their own
        const bool keys = i >= 6;
        const int64_t tokens = keys ? (a->cu_k ? a->total_k : a->max_k) : a->cu_q ? a->total_q : a->max_q;
        if ((backward ? i >= 5 : i == 3) && ((strides[i][0] == 0 && a->B > 1 && !(keys ? a->cu_k : a->cu_q)) ||
            (strides[i][1] == 0 && tokens > 1) || (strides[i][2] == 0 && (keys ? a->Hkv : a->Hq) > 1))) return SDROP_ESHAPE;
    }
    P = AttnParams();
    P.q_b = 2 * a->q_b; P.q_t = 2 * a->q_t; P.q_h = 2 * a->q_h;
    P.k_b = 2 * a->k_b; P.k_t = 2 * a->k_t; P.k_h = 2 * a->k_h;
    P.v_b = 2 * a->v_b; P.v_t = 2 * a->v_t; P.v_h = 2 * a->v_h;
    P.o_b = 2 * a->o_b; P.o_t = 2 * a->o_t; P.o_h = 2 * a->o_h;
    P.do_b = 2 * a->do_b; P.do_t = 2 * a->do_t; P.do_h = 2 * a->do_h;
    P.dq_b = 2 * a->dq_b; P.dq_t = 2 * a->dq_t; P.dq_h = 2 * a->dq_h;
    P.dk_b = 2 * a->dk_b; P.dk_t = 2 * a->dk_t; P.dk_h = 2 * a->dk_h;
    P.dv_b = 2 * a->dv_b; P.dv_t = 2 * a->dv_t; P.dv_h = 2 * a->dv_h;
    P.cu_q = a->cu_q;
    P.cu_k = a->cu_k;
    P.k_len = a->k_len;
    P.total_q = a->total_q;
    P.total_k = a->total_k;
    P.B = (int32_t)a->B;
    P.max_q = (int32_t)a->max_q;
    P.max_k = (int32_t)a->max_k;
    P.Hq = (int32_t)a->Hq;
    P.Hkv = (int32_t)a->Hkv;
    P.G = P.Hq / P.Hkv;
    P.D = (int32_t)a->D;
    P.causal = a->causal;
    P.max_rows = P.max_q * P.G;
    // r / G by a multiplication (Granlund, Montgomery 1994): exact for r < 2^31
    while ((1 << P.g_shift) < P.G) ++P.g_shift;
    P.g_mul = (uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << P.g_shift) - (uint64_t)P.G)) / (uint64_t)P.G + 1);
    P.scale = (float)a->scale;
    P.c = (float)(a->scale * 1.4426950408889634);
    if (!(P.c >= 0x1p-100f && P.c < INFINITY)) return SDROP_EINVAL;         // (the backward pass divides lse by it)
    P.status = device_status_word();
    return SDROP_OK;
}

}  // namespace sdrop

using namespace sdrop;

extern "C" {

size_t sdrop_attn_workspace_bytes(const sdrop_attn_t *a)
{
    AttnParams P;
    if (attn_params(a, false, P) != SDROP_OK) return 0;
    return part_bytes(P, fwd_plan(P));
}

int sdrop_attn(const void *q, const void *k, const void *v, void *o, void *o_rest, float *lse, const sdrop_attn_t *a, void *ws,
               size_t ws_bytes, void *stream)
{
    if (!q || !k || !v || !o) return SDROP_EINVAL;
    AttnParams P;
    const int rc = attn_params(a, false, P);
    if (rc != SDROP_OK) return rc;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(o_rest) || reinterpret_cast<uintptr_t>(lse) % 4)
        return SDROP_EALIGN;
    const FwdPlan p = fwd_plan(P);
    const size_t need = part_bytes(P, p);
    if (ws_bytes < need || (need && (!ws || !aligned16(ws)))) return SDROP_EWORKSPACE;
    if ((int64_t)P.B * P.Hkv * p.tiles * p.splits > (int64_t(1) << 24) - 1) return SDROP_ESHAPE;      // (a launch counts its threads in 32 bits)
    P.q = static_cast<const char *>(q);
    P.k = static_cast<const char *>(k);
    P.v = static_cast<const char *>(v);
    P.out = static_cast<char *>(o);
    P.out_rest = static_cast<char *>(o_rest);
    P.lse = lse;
    P.tiles = (int32_t)p.tiles;
    P.splits = (int32_t)p.splits;
    P.part_o = static_cast<float *>(ws);
    P.part_lse = P.splits > 1 ? P.part_o + (int64_t)P.splits * P.B * P.Hkv * P.max_rows * P.D : nullptr;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a->dtype == SDROP_F16) return P.D <= 64 ? launch_fwd<F16, 64>(P, p, st) : launch_fwd<F16, 128>(P, p, st);
    return P.D <= 64 ? launch_fwd<BF16, 64>(P, p, st) : launch_fwd<BF16, 128>(P, p, st);
}

}  // extern "C"
