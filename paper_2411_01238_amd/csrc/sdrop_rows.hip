// Element dropout and layer norm around the substituted layers (the paper's baseline, arxiv 2411.01238 Section 2.1, and the
// norms of its transformer blocks, Section 4.2): row-wise operators, all of them bound by memory.
//
//     dropout    y = r + m x / (1 - p)                                   dx = m dy / (1 - p), m drawn again
//     norm       h = r + m x / (1 - p)  (or x itself), rounded to its type
//                mu = mean(h), rs = 1 / sqrt(var(h) + eps), z = (h - mu) rs, y = z gamma + beta
//     backward   w = dy gamma,  dr = dh + rs (w - mean(w) - z mean(w z)),  dx = m dr / (1 - p)
//                dgamma = sum over rows of dy z,  dbeta = sum over rows of dy
//
// Everything between load and store is fp32; sums over a row and over rows are in an order that depends on the shape alone.
#include "rows_common.h"
#include <math.h>

namespace sdrop {
namespace {

// ---- dropout ----

struct DropoutArgs {
    const char *x, *r;
    char *y;
    int64_t chunks;                 // 8-element chunks of all rows
    int64_t ld_x, ld_r, ld_y;       // elements
    int64_t drow;                   // chunks a thread moves on per step: drow rows and dcol chunks
    int32_t N, per_row, dcol;
    ElementMask mask;
};

template <class T, bool TAIL, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs A)
{
    const int64_t step = (int64_t)gridDim.x * 256;
    int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    int64_t row = c / A.per_row;
    int col = (int)(c - row * A.per_row);
    for (; c < A.chunks; c += step) {
        const int n = A.N - col * 8;
        float x[8], f[8], r[8];
        load8<T, TAIL>(reinterpret_cast<const T *>(A.x) + row * A.ld_x + col * 8, n, x);
        if constexpr (RES) load8<T, TAIL>(reinterpret_cast<const T *>(A.r) + row * A.ld_r + col * 8, n, r);
        mask8(A.mask, (uint64_t)c, f);
        // (a dropped element is 0 whatever x holds there, an infinity or NaN too)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (f[i] != 0.f ? x[i] * f[i] : 0.f) + (RES ? r[i] : 0.f);
        store8<T, TAIL>(reinterpret_cast<T *>(A.y) + row * A.ld_y + col * 8, n, x);
        row += A.drow;
        col += A.dcol;
        if (col >= A.per_row) { col -= A.per_row; ++row; }
    }
}

template <class T> void launch_dropout(const DropoutArgs &A, unsigned grid, hipStream_t st)
{
    const bool tail = A.N % 8 != 0;
    if (A.r) {
        if (tail) hipLaunchKernelGGL((dropout_kernel<T, true, true>), dim3(grid), dim3(256), 0, st, A);
        else hipLaunchKernelGGL((dropout_kernel<T, false, true>), dim3(grid), dim3(256), 0, st, A);
    } else {
        if (tail) hipLaunchKernelGGL((dropout_kernel<T, true, false>), dim3(grid), dim3(256), 0, st, A);
        else hipLaunchKernelGGL((dropout_kernel<T, false, false>), dim3(grid), dim3(256), 0, st, A);
    }
}

// ---- layer norm ----

struct NormArgs {
    // forward: x, r (may be null) -> h (may be null), y.   backward: dy, dh (may be null), h -> dr, dx (either may be null)
    const char *x, *r, *gamma, *beta, *dy, *dh;
    char *h, *y, *dr, *dx;
    float *mean, *rstd;             // forward: may be null
    float *part;                    // backward: fp32 rows [parts][2][N] of dgamma and dbeta; null: not wanted
    int64_t M, ld_x, ld_r, ld_h, ld_y, ld_dy, ld_dh, ld_dr, ld_dx;
    int64_t rows_per_part;          // column sums of the longest rows
    int32_t N, per_row, w32;        // per_row: chunks of a row; w32: gamma and beta are fp32
    float eps, inv_n;
    ElementMask mask;
};

// eight weights of type T, or fp32 ones
template <class T, bool TAIL> __device__ __forceinline__ void load_weight8(const char *p, int w32, int col, int n, float (&v)[8])
{
    if (sizeof(T) == 4 || w32) load8<float, TAIL>(reinterpret_cast<const float *>(p) + col, n, v);
    else load8<T, TAIL>(reinterpret_cast<const T *>(p) + col, n, v);
}

// Sum over the WPR wavefronts of a row, in every lane.  `red`: WPR floats of LDS that no one else writes until the next barrier.
template <int WPR> __device__ __forceinline__ float row_sum(float v, float *red, int wave)
{
    v = wave_sum(v);
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int i = 1; i < WPR; ++i) v += red[i];
    }
    return v;
}

// h of one chunk: x, plus dropout and residual where the call has them; written to H, and rounded, where it is a tensor of its own
template <class T, bool TAIL> __device__ __forceinline__ void chunk_h(const NormArgs &A, int64_t row, int col, int n, float (&h)[8])
{
    load8<T, TAIL>(reinterpret_cast<const T *>(A.x) + row * A.ld_x + col, n, h);
    if (!A.h) return;
    float r[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (A.r) load8<T, TAIL>(reinterpret_cast<const T *>(A.r) + row * A.ld_r + col, n, r);
    if (A.mask.threshold) {
        float f[8];
        mask8(A.mask, (uint64_t)row * (uint64_t)A.per_row + (uint64_t)(col >> 3), f);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = (f[i] != 0.f ? h[i] * f[i] : 0.f) + r[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += r[i];
    }
    store8<T, TAIL>(reinterpret_cast<T *>(A.h) + row * A.ld_h + col, n, h);
}

template <class T, bool TAIL> __device__ __forceinline__ void chunk_y(const NormArgs &A, int64_t row, int col, int n, const float (&h)[8], float mu, float rs)
{
    float g[8], b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, y[8];
    load_weight8<T, TAIL>(A.gamma, A.w32, col, n, g);
    if (A.beta) load_weight8<T, TAIL>(A.beta, A.w32, col, n, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (h[i] - mu) * rs * g[i] + b[i];
    store8<T, TAIL>(reinterpret_cast<T *>(A.y) + row * A.ld_y + col, n, y);
}

// A row in the registers of WPR wavefronts, C chunks per lane: read once, the variance from the deviations.
template <class T, int WPR, int C, bool TAIL>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void norm_fwd_kernel(NormArgs A)
{
    __shared__ float red[2][WPR];
    const int wave = threadIdx.x >> 6;
    const int t = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
    int64_t row = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    while (row < A.M) {
        float h[C][8], s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * 64 * WPR + t) * 8;
            if (col < A.N) {
                chunk_h<T, TAIL>(A, row, col, A.N - col, h[c]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = 0.f;
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += h[c][i];
        const float mu = row_sum<WPR>(s, red[0], wave) * A.inv_n;
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int n = A.N - (c * 64 * WPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = h[c][i] - mu;
                if (TAIL ? i < n : 0 < n) q += d * d;
            }
        }
        const float rs = 1.f / sqrtf(row_sum<WPR>(q, red[1], wave) * A.inv_n + A.eps);
        if (t == 0) {
            if (A.mean) A.mean[row] = mu;
            if (A.rstd) A.rstd[row] = rs;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * 64 * WPR + t) * 8;
            if (col < A.N) chunk_y<T, TAIL>(A, row, col, A.N - col, h[c], mu, rs);
        }
        row += (int64_t)gridDim.x * (WPR == 1 ? 4 : 1);
        if (WPR > 1 && row < A.M) __syncthreads();      // (the next row's sums go where this one's were read)
    }
}

// Rows too long for registers: a workgroup per row reads it twice (the second time from the cache, mostly).  Mean and squared
// deviations are joined chunk by chunk (Chan, Golub, LeVeque 1979), not as a difference of two large sums.
template <class T, bool TAIL>
__global__ __launch_bounds__(256) void norm_fwd_long_kernel(NormArgs A)
{
    __shared__ float red[2][4];
    const int wave = threadIdx.x >> 6;
    for (int64_t row = blockIdx.x; row < A.M; row += gridDim.x) {
        if (row != (int64_t)blockIdx.x) __syncthreads();        // (the last row's sums have been read)
        float cnt = 0.f, mean = 0.f, m2 = 0.f;
        for (int col = threadIdx.x * 8; col < A.N; col += 256 * 8) {
            const int n = A.N - col < 8 ? A.N - col : 8;
            float h[8], s = 0.f, q = 0.f;
            chunk_h<T, TAIL>(A, row, col, n, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += h[i];
            const float cm = s / (float)n;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!TAIL || i < n) q += (h[i] - cm) * (h[i] - cm);
            const float tot = cnt + (float)n, d = cm - mean;
            mean += d * ((float)n / tot);
            m2 += q + d * d * (cnt * (float)n / tot);
            cnt = tot;
        }
        const float mu = row_sum<4>(mean * cnt, red[0], wave) * A.inv_n;
        const float q = row_sum<4>(m2 + cnt * (mean - mu) * (mean - mu), red[1], wave);
        const float rs = 1.f / sqrtf(q * A.inv_n + A.eps);
        if (threadIdx.x == 0) {
            if (A.mean) A.mean[row] = mu;
            if (A.rstd) A.rstd[row] = rs;
        }
        // every thread reads back what it wrote itself
        const T *src = reinterpret_cast<const T *>(A.h ? A.h : A.x) + row * (A.h ? A.ld_h : A.ld_x);
        for (int col = threadIdx.x * 8; col < A.N; col += 256 * 8) {
            const int n = A.N - col;
            float h[8];
            load8<T, TAIL>(src + col, n, h);
            chunk_y<T, TAIL>(A, row, col, n, h, mu, rs);
        }
    }
}

// dr of one chunk from w = dy gamma and z, and what follows from it
template <class T, bool TAIL>
__device__ __forceinline__ void chunk_dr(const NormArgs &A, int64_t row, int col, int n, const float (&w)[8], const float (&z)[8], float rs, float c1, float c2)
{
    float d[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (A.dh) load8<T, TAIL>(reinterpret_cast<const T *>(A.dh) + row * A.ld_dh + col, n, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] += rs * (w[i] - c1 - z[i] * c2);
    if (A.dx) {
        float f[8];
        mask8(A.mask, (uint64_t)row * (uint64_t)A.per_row + (uint64_t)(col >> 3), f);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] != 0.f ? d[i] * f[i] : 0.f;
        store8<T, TAIL>(reinterpret_cast<T *>(A.dx) + row * A.ld_dx + col, n, f);
    }
    if (A.dr) store8<T, TAIL>(reinterpret_cast<T *>(A.dr) + row * A.ld_dr + col, n, d);
}

constexpr int kBwdWaves = 8;        // wavefronts of a backward workgroup

// Each workgroup walks every gridDim.x-th group of 8 / WPR rows and keeps the column sums of its rows in registers: dy and h
// are read once for both.  An fp32 row of sums per workgroup goes to the workspace, which norm_finish_kernel adds in order.
template <class T, int WPR, int C, bool TAIL>
__global__ __launch_bounds__(64 * kBwdWaves) void norm_bwd_kernel(NormArgs A)
{
    constexpr int GROUPS = kBwdWaves / WPR;         // rows at a time
    __shared__ float red[2][GROUPS][2][WPR];
    __shared__ float join[GROUPS > 1 ? GROUPS / 2 : 1][C * 64 * WPR * 8 + 4];
    const int group = threadIdx.x / (64 * WPR), t = threadIdx.x % (64 * WPR), wave = t >> 6;
    float dg[C][8], db[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = db[c][i] = 0.f;
    int odd = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * GROUPS; r0 < A.M; r0 += (int64_t)gridDim.x * GROUPS, odd ^= 1) {
        const int64_t row = r0 + group;
        const bool live = row < A.M;                // (the same in a row's wavefronts; all of them meet at the barrier)
        float w[C][8], z[C][8], s1 = 0.f, s2 = 0.f, mu = 0.f, rs = 0.f;
        if (live) {
            mu = A.mean[row];
            rs = A.rstd[row];
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * 64 * WPR + t) * 8, n = A.N - col;
            if (live && n > 0) {
                float g[8];
                load8<T, TAIL>(reinterpret_cast<const T *>(A.dy) + row * A.ld_dy + col, n, w[c]);
                load8<T, TAIL>(reinterpret_cast<const T *>(A.h) + row * A.ld_h + col, n, z[c]);
                load_weight8<T, TAIL>(A.gamma, A.w32, col, n, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[c][i] = (z[c][i] - mu) * rs;
                    // (beyond the row's end dy and gamma are 0, z is not, and has no part in anything)
                    dg[c][i] += w[c][i] * z[c][i];
                    db[c][i] += w[c][i];
                    w[c][i] *= g[i];
                    s1 += w[c][i];
                    s2 += w[c][i] * z[c][i];
                }
            }
        }
        if constexpr (WPR == 1) {
            s1 = wave_sum(s1);
            s2 = wave_sum(s2);
        } else {
            // one barrier per row: the other set of sums is read behind the next one
            s1 = wave_sum(s1);
            s2 = wave_sum(s2);
            if ((t & 63) == 0) { red[odd][group][0][wave] = s1; red[odd][group][1][wave] = s2; }
            __syncthreads();
            s1 = red[odd][group][0][0];
            s2 = red[odd][group][1][0];
#pragma unroll
            for (int i = 1; i < WPR; ++i) { s1 += red[odd][group][0][i]; s2 += red[odd][group][1][i]; }
        }
        s1 *= A.inv_n;
        s2 *= A.inv_n;
        if (A.dr || A.dx) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * 64 * WPR + t) * 8;
                if (live && col < A.N) chunk_dr<T, TAIL>(A, row, col, A.N - col, w[c], z[c], rs, s1, s2);
            }
        }
    }
    if (!A.part) return;
    // the row groups' sums, halved until one is left
#pragma unroll
    for (int what = 0; what < 2; ++what) {
        auto &acc = what ? db : dg;
#pragma unroll
        for (int half = GROUPS / 2; half >= 1; half /= 2) {
            __syncthreads();
            if (group >= half && group < 2 * half) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) join[group - half][(c * 8 + i) * 64 * WPR + t] = acc[c][i];
            }
            __syncthreads();
            if (group < half) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[c][i] += join[group][(c * 8 + i) * 64 * WPR + t];
            }
        }
        if (group == 0) {
            float *dst = A.part + ((int64_t)blockIdx.x * 2 + what) * A.N;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * 64 * WPR + t) * 8;
                if (col < A.N) store8<float, TAIL>(dst + col, A.N - col, acc[c]);
            }
        }
    }
}

// Rows too long for registers: dr by a workgroup per row that reads it twice; the column sums by norm_colsum_kernel.
template <class T, bool TAIL>
__global__ __launch_bounds__(256) void norm_bwd_long_kernel(NormArgs A)
{
    __shared__ float red[2][4];
    const int wave = threadIdx.x >> 6;
    for (int64_t row = blockIdx.x; row < A.M; row += gridDim.x) {
        if (row != (int64_t)blockIdx.x) __syncthreads();        // (the last row's sums have been read)
        const T *dy = reinterpret_cast<const T *>(A.dy) + row * A.ld_dy, *h = reinterpret_cast<const T *>(A.h) + row * A.ld_h;
        const float mu = A.mean[row], rs = A.rstd[row];
        float s1 = 0.f, s2 = 0.f;
        auto chunk = [&](int col, float (&w)[8], float (&z)[8]) __attribute__((always_inline)) {
            float g[8];
            load8<T, TAIL>(dy + col, A.N - col, w);
            load8<T, TAIL>(h + col, A.N - col, z);
            load_weight8<T, TAIL>(A.gamma, A.w32, col, A.N - col, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[i] = (z[i] - mu) * rs;
                w[i] *= g[i];
            }
        };
        for (int col = threadIdx.x * 8; col < A.N; col += 256 * 8) {
            float w[8], z[8];
            chunk(col, w, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) { s1 += w[i]; s2 += w[i] * z[i]; }
        }
        s1 = row_sum<4>(s1, red[0], wave) * A.inv_n;
        s2 = row_sum<4>(s2, red[1], wave) * A.inv_n;
        for (int col = threadIdx.x * 8; col < A.N; col += 256 * 8) {
            float w[8], z[8];
            chunk(col, w, z);
            chunk_dr<T, TAIL>(A, row, col, A.N - col, w, z, rs, s1, s2);
        }
    }
}

// part[blockIdx.y] = column sums of dy z and of dy over rows_per_part rows; a thread owns 8 columns
template <class T, bool TAIL>
__global__ __launch_bounds__(256) void norm_colsum_kernel(NormArgs A)
{
    const int col = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= A.N) return;
    const int64_t r0 = (int64_t)blockIdx.y * A.rows_per_part, r1 = r0 + A.rows_per_part < A.M ? r0 + A.rows_per_part : A.M;
    float dg[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, db[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int64_t row = r0; row < r1; ++row) {
        float w[8], z[8];
        load8<T, TAIL>(reinterpret_cast<const T *>(A.dy) + row * A.ld_dy + col, A.N - col, w);
        load8<T, TAIL>(reinterpret_cast<const T *>(A.h) + row * A.ld_h + col, A.N - col, z);
        const float mu = A.mean[row], rs = A.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dg[i] += w[i] * ((z[i] - mu) * rs);
            db[i] += w[i];
        }
    }
    float *dst = A.part + (int64_t)blockIdx.y * 2 * A.N + col;
    store8<float, TAIL>(dst, A.N - col, dg);
    store8<float, TAIL>(dst + A.N, A.N - col, db);
}

// dgamma and dbeta: the parts' rows in a fixed order, 16 columns and 16 groups of parts per workgroup
template <class W>
__global__ __launch_bounds__(256) void norm_finish_kernel(const float *part, W *dgamma, W *dbeta, int N, int parts)
{
    __shared__ float red[16][17];
    const int lane = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + lane;       // of the 2 N columns of a part
    float s = 0.f;
    if (col < 2 * (int64_t)N) {
        const float *p = part + col;
        int i = g;
        for (; i + 15 * 16 < parts; i += 16 * 16) {
            float v[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = p[(int64_t)(i + 16 * u) * 2 * N];
#pragma unroll
            for (int u = 0; u < 16; ++u) s += v[u];
        }
        for (; i < parts; i += 16) s += p[(int64_t)i * 2 * N];
    }
    red[g][lane] = s;
    __syncthreads();
    if (g == 0 && col < 2 * (int64_t)N) {
        float t = red[0][lane];
#pragma unroll
        for (int i = 1; i < 16; ++i) t += red[i][lane];
        W *dst = col < N ? dgamma : dbeta;
        if (dst) dst[col < N ? col : col - N] = static_cast<W>(t);
    }
}

// How a row lies in registers: the fewest wavefronts that leave a lane at most two chunks, since the backward pass holds five values for
// each of its elements (32768 x 2048 bf16 on one wavefront, four chunks a lane: 102 us for dX alone, on four wavefronts 73; 8192 x 8192
// on four wavefronts 91, on eight 74).  waves 0: it does not.
struct RowPlan { int waves, chunks; };
RowPlan row_plan(int64_t N)
{
    if (N <= 512) return {1, 1};
    if (N <= 1024) return {1, 2};
    if (N <= 2048) return {4, 1};
    if (N <= 4096) return {4, 2};
    if (N <= 8192) return {8, 2};
    if (N <= 16384) return {8, 4};
    return {0, 0};
}

// Parts of the column sums: two workgroups per CU, no more than there are groups of rows (or, for rows too long for
// registers, than parts of 16 rows).  us of the backward pass with one / two / four per CU: 32768 x 2048 bf16 102 / 80 / 88, 65536 x 512 58 / 42 / 46,
// 16384 x 1024 24.4 / 23.3 / 27.4, 8192 x 8192 102 / 92 / 105; but 4096 x 1024 13.0 / 14.8 / 14.7, 2048 x 4096 19 / 22 / 30.
int64_t norm_parts(int64_t M, int64_t N)
{
    const RowPlan p = row_plan(N);
    if (p.waves == 0) {
        const int64_t tiles = ((N + 7) / 8 + 255) / 256;
        int64_t parts = (4 * (int64_t)cu_count() + tiles - 1) / tiles;
        if (parts > (M + 15) / 16) parts = (M + 15) / 16;
        const int64_t rows = (M + parts - 1) / parts;
        return (M + rows - 1) / rows;
    }
    const int64_t groups = kBwdWaves / p.waves, most = (M + groups - 1) / groups;
    return most < 2 * cu_count() ? most : 2 * cu_count();
}

// A launch counts its threads in 32 bits: kernels with a workgroup per row or per four rows walk on where there are more.  (Not
// earlier: with 2048 workgroups, eight per CU, that walk over the rows 32768 x 2048 bf16 takes 128 us instead of 108.)
constexpr int64_t kMostGroups = int64_t(1) << 22;
unsigned groups_for(int64_t n) { return (unsigned)(n < kMostGroups ? n : kMostGroups); }

template <class T, bool TAIL> void launch_norm_fwd(const NormArgs &A, hipStream_t st)
{
    const RowPlan p = row_plan(A.N);
    const dim3 wave_rows(groups_for((A.M + 3) / 4)), rows(groups_for(A.M)), block(256);
    if (p.waves == 1 && p.chunks == 1) hipLaunchKernelGGL((norm_fwd_kernel<T, 1, 1, TAIL>), wave_rows, block, 0, st, A);
    else if (p.waves == 1 && p.chunks == 2) hipLaunchKernelGGL((norm_fwd_kernel<T, 1, 2, TAIL>), wave_rows, block, 0, st, A);
    else if (p.waves == 4 && p.chunks == 1) hipLaunchKernelGGL((norm_fwd_kernel<T, 4, 1, TAIL>), rows, block, 0, st, A);
    else if (p.waves == 4) hipLaunchKernelGGL((norm_fwd_kernel<T, 4, 2, TAIL>), rows, block, 0, st, A);
    else if (p.waves == 8 && p.chunks == 2) hipLaunchKernelGGL((norm_fwd_kernel<T, 8, 2, TAIL>), rows, dim3(512), 0, st, A);
    else if (p.waves == 8) hipLaunchKernelGGL((norm_fwd_kernel<T, 8, 4, TAIL>), rows, dim3(512), 0, st, A);
    else hipLaunchKernelGGL((norm_fwd_long_kernel<T, TAIL>), rows, block, 0, st, A);
}

template <class T, bool TAIL> void launch_norm_bwd(NormArgs A, int64_t parts, hipStream_t st)
{
    const RowPlan p = row_plan(A.N);
    const dim3 grid((unsigned)parts), block(64 * kBwdWaves);
    if (p.waves == 1 && p.chunks == 1) hipLaunchKernelGGL((norm_bwd_kernel<T, 1, 1, TAIL>), grid, block, 0, st, A);
    else if (p.waves == 1 && p.chunks == 2) hipLaunchKernelGGL((norm_bwd_kernel<T, 1, 2, TAIL>), grid, block, 0, st, A);
    else if (p.waves == 4 && p.chunks == 1) hipLaunchKernelGGL((norm_bwd_kernel<T, 4, 1, TAIL>), grid, block, 0, st, A);
    else if (p.waves == 4) hipLaunchKernelGGL((norm_bwd_kernel<T, 4, 2, TAIL>), grid, block, 0, st, A);
    else if (p.waves == 8 && p.chunks == 2) hipLaunchKernelGGL((norm_bwd_kernel<T, 8, 2, TAIL>), grid, block, 0, st, A);
    else if (p.waves == 8) hipLaunchKernelGGL((norm_bwd_kernel<T, 8, 4, TAIL>), grid, block, 0, st, A);
    else {
        // the sums first: dr may be written over dy
        if (A.part) {
            A.rows_per_part = (A.M + parts - 1) / parts;
            hipLaunchKernelGGL((norm_colsum_kernel<T, TAIL>), dim3((unsigned)((A.per_row + 255) / 256), (unsigned)parts), dim3(256), 0, st, A);
        }
        if (A.dr || A.dx) hipLaunchKernelGGL((norm_bwd_long_kernel<T, TAIL>), dim3(groups_for(A.M)), dim3(256), 0, st, A);
    }
}

}  // namespace
}  // namespace sdrop

using namespace sdrop;

extern "C" {

int sdrop_dropout(const void *X, const void *R, void *Y, int64_t M, int64_t N, double p, uint64_t seed, uint64_t rng_stream,
                  int dtype, int64_t ld_x, int64_t ld_r, int64_t ld_y, void *stream)
{
    if (!X || !Y || !(p >= 0.0 && p <= 1.0)) return SDROP_EINVAL;
    if (!rows_shape_ok(M, N) || !row_ld_ok(ld_x, N) || !row_ld_ok(ld_r, N) || !row_ld_ok(ld_y, N)) return SDROP_ESHAPE;
    if (!type_ok(dtype)) return SDROP_EDTYPE;
    const size_t sz = type_size(dtype);
    if (!aligned(X, sz) || !aligned(R, sz) || !aligned(Y, sz)) return SDROP_EALIGN;
    DropoutArgs A;
    A.x = static_cast<const char *>(X);
    A.r = static_cast<const char *>(R);
    A.y = static_cast<char *>(Y);
    A.N = (int32_t)N;
    A.per_row = (int32_t)((N + 7) / 8);
    A.chunks = M * A.per_row;
    A.ld_x = ld_x ? ld_x : N;
    A.ld_r = ld_r ? ld_r : N;
    A.ld_y = ld_y ? ld_y : N;
    A.mask = element_mask(p, seed, rng_stream);
    // eight workgroups per CU fill it; each then strides over the rest
    int64_t grid = (A.chunks + 255) / 256;
    if (grid > 8 * (int64_t)cu_count()) grid = 8 * (int64_t)cu_count();
    A.drow = grid * 256 / A.per_row;
    A.dcol = (int32_t)(grid * 256 % A.per_row);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == SDROP_F16) launch_dropout<_Float16>(A, (unsigned)grid, st);
    else if (dtype == SDROP_BF16) launch_dropout<__bf16>(A, (unsigned)grid, st);
    else launch_dropout<float>(A, (unsigned)grid, st);
    return hip_status(hipGetLastError());
}

int sdrop_layer_norm(const void *X, const void *R, const void *gamma, const void *beta, void *H, void *Y, float *mean, float *rstd,
                     int64_t M, int64_t N, double eps, double p, uint64_t seed, uint64_t rng_stream, int dtype, int w_dtype,
                     int64_t ld_x, int64_t ld_r, int64_t ld_h, int64_t ld_y, void *stream)
{
    if (!X || !gamma || !Y || !(p >= 0.0 && p <= 1.0) || !(eps >= 0.0 && eps < INFINITY)) return SDROP_EINVAL;
    if ((R || p > 0.0) && !H) return SDROP_EINVAL;
    if (!rows_shape_ok(M, N) || !row_ld_ok(ld_x, N) || !row_ld_ok(ld_r, N) || !row_ld_ok(ld_h, N) || !row_ld_ok(ld_y, N)) return SDROP_ESHAPE;
    if (!type_ok(dtype) || (w_dtype != dtype && w_dtype != SDROP_F32)) return SDROP_EDTYPE;
    const size_t sz = type_size(dtype), wsz = type_size(w_dtype);
    if (!aligned(X, sz) || !aligned(R, sz) || !aligned(H, sz) || !aligned(Y, sz) || !aligned(gamma, wsz) || !aligned(beta, wsz) ||
        !aligned(mean, 4) || !aligned(rstd, 4)) return SDROP_EALIGN;
    NormArgs A = {};
    A.x = static_cast<const char *>(X);
    A.r = static_cast<const char *>(R);
    A.gamma = static_cast<const char *>(gamma);
    A.beta = static_cast<const char *>(beta);
    A.h = static_cast<char *>(H);
    A.y = static_cast<char *>(Y);
    A.mean = mean;
    A.rstd = rstd;
    A.M = M;
    A.N = (int32_t)N;
    A.per_row = (int32_t)((N + 7) / 8);
    A.ld_x = ld_x ? ld_x : N;
    A.ld_r = ld_r ? ld_r : N;
    A.ld_h = ld_h ? ld_h : N;
    A.ld_y = ld_y ? ld_y : N;
    A.w32 = w_dtype == SDROP_F32;
    A.eps = (float)eps;
    A.inv_n = 1.f / (float)N;
    A.mask = element_mask(p, seed, rng_stream);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool tail = N % 8 != 0;
    if (dtype == SDROP_F16) tail ? launch_norm_fwd<_Float16, true>(A, st) : launch_norm_fwd<_Float16, false>(A, st);
    else if (dtype == SDROP_BF16) tail ? launch_norm_fwd<__bf16, true>(A, st) : launch_norm_fwd<__bf16, false>(A, st);
    else tail ? launch_norm_fwd<float, true>(A, st) : launch_norm_fwd<float, false>(A, st);
    return hip_status(hipGetLastError());
}

size_t sdrop_layer_norm_bwd_workspace_bytes(int64_t M, int64_t N)
{
    return rows_shape_ok(M, N) ? (size_t)norm_parts(M, N) * 2 * (size_t)N * sizeof(float) : 0;
}

int sdrop_layer_norm_bwd(const void *dY, const void *dH, const void *H, const void *gamma, const float *mean, const float *rstd,
                         void *dR, void *dX, void *dgamma, void *dbeta, int64_t M, int64_t N, double p, uint64_t seed,
                         uint64_t rng_stream, int dtype, int w_dtype, int64_t ld_dy, int64_t ld_dh, int64_t ld_h, int64_t ld_dr,
                         int64_t ld_dx, void *ws, size_t ws_bytes, void *stream)
{
    if (!dY || !H || !gamma || !mean || !rstd || !(p >= 0.0 && p <= 1.0) || (!dR && !dX && !dgamma && !dbeta)) return SDROP_EINVAL;
    if (!rows_shape_ok(M, N) || !row_ld_ok(ld_dy, N) || !row_ld_ok(ld_dh, N) || !row_ld_ok(ld_h, N) || !row_ld_ok(ld_dr, N) ||
        !row_ld_ok(ld_dx, N)) return SDROP_ESHAPE;
    if (!type_ok(dtype) || (w_dtype != dtype && w_dtype != SDROP_F32)) return SDROP_EDTYPE;
    const size_t sz = type_size(dtype), wsz = type_size(w_dtype);
    if (!aligned(dY, sz) || !aligned(dH, sz) || !aligned(H, sz) || !aligned(dR, sz) || !aligned(dX, sz) || !aligned(gamma, wsz) ||
        !aligned(dgamma, wsz) || !aligned(dbeta, wsz) || !aligned(mean, 4) || !aligned(rstd, 4)) return SDROP_EALIGN;
    const bool sums = dgamma || dbeta;
    if (sums && (!ws || ws_bytes < sdrop_layer_norm_bwd_workspace_bytes(M, N) || !aligned(ws, 16))) return SDROP_EWORKSPACE;
    NormArgs A = {};
    A.dy = static_cast<const char *>(dY);
    A.dh = static_cast<const char *>(dH);
    A.h = static_cast<char *>(const_cast<void *>(H));
    A.gamma = static_cast<const char *>(gamma);
    A.mean = const_cast<float *>(mean);
    A.rstd = const_cast<float *>(rstd);
    A.dr = static_cast<char *>(dR);
    A.dx = static_cast<char *>(dX);
    A.part = sums ? static_cast<float *>(ws) : nullptr;
    A.M = M;
    A.N = (int32_t)N;
    A.per_row = (int32_t)((N + 7) / 8);
    A.ld_dy = ld_dy ? ld_dy : N;
    A.ld_dh = ld_dh ? ld_dh : N;
    A.ld_h = ld_h ? ld_h : N;
    A.ld_dr = ld_dr ? ld_dr : N;
    A.ld_dx = ld_dx ? ld_dx : N;
    A.w32 = w_dtype == SDROP_F32;
    A.inv_n = 1.f / (float)N;
    A.mask = element_mask(p, seed, rng_stream);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t parts = norm_parts(M, N);
    const bool tail = N % 8 != 0;
    if (dtype == SDROP_F16) tail ? launch_norm_bwd<_Float16, true>(A, parts, st) : launch_norm_bwd<_Float16, false>(A, parts, st);
    else if (dtype == SDROP_BF16) tail ? launch_norm_bwd<__bf16, true>(A, parts, st) : launch_norm_bwd<__bf16, false>(A, parts, st);
    else tail ? launch_norm_bwd<float, true>(A, parts, st) : launch_norm_bwd<float, false>(A, parts, st);
    int rc = hip_status(hipGetLastError());
    if (rc != SDROP_OK || !sums) return rc;
    const dim3 grid((unsigned)((2 * N + 15) / 16)), block(256);
    const float *part = static_cast<const float *>(ws);
    if (w_dtype == SDROP_F16)
        hipLaunchKernelGGL(norm_finish_kernel<_Float16>, grid, block, 0, st, part, static_cast<_Float16 *>(dgamma), static_cast<_Float16 *>(dbeta), (int)N, (int)parts);
    else if (w_dtype == SDROP_BF16)
        hipLaunchKernelGGL(norm_finish_kernel<__bf16>, grid, block, 0, st, part, static_cast<__bf16 *>(dgamma), static_cast<__bf16 *>(dbeta), (int)N, (int)parts);
    else
        hipLaunchKernelGGL(norm_finish_kernel<float>, grid, block, 0, st, part, static_cast<float *>(dgamma), static_cast<float *>(dbeta), (int)N, (int)parts);
    return hip_status(hipGetLastError());
}

}  // extern "C"
