// Layer norm between the products of a network (Sec. VI "Kernel Fusion" counts Add-bias + LayerNorm among what eats a sparse
// product's gain; the addition rides in the product's epilogue, this is the rest).
//
//   mu = mean_n x[n],  rstd = 1 / sqrt(mean_n (x[n] - mu)^2 + eps),  y[n] = (x[n] - mu) rstd gamma[n] + beta[n]
//   backward, with xh = (x - mu) rstd and g = dy gamma:
//     dx = rstd (g - mean_n g - xh mean_n(g xh)),   dgamma[n] = sum_m dy xh,   dbeta[n] = sum_m dy
//
// All of it is bound by memory: forward 4 bytes an element, backward 6.  A row is read once and waits in registers for its
// statistics; everything is fp32, rounded once at the store.
//
// The mean comes in two steps, mu0 = fl(sum x / N) and the rest r = sum (x - mu0) / N: a step of fp32 at 60000 is 0.004, which the 1 / sqrt(eps) of a
// row that hardly varies makes 1.2.  x - mu0 is exact for such rows, so (x - mu0) - r has the error of its own size, not of x's, and the variance
// is sum (x - mu0)^2 / N - r^2, the difference of a sum about the mean and next to nothing (for most rows r is below a step of mu0).
// The first step is a division: a constant row whose sum is exact has itself as its mean then, and the product with fl(1 / N)
// misses it for many N.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/tw.h"
#include "tw_device.hpp"

namespace {

typedef unsigned short us;

struct LnParams {
    const us* x;
    const us* gamma;            // null: ones
    const us* beta;             // null: zeros
    us* y;
    float* mean;                // null: not wanted
    float* rstd;
    long ldx, ldy;
    int M, N;
    float eps;
    int stream;                 // rows of y start on 128-byte boundaries: whole lines go out as streaming stores
};

// Lanes exchanged by the vector unit alone: within rows of 16 lanes (CTRL: 0xB1 lane ^ 1, 0x4E lane ^ 2, 0x141 the other four of eight, 0x140 the other
// eight, 0x128 lane ^ 8), and whole rows or halves.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// In lanes of even rows (of the lower half) a summed over the pair of rows (both halves), in the others b.
__device__ __forceinline__ float rows_sum(float a, float b) {
    const auto both = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned even = both[0], odd = both[1];            // (copies: the builtin cast of a vector's element takes the first one)
    return __builtin_bit_cast(float, even) + __builtin_bit_cast(float, odd);
}
__device__ __forceinline__ float halves_sum(float a, float b) {
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned low = both[0], high = both[1];
    return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
}
// Sum over groups of TPR consecutive lanes, the same bits in every lane of the group.
template <int TPR>
__device__ __forceinline__ float group_sum(float v) {
    static_assert(TPR >= 16, "");
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    if constexpr (TPR >= 32) v = rows_sum(v, v);
    if constexpr (TPR >= 64) v = halves_sum(v, v);
    return v;
}

template <int DT>
__device__ __forceinline__ void unpack8(tw_u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = tw_to_f32<DT>((us)(v[i] & 0xFFFFu));
        f[2 * i + 1] = tw_to_f32<DT>((us)(v[i] >> 16));
    }
}
template <int DT>
__device__ __forceinline__ tw_u32x4 pack8(const float (&f)[8]) {
    tw_u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (unsigned)tw_cvt<DT>(f[2 * i]) | ((unsigned)tw_cvt<DT>(f[2 * i + 1]) << 16);
    return v;
}
// Eight parameters from index c on as they lie in memory; those from N on are zero and not read, all are `none` without a source.
template <bool TAIL>
__device__ __forceinline__ tw_u32x4 params8(const us* src, int c, int N, unsigned none) {
    if (!src) return tw_u32x4{none, none, none, none};
    if (c >= N) return tw_u32x4{0u, 0u, 0u, 0u};
    if (!TAIL || c + 8 <= N) return *(const tw_u32x4*)(src + c);
    unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (c + e < N) w[e >> 1] |= (unsigned)src[c + e] << (16 * (e & 1));
    return tw_u32x4{w[0], w[1], w[2], w[3]};
}
template <int DT> constexpr unsigned ones() { return DT == TW_F16 ? 0x3C003C00u : 0x3F803F80u; }
template <bool TAIL>
__device__ __forceinline__ void put8(us* dst, int left, tw_u32x4 v) {   // left: elements up to the row's end
    if (!TAIL || left >= 8) {
        *(tw_u32x4*)dst = v;
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) dst[e] = (us)(v[e >> 1] >> (16 * (e & 1)));
    }
}

// Sum over the TPR threads of a row: lanes of a wave, or the four waves of a workgroup (`red`: rows of four floats, used in turn).
template <int TPR, int ROWS>
__device__ __forceinline__ float row_sum(float v, float (&red)[ROWS][4], int turn) {
    v = group_sum<TPR>(v);
    if constexpr (TPR == 256) {
        if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        v = (red[turn][0] + red[turn][1]) + (red[turn][2] + red[turn][3]);
    }
    return v;
}

// The same for two sums at once: rows `turn` and `turn` + 1 of `red`.
template <int TPR>
__device__ __forceinline__ void row_sum2(float& v, float& w, float (&red)[3][4], int turn) {
    v = group_sum<TPR>(v);
    w = group_sum<TPR>(w);
    if constexpr (TPR == 256) {
        if ((threadIdx.x & 63) == 0) {
            red[turn][threadIdx.x >> 6] = v;
            red[turn + 1][threadIdx.x >> 6] = w;
        }
        __syncthreads();
        v = (red[turn][0] + red[turn][1]) + (red[turn][2] + red[turn][3]);
        w = (red[turn + 1][0] + red[turn + 1][1]) + (red[turn + 1][2] + red[turn + 1][3]);
    }
}
// 1 / deviation from the sums of squares about a value that misses the mean by `rest`.  (The comparison keeps NaN.)
__device__ __forceinline__ float deviation(float squares, float rest, float inv_n, float eps) {
    const float var = squares * inv_n - rest * rest;
    return 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);
}

// The mean of both steps.  (The rest about an infinity is NaN, the mean that infinity.)
__device__ __forceinline__ float both_steps(float mean, float rest) { return __builtin_fabsf(mean) < __builtin_inff() ? mean + rest : mean; }

// Row-major, 16-byte pieces.  TPR threads of a workgroup of 256 share a row, thread t of them the pieces t, t + TPR, .. (PER of
// them); TAIL: N is no multiple of 8, the last piece reaches into the row's pitch.
// (16384 x 4096: 40 us, 6.7 TB/s with part of the data in the last-level cache; 512 x 768: 3.6 us, an empty kernel takes 2.4.)
template <int DT, int TPR, int PER, bool TAIL>
__global__ __launch_bounds__(256) void tw_ln_kernel(const LnParams p) {
    constexpr int kGroups = 256 / TPR;
    __shared__ float red[3][4];
    const int t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
    const float inv_n = 1.f / (float)p.N;
    tw_u32x4 ga[PER], be[PER];                               // (asked for with the first row, not behind its statistics)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        ga[i] = params8<TAIL>(p.gamma, 8 * (t + i * TPR), p.N, ones<DT>());
        be[i] = params8<TAIL>(p.beta, 8 * (t + i * TPR), p.N, 0u);
    }
    for (long m0 = (long)blockIdx.x * kGroups; m0 < p.M; m0 += (long)gridDim.x * kGroups) {   // (uniform: the barriers are met by all)
        const long m = m0 + grp < p.M ? m0 + grp : p.M - 1;   // (groups behind the last row repeat it and store nothing)
        const bool mine = m0 + grp < p.M;
        const us* row = p.x + m * p.ldx;
        float v[PER][8];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
            tw_u32x4 w{0u, 0u, 0u, 0u};
            if (c < p.N) w = *(const tw_u32x4*)(row + c);
            unpack8<DT>(w, v[i]);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (TAIL && c + e >= p.N) v[i][e] = 0.f;
                s += v[i][e];
            }
        }
        const float mean = row_sum<TPR>(s, red, 0) / (float)p.N;
        float q = 0.f, r = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
            if (c < p.N) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[i][e] -= mean;
                    if (!TAIL || c + e < p.N) {
                        q = __builtin_fmaf(v[i][e], v[i][e], q);
                        r += v[i][e];
                    }
                }
            }
        }
        row_sum2<TPR>(q, r, red, 1);
        r *= inv_n;
        const float rstd = deviation(q, r, inv_n, p.eps);
        if (mine && t == 0) {
            if (p.mean) p.mean[m] = both_steps(mean, r);
            if (p.rstd) p.rstd[m] = rstd;
        }
        us* out = p.y + m * p.ldy;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
            if (c < p.N && mine) {
                float g[8], b[8];
                unpack8<DT>(ga[i], g);
                unpack8<DT>(be[i], b);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf((v[i][e] - r) * rstd, g[e], b[e]);
                put8<TAIL>(out + c, p.N - c, pack8<DT>(v[i]));
            }
        }
    }
}

// Row-major, any pitch, any alignment, any N: a workgroup per row reads it three times, element by element (from the caches after the
// first).
template <int DT>
__global__ __launch_bounds__(256) void tw_ln_any_kernel(const LnParams p) {
    __shared__ float red[3][4];
    const float inv_n = 1.f / (float)p.N;
    for (long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const us* row = p.x + m * p.ldx;
        float s = 0.f;
        for (int c = threadIdx.x; c < p.N; c += 256) s += tw_to_f32<DT>(row[c]);
        const float mean = row_sum<256>(s, red, 0) / (float)p.N;
        float q = 0.f, r = 0.f;
        for (int c = threadIdx.x; c < p.N; c += 256) {
            const float d = tw_to_f32<DT>(row[c]) - mean;
            q = __builtin_fmaf(d, d, q);
            r += d;
        }
        row_sum2<256>(q, r, red, 1);
        r *= inv_n;
        const float rstd = deviation(q, r, inv_n, p.eps);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[m] = both_steps(mean, r);
            if (p.rstd) p.rstd[m] = rstd;
        }
        us* out = p.y + m * p.ldy;
        for (int c = threadIdx.x; c < p.N; c += 256) {
            const float g = p.gamma ? tw_to_f32<DT>(p.gamma[c]) : 1.f, b = p.beta ? tw_to_f32<DT>(p.beta[c]) : 0.f;
            out[c] = tw_cvt<DT>(__builtin_fmaf(((tw_to_f32<DT>(row[c]) - mean) - r) * rstd, g, b));
        }
    }
}

// The same pieces, as ones the compiler knows nothing of: it then unpacks them again where they are used, and does not keep the
// unpacked values (eight registers a piece instead of four) from one phase to the next.
template <int PER>
__device__ __forceinline__ void forget(tw_u32x4 (&w)[PER]) {
#pragma unroll
    for (int i = 0; i < PER; ++i) asm volatile("" : "+v"(w[i]));
}

constexpr int PCS = 8;                                       // 16-byte pieces of a row that a workgroup takes: a token for each lane of a wave
// Statistics of the block's tokens.  A lane has sums of eight tokens over its rows; `leave` sums them over the eight lanes of the wave that hold the
// same piece, each of which ends with one token and leaves it in LDS, where the block's tokens lie in order.  Behind a barrier lane t of every wave has
// `waves_sum` of token t, and what all lanes make of those goes round through the wave's own part of LDS: `give` puts a lane's value there,
// `get` takes the eight of its piece.  (Sums of all eight
// tokens in every lane, 24 exchanges through LDS and 64 reads of it each: 17.2 us on 16384 x 768, 13.4 so.)
__device__ __forceinline__ void leave(const float (&s)[8], float (&red)[8 * PCS], int lane) {
    const float a = halves_sum(s[0], s[4]), b = halves_sum(s[1], s[5]), c = halves_sum(s[2], s[6]), d = halves_sum(s[3], s[7]);
    float x = rows_sum(a, c), y = rows_sum(b, d);
    x += dpp<0x128>(x);                                      // (both by every lane: lanes that a branch leaves out give nothing)
    y += dpp<0x128>(y);
    red[8 * (lane % PCS) + 4 * (lane >> 5) + 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1)] = (lane & 8) == 0 ? x : y;
}
template <int WAVES>
__device__ __forceinline__ float waves_sum(const float (&red)[WAVES][8 * PCS], int lane) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) s += red[k][lane];
    return s;
}
__device__ __forceinline__ void give(float v, float (&own)[8 * PCS], int lane) { own[lane] = v; }
__device__ __forceinline__ void get(float (&v)[8], const float (&own)[8 * PCS], int lane) {
    asm volatile("" ::: "memory");                           // (the LDS executes a wave's instructions in order)
    const float4 a = *(const float4*)&own[8 * (lane % PCS)], b = *(const float4*)&own[8 * (lane % PCS) + 4];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    asm volatile("" ::: "memory");
}
// Transposed boundary: features are rows, tokens columns.  A workgroup takes 8 * PCS tokens, a lane the 16-byte piece lane % PCS of the rows
// lane / PCS + 64 / PCS * wave + 64 / PCS * WAVES * i, PER of them, which wait in registers as they were read.  A token's sums meet across
// the lanes of a wave that hold its piece and, through LDS, across the waves.  64 tokens are whole 128-byte lines, which go out as
// streaming stores: 16384 x 768 in 13.4 us (3.8 TB/s); 32 tokens a workgroup, twice as many of them: 24.7 us, half lines.
template <int DT, int WAVES, int PER>
__global__ __launch_bounds__(64 * WAVES) void tw_ln_t_kernel(const LnParams p) {
    constexpr int kRows = 64 / PCS * WAVES;
    __shared__ float red[3][WAVES][8 * PCS];
    __shared__ __attribute__((aligned(16))) float own[WAVES][2][8 * PCS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pc = lane % PCS;
    const long m0 = (long)blockIdx.x * (8 * PCS) + 8 * pc;
    const int n0 = 64 / PCS * wave + lane / PCS;
    const bool here = m0 < p.M;
    const float inv_n = 1.f / (float)p.N;
    tw_u32x4 w[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        w[i] = tw_u32x4{0u, 0u, 0u, 0u};
        if (here && n0 + kRows * i < p.N) w[i] = tw_load16_stream(p.x + (long)(n0 + kRows * i) * p.ldx + m0);
    }
    float mean[8] = {}, rstd[8] = {}, rest[8] = {};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        float f[8];
        unpack8<DT>(w[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) mean[e] += f[e];
        __builtin_amdgcn_sched_barrier(0);
    }
    leave(mean, red[0][wave], lane);
    __syncthreads();
    const float my_mean = waves_sum(red[0], lane) / (float)p.N;
    give(my_mean, own[wave][0], lane);
    get(mean, own[wave][0], lane);
    forget(w);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        float f[8];
        unpack8<DT>(w[i], f);
        if (n0 + kRows * i < p.N) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = f[e] - mean[e];
                rstd[e] = __builtin_fmaf(d, d, rstd[e]);
                rest[e] += d;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    leave(rstd, red[1][wave], lane);
    leave(rest, red[2][wave], lane);
    __syncthreads();
    const float my_rest = waves_sum(red[2], lane) * inv_n, my_rstd = deviation(waves_sum(red[1], lane), my_rest, inv_n, p.eps);
    const long token = (long)blockIdx.x * (8 * PCS) + lane;
    if (wave == 0 && token < p.M) {
        if (p.mean) p.mean[token] = both_steps(my_mean, my_rest);
        if (p.rstd) p.rstd[token] = my_rstd;
    }
    give(my_rstd, own[wave][0], lane);
    give(my_rest, own[wave][1], lane);
    get(rstd, own[wave][0], lane);
    get(rest, own[wave][1], lane);
    forget(w);
    if (!here) return;
    const int left = p.M - m0 < 8 ? (int)(p.M - m0) : 8;
#pragma unroll
    for (int i0 = 0; i0 < PER; i0 += 4) {                    // (four rows at a time: unpacked all at once they would not fit)
        float g[4], b[4];
#pragma unroll
        for (int i = 0; i < 4 && i0 + i < PER; ++i) {
            const int n = n0 + kRows * (i0 + i), at = n < p.N ? n : p.N - 1;
            g[i] = p.gamma ? tw_to_f32<DT>(p.gamma[at]) : 1.f;
            b[i] = p.beta ? tw_to_f32<DT>(p.beta[at]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4 && i0 + i < PER; ++i) {
            const int n = n0 + kRows * (i0 + i);
            float f[8];
            unpack8<DT>(w[i0 + i], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __builtin_fmaf(((f[e] - mean[e]) - rest[e]) * rstd[e], g[i], b[i]);
            if (n >= p.N) continue;
            if (p.stream && left == 8) tw_store16_stream(p.y + (long)n * p.ldy + m0, pack8<DT>(f));
            else put8<true>(tw_opaque(p.y) + (long)n * p.ldy + m0, left, pack8<DT>(f));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The same for rows that do not fit the registers: they are read three times (from the caches after the first), four requests of a lane at a time.
template <int DT>
__global__ __launch_bounds__(1024) void tw_ln_t_loop_kernel(const LnParams p) {
    constexpr int WAVES = 16, kRows = 64 / PCS * WAVES;
    __shared__ float red[3][WAVES][8 * PCS];
    __shared__ __attribute__((aligned(16))) float own[WAVES][2][8 * PCS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pc = lane % PCS;
    const long m0 = (long)blockIdx.x * (8 * PCS) + 8 * pc;
    const int n0 = 64 / PCS * wave + lane / PCS;
    const bool here = m0 < p.M;
    const float inv_n = 1.f / (float)p.N;
    auto rows = [&](auto use) {                              // use(row, its piece) for this lane's rows
        for (int n = n0; n < p.N; n += 4 * kRows) {
            tw_u32x4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = tw_u32x4{0u, 0u, 0u, 0u};
                if (here && n + i * kRows < p.N) w[i] = *(const tw_u32x4*)(p.x + (long)(n + i * kRows) * p.ldx + m0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i * kRows < p.N) use(n + i * kRows, w[i]);
        }
    };
    float mean[8] = {}, rstd[8] = {}, rest[8] = {};
    rows([&](int, tw_u32x4 w) {
        float f[8];
        unpack8<DT>(w, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) mean[e] += f[e];
    });
    leave(mean, red[0][wave], lane);
    __syncthreads();
    const float my_mean = waves_sum(red[0], lane) / (float)p.N;
    give(my_mean, own[wave][0], lane);
    get(mean, own[wave][0], lane);
    rows([&](int, tw_u32x4 w) {
        float f[8];
        unpack8<DT>(w, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = f[e] - mean[e];
            rstd[e] = __builtin_fmaf(d, d, rstd[e]);
            rest[e] += d;
        }
    });
    leave(rstd, red[1][wave], lane);
    leave(rest, red[2][wave], lane);
    __syncthreads();
    const float my_rest = waves_sum(red[2], lane) * inv_n, my_rstd = deviation(waves_sum(red[1], lane), my_rest, inv_n, p.eps);
    const long token = (long)blockIdx.x * (8 * PCS) + lane;
    if (wave == 0 && token < p.M) {
        if (p.mean) p.mean[token] = both_steps(my_mean, my_rest);
        if (p.rstd) p.rstd[token] = my_rstd;
    }
    give(my_rstd, own[wave][0], lane);
    give(my_rest, own[wave][1], lane);
    get(rstd, own[wave][0], lane);
    get(rest, own[wave][1], lane);
    if (!here) return;
    const int left = p.M - m0 < 8 ? (int)(p.M - m0) : 8;
    rows([&](int n, tw_u32x4 w) {
        const float g = p.gamma ? tw_to_f32<DT>(p.gamma[n]) : 1.f, b = p.beta ? tw_to_f32<DT>(p.beta[n]) : 0.f;
        float f[8];
        unpack8<DT>(w, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __builtin_fmaf(((f[e] - mean[e]) - rest[e]) * rstd[e], g, b);
        put8<true>(p.y + (long)n * p.ldy + m0, left, pack8<DT>(f));
    });
}

// Transposed boundary, any pitch, alignment and N: a lane per token, the rows dealt out to the waves, read three times.
template <int DT>
__global__ __launch_bounds__(1024) void tw_ln_t_any_kernel(const LnParams p) {
    __shared__ float red[3][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long m = (long)blockIdx.x * 64 + lane;
    const long mc = m < p.M ? m : p.M - 1;
    const float inv_n = 1.f / (float)p.N;
    auto sum = [&](int turn) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) s += red[turn][k][lane];
        return s;
    };
    float s = 0.f;
    for (int n = wave; n < p.N; n += 16) s += tw_to_f32<DT>(p.x[(long)n * p.ldx + mc]);
    red[0][wave][lane] = s;
    __syncthreads();
    const float mean = sum(0) / (float)p.N;
    float rest = 0.f;
    s = 0.f;
    for (int n = wave; n < p.N; n += 16) {
        const float d = tw_to_f32<DT>(p.x[(long)n * p.ldx + mc]) - mean;
        s = __builtin_fmaf(d, d, s);
        rest += d;
    }
    red[1][wave][lane] = s;
    red[2][wave][lane] = rest;
    __syncthreads();
    rest = sum(2) * inv_n;
    const float rstd = deviation(sum(1), rest, inv_n, p.eps);
    if (m >= p.M) return;
    if (wave == 0) {
        if (p.mean) p.mean[m] = both_steps(mean, rest);
        if (p.rstd) p.rstd[m] = rstd;
    }
    for (int n = wave; n < p.N; n += 16) {
        const float g = p.gamma ? tw_to_f32<DT>(p.gamma[n]) : 1.f, b = p.beta ? tw_to_f32<DT>(p.beta[n]) : 0.f;
        p.y[(long)n * p.ldy + m] = tw_cvt<DT>(__builtin_fmaf(((tw_to_f32<DT>(p.x[(long)n * p.ldx + m]) - mean) - rest) * rstd, g, b));
    }
}

// ------------------------------------------------------------------------------------------------ backward
struct LnGradParams {
    const us* dy;
    const us* x;
    const us* gamma;
    const float* mean;
    const float* rstd;
    us* dx;
    float* part_gamma;          // [n_parts][N]: a workgroup's sums over its rows
    float* part_beta;
    float* row_stats;           // tw_ln_grad_rows_kernel: [M][2]: mean g, mean g xh
    long lddy, ldx, lddx;
    int M, N, rows_per_part;
};

// Row-major, 16-byte pieces, threads and pieces as tw_ln_kernel.  A workgroup walks its rows; a thread's share of dgamma and
// dbeta stays in registers all the way, the shares of the workgroup's row groups meet in LDS at the end, and the
// workgroups' sums are added by a second kernel in a fixed order (no atomics: repeated calls give the same bits).
// 16384 x 768: 17.4 us (4.3 TB/s), 19.1 without the next row on its way; the second kernel 4.
template <int DT, int TPR, int PER, bool TAIL>
__global__ __launch_bounds__(256) void tw_ln_grad_kernel(const LnGradParams p) {
    constexpr int kGroups = 256 / TPR;
    __shared__ float red[2][4];
    extern __shared__ __attribute__((aligned(16))) float share[];            // [kGroups][TPR * PER * 8]
    const int t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
    const float inv_n = 1.f / (float)p.N;
    const long first = (long)blockIdx.x * p.rows_per_part;
    const long last = first + p.rows_per_part < p.M ? first + p.rows_per_part : p.M;
    float sg[PER][8], sb[PER][8];
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sg[i][e] = sb[i][e] = 0.f;
    tw_u32x4 ga[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) ga[i] = params8<TAIL>(p.gamma, 8 * (t + i * TPR), p.N, ones<DT>());
    tw_u32x4 wx[PER], wd[PER];                               // the row that comes next, on its way while one is worked on
    float next_mean, next_rstd;
    auto request = [&](long m0) {
        const long m = m0 + grp < last ? m0 + grp : last - 1;
        next_mean = p.mean[m];
        next_rstd = p.rstd[m];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
            wx[i] = wd[i] = tw_u32x4{0u, 0u, 0u, 0u};
            if (c < p.N) {
                wx[i] = *(const tw_u32x4*)(p.x + m * p.ldx + c);
                wd[i] = *(const tw_u32x4*)(p.dy + m * p.lddy + c);
            }
        }
    };
    request(first);
    for (long m0 = first; m0 < last; m0 += kGroups) {
        const bool mine = m0 + grp < last;
        const long m = m0 + grp;
        const float mean = next_mean, rstd = next_rstd;
        float c1 = 0.f, c2 = 0.f;
        float xh[PER][8], g[PER][8];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
            if (c < p.N) {
                float f[8], d[8], gv[8];
                unpack8<DT>(wx[i], f);
                unpack8<DT>(wd[i], d);
                unpack8<DT>(ga[i], gv);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (TAIL && c + e >= p.N) f[e] = mean, d[e] = 0.f;
                    xh[i][e] = (f[e] - mean) * rstd;
                    g[i][e] = d[e] * gv[e];
                    if (mine) {
                        sg[i][e] = __builtin_fmaf(d[e], xh[i][e], sg[i][e]);
                        sb[i][e] += d[e];
                    }
                    c1 += g[i][e];
                    c2 = __builtin_fmaf(g[i][e], xh[i][e], c2);
                }
            }
        }
        if (m0 + kGroups < last) request(m0 + kGroups);
        if constexpr (TPR == 256) {
            c1 = group_sum<64>(c1);
            c2 = group_sum<64>(c2);
            __syncthreads();                                 // everyone is through with the last row's sums
            if ((threadIdx.x & 63) == 0) {
                red[0][threadIdx.x >> 6] = c1;
                red[1][threadIdx.x >> 6] = c2;
            }
            __syncthreads();
            c1 = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
            c2 = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
        } else {
            c1 = group_sum<TPR>(c1);
            c2 = group_sum<TPR>(c2);
        }
        c1 *= inv_n;
        c2 *= inv_n;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 8 * (t + i * TPR);
            if (c < p.N && mine) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = rstd * (g[i][e] - c1 - xh[i][e] * c2);
                put8<TAIL>(p.dx + m * p.lddx + c, p.N - c, pack8<DT>(o));
            }
        }
    }
    if constexpr (TPR == 256) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = 8 * (t + i * TPR) + e;
                if (c < p.N) {
                    p.part_gamma[(long)blockIdx.x * p.N + c] = sg[i][e];
                    p.part_beta[(long)blockIdx.x * p.N + c] = sb[i][e];
                }
            }
    } else {
        constexpr int kCols = TPR * PER * 8;
        auto meet = [&](const float (&s)[PER][8], float* out) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) share[grp * kCols + 8 * (t + i * TPR) + e] = s[i][e];
            __syncthreads();
            for (int c = threadIdx.x; c < p.N; c += 256) {
                float v = 0.f;
#pragma unroll
                for (int k = 0; k < kGroups; ++k) v += share[k * kCols + c];
                out[(long)blockIdx.x * p.N + c] = v;
            }
        };
        meet(sg, p.part_gamma);
        meet(sb, p.part_beta);
    }
}

// Any pitch, alignment and N, two kernels: the rows' two means, then a thread per column that walks a run of rows.
template <int DT>
__global__ __launch_bounds__(256) void tw_ln_grad_rows_kernel(const LnGradParams p) {
    __shared__ float red[2][4];
    const float inv_n = 1.f / (float)p.N;
    for (long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const float mean = p.mean[m], rstd = p.rstd[m];
        float c1 = 0.f, c2 = 0.f;
        for (int c = threadIdx.x; c < p.N; c += 256) {
            const float g = tw_to_f32<DT>(p.dy[m * p.lddy + c]) * (p.gamma ? tw_to_f32<DT>(p.gamma[c]) : 1.f);
            c1 += g;
            c2 = __builtin_fmaf(g, (tw_to_f32<DT>(p.x[m * p.ldx + c]) - mean) * rstd, c2);
        }
        c1 = row_sum<256>(c1, red, 0);
        c2 = row_sum<256>(c2, red, 1);
        if (threadIdx.x == 0) {
            p.row_stats[2 * m] = c1 * inv_n;
            p.row_stats[2 * m + 1] = c2 * inv_n;
        }
    }
}
template <int DT>
__global__ __launch_bounds__(256) void tw_ln_grad_cols_kernel(const LnGradParams p) {
    const long c = (long)blockIdx.y * 256 + threadIdx.x;
    if (c >= p.N) return;
    const long first = (long)blockIdx.x * p.rows_per_part;
    const long last = first + p.rows_per_part < p.M ? first + p.rows_per_part : p.M;
    const float ga = p.gamma ? tw_to_f32<DT>(p.gamma[c]) : 1.f;
    float sg = 0.f, sb = 0.f;
    for (long m = first; m < last; ++m) {
        const float d = tw_to_f32<DT>(p.dy[m * p.lddy + c]), rstd = p.rstd[m];
        const float xh = (tw_to_f32<DT>(p.x[m * p.ldx + c]) - p.mean[m]) * rstd;
        sg = __builtin_fmaf(d, xh, sg);
        sb += d;
        p.dx[m * p.lddx + c] = tw_cvt<DT>(rstd * (d * ga - p.row_stats[2 * m] - xh * p.row_stats[2 * m + 1]));
    }
    p.part_gamma[(long)blockIdx.x * p.N + c] = sg;
    p.part_beta[(long)blockIdx.x * p.N + c] = sb;
}

// dst[n] = sum over the parts: 32 columns to a workgroup, every 32nd part to half a wave, eight requests on their way, then the halves' sums in
// order.  blockIdx.y: dgamma or dbeta.  (64 columns and four waves, a request at a time: 32 us for 512 parts of 768 columns.)
__global__ __launch_bounds__(1024) void tw_ln_grad_sum_kernel(const float* part_gamma, const float* part_beta, int n_parts, int N,
                                                              float* dgamma, float* dbeta) {
    __shared__ float red[32][32];
    const float* src = blockIdx.y ? part_beta : part_gamma;
    float* dst = blockIdx.y ? dbeta : dgamma;
    if (!dst) return;                                        // (uniform)
    const int col = threadIdx.x & 31, half = threadIdx.x >> 5;
    const long c = (long)blockIdx.x * 32 + col;
    float s = 0.f;
    if (c < N) {
        int k = half;
        for (; k + 7 * 32 < n_parts; k += 8 * 32) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = src[(long)(k + 32 * i) * N + c];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        for (; k < n_parts; k += 32) s += src[(long)k * N + c];
    }
    red[half][col] = s;
    __syncthreads();
    if (half == 0 && c < N) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += red[i][col];
        dst[c] = t;
    }
}

// ------------------------------------------------------------------------------------------------ host
constexpr int kMaxFeatures = (1 << 24) - 256;   // (65535 workgroups of 256 columns; half a million of 1024 threads)

// Threads of a row and 16-byte pieces of a thread for N features; false: the row does not fit the registers of 256 threads.
bool row_shape(int N, int& tpr, int& per) {
    const int pieces = (N - 1) / 8 + 1;
    if (pieces <= 16) { tpr = 16; per = 1; }
    else if (pieces <= 32) { tpr = 32; per = 1; }
    else if (pieces <= 256) { tpr = 64; per = (pieces + 63) / 64; }
    else if (pieces <= 512) { tpr = 256; per = 2; }
    else if (pieces <= 1024) { tpr = 256; per = 4; }
    else if (pieces <= 2048) { tpr = 256; per = 8; }
    else return false;
    return true;
}

template <template <int, int, int, bool> class K, int DT, bool TAIL>
const void* pick_shape(int tpr, int per) {
    if (tpr == 16) return K<DT, 16, 1, TAIL>::fn();
    if (tpr == 32) return K<DT, 32, 1, TAIL>::fn();
    if (tpr == 64) return per == 1 ? K<DT, 64, 1, TAIL>::fn() : per == 2 ? K<DT, 64, 2, TAIL>::fn() : per == 3 ? K<DT, 64, 3, TAIL>::fn() : K<DT, 64, 4, TAIL>::fn();
    return per == 2 ? K<DT, 256, 2, TAIL>::fn() : per == 4 ? K<DT, 256, 4, TAIL>::fn() : K<DT, 256, 8, TAIL>::fn();
}
template <template <int, int, int, bool> class K>
const void* pick(tw_dtype dt, int tpr, int per, bool tail) {
    if (dt == TW_F16) return tail ? pick_shape<K, TW_F16, true>(tpr, per) : pick_shape<K, TW_F16, false>(tpr, per);
    return tail ? pick_shape<K, TW_BF16, true>(tpr, per) : pick_shape<K, TW_BF16, false>(tpr, per);
}
template <int DT, int TPR, int PER, bool TAIL> struct Forward {
    static const void* fn() { return (const void*)tw_ln_kernel<DT, TPR, PER, TAIL>; }
};
template <int DT, int TPR, int PER, bool TAIL> struct Backward {
    static const void* fn() { return (const void*)tw_ln_grad_kernel<DT, TPR, PER, TAIL>; }
};

template <int DT>
const void* pick_t(int N) {
    if (N <= 256) return (const void*)tw_ln_t_kernel<DT, 8, 4>;
    if (N <= 512) return (const void*)tw_ln_t_kernel<DT, 8, 8>;
    if (N <= 768) return (const void*)tw_ln_t_kernel<DT, 8, 12>;
    if (N <= 1024) return (const void*)tw_ln_t_kernel<DT, 8, 16>;
    return N <= 2048 ? (const void*)tw_ln_t_kernel<DT, 8, 32> : (const void*)tw_ln_t_loop_kernel<DT>;
}

bool odd(const void* q) { return ((uintptr_t)q & 1) != 0; }
bool vec16(const void* q) { return ((uintptr_t)q & 15) == 0; }

// A result that starts where an operand does is that operand only with the same pitch: else its rows lie over rows that are still to be read.
bool over_other_rows(const void* out, int ld_out, const void* in, int ld_in, int rows) { return out == in && ld_out != ld_in && rows > 1; }

// (rows, inner: how many rows the matrices have and the elements of one)
int check_forward(const void* X, int ldx, int M, int N, const void* gamma, const void* beta, float eps, const void* Y, int ldy,
                  const float* mean, const float* rstd, tw_dtype dt, int rows, int inner) {
    if ((M > 0 && (!X || !Y)) || M < 0 || N <= 0 || ldx < inner || ldy < inner) return TW_ERR_ARG;
    if (dt != TW_F16 && dt != TW_BF16) return TW_ERR_ARG;
    if (!(eps >= 0.f) || std::isinf(eps)) return TW_ERR_ARG;
    if (M > 0 && over_other_rows(Y, ldy, X, ldx, rows)) return TW_ERR_ARG;
    if (N > kMaxFeatures) return TW_ERR_UNSUPPORTED;
    if (odd(X) || odd(Y) || odd(gamma) || odd(beta) || ((uintptr_t)mean & 3) != 0 || ((uintptr_t)rstd & 3) != 0) return TW_ERR_ALIGN;
    return TW_OK;
}
// Grids in the first dimension are capped (the kernels over rows walk on): a launch holds fewer than 2^32 threads there.
unsigned capped(long blocks) { return (unsigned)(blocks < (1L << 22) ? blocks : (1L << 22)); }

int launch(const void* fn, dim3 grid, dim3 block, void* params, size_t lds, void* stream) {
    void* args[] = {params};
    return hipLaunchKernel(fn, grid, block, args, lds, (hipStream_t)stream) == hipSuccess ? TW_OK : TW_ERR_HIP;
}

// Workgroups of the backward pass: each leaves N sums of dgamma and of dbeta.
int grad_parts(int M) {
    return M < 8 * 512 ? (M + 7) / 8 : 512;
}
}  // namespace

extern "C" int tw_layernorm(const void* X, int ldx, int M, int N, const void* gamma, const void* beta, float eps, void* Y, int ldy,
                            float* mean, float* rstd, tw_dtype dt, void* hip_stream) {
    const int rc = check_forward(X, ldx, M, N, gamma, beta, eps, Y, ldy, mean, rstd, dt, M, N);
    if (rc) return rc;
    if (M == 0) return TW_OK;
    LnParams p{(const us*)X, (const us*)gamma, (const us*)beta, (us*)Y, mean, rstd, ldx, ldy, M, N, eps, 0};
    int tpr = 0, per = 0;
    const bool vec = vec16(X) && vec16(Y) && vec16(gamma) && vec16(beta) && (ldx & 7) == 0 && (ldy & 7) == 0;
    if (vec && row_shape(N, tpr, per)) {
        const long groups = 256 / tpr, blocks = (M + groups - 1) / groups;
        return launch(pick<Forward>(dt, tpr, per, (N & 7) != 0), dim3(capped(blocks)), dim3(256), &p, 0, hip_stream);
    }
    const void* fn = dt == TW_F16 ? (const void*)tw_ln_any_kernel<TW_F16> : (const void*)tw_ln_any_kernel<TW_BF16>;
    return launch(fn, dim3(capped(M)), dim3(256), &p, 0, hip_stream);
}

extern "C" int tw_layernorm_t(const void* Xt, int ldxt, int M, int N, const void* gamma, const void* beta, float eps, void* Yt, int ldyt,
                              float* mean, float* rstd, tw_dtype dt, void* hip_stream) {
    const int rc = check_forward(Xt, ldxt, M, N, gamma, beta, eps, Yt, ldyt, mean, rstd, dt, N, M);
    if (rc) return rc;
    if (M == 0) return TW_OK;
    LnParams p{(const us*)Xt, (const us*)gamma, (const us*)beta, (us*)Yt, mean, rstd, ldxt, ldyt, M, N, eps,
               ((uintptr_t)Yt & 127) == 0 && (ldyt & 63) == 0};
    if (M > (1 << 27) - 64) return TW_ERR_UNSUPPORTED;       // (a workgroup of up to 1024 threads per 64 tokens)
    if (vec16(Xt) && vec16(Yt) && (ldxt & 7) == 0 && (ldyt & 7) == 0)
        return launch(dt == TW_F16 ? pick_t<TW_F16>(N) : pick_t<TW_BF16>(N), dim3((unsigned)((M + 8L * PCS - 1) / (8 * PCS))), dim3(N <= 2048 ? 512 : 1024), &p, 0, hip_stream);
    const dim3 grid((unsigned)((M + 63L) / 64));
    const void* fn = dt == TW_F16 ? (const void*)tw_ln_t_any_kernel<TW_F16> : (const void*)tw_ln_t_any_kernel<TW_BF16>;
    return launch(fn, grid, dim3(1024), &p, 0, hip_stream);
}

extern "C" int tw_layernorm_grad_workspace(int M, int N, size_t* ws_bytes) {
    if (!ws_bytes || M < 0 || N <= 0) return TW_ERR_ARG;
    *ws_bytes = 4 * ((size_t)grad_parts(M) * 2 * (size_t)N + 2 * (size_t)M);
    return TW_OK;
}

extern "C" int tw_layernorm_grad(const void* dY, int lddy, const void* X, int ldx, int M, int N, const void* gamma, const float* mean,
                                 const float* rstd, void* dX, int lddx, float* dgamma, float* dbeta, void* workspace, size_t ws_bytes,
                                 tw_dtype dt, void* hip_stream) {
    if ((M > 0 && (!dY || !X || !mean || !rstd || !dX || !workspace)) || M < 0 || N <= 0) return TW_ERR_ARG;
    if (dt != TW_F16 && dt != TW_BF16) return TW_ERR_ARG;
    if (lddy < N || ldx < N || lddx < N) return TW_ERR_ARG;
    if (over_other_rows(dX, lddx, dY, lddy, M) || over_other_rows(dX, lddx, X, ldx, M)) return TW_ERR_ARG;
    if (N > kMaxFeatures) return TW_ERR_UNSUPPORTED;
    if (odd(dY) || odd(X) || odd(dX) || odd(gamma)) return TW_ERR_ALIGN;
    if ((((uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)dgamma | (uintptr_t)dbeta) & 3) != 0 || !vec16(workspace)) return TW_ERR_ALIGN;
    size_t need = 0;
    tw_layernorm_grad_workspace(M, N, &need);
    if (ws_bytes < need) return TW_ERR_BUF;
    const int parts = grad_parts(M);
    LnGradParams p;
    p.dy = (const us*)dY; p.x = (const us*)X; p.gamma = (const us*)gamma; p.mean = mean; p.rstd = rstd; p.dx = (us*)dX;
    p.part_gamma = (float*)workspace; p.part_beta = p.part_gamma + (size_t)parts * N; p.row_stats = p.part_beta + (size_t)parts * N;
    p.lddy = lddy; p.ldx = ldx; p.lddx = lddx; p.M = M; p.N = N;
    p.rows_per_part = parts > 0 ? (int)(((long)M + parts - 1) / parts) : 0;
    int rc = TW_OK;
    if (M > 0) {
        int tpr = 0, per = 0;
        const bool vec = vec16(dY) && vec16(X) && vec16(dX) && vec16(gamma) && ((lddy | ldx | lddx) & 7) == 0;
        if (vec && row_shape(N, tpr, per)) {
            const size_t lds = tpr == 256 ? 0 : (size_t)256 * per * 8 * 4;
            rc = launch(pick<Backward>(dt, tpr, per, (N & 7) != 0), dim3((unsigned)parts), dim3(256), &p, lds, hip_stream);
        } else {
            const unsigned gy = (unsigned)((N + 255) / 256);
            rc = launch(dt == TW_F16 ? (const void*)tw_ln_grad_rows_kernel<TW_F16> : (const void*)tw_ln_grad_rows_kernel<TW_BF16>,
                        dim3(capped(M)), dim3(256), &p, 0, hip_stream);
            if (!rc)
                rc = launch(dt == TW_F16 ? (const void*)tw_ln_grad_cols_kernel<TW_F16> : (const void*)tw_ln_grad_cols_kernel<TW_BF16>,
                            dim3((unsigned)parts, gy), dim3(256), &p, 0, hip_stream);
        }
        if (rc) return rc;
    }
    if (!dgamma && !dbeta) return TW_OK;
    int n_parts = parts, n = N;                              // (M = 0: no part, the sums are zero)
    const float* pg = p.part_gamma;
    const float* pb = p.part_beta;
    void* args[] = {(void*)&pg, (void*)&pb, (void*)&n_parts, (void*)&n, (void*)&dgamma, (void*)&dbeta};
    return hipLaunchKernel((const void*)tw_ln_grad_sum_kernel, dim3((unsigned)(((long)N + 31) / 32), 2), dim3(1024), args, 0,
                           (hipStream_t)hip_stream) == hipSuccess ? TW_OK : TW_ERR_HIP;
}
