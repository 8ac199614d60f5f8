// Attention over whole prompts between the fused QKV product and the output product of a Transformer layer: packed sequences of
// different lengths, heads of K and V shared by groups of heads of Q, causal or not.
//
//   O[i, h] = sum_j p_ij V[j, kv(h)],   p_ij = softmax over j of scale * Q[i, h] . K[j, kv(h)],   j in i's sequence, j <= i if causal
//
// One pass over the keys: with m the running maximum of a row's scores (times log2 e) and l the running sum of 2^(score - m), a tile of keys
// whose maximum is larger scales what has been summed by 2^(m_old - m_new).  m, l and the sums are fp32; the weights p are rounded to the
// storage type for the matrix unit (they multiply values of that type, and l sums them before that rounding).
//
// Tiles are cut through the PACKED tokens, not through the sequences: a tile is 128 consecutive rows, whatever sequences they belong to, and a
// row carries its own range of keys [lo, hi).  A short sequence then does not cost a tile of its own, the grid follows
// from the number of tokens alone, and a causal mask is hi = row + 1.  Keys run from the first row's lo to the last row's hi.
//
// Workgroup: four waves of 32 rows, one head.  A wave computes the TRANSPOSED scores S^T = K Q^T of 64 keys: its result layout (lane = row of Q,
// registers = keys) is, with the contraction slots renamed, the operand layout that O^T = V^T P^T wants, so the weights go from one product
// to the next in registers; a row's maximum and sum are the lane's own registers and one exchange between lane halves.  K and V tiles
// come into two LDS buffers by direct loads, on their way while the tile before is multiplied.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <type_traits>

#include "../../include/tw.h"
#include "tw_device.hpp"

namespace {

typedef unsigned short us;
typedef short i16x4 __attribute__((ext_vector_type(4)));
constexpr int kRowsPerTile = 128, kKeys = 64;
constexpr float kSlack = 8.f;
constexpr unsigned kOut = 0x80000000u;      // an offset out of a buffer descriptor's range: fetches zeros

struct AttnParams {
    const us* q;
    const us* k;
    const us* v;
    us* o;
    const int* seq_start;                   // n_seqs + 1 boundaries, or null: one sequence
    long ldq, ldk, ldv, ldo;
    int M, n_seqs, heads, group, d;         // group: heads of Q per head of K and V
    int n_tiles;
    float scale2;                           // scale * log2 e
    int causal;
};

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ tw_u32x4 descriptor(const us* base) {
    const uint64_t a = (uint64_t)base;
    return tw_u32x4{(unsigned)uni((int)(unsigned)a), (unsigned)uni((int)(unsigned)(a >> 32)) & 0xFFFFu, kOut, 0x00020000u};
}
__device__ __forceinline__ i16x4 read_tr(const unsigned char* a) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)a);
}

// Which tile and which head a workgroup takes.  Workgroups whose ids are equal modulo 8 share an XCD and its L2: each XCD gets whole heads where
// their number allows, so that a head's K and V are read into one L2.  Causal tiles cost more the later they lie: heavy ones go first.
__device__ __forceinline__ void place(const AttnParams& p, int& tile, int& head) {
    const int id = (int)blockIdx.x, total = (int)gridDim.x;
    if ((p.heads & 7) == 0) {
        const int per = p.heads >> 3, j = id >> 3;
        head = (id & 7) * per + j % per;
        tile = p.n_tiles - 1 - j / per;
    } else {
        // runs of consecutive (head, tile) for each XCD; tiles from both ends in turn, so that every run has light and heavy ones
        const int x = id & 7, q = total >> 3, r = total & 7;
        const int at = x * q + (x < r ? x : r) + (id >> 3);
        head = at / p.n_tiles;
        const int t = at - head * p.n_tiles;
        tile = t & 1 ? t >> 1 : p.n_tiles - 1 - (t >> 1);
    }
}

// KS: contraction steps of 16 that the head's width takes (d <= 16 * KS).  LDS rows of K and V: 32, 64 or 128 elements.
template <int DT, int KS>
__global__ __launch_bounds__(256, 2) void tw_attention_kernel(const AttnParams p) {
    constexpr int ROW = KS <= 2 ? 64 : KS <= 4 ? 128 : 256;            // bytes of a row in LDS
    constexpr int PIECES = ROW / 16, FB = KS / 2;                      // 16-byte pieces of a row, 32-feature blocks
    constexpr int TILE = kKeys * ROW, LOADS = TILE / 1024 / 4;         // requests of a wave per tile and matrix
    constexpr int OPITCH = KS * 32 + 16;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE > 4 * 32 * OPITCH ? 4 * TILE : 4 * 32 * OPITCH];
    __shared__ int s_first, s_next;
    __shared__ unsigned s_marks[4];
    __shared__ int s_range[4][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    int tile, head;
    place(p, tile, head);
    const int r0 = tile * kRowsPerTile, row = r0 + 32 * wave + l32;

    // This lane's row of Q, the second operand of the scores (contraction slots 16 s + 8 h ..).  Rows behind the last one repeat it.
    tw_u16x8 q[KS];
    {
        const us* src = p.q + (long)(row < p.M ? row : p.M - 1) * p.ldq + (long)head * p.d;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s] = tw_u16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (16 * s + 8 * h < p.d) q[s] = *(const tw_u16x8*)(src + 16 * s + 8 * h);
        }
    }

    // The row's keys [lo, hi): between the last boundary at or before it and the first one behind it.  Every thread looks at its share of
    // the boundaries: those inside the tile become marks, of the others the nearest on either side count.
    int lo = 0, hi = p.M;
    if (p.seq_start) {
        if (tid < 4) s_marks[tid] = 0u;
        if (tid == 4) { s_first = -1; s_next = INT_MAX; }
        __syncthreads();
        for (int i = tid; i <= p.n_seqs; i += 256) {
            const int b = min(max(p.seq_start[i], 0), p.M);
            if (b <= r0) atomicMax(&s_first, b);
            else if (b < r0 + kRowsPerTile) atomicOr(&s_marks[(b - r0) >> 5], 1u << ((b - r0) & 31));
            else atomicMin(&s_next, b);
        }
        __syncthreads();
        lo = s_first;
        hi = s_next;
        const int w0 = wave;
        const unsigned below = (2u << l32) - 1u;             // marks at or before the row, within its word
        for (int w = 0; w < w0; ++w)
            if (s_marks[w]) lo = r0 + 32 * w + 31 - __builtin_clz(s_marks[w]);
        const unsigned mine = s_marks[w0];
        if (mine & below) lo = r0 + 32 * w0 + 31 - __builtin_clz(mine & below);
        for (int w = 3; w > w0; --w)
            if (s_marks[w]) hi = r0 + 32 * w + __builtin_ctz(s_marks[w]);
        if (mine & ~below) hi = r0 + 32 * w0 + __builtin_ctz(mine & ~below);
    }
    const bool valid = row < p.M && lo >= 0 && hi != INT_MAX;   // the row belongs to a sequence
    hi = hi < p.M ? hi : p.M;
    if (p.causal) hi = row + 1;
    if (!valid) lo = hi = 0;
    // what the wave and the workgroup need of the keys: [first, last), and the part of it that every row of the wave sees
    int first = valid ? lo : INT_MAX, last = valid ? hi : 0, inner0 = valid ? lo : 0, inner1 = valid ? hi : INT_MAX;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        first = min(first, __shfl_xor(first, s));
        last = max(last, __shfl_xor(last, s));
        inner0 = max(inner0, __shfl_xor(inner0, s));
        inner1 = min(inner1, __shfl_xor(inner1, s));
    }
    first = uni(first); last = uni(last); inner0 = uni(inner0); inner1 = uni(inner1);
    if (lane == 0) { s_range[wave][0] = first; s_range[wave][1] = last; }
    __syncthreads();
    const int k_begin = uni(min(min(s_range[0][0], s_range[1][0]), min(s_range[2][0], s_range[3][0])));
    const int k_end = uni(max(max(s_range[0][1], s_range[1][1]), max(s_range[2][1], s_range[3][1])));
    if (k_begin >= k_end) return;                            // (uniform) no row of the tile belongs to a sequence

    // What this lane fetches of a tile: request i of the wave fills 1 KB, i.e. 1024 / ROW rows.  Slot s of row r holds piece s ^ f(r), with f such
    // that the lanes an LDS read serves together hit different banks: fk for 16-byte reads of 16 consecutive rows, fv for transposing
    // reads of four consecutive rows (and of the four behind them, by the other lane half).
    auto fk = [](int r) { return ROW == 64 ? (r >> 2) & 3 : ROW == 128 ? (r >> 1) & 7 : r & 15; };
    auto fv = [](int r) { return ROW == 64 ? ((r >> 2) & 1) << 1 : ROW == 128 ? (((r >> 1) & 1) << 2) ^ (((r >> 2) & 1) << 1) : ((r & 3) << 2) ^ (((r >> 2) & 1) << 1); };
    const int kvh = head / p.group;
    const us* kbase = p.k + (long)kvh * p.d;
    const us* vbase = p.v + (long)kvh * p.d;
    const unsigned ldk2 = 2u * (unsigned)p.ldk, ldv2 = 2u * (unsigned)p.ldv;
    constexpr int RPR = 1024 / ROW;                          // rows per request
    const int frow = lane / PIECES, fslot = lane % PIECES;
    auto issue = [&](int k0, int buf) {                      // the tile of keys k0 ..
        const tw_u32x4 dk = descriptor(kbase + (long)k0 * p.ldk), dv = descriptor(vbase + (long)k0 * p.ldv);
        const unsigned dst = lds0 + (unsigned)buf * (2 * TILE);
        const int left = p.M - k0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = (wave * LOADS + i) * RPR + frow;
            const int pk = fslot ^ fk(r), pv = fslot ^ fv(r);
            tw_load_lds<false>(dk, r < left && 8 * pk < p.d ? (unsigned)r * ldk2 + pk * 16 : kOut, dst + (wave * LOADS + i) * 1024u);
            tw_load_lds<false>(dv, r < left && 8 * pv < p.d ? (unsigned)r * ldv2 + pv * 16 : kOut, dst + TILE + (wave * LOADS + i) * 1024u);
        }
    };

    tw_f32x16 o[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] = 0.f;
    // ref: what the exponents are taken from, at least the running maximum less kSlack; l: this lane's share of the sum of weights
    float ref = -__builtin_inff(), l = 0.f;

    // Where this lane's operands lie in a tile.  Scores: row (key) 32 b + l32, piece (2 ks + h) ^ fk; values: rows 16 st + 4 h + j / 4 (+ 8), piece
    // (4 f + ..) ^ fv.  The swizzles repeat every 16 (8) rows, so blocks and steps are constant offsets, and ks and f flip bits.
    const int j = lane & 15;
    const unsigned ka = (unsigned)(l32 * ROW + ((h ^ fk(l32)) << 4));
    const int vr = 4 * h + (j >> 2);
    const unsigned va = (unsigned)(TILE + vr * ROW + (((2 * ((lane >> 4) & 1) + ((j & 3) >> 1)) ^ fv(vr)) << 4) + (j & 1) * 8);
    auto value_operand = [&](const unsigned char* buf, int st, int f) {
        const unsigned char* at = buf + (va ^ (unsigned)(f << 6)) + 16 * st * ROW;
        const i16x4 a = read_tr(at), c = read_tr(at + 8 * ROW);
        return tw_u16x8{(us)a[0], (us)a[1], (us)a[2], (us)a[3], (us)c[0], (us)c[1], (us)c[2], (us)c[3]};
    };

    // a scale of zero is taken into the scores: the mark of a key that is not seen, -inf, must not meet it
    const bool flat = p.scale2 == 0.f;
    const float scale2 = flat ? 1.f : p.scale2;

    auto work = [&](const unsigned char* buf, int k0) {
        const bool whole = k0 >= inner0 && k0 + kKeys <= inner1;          // every row sees every key (wave-uniform)
        tw_f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const tw_u16x8 a = *(const tw_u16x8*)(buf + (ka ^ (unsigned)(ks << 5)) + 32 * b * ROW);
                s[b] = tw_mfma<DT>(a, q[ks], s[b]);
            }
        if (flat) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] *= 0.f;
        }
        bool odd = false;                                    // (wave-uniform) values that are not finite beside keys that some row does not see
        if (!whole) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = k0 + 32 * b + 8 * (r >> 2) + 4 * h + (r & 3);
                    if ((unsigned)(key - lo) >= (unsigned)(hi - lo)) s[b][r] = -__builtin_inff();
                }
            constexpr us kInf = DT == TW_F16 ? 0x7C00 : 0x7F80;
            tw_u16x8 most{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int f = 0; f < FB; ++f) most = __builtin_elementwise_max(most, value_operand(buf, st, f) & (us)0x7FFF);
            bool mine = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) mine |= most[e] >= kInf;
            odd = __any(mine);
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[b][r]);
        top = __builtin_fmaxf(top, __shfl_xor(top, 32)) * scale2;
        // The exponents' reference moves only when some row's maximum has grown by more than kSlack powers of two: the weights stay below
        // 2^kSlack, which 16 bits hold as precisely, and most tiles scale nothing.
        if (__any(top > ref + kSlack)) {
            const float next = __builtin_fmaxf(ref, top);
            const float from = ref == -__builtin_inff() ? next : ref;     // (nothing summed yet; -inf twice: no key seen)
            const float fade = __builtin_amdgcn_exp2f(ref == next ? 0.f : from - next);
            ref = next;
            l *= fade;
#pragma unroll
            for (int f = 0; f < FB; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[f][r] *= fade;
        }
        const float base = ref == -__builtin_inff() ? 0.f : ref;          // (no key yet, or only scores of -inf: all weights 0)
        tw_u16x8 w[4];                                       // weights: operand of contraction step 2 b + r / 8
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], scale2, -base));
                sum[r & 3] += e;
                w[2 * b + (r >> 3)][r & 7] = tw_cvt<DT>(e);
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        // O^T += V^T P^T.  Slots 8 h + 0..3 and 8 h + 4..7 of step st are the keys 16 st + 4 h + 0..3 and 16 st + 8 + 4 h + 0..3
        if (!odd) {
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int f = 0; f < FB; ++f) o[f] = tw_mfma<DT>(value_operand(buf, st, f), w[st], o[f]);
        } else {                                             // rare: a weight of zero must not meet them; they reach the rows that see their key
            constexpr us kInf = DT == TW_F16 ? 0x7C00 : 0x7F80;
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int f = 0; f < FB; ++f) {
                    tw_u16x8 x = value_operand(buf, st, f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = (x[e] & 0x7FFF) >= kInf ? (us)0 : x[e];
                    o[f] = tw_mfma<DT>(x, w[st], o[f]);
                }
            for (int kk = 0; kk < kKeys; ++kk) {
                const bool sees = (unsigned)(k0 + kk - lo) < (unsigned)(hi - lo);
#pragma unroll
                for (int f = 0; f < FB; ++f)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int c = 32 * f + 8 * (r >> 2) + 4 * h + (r & 3);
                        const float x = tw_to_f32<DT>(*(const us*)(buf + TILE + kk * ROW + (((c >> 3) ^ fv(kk)) << 4) + (c & 7) * 2));
                        if (sees && !(__builtin_fabsf(x) < __builtin_inff())) o[f][r] += x;
                    }
            }
        }
    };

    issue(k_begin, 0);
    auto turn = [&](int k0, int buf) {                       // (buf: a constant)
        tw_lds_wait<0>();                                    // the tile has landed, and nobody reads the other buffer any more
        if (k0 + kKeys < k_end) issue(k0 + kKeys, buf ^ 1);
        if (k0 < last && k0 + kKeys > first) work(smem + buf * (2 * TILE), k0);   // (wave-uniform)
    };
    for (int k0 = k_begin; k0 < k_end; k0 += 2 * kKeys) {
        turn(k0, 0);
        if (k0 + kKeys < k_end) turn(k0 + kKeys, 1);
    }
    l += __shfl_xor(l, 32);
    const float inv = 1.f / l;
    __syncthreads();                                         // the staging areas of the results lie over the tiles
    unsigned char* stage = smem + wave * (32 * OPITCH);
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            tw_u32x2 v;
            v.x = (unsigned)tw_cvt<DT>(o[f][4 * c] * inv) | ((unsigned)tw_cvt<DT>(o[f][4 * c + 1] * inv) << 16);
            v.y = (unsigned)tw_cvt<DT>(o[f][4 * c + 2] * inv) | ((unsigned)tw_cvt<DT>(o[f][4 * c + 3] * inv) << 16);
            *(tw_u32x2*)(stage + l32 * OPITCH + (32 * f + 8 * c + 4 * h) * 2) = v;
        }
    const unsigned long long rows = __builtin_amdgcn_ballot_w64(valid);      // (both halves alike)
    asm volatile("" ::: "memory");                           // (the LDS executes a wave's instructions in order)
    constexpr int OP = 2 * KS;                               // 16-byte pieces of a result row
#pragma unroll
    for (int i = 0; i < 32 * OP / 64; ++i) {
        const int at = lane + 64 * i, r = at / OP, pc = at % OP;
        const tw_u32x4 v = *(const tw_u32x4*)(stage + r * OPITCH + pc * 16);
        if (((rows >> r) & 1) != 0 && 8 * pc < p.d) *(tw_u32x4*)(p.o + (long)(r0 + 32 * wave + r) * p.ldo + (long)head * p.d + 8 * pc) = v;
    }
}

template <int DT>
const void* pick(int d) {
    return d <= 32 ? (const void*)tw_attention_kernel<DT, 2> : d <= 64 ? (const void*)tw_attention_kernel<DT, 4>
           : d <= 96 ? (const void*)tw_attention_kernel<DT, 6> : (const void*)tw_attention_kernel<DT, 8>;
}
}  // namespace

extern "C" int tw_attention(const void* Q, int ldq, const void* K, int ldk, const void* V, int ldv, void* O, int ldo, int M,
                            const int* seq_start, int n_seqs, int heads, int kv_heads, int head_dim, float scale, int causal, tw_dtype dt,
                            void* hip_stream) {
    if ((M > 0 && (!Q || !K || !V || !O)) || M < 0 || n_seqs < 0 || heads <= 0 || kv_heads <= 0 || head_dim <= 0) return TW_ERR_ARG;
    if (dt != TW_F16 && dt != TW_BF16) return TW_ERR_ARG;
    if (heads % kv_heads != 0 || !(scale >= 0.f) || std::isinf(scale)) return TW_ERR_ARG;
    if (!seq_start && n_seqs > 1) return TW_ERR_ARG;
    if ((long)ldq < (long)heads * head_dim || (long)ldo < (long)heads * head_dim || (long)ldk < (long)kv_heads * head_dim || (long)ldv < (long)kv_heads * head_dim) return TW_ERR_ARG;
    if (head_dim > 128 || (head_dim & 7) != 0) return TW_ERR_UNSUPPORTED;
    if (((ldq | ldk | ldv | ldo) & 7) != 0) return TW_ERR_ALIGN;
    if ((((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O) & 15) != 0 || ((uintptr_t)seq_start & 3) != 0) return TW_ERR_ALIGN;
    // a tile's rows are addressed by 31-bit offsets; a launch holds fewer than 2^32 threads
    if (ldk >= (1 << 24) || ldv >= (1 << 24)) return TW_ERR_UNSUPPORTED;
    const long n_tiles = ((long)M + kRowsPerTile - 1) / kRowsPerTile;
    if (n_tiles * heads >= (1L << 24)) return TW_ERR_UNSUPPORTED;
    if (M == 0 || (seq_start && n_seqs == 0)) return TW_OK;
    AttnParams p;
    p.q = (const us*)Q; p.k = (const us*)K; p.v = (const us*)V; p.o = (us*)O; p.seq_start = seq_start;
    p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo;
    p.M = M; p.n_seqs = n_seqs; p.heads = heads; p.group = heads / kv_heads; p.d = head_dim;
    p.n_tiles = (int)n_tiles; p.scale2 = scale * 1.44269504f; p.causal = causal != 0;
    const void* fn = dt == TW_F16 ? pick<TW_F16>(head_dim) : pick<TW_BF16>(head_dim);
    void* args[] = {(void*)&p};
    return hipLaunchKernel(fn, dim3((unsigned)(n_tiles * heads)), dim3(256), args, 0, (hipStream_t)hip_stream) == hipSuccess ? TW_OK : TW_ERR_HIP;
}
