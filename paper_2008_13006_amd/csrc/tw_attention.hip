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
//
// Bound: 2 d multiply-adds a key and row on the matrix unit, and one exponential a key and row beside them.  One prompt of 8192 tokens, 16
// heads of 128, causal: 260 to 271 us from card to card, 1015 to 1060 TFLOP/s of what the mask leaves (a large bf16 product reaches 1256; f16
// takes 7 % longer).  The matrix unit is busy for 54 % of the cycles, the vector unit issues for 52 %.  What did not pay
// there: 32 keys at a time in three stages of one wave (353 us: what one wave issues to the matrix unit and to the vector unit does not
// overlap; what two waves issue does, and two workgroups share a compute unit), eight waves whose halves take turns at the two units
// (300 us, and twice the time on short prompts), higher wave priority around the products (no difference).
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
constexpr float kSlack = 8.f, kLog2e = 1.44269504f;
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
    int by_cost;                            // tiles are taken in the order of their numbers of keys
};

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ tw_u32x4 descriptor(const us* base) {
    const uint64_t a = (uint64_t)base;
    return tw_u32x4{(unsigned)uni((int)(unsigned)a), (unsigned)uni((int)(unsigned)(a >> 32)) & 0xFFFFu, kOut, 0x00020000u};
}
// The larger of a value and that of the other lane half (lane ^ 32).
__device__ __forceinline__ float max_halves(float x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned low = both[0], high = both[1];            // (copies: the builtin cast of a vector's element takes the first one)
    return __builtin_fmaxf(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high));
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

// Packed prompts of several tiles each: the tile with `rank` tiles of fewer keys (of equal ones the earlier counts as fewer), so that the heaviest
// start first and the last ones to end are short.  Every workgroup works the order out by itself, thread t for tile t: at most 256 tiles and 256
// boundaries (M up to 32768).  Keys and tile numbers are distinct pairs, so the ranks are a permutation whatever the boundaries are.
// 24 causal prompts of 12000 tokens, 16 heads of 128: 117 us in the order of the tokens, 102 so.
__device__ __forceinline__ int tile_by_cost(const AttnParams& p, int rank, unsigned char* smem, int& s_tile) {
    int* bounds = (int*)smem;
    int* costs = bounds + 256;
    const int t = (int)threadIdx.x;
    bounds[t] = t <= p.n_seqs ? min(max(p.seq_start[t], 0), p.M) : INT_MAX;
    __syncthreads();
    const int first = t * kRowsPerTile, last = min(first + kRowsPerTile, p.M) - 1;
    int begin = 0, next = INT_MAX;
    for (int i = 0; i <= p.n_seqs; i += 16) {                // (those behind the last one are INT_MAX)
        int4 b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) b[k] = ((const int4*)(bounds + i))[k];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            for (const int v : {b[k].x, b[k].y, b[k].z, b[k].w}) {
                begin = v <= first ? max(begin, v) : begin;
                next = v > last ? min(next, v) : next;
            }
    }
    const int keys = (p.causal || next == INT_MAX ? last + 1 : next) - begin;
    const int mine = t < p.n_tiles ? keys * 256 + t : INT_MAX;
    costs[t] = mine;
    __syncthreads();
    int fewer = 0;
    for (int i = 0; i < p.n_tiles; i += 32) {
        int4 c[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = ((const int4*)(costs + i))[k];
#pragma unroll
        for (int k = 0; k < 8; ++k) fewer += (c[k].x < mine) + (c[k].y < mine) + (c[k].z < mine) + (c[k].w < mine);
    }
    if (t < p.n_tiles && fewer == rank) s_tile = t;
    __syncthreads();
    return uni(s_tile);
}

// KS: contraction steps of 16 that the head's width takes (d <= 16 * KS).  LDS rows of K and V: 32, 64 or 128 elements.
template <int DT, int KS>
__global__ __launch_bounds__(256, 2) void tw_attention_kernel(const AttnParams p) {
    constexpr int ROW = KS <= 2 ? 64 : KS <= 4 ? 128 : 256;            // bytes of a row in LDS
    constexpr int PIECES = ROW / 16, FB = KS / 2;                      // 16-byte pieces of a row, 32-feature blocks
    constexpr int TILE = kKeys * ROW, LOADS = TILE / 1024 / 4;         // requests of a wave per tile and matrix
    constexpr int OPITCH = KS * 32 + 16;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE > 4 * 32 * OPITCH ? 4 * TILE : 4 * 32 * OPITCH];
    __shared__ int s_first, s_next, s_tile;
    __shared__ unsigned s_marks[4];
    __shared__ int s_range[4][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    int tile, head;
    place(p, tile, head);
    if (p.by_cost) tile = tile_by_cost(p, tile, smem, s_tile);
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
    // Request i of the tile of keys k0 .., the first LOADS of K, the others of V.  Rows behind the last key are out of range.
    auto request = [&](int k0, int buf, int i) __attribute__((always_inline)) {
        const bool of_v = i >= LOADS;
        const int n = of_v ? i - LOADS : i, r = (wave * LOADS + n) * RPR + frow, pc = fslot ^ (of_v ? fv(r) : fk(r));
        const us* base = of_v ? vbase + (long)k0 * p.ldv : kbase + (long)k0 * p.ldk;
        tw_load_lds<false>(descriptor(base), r < k_end - k0 && 8 * pc < p.d ? (unsigned)r * (of_v ? ldv2 : ldk2) + pc * 16 : kOut,
                           lds0 + (unsigned)buf * (2 * TILE) + (of_v ? TILE : 0) + (wave * LOADS + n) * 1024u);
    };

    tw_f32x16 o[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] = 0.f;
    // ref: what the exponents are taken from, between the running maximum less kSlack + kLift and that less kLift; l: this lane's share of the sum of weights.
    // f16 holds nothing below 2^-24, which thousands of keys that one outweighs may lie below: its weights are taken 2^7 times as large, so that the
    // largest lies between 2^7 and 2^15 and a small one is off by 2^-32 of it at most.
    constexpr float kLift = DT == TW_F16 ? 7.f : 0.f;
    float ref = -__builtin_inff(), l = 0.f;

    // Where this lane's operands lie in a tile.  Scores: row (key) 32 b + l32, piece (2 ks + h) ^ fk; values: rows 16 st + 4 h + j / 4 (+ 8), piece
    // (4 f + ..) ^ fv.  The swizzles repeat every 16 (8) rows, so blocks and steps are constant offsets, and ks and f flip bits.
    const int j = lane & 15;
    const unsigned ka = (unsigned)(l32 * ROW + ((h ^ fk(l32)) << 4));
    const int vr = 4 * h + (j >> 2);
    const unsigned va = (unsigned)(TILE + vr * ROW + (((2 * ((lane >> 4) & 1) + ((j & 3) >> 1)) ^ fv(vr)) << 4) + (j & 1) * 8);
    auto value_operand = [&](const unsigned char* buf, int st, int f) __attribute__((always_inline)) {
        const unsigned char* at = buf + (va ^ (unsigned)(f << 6)) + 16 * st * ROW;
        return __builtin_bit_cast(tw_u16x8, __builtin_shufflevector(read_tr(at), read_tr(at + 8 * ROW), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // a scale of zero is taken into the scores: the mark of a key that is not seen, -inf, must not meet it
    const bool flat = p.scale2 == 0.f;
    const float scale2 = flat ? 1.f : p.scale2;
    constexpr us kInf = DT == TW_F16 ? 0x7C00 : 0x7F80;
    bool odd = false;                                        // values that are not finite lie beside keys that some row does not see
    // From 2^20 on a score's product with scale2 is rounded before the reference is taken from it, as it was for the reference: the fused form
    // would leave that rounding, up to half a step of the product, in the exponent of the largest (2^24 and more: whole powers of two).
    bool large = false;
    constexpr float kLarge = 1048576.f;
    // operands are read that many products ahead (d = 128, one prompt of 8192: four 270 us, eight 262; of 64 there are two workgroups more
    // to a compute unit with the registers of four)
    constexpr int kAhead = KS >= 6 ? 8 : 4;

    // The tile of keys k0 .. in `buf`; next(i) makes request i for the tile after it.
    auto work = [&](const unsigned char* buf, int k0, auto next) __attribute__((always_inline)) {
        const bool whole = k0 >= inner0 && k0 + kKeys <= inner1;          // every row sees every key (wave-uniform)
        tw_f32x16 s[2];
        tw_u16x8 x[kAhead];
        auto key_operand = [&](int n) __attribute__((always_inline)) {
            return *(const tw_u16x8*)(buf + (ka ^ (unsigned)((n >> 1) << 5)) + 32 * (n & 1) * ROW);
        };
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
        for (int n = 0; n < kAhead && n < 2 * KS; ++n) x[n] = key_operand(n);
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
            __builtin_amdgcn_sched_barrier(0);
            s[n & 1] = tw_mfma<DT>(x[n % kAhead], q[n >> 1], s[n & 1]);
            __builtin_amdgcn_sched_barrier(0);
            if (n + kAhead < 2 * KS) x[n % kAhead] = key_operand(n + kAhead);
        }
        if (flat) {
            float zero = 0.f;
            asm volatile("" : "+v"(zero));                   // (or the products are made ahead of the branch, for every tile)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] *= zero;
        }
        if (!whole) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = k0 + 32 * b + 8 * (r >> 2) + 4 * h + (r & 3);
                    if ((unsigned)(key - lo) >= (unsigned)(hi - lo)) s[b][r] = -__builtin_inff();
                }
            // a weight of zero must not meet a value that is not finite: see the end
            tw_u16x8 most{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int f = 0; f < FB; ++f)
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(tw_u16x8, __builtin_bit_cast(tw_u32x4, value_operand(buf, st, f)) & 0x7FFF7FFFu));
            bool any = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) any |= most[e] >= kInf;
            odd |= __any(any) != 0;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[b][r]);
        top = max_halves(top) * scale2;
        // The exponents' reference moves only when some row's maximum has grown by more than kSlack powers of two: the weights stay below
        // 2^(kSlack + kLift), which 16 bits hold as precisely, and most tiles scale nothing.
        if (__any(top - ref > kSlack + kLift)) {             // (the difference: a step of the sum may be larger than the slack)
            const float next_ref = __builtin_fmaxf(ref, top - kLift);
            const float from = ref == -__builtin_inff() ? next_ref : ref;     // (nothing summed yet; -inf twice: no key seen)
            const float fade = __builtin_amdgcn_exp2f(ref == next_ref ? 0.f : from - next_ref);
            ref = next_ref;
            large |= __any(__builtin_fabsf(ref) > kLarge && __builtin_fabsf(ref) < __builtin_inff()) != 0;
            l *= fade;
#pragma unroll
            for (int f = 0; f < FB; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[f][r] *= fade;
        }
        const float base = ref == -__builtin_inff() ? 0.f : ref;          // (no key yet, or only scores of -inf: all weights 0)
        float factor = scale2;
        if (large) {
            asm volatile("" : "+v"(factor));                 // (as above)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] *= factor;
            factor = 1.f;
        }
        tw_u16x8 w[4];                                       // weights: operand of contraction step 2 b + r / 8
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        // A request for the next tile, then its share of the exponentials: a compute unit takes 64 bytes of requests a clock, and a wave that makes
        // all of its own at once waits for that.
        constexpr int kShare = 32 / (2 * LOADS);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int b = i >> 4, r = i & 15;
            if (i % kShare == 0) {
                __builtin_amdgcn_sched_barrier(0);
                next(i / kShare);
                __builtin_amdgcn_sched_barrier(0);
            }
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], factor, -base));
            sum[r & 3] += e;
            w[2 * b + (r >> 3)][r & 7] = tw_cvt<DT>(e);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        // O^T += V^T P^T.  Slots 8 h + 0..3 and 8 h + 4..7 of step st are the keys 16 st + 4 h + 0..3 and 16 st + 8 + 4 h + 0..3
#pragma unroll
        for (int n = 0; n < kAhead; ++n) x[n] = value_operand(buf, n / FB, n % FB);
#pragma unroll
        for (int n = 0; n < 4 * FB; ++n) {
            __builtin_amdgcn_sched_barrier(0);
            o[n % FB] = tw_mfma<DT>(x[n % kAhead], w[n / FB], o[n % FB]);
            __builtin_amdgcn_sched_barrier(0);
            if (n + kAhead < 4 * FB) x[n % kAhead] = value_operand(buf, (n + kAhead) / FB, (n + kAhead) % FB);
        }
    };

#pragma unroll
    for (int i = 0; i < 2 * LOADS; ++i) request(k_begin, 0, i);
    auto turn = [&](int k0, int buf) __attribute__((always_inline)) {     // (buf: a constant)
        tw_lds_wait<0>();                                    // the tile has landed, and nobody reads the other buffer any more
        // (behind the last tile the requests are out of range)
        auto next = [&](int i) __attribute__((always_inline)) { request(k0 + kKeys, buf ^ 1, i); };
        if (k0 < last && k0 + kKeys > first) {               // (wave-uniform)
            work(smem + buf * (2 * TILE), k0, next);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * LOADS; ++i) next(i);
        }
    };
    for (int k0 = k_begin; k0 < k_end; k0 += 2 * kKeys) {
        turn(k0, 0);
        if (k0 + kKeys < k_end) turn(k0 + kKeys, 1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // nothing on its way into LDS any more
    l += __shfl_xor(l, 32);
    // Rare: a value that is not finite, beside keys that some row of the wave does not see, has met a weight of zero there.  Everything is made
    // again, key by key, each row's own keys only.  (Not the sums with V alone: scores of 2^24 and more whose products are added in another
    // order have other weights than those that l has summed.)
    if (odd) {
        float most = -__builtin_inff(), weights = 0.f;
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[f][r] = 0.f;
#pragma unroll 1
        for (int key = first; key < last; ++key) {
            const us* krow = p.k + (long)key * p.ldk + (long)kvh * p.d;
            const us* vrow = p.v + (long)key * p.ldv + (long)kvh * p.d;
            float x = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                if (16 * ks + 8 * h < p.d) {
                    const tw_u16x8 kv = *(const tw_u16x8*)(krow + 16 * ks + 8 * h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x = __builtin_fmaf(tw_to_f32<DT>(kv[e]), tw_to_f32<DT>(q[ks][e]), x);
                }
            x += __shfl_xor(x, 32);
            if (flat) x *= 0.f;
            if ((unsigned)(key - lo) >= (unsigned)(hi - lo)) continue;
            x *= scale2;
            if (x > most) {
                const float fade = most == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(most - x);
                weights *= fade;
#pragma unroll
                for (int f = 0; f < FB; ++f)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[f][r] *= fade;
                most = x;
            }
            const float e = __builtin_amdgcn_exp2f(x - (most == -__builtin_inff() ? 0.f : most));
            weights += e;
#pragma unroll
            for (int f = 0; f < FB; ++f)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = 32 * f + 8 * (r >> 2) + 4 * h + (r & 3);
                    const float v = c < p.d ? tw_to_f32<DT>(vrow[c]) : 0.f;
                    o[f][r] += __builtin_fabsf(v) < __builtin_inff() ? e * v : v;
                }
        }
        l = weights;
    }
    const float inv = 1.f / l;
    // A mean of values that f16 holds is one itself, but the weights' rounding adds up to half a step of the largest: back to that one, unless
    // an infinity among the values made it.
    auto mean = [&](float sum) __attribute__((always_inline)) {
        const float x = sum * inv;
        if constexpr (DT == TW_F16) return __builtin_fabsf(x) < __builtin_inff() ? __builtin_fminf(__builtin_fmaxf(x, -65504.f), 65504.f) : x;
        else return x;
    };
    __syncthreads();                                         // the staging areas of the results lie over the tiles
    unsigned char* stage = smem + wave * (32 * OPITCH);
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            tw_u32x2 v;
            v.x = (unsigned)tw_cvt<DT>(mean(o[f][4 * c])) | ((unsigned)tw_cvt<DT>(mean(o[f][4 * c + 1])) << 16);
            v.y = (unsigned)tw_cvt<DT>(mean(o[f][4 * c + 2])) | ((unsigned)tw_cvt<DT>(mean(o[f][4 * c + 3])) << 16);
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
    if (head_dim > 128 || (head_dim & 7) != 0 || std::isinf(scale * kLog2e)) return TW_ERR_UNSUPPORTED;
    if (((ldq | ldk | ldv | ldo) & 7) != 0) return TW_ERR_ALIGN;
    if ((((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O) & 15) != 0 || ((uintptr_t)seq_start & 3) != 0) return TW_ERR_ALIGN;
    if (O == Q && ldo != ldq && M > 1) return TW_ERR_ARG;    // (O's rows would lie over rows of Q that are still to be read)
    // a tile's rows are addressed by 31-bit offsets; a launch holds fewer than 2^32 threads
    if (ldk >= (1 << 24) || ldv >= (1 << 24)) return TW_ERR_UNSUPPORTED;
    const long n_tiles = ((long)M + kRowsPerTile - 1) / kRowsPerTile;
    if (n_tiles * heads >= (1L << 24)) return TW_ERR_UNSUPPORTED;
    if (M == 0 || (seq_start && n_seqs == 0)) return TW_OK;
    AttnParams p;
    p.q = (const us*)Q; p.k = (const us*)K; p.v = (const us*)V; p.o = (us*)O; p.seq_start = seq_start;
    p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo;
    p.M = M; p.n_seqs = n_seqs; p.heads = heads; p.group = heads / kv_heads; p.d = head_dim;
    p.n_tiles = (int)n_tiles; p.scale2 = scale * kLog2e; p.causal = causal != 0;
    // Working out the order costs a workgroup 2 to 3 us.  It pays for few long prompts of different lengths and wide heads, 24 and 10 of 522 and 1800
    // tokens on average, 16 heads of 128: 90 -> 85 and 228 -> 204 us causal, 124 -> 113 and 390 -> 340 not; of equal lengths it costs 0 to 2 % and 2 to
    // 8 %.  Short prompts (60 of 295 on average: 109 -> 118 us) and heads of 64 (50 -> 53, 130 -> 131 us), of which four workgroups share
    // a compute unit, lose.  A launch that fits the card at once has no order.
    p.by_cost = seq_start && n_seqs > 1 && n_seqs < 256 && n_tiles <= 256 && head_dim > 64 && M >= 3L * kRowsPerTile * n_seqs && n_tiles * heads > 512;
    const void* fn = dt == TW_F16 ? pick<TW_F16>(head_dim) : pick<TW_BF16>(head_dim);
    void* args[] = {(void*)&p};
    return hipLaunchKernel(fn, dim3((unsigned)(n_tiles * heads)), dim3(256), args, 0, (hipStream_t)hip_stream) == hipSuccess ? TW_OK : TW_ERR_HIP;
}
