// Attention of new queries over the 8-bit cache, for gfx950.
//
//   S = (q k8^T) * scale * s_k,  O = softmax(S) (s_v v8)
// with one s_k and s_v per block of tokens and head.  Every code is exactly a
// bf16 number, so the products run on bf16 matrix instructions without any
// rounding of K, V or Q: s_k is a factor of the scores of a block, s_v one of
// its probabilities, which are rounded to bf16 once after it (in tiles of 16
// rows to two bf16, hardly at all).  Scores, the running maximum and sum of the
// softmax (in units of log 2) and the output accumulate in fp32.
//
// A call is cut into items: (sequence, head, tile of query rows, part of the
// walk over its tokens).  Two kernels take them by the rows of a tile, and
// join_kernel joins the parts of a walk:
//   rows_kernel   16 or 32 rows: few rows, bound by reading the cache, or calls
//                 too small to fill the chip, bound by the turns of a walk;
//   tile_kernel   64, 128 or 256 rows: bound by the card's power, which the
//                 conversions of the codes share with the matrix products.
// Without lists the query heads of a key/value head share a tile (their rows
// are consecutive in memory).
//
// rows_kernel: the waves of a work-group take steps of 32 tokens in turn, each
// with a softmax state of its own, and are joined at the end.  A wave keeps
// everything in registers, without LDS or a barrier in its loop, and has the
// codes of its next step under way while it computes one:
//   S^T (tokens x rows) = K Q^T   v_mfma_f32_16x16x32_bf16: a lane loads 16
//       consecutive bytes of one token's K; which channels meet in a matrix
//       step is free as long as Q is laid out alike;
//   O^T (channels x rows) += V^T P^T: the 8 tokens that a lane's scores
//       belong to are those whose V it loads (D/16 consecutive channels
//       each), so P needs no exchange between lanes and V^T is formed by
//       byte permutes of the lane's own loads.
// One query over 24 heads of 118,800 tokens of 128 channels (730 MB) takes 131
// us: 5.6 TB/s, where a large copy moves 4.9; over lists of a quarter of the
// blocks 35 us (5.2).  With one step's codes and no more under way the first took
// 177 us.
// A wave that meets a value scale under 2^-64 walks its steps twice (see
// small_scale): products apart from the accumulators in the one loop cost 6% of a
// call with 16 rows and 19% of one with 32.
#include "moddit_internal.h"

#include <algorithm>
#include <type_traits>

namespace moddit {
namespace {

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
typedef __bf16 bf16x8 __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef short s16x4 __attribute__((__vector_size__(4 * sizeof(short))));
typedef short s16x8 __attribute__((__vector_size__(8 * sizeof(short))));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4_t;
typedef __attribute__((address_space(3))) const uint4 lds_u4_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kXcds = 8;
constexpr int kStep = 32;          // tokens of a wave's step
constexpr float kSumLimit = 256.0f; // bound on a lane's probability sum per unit while its maximum is kept

template <class F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(f, std::make_integer_sequence<int, N>{});
}

constexpr int kRowWaves = 8;       // waves of a work-group of rows_kernel
template <int ROWS>
constexpr int kTileWaves = ROWS == 256 ? 8 : 4;   // of tile_kernel

struct AttnArgs {
    const uint16_t* q;
    const uint8_t *k, *v;
    const float *ks, *vs;
    const int32_t *len, *idx, *cnt;
    uint16_t* o;
    float* lse;
    float* part;               // C > 1: O / l of every item, then its log2-sum-exp2
    int B, Hq, H, Lq, cap, ncap, max_len, n, nq, block;
    int shift;                 // block = 1 << shift
    int group;                 // query heads per key/value head
    int tiles;                 // row tiles per head and query block (lists) or key/value head
    int heads;                 // heads that items count: Hq with lists, H without
    int C;                     // parts of a walk
    int stretch;               // consecutive items of a die
    int units;                 // B * heads * (lists: nq) * tiles
    float c2;                  // scale * log2(e)
};

// Two consecutive codes of w (bytes 0, 1 or 2, 3) as a pair of bf16.
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w) {
    if constexpr (FMT == MOD_CACHE_E4M3) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    } else {
        const float a = (float)(int8_t)(w >> (HI ? 16 : 0)), b = (float)(int8_t)(w >> (HI ? 24 : 8));
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);   // exact: 8 bits
    }
}

// Eight consecutive codes as a matrix operand.
template <int FMT>
__device__ __forceinline__ bf16x8 operand8(uint32_t w0, uint32_t w1) {
    const u32x4 r = {bf16_pair<FMT, false>(w0), bf16_pair<FMT, true>(w0), bf16_pair<FMT, false>(w1),
                     bf16_pair<FMT, true>(w1)};
    return __builtin_bit_cast(bf16x8, r);
}

// Code F of a and of b as a pair of bf16.
template <int FMT, int F>
__device__ __forceinline__ uint32_t column_pair(uint32_t a, uint32_t b) {
    if constexpr (FMT == MOD_CACHE_E4M3) {
        const uint32_t x = __builtin_amdgcn_perm(b, a, F < 2 ? 0x05010400u : 0x07030602u);
        return bf16_pair<FMT, F % 2 == 1>(x);
    } else {
        const float x = (float)(int8_t)(a >> (8 * F)), y = (float)(int8_t)(b >> (8 * F));
        return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const bf16x2 r = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};   // one instruction
    return __builtin_bit_cast(uint32_t, r);
}

// max / sum over the four lanes that hold a query row's tokens (16 apart): a
// swap with x in both operands leaves both lanes' values in its results
__device__ __forceinline__ float max4(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum4(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A value that all lanes share, in a scalar register.
__device__ __forceinline__ float uniform(float x) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

// Value scales under 2^-64 (a write gives 2^-126 on): their products with
// probabilities below one may be subnormal bf16, of fewer bits.  They enter
// 2^64 times as large, and 2^-64 elsewhere: exact.
__device__ __forceinline__ bool small_scale(float s) { return s > 0.0f && s < 0x1p-64f; }
constexpr uint32_t kSmallScale = 0x1f800000u;   // 2^-64: the bits of positive numbers have their order

__device__ __forceinline__ int clamp_len(const AttnArgs& a, int b) {
    return a.len ? min(max(a.len[b], 0), a.max_len) : a.max_len;
}

// Item `u` of the launch: which rows it has.
struct Rows {
    int b, head, kv, i;        // sequence, query head (lists), key/value head, query block
    long row0;                 // first row of q, o and lse
    int count;                 // rows of the tile that exist
};
template <int ROWS, bool LISTS>
__device__ __forceinline__ Rows rows_of(const AttnArgs& a, int u) {
    Rows r;
    const int t = u % a.tiles;
    u /= a.tiles;
    r.i = 0;
    if (LISTS) {
        r.i = u % a.nq;
        u /= a.nq;
    }
    r.head = u % a.heads;
    r.b = u / a.heads;
    const int group = a.group;
    r.kv = LISTS ? r.head / group : r.head;
    const int all = LISTS ? min(a.block, a.Lq - r.i * a.block) : group * a.Lq;
    r.row0 = (LISTS ? ((long)r.b * a.Hq + r.head) * a.Lq + (long)r.i * a.block
                    : ((long)r.b * a.Hq + (long)r.head * group) * a.Lq) + (long)t * ROWS;
    r.count = all - t * ROWS;
    return r;
}

// This work-group's item; false: none.  Items are ordered by head, part of the
// walk, then the tiles that share it.  Consecutive work-groups go to the dies
// in turn; a die takes `stretch` consecutive items (an eighth of the tiles of a
// part, which read the same or nearly the same tokens), then every eighth such
// stretch: heads and sequences of different lengths spread over all dies.
template <bool LISTS>
__device__ __forceinline__ bool item_of(const AttnArgs& a, int& unit, int& part) {
    const int i = (int)(blockIdx.x / kXcds), x = (int)(blockIdx.x % kXcds);
    const int w = (i / a.stretch * kXcds + x) * a.stretch + i % a.stretch;
    const int tiles = (LISTS ? a.nq : 1) * a.tiles;
    const int hb = w / (tiles * a.C), rest = w % (tiles * a.C);
    part = rest / tiles;
    unit = hb * tiles + rest % tiles;
    return w < a.units * a.C;
}

template <int D, int FMT, int RT, bool LISTS>
__global__ __launch_bounds__(64 * kRowWaves, 1) void rows_kernel(AttnArgs a) {
    constexpr int ROWS = 16 * RT, WAVES = kRowWaves;
    // With 16 rows the memory bounds the kernel: P enters as two bf16, its
    // rounding and what that left off, so that the output's own rounding is the
    // only one that counts (132 -> 133 us on 24 heads of 118,800 tokens; 52 -> 56
    // us with 32 rows, four sequences of 32768, where P is one bf16).
    constexpr bool TWICE = RT == 1;
    constexpr int KC = D / 64;          // 16-byte chunks of a token's K per lane
    constexpr int VF = D / 16;          // channels of V per lane, 16-channel tiles of O^T
    constexpr int VW = VF / 4;          // dwords of V per token and lane
    constexpr int LDO = D + 4;
    __shared__ float obuf[WAVES][16][LDO];
    __shared__ float mbuf[WAVES][ROWS], lbuf[WAVES][ROWS];

    int unit, part;
    if (!item_of<LISTS>(a, unit, part)) return;
    const Rows r = rows_of<ROWS, LISTS>(a, unit);
    if (r.count <= 0) return;           // a tile past a short query block

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int len = clamp_len(a, r.b);
    const size_t hk = (size_t)r.b * a.H + r.kv;
    const uint8_t* kp = a.k + hk * a.cap * D;
    const uint8_t* vp = a.v + hk * a.cap * D;
    const float* ksp = a.ks + hk * a.ncap;
    const float* vsp = a.vs + hk * a.ncap;
    const int ps = a.shift - 5;         // steps per block: 1 << ps
    const int32_t* list = nullptr;
    int steps = (len + kStep - 1) / kStep;
    if (LISTS) {
        const long lrow = ((long)r.b * a.Hq + r.head) * a.nq + r.i;
        list = a.idx + lrow * a.n;
        steps = min(max(a.cnt[lrow], 0), a.n) << ps;
    }
    const int s0 = (int)((long)steps * part / a.C), s1 = (int)((long)steps * (part + 1) / a.C);

    // A step's codes and scales; t0: its first token, -1 where there is none.
    struct Step {
        uint4 k[2][KC];
        uint32_t v[8][VW];
        float ks, vs;
        int t0;
    };
    auto entry_of = [&](int s) __attribute__((always_inline)) { return LISTS && s < s1 ? list[s >> ps] : 0; };
    auto load = [&](Step& x, int s, int j) __attribute__((always_inline)) {
        int t0 = s * kStep;
        if (LISTS) {
            j = __builtin_amdgcn_readfirstlane(j);
            t0 = j * a.block + (s & ((1 << ps) - 1)) * kStep;
            if (j < 0 || j >= a.n || t0 >= len) t0 = -1;
        }
        if (s >= s1) t0 = -1;
        x.t0 = t0;
        if (t0 < 0) return;
        const int last = len - 1 - t0;   // tokens past the end: masked
        const uint8_t* kb = kp + (size_t)t0 * D;
        const uint8_t* vb = vp + (size_t)t0 * D;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < KC; ++c)
                x.k[t][c] = *reinterpret_cast<const uint4*>(kb + (uint32_t)(min(16 * t + l16, last) * D + 64 * c + 16 * g));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint8_t* p = vb + (uint32_t)(min(16 * (e / 4) + 4 * g + e % 4, last) * D + VF * l16);
            if constexpr (VW == 2) {
                const uint2 y = *reinterpret_cast<const uint2*>(p);
                x.v[e][0] = y.x;
                x.v[e][1] = y.y;
            } else {
                x.v[e][0] = *reinterpret_cast<const uint32_t*>(p);
            }
        }
        x.ks = ksp[t0 >> a.shift];
        x.vs = vsp[t0 >> a.shift];
    };
    // two steps are under way: the codes of the next arrive while one is computed
    Step even, odd;
    load(even, s0 + wave, entry_of(s0 + wave));

    // Q as the second operand: row l16 of tile rt, the channels that a lane of
    // group g loads of K
    bf16x8 qf[RT][2 * KC];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = 16 * rt + l16;
#pragma unroll
        for (int c = 0; c < 2 * KC; ++c) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (row < r.count)
                x = *reinterpret_cast<const uint4*>(a.q + (r.row0 + row) * D + 64 * (c / 2) + 16 * g + 8 * (c % 2));
            qf[rt][c] = __builtin_bit_cast(bf16x8, x);
        }
    }
    f32x4 acc[RT][VF];
    float m[RT], l[RT];
    uint32_t least = ~0u;               // bits of the smallest value scale but zero, less one

    // SMALL: value scales of any size (see small_scale)
    auto compute = [&](const Step& y, auto small_tag) __attribute__((always_inline)) {
        constexpr bool SMALL = decltype(small_tag)::value;
        const int t0 = __builtin_amdgcn_readfirstlane(y.t0);
        if (t0 < 0) return;
        const float sc = y.ks * a.c2;
        const bool up = SMALL && small_scale(y.vs);
        const float vs = up ? y.vs * 0x1p64f : y.vs, down = up ? 0x1p-64f : 1.0f;
        if constexpr (!SMALL) least = min(least, (uint32_t)__builtin_amdgcn_readfirstlane(__float_as_uint(y.vs)) - 1);
        f32x4 st[RT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 2 * KC; ++c) {
                const uint4 x = y.k[t][c / 2];
                const bf16x8 kf = c % 2 == 0 ? operand8<FMT>(x.x, x.y) : operand8<FMT>(x.z, x.w);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    st[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        kf, qf[rt][c], c == 0 ? f32x4{0, 0, 0, 0} : st[rt][t], 0, 0, 0);
            }
        bf16x8 pf[RT], pl[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float x[8], mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = st[rt][e / 4][e % 4] * sc;
            if (t0 + kStep > len) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (t0 + 16 * (e / 4) + 4 * g + e % 4 >= len) x[e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[e]);
            const float mn = fmaxf(m[rt], max4(mx));
            if (__any(mn > m[rt])) {
                const float alpha = mn > m[rt] ? __builtin_amdgcn_exp2f(m[rt] - mn) : 1.0f;
                m[rt] = mn;
                l[rt] *= alpha;
#pragma unroll
                for (int f = 0; f < VF; ++f) acc[rt][f] *= alpha;
            }
            const float mb = mn == -INFINITY ? 0.0f : mn;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p = __builtin_amdgcn_exp2f(x[e] - mb);
                l[rt] += p;
                pf[rt][e] = static_cast<__bf16>(p * vs);
                if constexpr (TWICE) pl[rt][e] = static_cast<__bf16>(p * vs - static_cast<float>(pf[rt][e]));
            }
        }
        static_for<VF>([&](auto f_tag) __attribute__((always_inline)) {
            constexpr int F = decltype(f_tag)::value, W = F / 4, BY = F % 4;
            const u32x4 x = {column_pair<FMT, BY>(y.v[0][W], y.v[1][W]), column_pair<FMT, BY>(y.v[2][W], y.v[3][W]),
                             column_pair<FMT, BY>(y.v[4][W], y.v[5][W]), column_pair<FMT, BY>(y.v[6][W], y.v[7][W])};
            const bf16x8 vf = __builtin_bit_cast(bf16x8, x);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                f32x4 sum = SMALL ? f32x4{0, 0, 0, 0} : acc[rt][F];
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt], sum, 0, 0, 0);
                if constexpr (TWICE) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[rt], sum, 0, 0, 0);
                acc[rt][F] = SMALL ? acc[rt][F] + sum * down : sum;
            }
        });
    };
    // the wave's steps, the first one's codes under way
    auto walk = [&](auto small_tag) __attribute__((always_inline)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = 0.0f;
#pragma unroll
            for (int f = 0; f < VF; ++f) acc[rt][f] = f32x4{0, 0, 0, 0};
        }
        int s = s0 + wave, jn = entry_of(s + WAVES);
        while (s < s1) {
            load(odd, s + WAVES, jn);
            jn = entry_of(s + 2 * WAVES);
            compute(even, small_tag);
            s += 2 * WAVES;
            load(even, s, jn);
            jn = entry_of(s + WAVES);
            compute(odd, small_tag);
        }
    };
    walk(std::false_type{});
    if (least < kSmallScale - 1) {      // rare: once more
        load(even, s0 + wave, entry_of(s0 + wave));
        walk(std::true_type{});
    }

    // join the waves
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] = sum4(l[rt]);
        if (g == 0) {
            mbuf[wave][16 * rt + l16] = m[rt];
            lbuf[wave][16 * rt + l16] = l[rt];
        }
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = mbuf[0][16 * rt + l16];
#pragma unroll
        for (int wv = 1; wv < WAVES; ++wv) top = fmaxf(top, mbuf[wv][16 * rt + l16]);
        const float mine = m[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[rt] - top);
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
            for (int f = 0; f < VF; f += 4)
                *reinterpret_cast<float4*>(&obuf[wave][l16][4 * VF * g + VF * rr + f]) =
                    make_float4(acc[rt][f][rr] * mine, acc[rt][f + 1][rr] * mine, acc[rt][f + 2][rr] * mine,
                                acc[rt][f + 3][rr] * mine);
        __syncthreads();
        constexpr int W = D / (4 * WAVES);   // channels per thread
        const int orow = tid / (4 * WAVES), ch = tid % (4 * WAVES) * W, tr = 16 * rt + orow;
        float tt = mbuf[0][tr];
#pragma unroll
        for (int wv = 1; wv < WAVES; ++wv) tt = fmaxf(tt, mbuf[wv][tr]);
        float sum = 0.0f, out[W];
#pragma unroll
        for (int e = 0; e < W; ++e) out[e] = 0.0f;
#pragma unroll
        for (int wv = 0; wv < WAVES; ++wv) {
            if (lbuf[wv][tr] != 0.0f)   // 0: that wave kept no token (its maximum may be -inf)
                sum += lbuf[wv][tr] * __builtin_amdgcn_exp2f(mbuf[wv][tr] - tt);
#pragma unroll
            for (int e = 0; e < W; ++e) out[e] += obuf[wv][orow][ch + e];
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const float lse2 = sum == 0.0f ? -INFINITY : tt + __builtin_amdgcn_logf(sum);   // log2
        if (tr >= r.count) {
        } else if (a.C > 1) {
            const long slot = ((long)unit * a.C + part) * ROWS + tr;
            float* po = a.part + slot * D + ch;
#pragma unroll
            for (int e = 0; e < W; ++e) po[e] = out[e] * inv;
            if (tid % (4 * WAVES) == 0) (a.part + (long)a.units * a.C * ROWS * D)[slot] = lse2;
        } else {
            uint32_t* po = reinterpret_cast<uint32_t*>(a.o + (r.row0 + tr) * D + ch);
#pragma unroll
            for (int e = 0; e < W; e += 2) po[e / 2] = pack_bf16(out[e] * inv, out[e + 1] * inv);
            if (a.lse && tid % (4 * WAVES) == 0) a.lse[r.row0 + tr] = lse2 * kLn2;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// tile_kernel: tiles of 64, 128 or 256 query rows of a head, for calls with more.
// The work-group brings the walk's tokens into LDS as bf16, 64 at a time (a
// "unit"), so a code is converted once for all rows of the tile; a wave owns 32
// rows (64-row tiles: two waves do, each half of the tokens).  It works on
// halves of a unit (32 tokens) as a pipeline of three:
//   scores    S^T (32 tokens x 32 rows) = K Q^T of one half,
//   softmax   of the half before it (P stays in the lanes that the product
//             wants it in),
//   product   O^T += V^T P^T of the half before that,
// with v_mfma_f32_32x32x16_bf16; V^T comes from the row-major tile through
// transposing LDS reads.  A wave issues an instruction every five cycles or so
// and a matrix instruction takes 32, so the matrix instructions of a half
// ("slots") are spaced out by its vector instructions: the softmax, and the
// conversion of the codes of the next unit, which were loaded one unit earlier.
// K and V tiles are double-buffered, V one unit behind K: one barrier a unit.
// With 256 rows one work-group fills a compute unit, with fewer two share it
// (three at d = 64).
//
// 10,800 queries over 24 heads of 118,800 tokens (15.8 TFLOP): int8 15.5 ms,
// 1.02 PFLOP/s (e4m3 14.6, 1.08), where a bf16 matrix product of 16384 reaches
// 1.38.  The matrix cores are busy in half of the cycles at 2.0 GHz, beside 7.7
// vector instructions to a matrix instruction: every tile converts the codes it
// reads again, through registers and LDS writes.  (This library's attention over
// bf16, which copies tiles into LDS as they are, has 4.1, 0.73 and 1.53 GHz.)
// Changes that leave the conversions cost what they saved at a lower clock:
// three buffers with the barrier off the critical path saved 6% of the cycles and
// no time, reads further ahead, priorities, other orders of a half and a layout
// without the staging writes' bank conflicts (a sixth of the LDS cycles)
// nothing.  Phases of scores
// and softmax behind barriers took 17.1 ms, rows_kernel alone 28.6; unrolling
// the loop by buffer spilled and took 35.
// 8-bit products of the codes of K with q as two E4M3 parts (exact down to 2^-21
// of a row's largest) would save K's conversions: 5 to 9% of E4M3 calls over
// lists.  But v_mfma_*_f8f6f4 sums 64 products with errors up to 2^-15 of their
// magnitudes (measured; the bf16 instruction's 2^-24), and scores are sums that
// are to hold 32 bits.
// ---------------------------------------------------------------------------
constexpr int kUnit = 64;

// What the softmax needs to know of a unit.
struct Unit {
    float sc;       // scale * s_k, in units of log 2
    float lv, ivs;  // log2 s and 1 / s of the value scale's part s that stands in the exponent
    int valid;      // tokens of the unit that exist
};

// The part of a value scale that goes into the values: 1, or a power of two
// that leaves between 2^-64 and 2^64 for the exponent (so the values stay exact
// and the probabilities normal), or 0 and NaN themselves.  For scales outside that
// range:
__device__ __forceinline__ float value_part(float s) {
    return small_scale(s) ? 0x1p-64f : s > 0x1p64f && s < INFINITY ? 0x1p64f : s;
}

template <int D, int FMT, bool LISTS, int ROWS>
__global__ __launch_bounds__(64 * kTileWaves<ROWS>, 2) void tile_kernel(AttnArgs a) {
    constexpr int WAVES = kTileWaves<ROWS>;
    constexpr bool SPLIT = ROWS == 64;           // two waves to 32 rows, each its half of every unit
    constexpr int DT = D / 32, KK = D / 16;
    constexpr int SLOTS = KK + 2 * DT;           // matrix instructions of a half
    // LDS rows of K are 16 bytes longer than their 2 D bytes, so that the 16 rows
    // that an operand read takes at once lie in different banks; those of V 64
    // bytes, for the 4 rows of 64 bytes of a transposing read.  (A swizzle
    // instead would need an address register per operand of a half.)
    constexpr int KROW = 2 * D + 16, VROW = 2 * D + 64;
    constexpr int KTILE = kUnit * KROW, VTILE = kUnit * VROW;
    constexpr int CPT = D / WAVES;               // codes of a tile that a thread brings:
    constexpr int PIECE = 16, PW = PIECE / 4;    // in pieces of one load,
    constexpr int NP = CPT / PIECE;              // each of a token TPP after the other's
    constexpr int TPR = D / PIECE, TPP = 64 * WAVES / TPR;
    __shared__ __align__(1024) char lds[2 * KTILE + 2 * VTILE];   // K, K, V, V

    int unit, part;
    if (!item_of<LISTS>(a, unit, part)) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int qw = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    const int th = SPLIT ? qw >> 1 : 0;          // the wave's half of the units
    const Rows r = rows_of<ROWS, LISTS>(a, unit);
    if (r.count <= 0) return;                    // a tile past a short query block

    const int len = clamp_len(a, r.b);
    const size_t hk = (size_t)r.b * a.H + r.kv;
    const uint8_t* kcodes = a.k + hk * a.cap * D;
    const uint8_t* vcodes = a.v + hk * a.cap * D;
    const float* ksp = a.ks + hk * a.ncap;
    const float* vsp = a.vs + hk * a.ncap;
    const int us = a.shift - 6;                  // units per block: 1 << us
    const int32_t* list = nullptr;
    int steps = (len + kUnit - 1) / kUnit;
    if (LISTS) {
        const long lrow = ((long)r.b * a.Hq + r.head) * a.nq + r.i;
        list = a.idx + lrow * a.n;
        steps = len > 0 ? min(max(a.cnt[lrow], 0), a.n) << us : 0;
    }
    const int u0 = (int)((long)steps * part / a.C);
    const int T = __builtin_amdgcn_readfirstlane((int)((long)steps * (part + 1) / a.C) - u0);   // units of this item

    const int row = 32 * (SPLIT ? qw & 1 : qw) + l32;   // the lane's row of the tile
    bf16x8 qreg[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (row < r.count) x = *reinterpret_cast<const uint4*>(a.q + (r.row0 + row) * D + 16 * kk + 8 * h);
        qreg[kk] = __builtin_bit_cast(bf16x8, x);
    }
    f32x16 oacc[DT], sacc[2];
    u32x4 pf[2][2];                              // P of either half, pairs of bf16
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x16{};
    float m = -INFINITY, l = 0.0f;

    // LDS addresses of the operands in the first buffers
    const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)lds;
    const int s16 = lane & 15;
    const uint32_t kad = lds0 + (uint32_t)((32 * th + l32) * KROW + 16 * h);
    const uint32_t vad = lds0 + (uint32_t)(2 * KTILE + (32 * th + 4 * h + (s16 >> 2)) * VROW + 32 * (lane >> 4 & 1) + 8 * (s16 & 3));

    // staging: thread tid brings 16 codes of a token, two 16-byte chunks of its
    // LDS row
    const int scol = tid % TPR, srow = tid / TPR;
    char* const kst = lds + srow * KROW + 2 * PIECE * scol;
    char* const vst = lds + 2 * KTILE + srow * VROW + 2 * PIECE * scol;
    uint32_t kr[NP][PW], vr[NP][PW];
    auto entry_of = [&](int u) __attribute__((always_inline)) { return LISTS ? list[(u0 + u) >> us] : 0; };
    // first token of unit u, whose list entry is j; -1: nothing to read
    auto token_of = [&](int u, int j) __attribute__((always_inline)) {
        u += u0;
        if (!LISTS) return u * kUnit;
        j = __builtin_amdgcn_readfirstlane(j);
        const int t = j * a.block + (u & ((1 << us) - 1)) * kUnit;
        return (j < 0 || j >= a.n || t >= len) ? -1 : t;
    };
    auto load = [&](const uint8_t* p, int t0, uint32_t (&x)[NP][PW]) __attribute__((always_inline)) {
        if (t0 < 0) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int q = 0; q < PW; ++q) x[i][q] = 0;
            return;
        }
        const uint8_t* base = p + (size_t)t0 * D;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int t = min(srow + TPP * i, len - 1 - t0);       // rows past the end: masked
            const uint32_t off = (uint32_t)(t * D + PIECE * scol);
            const uint4 v = *reinterpret_cast<const uint4*>(base + off);
            x[i][0] = v.x, x[i][1] = v.y, x[i][2] = v.z, x[i][3] = v.w;
        }
    };
    auto fetch_scales = [&](int t0, float& ks, float& vs) __attribute__((always_inline)) {
        ks = vs = 1.0f;
        if (t0 >= 0) {
            ks = ksp[t0 >> a.shift];
            vs = vsp[t0 >> a.shift];
        }
    };
    // pair q of the thread's codes; after a chunk's last pair the chunk goes to LDS
    // (`to`: the thread's place in the buffer, whose rows are ROW bytes apart)
    using No = std::false_type;
    using Yes = std::true_type;
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using KR = std::integral_constant<int, KROW>;
    using VR = std::integral_constant<int, VROW>;
    uint32_t kconv[4], vconv[4];
    auto convert = [&](auto q_tag, auto row_tag, uint32_t (&x)[NP][PW], char* to, uint32_t (&conv)[4])
                       __attribute__((always_inline)) {
        constexpr int Q = decltype(q_tag)::value, I = Q / (2 * PW), W = Q / 2 % PW, ROW = decltype(row_tag)::value;
        asm volatile("" : "+v"(x[I][W]));        // (keeps the conversion in its slot)
        conv[Q % 4] = bf16_pair<FMT, Q % 2 == 1>(x[I][W]);
        asm volatile("" : "+v"(conv[Q % 4]));
        if constexpr (Q % 4 == 3)
            *reinterpret_cast<uint4*>(to + TPP * I * ROW + 16 * (Q / 4 % (PW / 2))) =
                make_uint4(conv[0], conv[1], conv[2], conv[3]);
    };
    constexpr int PAIRS = CPT / 2;               // pairs of codes per thread and tile
    // V times the part of its scale that goes into the values
    auto stage_scaled = [&](char* to, float s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int c = 0; c < PW / 2; ++c) {
                uint32_t out[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t wd = vr[i][2 * c + q / 2];
                    const uint32_t pr = q % 2 ? bf16_pair<FMT, true>(wd) : bf16_pair<FMT, false>(wd);
                    out[q] = pack_bf16(__uint_as_float(pr << 16) * s, __uint_as_float(pr & 0xffff0000u) * s);
                }
                *reinterpret_cast<uint4*>(to + TPP * i * VROW + 16 * c) = make_uint4(out[0], out[1], out[2], out[3]);
            }
    };
    auto barrier = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    // Operands that were read ahead for the next half.
    constexpr int AHEAD = 2;                     // operand reads ahead, of either kind
    bf16x8 nk[AHEAD];
    s16x4 nv0[AHEAD], nv1[AHEAD];
    auto read_k = [&](uint32_t ka, auto i) __attribute__((always_inline)) {
        return __builtin_bit_cast(bf16x8, *(lds_u4_t*)(uintptr_t)(ka + (uint32_t)(32 * decltype(i)::value)));
    };
    auto read_v = [&](uint32_t va, auto i, s16x4& x0, s16x4& x1) __attribute__((always_inline)) {
        constexpr uint32_t at = 16 * (decltype(i)::value / DT) * VROW + 64 * (decltype(i)::value % DT);
        x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)(va + at));
        x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)(va + at + 8 * VROW));
    };
    auto read_ahead = [&](uint32_t ka, uint32_t va) __attribute__((always_inline)) {
        static_for<AHEAD>([&](auto i) __attribute__((always_inline)) {
            nk[decltype(i)::value] = read_k(ka, i);
            read_v(va, i, nv0[decltype(i)::value], nv1[decltype(i)::value]);
        });
    };

    // One half: scores of the half SUB at ka (QK), softmax of the half before it,
    // half 1 - SUB of unit `u` (SM), product of the one before that, at va (PV),
    // and the conversion of K and V codes to kto and vto (KC, VC).  NEXT: reads
    // the next half's first operands, at kn and vn, ahead.
    auto half = [&](auto sub_tag, uint32_t ka, uint32_t va, auto qk_tag, auto sm_tag, auto pv_tag, auto kc_tag,
                    auto vc_tag, auto next_tag, Unit u, char* kto, char* vto, uint32_t kn, uint32_t vn)
                    __attribute__((always_inline)) {
        constexpr int SUB = decltype(sub_tag)::value;
        constexpr bool QK = decltype(qk_tag)::value, SM = decltype(sm_tag)::value, PV = decltype(pv_tag)::value;
        constexpr bool KC = decltype(kc_tag)::value, VC = decltype(vc_tag)::value, NEXT = decltype(next_tag)::value;
        constexpr int PS = 1 - SUB;              // the half whose softmax this is
        constexpr int EPS = 16 / SLOTS;          // scores of a lane per slot
        float sc = u.sc;
        if constexpr (SM) {
            const int lim = u.valid - 32 * (SPLIT ? th : PS);
            if (lim < 32) {
                const int mine = lim - 4 * h;
#pragma unroll
                for (int ii = 0; ii < 16; ++ii)
                    sacc[PS][ii] = 8 * (ii >> 2) + (ii & 3) >= mine ? -INFINITY : sacc[PS][ii] * sc;
                sc = 1.0f;
            }
        }
        float ps0 = 0.0f, ps1 = 0.0f, off = u.lv - (m == -INFINITY ? 0.0f : m);
        bf16x8 ak[KK];
        s16x4 v0[2 * DT], v1[2 * DT];
        float pr[16];
        uint32_t pb[8];
        // sums and pairs of scores [e0, e1), whose exponentials the slot before took
        auto gather = [&](auto e0, auto e1) __attribute__((always_inline)) {
#pragma unroll
            for (int e = decltype(e0)::value; e < decltype(e1)::value; ++e) {
                (e % 2 ? ps1 : ps0) += pr[e];
                if (e % 2 == 1) {
                    pb[e / 2] = pack_bf16(pr[e - 1], pr[e]);
                    asm volatile("" : "+v"(pb[e / 2]));
                }
            }
        };
        static_for<AHEAD>([&](auto i) __attribute__((always_inline)) {
            constexpr int I = decltype(i)::value;
            ak[I] = nk[I];
            v0[I] = nv0[I];
            v1[I] = nv1[I];
        });
        static_for<SLOTS>([&](auto s_tag) __attribute__((always_inline)) {
            constexpr int S = decltype(s_tag)::value, I = S / 2, J = I + AHEAD;
            if constexpr (S % 2 == 0) {
                if constexpr (QK)
                    sacc[SUB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ak[I], qreg[I], I == 0 ? f32x16{} : sacc[SUB], 0,
                                                                        0, 0);
                if constexpr (J < KK && QK) ak[J] = read_k(ka, std::integral_constant<int, J>{});
                if constexpr (J >= KK && NEXT) nk[J - KK] = read_k(kn, std::integral_constant<int, J - KK>{});
            } else {
                if constexpr (PV) {
                    const s16x8 v8 = {v0[I][0], v0[I][1], v0[I][2], v0[I][3], v1[I][0], v1[I][1], v1[I][2], v1[I][3]};
                    oacc[I % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v8),
                                                                           __builtin_bit_cast(bf16x8, pf[SUB][I / DT]),
                                                                           oacc[I % DT], 0, 0, 0);
                }
                if constexpr (J < 2 * DT && PV) read_v(va, std::integral_constant<int, J>{}, v0[J], v1[J]);
                if constexpr (J >= 2 * DT && NEXT)
                    read_v(vn, std::integral_constant<int, J - 2 * DT>{}, nv0[J - 2 * DT], nv1[J - 2 * DT]);
            }
            if constexpr (SM) {
                // the slot's scores, and the sums of the slot before (the empty
                // statements keep them in their slot)
                asm volatile("" : "+v"(off));
                float arg[EPS];
#pragma unroll
                for (int e = 0; e < EPS; ++e) arg[e] = __builtin_fmaf(sacc[PS][S * EPS + e], sc, off);
#pragma unroll
                for (int e = 0; e < EPS; ++e) pr[S * EPS + e] = __builtin_amdgcn_exp2f(arg[e]);
                if constexpr (S > 0)
                    gather(std::integral_constant<int, (S - 1) * EPS>{}, std::integral_constant<int, S * EPS>{});
#pragma unroll
                for (int e = S * EPS; e < (S + 1) * EPS; ++e) asm volatile("" : "+v"(pr[e]));
                asm volatile("" : "+v"(ps0), "+v"(ps1));
            }
            constexpr int Q0 = S * PAIRS / SLOTS, Q1 = (S + 1) * PAIRS / SLOTS;
            static_for<Q1 - Q0>([&](auto q) __attribute__((always_inline)) {
                using Q = std::integral_constant<int, Q0 + decltype(q)::value>;
                if constexpr (KC) convert(Q{}, KR{}, kr, kto, kconv);
                if constexpr (VC) convert(Q{}, VR{}, vr, vto, vconv);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (SM) {
            gather(std::integral_constant<int, 16 - EPS>{}, std::integral_constant<int, 16>{});
            // The running maximum is kept while no lane's probabilities sum past
            // kSumLimit; the first half and the rare others take the half's
            // maximum and rescale.  The other rows of the wave keep theirs: a row
            // does not depend on its neighbours.
            int move = !(m > -INFINITY) || !((ps0 + ps1) * u.ivs <= kSumLimit);
            if (__any(move)) {
                float mx = -INFINITY;
#pragma unroll
                for (int ii = 0; ii < 16; ++ii) mx = fmaxf(mx, sacc[PS][ii] * sc);
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                move |= __shfl_xor(move, 32);
                const float mn = move ? fmaxf(m, mx) : m;
                const float alpha = mn == m ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
                l *= alpha;
                m = mn;
                off = u.lv - (m == -INFINITY ? 0.0f : m);
                ps0 = ps1 = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    pr[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[PS][e], sc, off));
                    if (e % 2 == 1) pb[e / 2] = pack_bf16(pr[e - 1], pr[e]);
                    (e % 2 ? ps1 : ps0) += pr[e];
                }
            }
            l += (ps0 + ps1) * u.ivs;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                pf[PS][c] = u32x4{pb[4 * c], pb[4 * c + 1], pb[4 * c + 2], pb[4 * c + 3]};
                asm volatile("" : "+v"(pf[PS][c]));
            }
        }
    };
    // a unit's scales; of the value scale `vs` only what goes into the values is left
    auto unit_of = [&](int t0, float ks, float& vs) __attribute__((always_inline)) {
        float in_p = uniform(vs);
        vs = 1.0f;
        if (!(in_p >= 0x1p-64f && in_p <= 0x1p64f)) {
            vs = uniform(value_part(in_p));
            in_p = uniform(vs == 0x1p-64f ? in_p * 0x1p64f : vs == 0x1p64f ? in_p * 0x1p-64f : 1.0f);
        }
        return Unit{uniform(ks * a.c2), uniform(__builtin_amdgcn_logf(in_p)), uniform(__builtin_amdgcn_rcpf(in_p)),
                    t0 < 0 ? 0 : len - t0};
    };
    // first tokens of this unit and the next, list entry of the one after
    int tc = -1, tn = -1, jn = 0;
    float ks = 1.0f, vs = 1.0f, vnow = 1.0f;
    Unit before{}, now{};
    // One unit, its K at kc and the V of the unit before at vp: its scores, the
    // rest of the unit before, and half of its softmax.
    int kc = 0, vp = VTILE;
    auto iterate = [&](int t, auto first_tag) __attribute__((always_inline)) {
        using Rest = std::bool_constant<!decltype(first_tag)::value>;
        const int kn = KTILE - kc, vc = VTILE - vp;
        const uint32_t ka = kad + kc, va = vad + vp;
        char* const vto = vst + vc;
        float ksn, vsn;
        fetch_scales(tn, ksn, vsn);
        half(I0{}, ka, va, Yes{}, Rest{}, Rest{}, Yes{}, No{}, Yes{}, before, kst + kn, vto, ka + 32 * KROW,
             va + 32 * VROW);
        int tnn = -1;
        if (t + 2 < T) {
            tnn = token_of(t + 2, jn);
            load(kcodes, tnn, kr);
            if (t + 3 < T) jn = entry_of(t + 3);
        }
        half(I1{}, ka + 32 * KROW, va + 32 * VROW, Yes{}, Yes{}, Rest{}, No{}, Yes{}, No{}, now, kst, vto, 0, 0);
        if (vs != 1.0f) stage_scaled(vto, vs);
        if (t + 1 < T) load(vcodes, tn, vr);
        barrier();
        read_ahead(kad + kn, vad + vc);
        before = now;
        now = unit_of(tn, ksn, vsn);
        vs = vsn;
        tn = tnn;
        kc = kn;
        vp = vc;
    };
    if constexpr (SPLIT) {
        // Here the pipeline runs over units: step j takes the scores of unit j, the
        // softmax of j - 1 and the product of j - 2 (units before the first and
        // past the last count as masked), from and into buffers j % 2, and
        // converts K of j + 1 and V of j - 1 into the others.
        auto step = [&](int j, auto sub_tag) __attribute__((always_inline)) {
            constexpr int SUB = decltype(sub_tag)::value, OTHER = 1 - SUB;
            char* const vto = vst + OTHER * VTILE;
            float ksn, vsn;
            fetch_scales(tn, ksn, vsn);
            half(sub_tag, kad + SUB * KTILE, vad + SUB * VTILE, Yes{}, Yes{}, Yes{}, Yes{}, Yes{}, No{}, before,
                 kst + OTHER * KTILE, vto, 0, 0);
            if (vs != 1.0f) stage_scaled(vto, vs);
            load(vcodes, tc, vr);
            int tnn = -1;
            if (j + 2 < T) {
                tnn = token_of(j + 2, jn);
                load(kcodes, tnn, kr);
                if (j + 3 < T) jn = entry_of(j + 3);
            }
            barrier();
            read_ahead(kad + OTHER * KTILE, vad + OTHER * VTILE);
            before = now;
            vs = vnow;
            now = unit_of(tn, ksn, vsn);
            vnow = vsn;
            tc = tn;
            tn = tnn;
        };
        if (T > 0) {
            for (int i = tid; i < 2 * VTILE / 16; i += 64 * WAVES)     // (P of no unit is 0, and so has V to be)
                *reinterpret_cast<uint4*>(lds + 2 * KTILE + 16 * i) = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < 2; ++c) pf[0][c] = pf[1][c] = u32x4{0, 0, 0, 0};
            sacc[1] = f32x16{};
            tc = token_of(0, entry_of(0));
            load(kcodes, tc, kr);
            fetch_scales(tc, ks, vnow);
            now = unit_of(tc, ks, vnow);
            before = Unit{0.0f, 0.0f, 1.0f, 0};
            static_for<PAIRS>([&](auto q) __attribute__((always_inline)) { convert(q, KR{}, kr, kst, kconv); });
            if (T > 1) {
                tn = token_of(1, entry_of(1));
                load(kcodes, tn, kr);
            }
            load(vcodes, -1, vr);
            if (T > 2) jn = entry_of(2);
            barrier();
            read_ahead(kad, vad);
            for (int j = 0; j < T + 2; j += 2) {
                step(j, I0{});
                step(j + 1, I1{});
            }
        }
        // join the two waves of a row: the second half's through LDS
        l += __shfl_xor(l, 32);
        float* const other = reinterpret_cast<float*>(lds) + (qw & 1) * (16 * DT + 2) * 64 + lane;
        __syncthreads();
        if (th == 1) {
            other[0] = m;
            other[64] = l;
#pragma unroll
            for (int i = 0; i < 16 * DT; ++i) other[(2 + i) * 64] = oacc[i / 16][i % 16];
        }
        __syncthreads();
        if (th == 1) return;
        const float m1 = other[0], l1 = other[64], top = fmaxf(m, m1);
        const float w0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        const float w1 = m1 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m1 - top);
        // a half without a token adds nothing; NaN of either passes on
        l = (l == 0.0f ? 0.0f : l * w0) + (l1 == 0.0f ? 0.0f : l1 * w1);
        m = top;
#pragma unroll
        for (int i = 0; i < 16 * DT; ++i)
            oacc[i / 16][i % 16] = oacc[i / 16][i % 16] * w0 + other[(2 + i) * 64] * w1;
    } else if (T > 0) {
        tc = token_of(0, entry_of(0));
        load(kcodes, tc, kr);
        fetch_scales(tc, ks, vs);
        now = unit_of(tc, ks, vs);
        static_for<PAIRS>([&](auto q) __attribute__((always_inline)) { convert(q, KR{}, kr, kst, kconv); });
        if (T > 1) {
            tn = token_of(1, entry_of(1));
            load(kcodes, tn, kr);
        }
        load(vcodes, tc, vr);
        if (T > 2) jn = entry_of(2);
        barrier();
        read_ahead(kad, vad);                    // (the V of no unit: not used)
        iterate(0, Yes{});
        for (int t = 1; t < T; ++t) iterate(t, No{});
        const uint32_t va = vad + vp;
        half(I0{}, kad, va, No{}, Yes{}, Yes{}, No{}, No{}, Yes{}, before, kst, vst, kad, va + 32 * VROW);
        half(I1{}, kad, va + 32 * VROW, No{}, No{}, Yes{}, No{}, No{}, No{}, before, kst, vst, kad, vad);
    }

    // the lane's channels: 32 dt + 8 gq + 4 h + 0..3 of its row
    if constexpr (!SPLIT) l += __shfl_xor(l, 32);
    if (row >= r.count) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const float lse2 = l == 0.0f ? -INFINITY : m + __builtin_amdgcn_logf(l);
    if (a.C > 1) {
        const long slot = ((long)unit * a.C + part) * ROWS + row;
        float* po = a.part + slot * D + 4 * h;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq)
                *reinterpret_cast<float4*>(po + 32 * dt + 8 * gq) =
                    make_float4(oacc[dt][4 * gq] * inv, oacc[dt][4 * gq + 1] * inv, oacc[dt][4 * gq + 2] * inv,
                                oacc[dt][4 * gq + 3] * inv);
        if (h == 0) (a.part + (long)a.units * a.C * ROWS * D)[slot] = lse2;
    } else {
        uint16_t* po = a.o + (r.row0 + row) * D + 4 * h;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq)
                *reinterpret_cast<uint2*>(po + 32 * dt + 8 * gq) =
                    make_uint2(pack_bf16(oacc[dt][4 * gq] * inv, oacc[dt][4 * gq + 1] * inv),
                               pack_bf16(oacc[dt][4 * gq + 2] * inv, oacc[dt][4 * gq + 3] * inv));
        if (a.lse && h == 0) a.lse[r.row0 + row] = lse2 * kLn2;
    }
}

// Joins the parts of every row in a fixed order.  D/4 lanes per row and slice of
// the parts; SLICES slices (8 where a row has many parts) take every eighth
// part each, and are joined through LDS.
template <int D, int ROWS, bool LISTS, int SLICES>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
    constexpr int LPR = D / 4, RPG = 256 / (LPR * SLICES);
    __shared__ float4 obuf[SLICES > 1 ? 256 : 1];
    __shared__ float mbuf[SLICES > 1 ? 256 : 1], lbuf[SLICES > 1 ? 256 : 1];
    const int tid = threadIdx.x, slice = tid / LPR % SLICES;
    const int row = (int)blockIdx.x * RPG + tid / (LPR * SLICES), unit = row / ROWS;
    const int tr = row % ROWS, ch = tid % LPR * 4;
    Rows r{};
    if (unit < a.units) r = rows_of<ROWS, LISTS>(a, unit);
    const bool live = unit < a.units && tr < r.count;
    const float* lse2 = a.part + (long)a.units * a.C * ROWS * D + (long)unit * a.C * ROWS + tr;
    const float* po = a.part + ((long)unit * a.C * ROWS + tr) * D + ch;
    float top = -INFINITY, sum = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    if (live) {
        // eight parts at once, their loads together (a part past the last: the last,
        // without weight)
        for (int c0 = slice; c0 < a.C; c0 += 8 * SLICES) {
            float x[8];
            f32x4 y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long c = min(c0 + i * SLICES, a.C - 1);
                x[i] = lse2[c * ROWS];
                y[i] = *reinterpret_cast<const f32x4*>(po + c * ROWS * D);
            }
            float mn = top;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (c0 + i * SLICES >= a.C) x[i] = -INFINITY;
                mn = fmaxf(mn, x[i]);
            }
            const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - mn);
            top = mn;
            sum *= keep;
            o *= keep;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = x[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x[i] - mn);   // no token: O is 0
                sum += w;
                o += y[i] * w;
            }
        }
    }
    if constexpr (SLICES > 1) {
        obuf[tid] = make_float4(o[0], o[1], o[2], o[3]);
        mbuf[tid] = top;
        lbuf[tid] = sum;
        __syncthreads();
        if (slice != 0) return;
        for (int t = 1; t < SLICES; ++t) {
            const int at = tid + t * LPR;
            const float x = mbuf[at], mn = fmaxf(top, x);
            const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - mn);
            const float w = x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x - mn);
            const float4 y = obuf[at];
            top = mn;
            sum = lbuf[at] != 0.0f ? sum * keep + lbuf[at] * w : sum;
            if (lbuf[at] != 0.0f) o = o * keep + f32x4{y.x, y.y, y.z, y.w} * w;
        }
    }
    if (!live) return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<uint2*>(a.o + (r.row0 + tr) * D + ch) =
        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    if (a.lse && tid % LPR == 0)
        a.lse[r.row0 + tr] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// What an estimate of a call's time needs to know of a tile's kernel, in
// microseconds: a turn of a work-group (a step of all its waves, a unit), what
// each work-group per compute unit adds to it, its start and end, and how much of
// a turn d = 64 takes.  A fit to 11,000 calls with 1 to 16,384 queries, 64 to
// 185,000 tokens, with and without lists, each with up to 60 ways to cut it up:
// the way chosen by it was 2% slower than the best one measured, on average,
// before workspace had a price.
struct TileCost {
    int rows;
    double turn, more, start, half;
};
constexpr TileCost kTileCosts[] = {{256, 1.5, 0.26, 8.5, 1.0},
                                   {128, 1.45, 0.4, 7.3, 0.76},
                                   {64, 1.25, 0.16, 11.0, 0.71},
                                   {32, 2.35, 0.0, 7.0, 0.5},
                                   {16, 2.0, 0.55, 4.0, 0.6}};

}  // namespace

CacheAttnPlan plan_cache_attn(int B, int H, int d, int block, int Hq, int Lq, int max_len, bool lists) {
    const int rows = lists ? std::min(block, Lq) : (int)std::min<long>((long)(Hq / H) * Lq, 1L << 30);
    CacheAttnPlan best{};
    double least = 0.0;
    // bytes of the call's codes, q and o (small calls: 256 MB, a thousandth of the memory)
    const double room = std::max(256e6, (2.0 * H * max_len + 4.0 * Hq * Lq) * B * d);
    // Work-groups run in rounds; the rows of a tile and the parts of a walk are
    // chosen so that the rounds end first by this estimate.  The lengths of lists
    // are not known here: they are taken to keep a quarter.  What the choice does:
    // one query over 24 heads of 118,800 tokens 801 us whole, 227 in 4 parts, 139
    // in 10 (240 work-groups, taken), 160 in 16; 8 heads of 8192 54 us whole, 10.0 in
    // 32 parts (taken).  1024 queries over 8 heads of 1024: 17.6 us in tiles of 32
    // (taken), 22.9 in tiles of 128 and three parts.  One frame of 3600 queries over
    // 24 heads' lists is 696 tiles of 128, two rounds, the second short: 1.64 ms
    // whole, 1.52 in two parts, 1.51 in five (taken).
    for (const TileCost& t : kTileCosts) {
        // a tile more than half empty is never better; d = 64: three work-groups of
        // 128 rows share a compute unit and one of 256 leaves a third of it empty
        // (10,800 queries, 24 x 118,800 tokens 9.2 ms, 10.0 with 256 rows; d = 128,
        // int8 16.2 with 256, 17.6 with 128)
        if ((t.rows > 16 && t.rows >= 2 * rows) || (t.rows == 256 && (lists || d == 64))) continue;
        CacheAttnPlan p{};
        p.rows = t.rows;
        p.tiles = (rows + t.rows - 1) / t.rows;
        p.heads = lists ? Hq : H;
        const long blocks = lists ? (Lq + block - 1) / block : 1, units = B * p.heads * blocks * p.tiles;
        p.stretch = (int)((blocks * p.tiles + kXcds - 1) / kXcds);
        const bool small = t.rows <= 32;
        // resident work-groups; turns of a whole walk
        const int slots = small || t.rows == 256 ? 256 : d == 64 ? 768 : 512;
        const double walk = std::max(1.0, (lists ? 0.25 : 1.0) * max_len / (small ? kStep * kRowWaves : kUnit));
        auto weigh = [&](int c) {
            const long items = units * c;
            // past 64 rounds parts save nothing; a launch's work-groups keep to their
            // limit, as those of the first tile, whole, do
            if (least != 0.0 && items > (c > 1 ? 1L << 14 : 1L << 18)) return;
            // of the die that gets the most
            const long share = (items + kXcds * p.stretch - 1) / (kXcds * p.stretch) * p.stretch;
            const double rounds = (double)((share + slots / kXcds - 1) / (slots / kXcds));
            const double us = (t.turn + t.more * (double)std::min<long>(items, slots) / 256) * (d == 64 ? t.half : 1.0);
            const double join = c == 1 ? 0.0 : 5.0 + 0.02 * c + 1.3e-6 * items * std::min(t.rows, rows) * d;
            // Parts have to save 1%, and 1% more for every quarter of the call's bytes
            // that they take as workspace past the first: each graph or stream keeps
            // one.  10,800 queries, 24 heads of 118,800 tokens (863 MB): four parts, 545
            // MB, 15.8 ms; six took 818 MB and 15.7 ms, whole tiles 18.2.
            const double held = (double)items * t.rows * (d + 1) * 4 / room;
            const double extra = c == 1 ? 0.0 : 0.01 + std::max(0.0, 0.04 * (held - 0.25));
            const double cost = (rounds * (walk / c * us + t.start) + join) * (1.0 + extra);
            if (least == 0.0 || cost < least) {
                least = cost;
                best = p;
                best.units = (int)units;
                best.C = c;
            }
        };
        // whole, a few parts, and the most that one, two ... rounds hold
        const int most = std::min((int)walk, 256);
        for (int c = 1; c <= std::min(most, 8); ++c) weigh(c);
        for (int r = 1, c = 8; r <= 8 && c < most; ++r)
            if (r * slots / units > 8) weigh(c = (int)std::min<long>(most, r * slots / units));
    }
    return best;
}

size_t cache_attn_plan_bytes(const CacheAttnPlan& p, int d) {
    return p.C == 1 ? 0 : (size_t)p.units * p.C * p.rows * (d + 1) * sizeof(float);
}

namespace {

template <int D, int FMT, int ROWS, bool LISTS>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
    const int round = kXcds * a.stretch;
    const dim3 grid((unsigned)((a.units * a.C + round - 1) / round * round));
    if constexpr (ROWS >= 64)
        hipLaunchKernelGGL((tile_kernel<D, FMT, LISTS, ROWS>), grid, dim3(64 * kTileWaves<ROWS>), 0, s, a);
    else
        hipLaunchKernelGGL((rows_kernel<D, FMT, ROWS / 16, LISTS>), grid, dim3(64 * kRowWaves), 0, s, a);
    if (a.C > 1) {
        auto join = [&](auto slices) {
            constexpr int SL = decltype(slices)::value, RPG = 256 / (D / 4 * SL);
            hipLaunchKernelGGL((join_kernel<D, ROWS, LISTS, SL>), dim3((unsigned)((a.units * ROWS + RPG - 1) / RPG)),
                               dim3(256), 0, s, a);
        };
        if (a.C > 8) join(std::integral_constant<int, 8>{});
        else join(std::integral_constant<int, 1>{});
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnPlan& p, const CacheView& c, const uint16_t* q, int Hq, int Lq,
                             int max_len, const int32_t* kv_len, const int32_t* kv_idx, const int32_t* kv_cnt,
                             float scale, uint16_t* o, float* lse, void* ws, hipStream_t s) {
    const bool lists = kv_idx != nullptr;
    AttnArgs a{q, c.k, c.v, c.ks, c.vs, kv_len, kv_idx, kv_cnt, o, lse, static_cast<float*>(ws),
               c.B, Hq, c.H, Lq, c.cap, c.n, max_len, (max_len + c.block - 1) / c.block,
               (Lq + c.block - 1) / c.block, c.block, c.block == 128 ? 7 : 6, Hq / c.H, p.tiles, p.heads, p.C,
               p.stretch, p.units, scale * kLog2e};
    hipError_t e = hipErrorInvalidValue;
    auto with_rt = [&](auto d, auto fmt, auto ls) {
        constexpr int D = decltype(d)::value, FMT = decltype(fmt)::value;
        constexpr bool LISTS = decltype(ls)::value;
        if (p.rows == 16) e = launch<D, FMT, 16, LISTS>(a, s);
        else if (p.rows == 32) e = launch<D, FMT, 32, LISTS>(a, s);
        else if (p.rows == 64) e = launch<D, FMT, 64, LISTS>(a, s);
        else if (p.rows == 128) e = launch<D, FMT, 128, LISTS>(a, s);
        else if constexpr (!LISTS && D == 128) e = launch<D, FMT, 256, LISTS>(a, s);
    };
    auto with_fmt = [&](auto d, auto fmt) {
        if (lists) with_rt(d, fmt, std::true_type{});
        else with_rt(d, fmt, std::false_type{});
    };
    auto with_d = [&](auto d) {
        if (c.format == MOD_CACHE_INT8) with_fmt(d, std::integral_constant<int, MOD_CACHE_INT8>{});
        else with_fmt(d, std::integral_constant<int, MOD_CACHE_E4M3>{});
    };
    if (c.d == 128) with_d(std::integral_constant<int, 128>{});
    else with_d(std::integral_constant<int, 64>{});
    return e;
}

}  // namespace moddit
