// Attention of new queries over the 8-bit cache, for gfx950.
//
//   S = (q k8^T) * scale * s_k,  O = softmax(S) (s_v v8)
// with one s_k and s_v per block of tokens and head.  Every code is exactly a
// bf16 number, so the products run on bf16 matrix instructions without any
// rounding of K, V or Q: s_k is a factor of the scores of a block, s_v one of
// its probabilities, which are rounded to bf16 once after it.  Scores, the
// running maximum and sum of the softmax (in units of log 2) and the output
// accumulate in fp32.
//
// rows_kernel: a work item is (sequence, head, tile of 16 RT query rows, part
// of the walk over the tokens); its four waves take steps of 32 tokens in turn,
// each with a softmax state of its own, and are joined at the end.  A wave
// keeps everything in registers:
//   S^T (tokens x rows) = K Q^T   v_mfma_f32_16x16x32_bf16: a lane loads 16
//       consecutive bytes of one token's K; which channels meet in a matrix
//       step is free as long as Q is laid out alike;
//   O^T (channels x rows) += V^T P^T: the 8 tokens that a lane's scores
//       belong to are those whose V it loads (D/16 consecutive channels
//       each), so P needs no exchange between lanes and V^T is formed by
//       byte permutes of the lane's own loads.
// No LDS and no barrier in the loop.  Without lists the query heads of a
// key/value head share the item (their rows are consecutive in memory).
#include "moddit_internal.h"

#include <algorithm>
#include <type_traits>

namespace moddit {
namespace {

typedef __bf16 bf16x8 __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kXcds = 8;
constexpr int kStep = 32;          // tokens of a wave's step

struct AttnArgs {
    const uint16_t* q;
    const uint8_t *k, *v;
    const float *ks, *vs;
    const int32_t *len, *idx, *cnt;
    uint16_t* o;
    float* lse;
    float* part;               // C > 1: O / l of every item, then its log2-sum-exp2
    int B, Hq, H, Lq, cap, ncap, max_len, n, nq, block;
    int tiles;                 // row tiles per head and query block (lists) or key/value head
    int heads;                 // heads that items count: Hq with lists, H without
    int C;                     // parts of a walk
    long units;                // B * heads * (lists: nq) * tiles
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

// max / sum over the four lanes that hold a query row's tokens (16 apart)
__device__ __forceinline__ float max4(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum4(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

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
__device__ __forceinline__ Rows rows_of(const AttnArgs& a, long u) {
    Rows r;
    const int t = (int)(u % a.tiles);
    u /= a.tiles;
    r.i = 0;
    if (LISTS) {
        r.i = (int)(u % a.nq);
        u /= a.nq;
    }
    r.head = (int)(u % a.heads);
    r.b = (int)(u / a.heads);
    const int group = a.Hq / a.H;
    r.kv = LISTS ? r.head / group : r.head;
    const int all = LISTS ? min(a.block, a.Lq - r.i * a.block) : group * a.Lq;
    r.row0 = (LISTS ? ((long)r.b * a.Hq + r.head) * a.Lq + (long)r.i * a.block
                    : ((long)r.b * a.Hq + (long)r.head * group) * a.Lq) + (long)t * ROWS;
    r.count = all - t * ROWS;
    return r;
}

template <int D, int FMT, int RT, bool LISTS>
__global__ __launch_bounds__(256, RT == 4 ? 1 : 2) void rows_kernel(AttnArgs a) {
    constexpr int ROWS = 16 * RT;
    constexpr int KC = D / 64;          // 16-byte chunks of a token's K per lane
    constexpr int VF = D / 16;          // channels of V per lane, 16-channel tiles of O^T
    constexpr int VW = VF / 4;          // dwords of V per token and lane
    constexpr int LDO = D + 4;
    __shared__ float obuf[4][16][LDO];
    __shared__ float mbuf[4][ROWS], lbuf[4][ROWS];

    const long total = a.units * a.C;
    // consecutive work-groups go to the dies in turn: a die takes one stretch of
    // the items, whose neighbours read the same tokens
    const long per = (total + kXcds - 1) / kXcds;
    const long w = (long)(blockIdx.x % kXcds) * per + blockIdx.x / kXcds;
    if (blockIdx.x / kXcds >= per || w >= total) return;
    // order: head, part of the walk, then the tiles that share it
    const long tiles = (LISTS ? (long)a.nq : 1) * a.tiles;
    const long hb = w / (tiles * a.C);
    const int part = (int)(w / tiles % a.C);
    const long unit = hb * tiles + w % tiles;
    const Rows r = rows_of<ROWS, LISTS>(a, unit);
    if (r.count <= 0) return;           // a tile past a short query block

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int len = clamp_len(a, r.b);
    const size_t hk = (size_t)r.b * a.H + r.kv;
    const uint8_t* kp = a.k + hk * a.cap * D + 16 * g;
    const uint8_t* vp = a.v + hk * a.cap * D + VF * l16;
    const float* ksp = a.ks + hk * a.ncap;
    const float* vsp = a.vs + hk * a.ncap;
    const int per_block = a.block / kStep;
    const int32_t* list = nullptr;
    long steps;
    if (LISTS) {
        const long lrow = ((long)r.b * a.Hq + r.head) * a.nq + r.i;
        list = a.idx + lrow * a.n;
        steps = (long)min(max(a.cnt[lrow], 0), a.n) * per_block;
    } else {
        steps = (len + kStep - 1) / kStep;
    }
    const int s0 = (int)(steps * part / a.C), s1 = (int)(steps * (part + 1) / a.C);

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
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.0f;
#pragma unroll
        for (int f = 0; f < VF; ++f) acc[rt][f] = f32x4{0, 0, 0, 0};
    }

    // first token of step s, or -1 where there is none
    auto token_of = [&](int s) {
        if (!LISTS) return s * kStep;
        const int j = list[s / per_block];
        const int t = j * a.block + s % per_block * kStep;
        return (j < 0 || j >= a.n || t >= len) ? -1 : t;
    };
    uint4 kw[2][KC];
    uint32_t vw[8][VW];
    float ksc = 0.0f, vsc = 0.0f;
    auto load = [&](int t0) {
        const int last = len - 1;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const size_t row = (size_t)min(t0 + 16 * t + l16, last) * D;
#pragma unroll
            for (int c = 0; c < KC; ++c) kw[t][c] = *reinterpret_cast<const uint4*>(kp + row + 64 * c);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const size_t row = (size_t)min(t0 + 16 * (e / 4) + 4 * g + e % 4, last) * D;
            if constexpr (VW == 2) {
                const uint2 x = *reinterpret_cast<const uint2*>(vp + row);
                vw[e][0] = x.x;
                vw[e][1] = x.y;
            } else {
                vw[e][0] = *reinterpret_cast<const uint32_t*>(vp + row);
            }
        }
        ksc = ksp[t0 / a.block];
        vsc = vsp[t0 / a.block];
    };

    for (int s = s0 + wave; s < s1; s += 4) {
        const int t0 = __builtin_amdgcn_readfirstlane(token_of(s));
        if (t0 < 0) continue;
        load(t0);
        const float sc = ksc * a.c2;
        f32x4 st[RT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 2 * KC; ++c) {
                const uint4 x = kw[t][c / 2];
                const bf16x8 kf = c % 2 == 0 ? operand8<FMT>(x.x, x.y) : operand8<FMT>(x.z, x.w);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    st[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        kf, qf[rt][c], c == 0 ? f32x4{0, 0, 0, 0} : st[rt][t], 0, 0, 0);
            }
        bf16x8 pf[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float x[8], mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = st[rt][e / 4][e % 4] * sc;
                if (t0 + 16 * (e / 4) + 4 * g + e % 4 >= len) x[e] = -INFINITY;
                mx = fmaxf(mx, x[e]);
            }
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
                pf[rt][e] = static_cast<__bf16>(p * vsc);
            }
        }
        auto product = [&](auto f_tag) __attribute__((always_inline)) {
            constexpr int F = decltype(f_tag)::value, W = F / 4, BY = F % 4;
            const u32x4 x = {column_pair<FMT, BY>(vw[0][W], vw[1][W]), column_pair<FMT, BY>(vw[2][W], vw[3][W]),
                             column_pair<FMT, BY>(vw[4][W], vw[5][W]), column_pair<FMT, BY>(vw[6][W], vw[7][W])};
            const bf16x8 vf = __builtin_bit_cast(bf16x8, x);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                acc[rt][F] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt], acc[rt][F], 0, 0, 0);
        };
        product(std::integral_constant<int, 0>{});
        product(std::integral_constant<int, 1>{});
        product(std::integral_constant<int, 2>{});
        product(std::integral_constant<int, 3>{});
        if constexpr (VF == 8) {
            product(std::integral_constant<int, 4>{});
            product(std::integral_constant<int, 5>{});
            product(std::integral_constant<int, 6>{});
            product(std::integral_constant<int, 7>{});
        }
    }

    // join the four waves
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
        const int row = 16 * rt + l16;
        float top = fmaxf(fmaxf(mbuf[0][row], mbuf[1][row]), fmaxf(mbuf[2][row], mbuf[3][row]));
        const float mine = m[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[rt] - top);
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
            for (int f = 0; f < VF; f += 4)
                *reinterpret_cast<float4*>(&obuf[wave][l16][4 * VF * g + VF * rr + f]) =
                    make_float4(acc[rt][f][rr] * mine, acc[rt][f + 1][rr] * mine, acc[rt][f + 2][rr] * mine,
                                acc[rt][f + 3][rr] * mine);
        __syncthreads();
        constexpr int W = D / 16;       // channels per thread
        const int orow = tid / 16, ch = tid % 16 * W, tr = 16 * rt + orow;
        const float tt = fmaxf(fmaxf(mbuf[0][tr], mbuf[1][tr]), fmaxf(mbuf[2][tr], mbuf[3][tr]));
        float sum = 0.0f;
#pragma unroll
        for (int wv = 0; wv < 4; ++wv)
            if (lbuf[wv][tr] != 0.0f)   // 0: that wave kept no token (its maximum may be -inf)
                sum += lbuf[wv][tr] * __builtin_amdgcn_exp2f(mbuf[wv][tr] - tt);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        float out[W];
#pragma unroll
        for (int e = 0; e < W; ++e)
            out[e] = (obuf[0][orow][ch + e] + obuf[1][orow][ch + e] + obuf[2][orow][ch + e] + obuf[3][orow][ch + e]) * inv;
        const float lse2 = sum == 0.0f ? -INFINITY : tt + __builtin_amdgcn_logf(sum);   // log2
        if (a.C > 1) {
            const long slot = (unit * a.C + part) * ROWS + tr;
            float* po = a.part + slot * D + ch;
#pragma unroll
            for (int e = 0; e < W; e += 4)
                *reinterpret_cast<float4*>(po + e) = make_float4(out[e], out[e + 1], out[e + 2], out[e + 3]);
            if (tid % 16 == 0) (a.part + a.units * a.C * ROWS * D)[slot] = lse2;
        } else if (tr < r.count) {
            uint32_t* po = reinterpret_cast<uint32_t*>(a.o + (r.row0 + tr) * D + ch);
#pragma unroll
            for (int e = 0; e < W; e += 2)
                po[e / 2] = (uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(out[e])) |
                            ((uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(out[e + 1])) << 16);
            if (a.lse && tid % 16 == 0) a.lse[r.row0 + tr] = lse2 * kLn2;
        }
        __syncthreads();
    }
}

// Joins the parts of every row in their order.  D/4 lanes per row.
template <int D, int ROWS, bool LISTS>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
    constexpr int LPR = D / 4, RPG = 256 / LPR;
    const int tid = threadIdx.x;
    const long row = (long)blockIdx.x * RPG + tid / LPR;
    const long unit = row / ROWS;
    if (unit >= a.units) return;
    const int tr = (int)(row % ROWS), ch = tid % LPR * 4;
    const Rows r = rows_of<ROWS, LISTS>(a, unit);
    if (tr >= r.count) return;
    const float* lse2 = a.part + a.units * a.C * ROWS * D + unit * a.C * ROWS + tr;
    const float* po = a.part + (unit * a.C * ROWS + tr) * D + ch;
    float top = -INFINITY;
    for (int c = 0; c < a.C; ++c) top = fmaxf(top, lse2[(long)c * ROWS]);
    float sum = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int c = 0; c < a.C; ++c) {
        const float x = lse2[(long)c * ROWS];
        if (x == -INFINITY) continue;      // that part kept no token
        const float w = __builtin_amdgcn_exp2f(x - top);
        sum += w;
        o += w * *reinterpret_cast<const f32x4*>(po + (long)c * ROWS * D);
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint2 pk;
    pk.x = (uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(o[0] * inv)) |
           ((uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(o[1] * inv)) << 16);
    pk.y = (uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(o[2] * inv)) |
           ((uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(o[3] * inv)) << 16);
    *reinterpret_cast<uint2*>(a.o + (r.row0 + tr) * D + ch) = pk;
    if (a.lse && tid % LPR == 0)
        a.lse[r.row0 + tr] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// How a call is cut up, from its host sizes alone.
struct Plan {
    int rt, C;
    int tiles, heads;
    long units;
};
Plan plan_of(int B, int H, int block, int Hq, int Lq, int max_len, bool lists) {
    Plan p;
    const int rows = lists ? std::min(block, Lq) : (int)std::min<long>((long)(Hq / H) * Lq, 1L << 30);
    p.rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.tiles = (rows + 16 * p.rt - 1) / (16 * p.rt);
    p.heads = lists ? Hq : H;
    p.units = (long)B * p.heads * (lists ? (Lq + block - 1) / block : 1) * p.tiles;
    // parts of a walk: until there are four work-groups per compute unit, each
    // with four steps per wave at least
    const long want = (1024 + p.units - 1) / p.units;
    const long most = std::max(1L, ((long)max_len + kStep - 1) / kStep / 16);
    p.C = (int)std::max(1L, std::min(want, most));
    return p;
}
size_t part_bytes(const Plan& p, int d) {
    return p.C == 1 ? 0 : (size_t)p.units * p.C * 16 * p.rt * (d + 1) * sizeof(float);
}

template <int D, int FMT, int RT, bool LISTS>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
    const long total = a.units * a.C;
    const unsigned grid = (unsigned)((total + kXcds - 1) / kXcds * kXcds);
    hipLaunchKernelGGL((rows_kernel<D, FMT, RT, LISTS>), dim3(grid), dim3(256), 0, s, a);
    if (a.C > 1) {
        constexpr int RPG = 256 / (D / 4);
        const long rows = a.units * 16 * RT;
        hipLaunchKernelGGL((join_kernel<D, 16 * RT, LISTS>), dim3((unsigned)((rows + RPG - 1) / RPG)), dim3(256), 0, s,
                           a);
    }
    return hipGetLastError();
}

}  // namespace

size_t cache_attn_ws_bytes(int B, int H, int d, int block, int Hq, int Lq, int max_len) {
    return std::max(part_bytes(plan_of(B, H, block, Hq, Lq, max_len, false), d),
                    part_bytes(plan_of(B, H, block, Hq, Lq, max_len, true), d));
}

hipError_t launch_cache_attn(const CacheView& c, const uint16_t* q, int Hq, int Lq, int max_len,
                             const int32_t* kv_len, const int32_t* kv_idx, const int32_t* kv_cnt, float scale,
                             uint16_t* o, float* lse, void* ws, hipStream_t s) {
    const bool lists = kv_idx != nullptr;
    const Plan p = plan_of(c.B, c.H, c.block, Hq, Lq, max_len, lists);
    AttnArgs a{q, c.k, c.v, c.ks, c.vs, kv_len, kv_idx, kv_cnt, o, lse, static_cast<float*>(ws),
               c.B, Hq, c.H, Lq, c.cap, c.n, max_len, (max_len + c.block - 1) / c.block,
               (Lq + c.block - 1) / c.block, c.block, p.tiles, p.heads, p.C, p.units, scale * kLog2e};
    hipError_t e = hipErrorInvalidValue;
    auto with_rt = [&](auto d, auto fmt, auto ls) {
        constexpr int D = decltype(d)::value, FMT = decltype(fmt)::value;
        constexpr bool LISTS = decltype(ls)::value;
        if (p.rt == 1) e = launch<D, FMT, 1, LISTS>(a, s);
        else if (p.rt == 2) e = launch<D, FMT, 2, LISTS>(a, s);
        else e = launch<D, FMT, 4, LISTS>(a, s);
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
