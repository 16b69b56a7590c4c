// Rotary positions over the axes of a video (time, height, width) and their
// gradient, for gfx950.
//
// The pair (x0, x1) of channels that belongs to frequency j of axis a turns by
// the angle pos_a * theta^(-2j/w_a):
//   y0 = x0 cos - x1 sin,   y1 = x1 cos + x0 sin     (backward: sin negated)
// cos and sin come from per-axis tables that the handle holds (fp32, computed
// in fp64 on the host: an fp32 angle of a far position would be off by
// position * 2^-24 radians).  The products and their sum are fp32; a value is
// rounded to bf16 once.
//
// Bound by memory: two bytes read and two written per channel.  A thread owns
// one 16-byte chunk of channels of one token and walks over heads, so the
// token's position, table entries and channel bookkeeping are looked up once
// for all of them; loads and stores are 16 bytes per lane, 16 (d = 128) or 8
// lanes to a token's row.
#include "moddit_internal.h"

#include <algorithm>

namespace moddit {
namespace {

struct RopeArgs {
    RopeTable t;
    Strided x, y;
    int H, L, Lv;              // Lv: tokens with a position
    int first;
    const int32_t* starts;
    float dir;                 // +1 forward, -1 backward
    int token_groups, heads;   // work-groups per sequence along the tokens; heads per thread
    int head_groups;
};

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const uint16_t a = __builtin_bit_cast(uint16_t, static_cast<__bf16>(lo));
    const uint16_t b = __builtin_bit_cast(uint16_t, static_cast<__bf16>(hi));
    return (uint32_t)a | ((uint32_t)b << 16);
}

// HALVES: the partner of a channel sits w/2 channels away, in general in
// another lane and not at a chunk boundary: the wave's rows go through LDS and
// the eight partners are read back one by one (9 LDS operations per 2 KB of
// HBM traffic of a wave, far under its time in memory).
template <int D, bool HALVES>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    constexpr int LPT = D / 8;          // lanes per token
    constexpr int TPG = 256 / LPT;      // tokens per work-group
    constexpr int U = 4;                // heads in flight
    __shared__ __align__(16) uint16_t rows[HALVES ? 4 * U * 512 : 8];
    const int tid = threadIdx.x, ch = tid % LPT;
    int wg = blockIdx.x;
    const int hg = wg % a.head_groups;
    wg /= a.head_groups;
    const int b = wg / a.token_groups;
    const int l = (wg % a.token_groups) * TPG + tid / LPT;
    const bool live = l < a.L;

    // position of the token along the axes
    int pos[3] = {0, 0, 0};
    bool placed = false, outside = false;
    if (live && l < a.Lv) {
        const long p = (long)a.first + (a.starts ? a.starts[b] : 0) + l;
        const int hw = a.t.height * a.t.width;
        placed = true;
        if (p < 0 || p >= (long)a.t.frames * hw) {
            outside = true;
        } else {
            pos[0] = (int)p / hw;
            const int r = (int)p % hw;
            pos[1] = r / a.t.width;
            pos[2] = r % a.t.width;
        }
    }
    // per channel: (cos, signed sin) and, HALVES, the partner channel
    constexpr int NC = HALVES ? 8 : 4;
    float c[NC], s[NC];
    bool turn[NC];
    int partner[NC];
#pragma unroll
    for (int e = 0; e < NC; ++e) {
        const int chan = 8 * ch + (HALVES ? e : 2 * e);
        int base = 0, ax = -1;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int w = 2 * a.t.half[k];
            if (ax < 0 && chan < base + w) ax = k;
            if (ax < 0) base += w;
        }
        turn[e] = placed && ax >= 0;
        c[e] = 1.0f;
        s[e] = 0.0f;
        partner[e] = chan;
        if (turn[e]) {
            const int half = ax == 0 ? a.t.half[0] : ax == 1 ? a.t.half[1] : a.t.half[2];
            const int at = ax == 0 ? pos[0] : ax == 1 ? pos[1] : pos[2];
            const int off = ax == 0 ? a.t.tab_off[0] : ax == 1 ? a.t.tab_off[1] : a.t.tab_off[2];
            const int rel = chan - base;
            const bool second = HALVES && rel >= half;
            const int j = HALVES ? (second ? rel - half : rel) : rel / 2;
            const float2 cs = a.t.table[off + (size_t)at * half + j];
            c[e] = outside ? NAN : cs.x;
            s[e] = (second ? cs.y : -cs.y) * a.dir;
            if (HALVES) partner[e] = second ? chan - half : chan + half;
        }
    }

    const int h0 = hg * a.heads, h1 = min(a.H, h0 + a.heads);
    const uint16_t* xp = a.x.p + b * a.x.b + (live ? l : 0) * a.x.l + 8 * ch;
    uint16_t* yp = a.y.p + b * a.y.b + (live ? l : 0) * a.y.l + 8 * ch;
    uint16_t* row = rows + (HALVES ? (tid / 64) * U * 512 : 0);   // the wave's
    const int row0 = HALVES ? (tid % 64) / LPT * D : 0;            // the token's row in it
    for (int h = h0; h < h1; h += U) {
        uint4 in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            in[u] = make_uint4(0, 0, 0, 0);
            if (live && h + u < h1) in[u] = *reinterpret_cast<const uint4*>(xp + (h + u) * a.x.h);
        }
        if constexpr (HALVES) {
#pragma unroll
            for (int u = 0; u < U; ++u) *reinterpret_cast<uint4*>(row + u * 512 + (tid % 64) * 8) = in[u];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t w[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
            uint32_t out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x0 = lo_bf16(w[i]), x1 = hi_bf16(w[i]);
                if constexpr (HALVES) {
                    const float p0 = lo_bf16(row[u * 512 + row0 + partner[2 * i]]);
                    const float p1 = lo_bf16(row[u * 512 + row0 + partner[2 * i + 1]]);
                    const uint32_t r = pack_bf16(fmaf(x0, c[2 * i], p0 * s[2 * i]),
                                                 fmaf(x1, c[2 * i + 1], p1 * s[2 * i + 1]));
                    out[i] = ((turn[2 * i] ? r : w[i]) & 0xffffu) | ((turn[2 * i + 1] ? r : w[i]) & 0xffff0000u);
                } else {
                    const uint32_t r = pack_bf16(fmaf(x0, c[i], x1 * s[i]), fmaf(x1, c[i], -(x0 * s[i])));
                    out[i] = turn[i] ? r : w[i];
                }
            }
            if (live && h + u < h1)
                *reinterpret_cast<uint4*>(yp + (h + u) * a.y.h) = make_uint4(out[0], out[1], out[2], out[3]);
        }
        if constexpr (HALVES) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

}  // namespace

hipError_t launch_rope(const RopeTable& t, const Strided& x, const Strided& y, int B, int H, int L, int d, int text,
                       int first, const int32_t* starts, bool backward, hipStream_t s) {
    RopeArgs a{t, x, y, H, L, L - text, first, starts, backward ? -1.0f : 1.0f, 0, 0, 0};
    const int tpg = 2048 / d;
    a.token_groups = (L + tpg - 1) / tpg;
    // heads are divided over work-groups while the tokens alone do not fill the chip
    const long groups = (long)B * a.token_groups;
    a.heads = H;
    while (a.heads > 4 && groups * ((H + a.heads - 1) / a.heads) < 2048) a.heads = std::max(4, a.heads / 2);
    a.head_groups = (H + a.heads - 1) / a.heads;
    const dim3 grid((unsigned)(groups * a.head_groups));
    if (d == 128) {
        if (t.halves) hipLaunchKernelGGL((rope_kernel<128, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((rope_kernel<128, false>), grid, dim3(256), 0, s, a);
    } else {
        if (t.halves) hipLaunchKernelGGL((rope_kernel<64, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((rope_kernel<64, false>), grid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace moddit
