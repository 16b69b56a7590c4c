// The 8-bit key/value cache for gfx950: quantisation of new tokens as they are
// written, and reading back.
//
// A block of tokens of one head shares a scale s; a code c stands for c * s.
// Writing takes the largest magnitude of what it puts into the block, the
// scale that it asks for (never less than the old one in a block that is
// continued), and rounds every x / s to the nearest code, ties to even:
//   E4M3   s is a power of two, so x / s is exact and the conversion rounds once;
//   INT8   r = rint(x * (1/s)) is at most one off, and only next to a border;
//          x - r s is exact in fp32 (both are multiples of the last place of
//          s, and it is at most about s), so comparing its double with s
//          decides the border as the real quotient does.
// Reading multiplies in fp32 and rounds to bf16: for E4M3 the product is exact, for
// INT8 (31 bits) its own rounding comes on top, 2^-16 of the second one.
// Bound by memory: per channel two bytes read and one written (write), or one
// read and two written (read).  One work-group per (sequence, head, block,
// K or V) keeps the block's new rows in registers between the maximum and the
// rounding, so they are read once.
#include "moddit_internal.h"

#include <type_traits>

namespace moddit {
namespace {

constexpr float kMinScale = 1.1754943508222875e-38f;   // 2^-126

struct StoreArgs {
    uint8_t* codes[2];
    float* scales[2];
    Strided x[2];              // bf16 tensors of the call; p may be null (not read)
    int H, cap, n, L, first;
    const int32_t* starts;
    const int32_t* counts;
    int groups;                // blocks a sequence's tokens can touch
};

// The sequence's tokens: positions [p0, p1) (empty where it takes none).
__device__ __forceinline__ void token_range(const StoreArgs& a, int b, int& p0, int& p1) {
    const long s = (long)a.first + (a.starts ? a.starts[b] : 0);
    int count = a.counts ? a.counts[b] : a.L;
    count = min(max(count, 0), a.L);
    if (s < 0 || s >= a.cap) {
        p0 = p1 = 0;
        return;
    }
    p0 = (int)s;
    p1 = (int)(s + count < a.cap ? s + count : a.cap);
}

// Scale that a largest magnitude (its bf16 bits) asks for.
template <int FMT>
__device__ __forceinline__ float scale_for(uint32_t amax_bits) {
    if (amax_bits == 0) return 0.0f;
    if (amax_bits >= 0x7f80u) return NAN;
    const float amax = __uint_as_float(amax_bits << 16);
    if constexpr (FMT == MOD_CACHE_INT8) {
        return fmaxf(__fdiv_rn(amax, 127.0f), kMinScale);
    } else {
        // amax = m 2^x, m in [1, 2): 448 = 1.75 * 2^8 holds amax / 2^(x-8) if m <= 1.75
        const int x = (int)(amax_bits >> 7) - 127, up = (amax_bits & 0x7fu) > 0x60u;
        return ldexpf(1.0f, max(x - 8 + up, -126));   // bf16 subnormals have x = -127: the minimum
    }
}

// Four codes of x[0..3] / s, lowest byte first; inv = 1 / s.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], float s, float inv) {
    if constexpr (FMT == MOD_CACHE_INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float r = rintf(x[i] * inv);
            const float rem = 2.0f * fmaf(-r, s, x[i]);
            const bool odd = ((int)r & 1) != 0;
            if (rem > s || (rem == s && odd)) r += 1.0f;
            if (rem < -s || (rem == -s && odd)) r -= 1.0f;
            r = fminf(fmaxf(r, -127.0f), 127.0f);
            w |= ((uint32_t)(int)r & 0xffu) << (8 * i);
        }
        return w;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
    }
}

// The numbers that the four codes of w are.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
    if constexpr (FMT == MOD_CACHE_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
    }
}

// Codes of an earlier token under a scale that grew: c s_old / s_new rounded to
// the nearest.  In fp64: the quotient of a 32-bit and a 24-bit number is
// either a border or further from it than its rounding.
template <int FMT>
__device__ __forceinline__ uint32_t requantise4(uint32_t w, float s_old, float s_new) {
    float x[4];
    decode4<FMT>(w, x);
    if constexpr (FMT == MOD_CACHE_INT8) {
        uint32_t r = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double z = rint((double)x[i] * (double)s_old / (double)s_new);
            r |= ((uint32_t)(int)fmin(fmax(z, -127.0), 127.0) & 0xffu) << (8 * i);
        }
        return r;
    } else {
        const float ratio = (float)((double)s_old / (double)s_new);   // powers of two, at most 1
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] *= ratio;
        return encode4<FMT>(x, 1.0f, 1.0f);
    }
}

template <int D, int BS, int FMT>
__global__ __launch_bounds__(256) void cache_write_kernel(StoreArgs a) {
    constexpr int LPT = D / 8;               // threads per token: 8 channels each
    constexpr int TPP = 256 / LPT;           // tokens per pass
    constexpr int NP = BS / TPP;             // passes
    __shared__ uint32_t wave_max[4];
    const int tid = threadIdx.x;
    int wg = blockIdx.x;
    const int kv = wg & 1;
    wg >>= 1;
    const int t = wg % a.groups;
    wg /= a.groups;
    const int h = wg % a.H, b = wg / a.H;
    int p0, p1;
    token_range(a, b, p0, p1);
    const int j = p0 / BS + t;
    const int lo = max(p0, j * BS), hi = min(p1, (j + 1) * BS);
    if (lo >= hi) return;                    // the same for the whole work-group

    const uint16_t* x = a.x[kv].p + b * a.x[kv].b + h * a.x[kv].h;
    const int c0 = 8 * (tid % LPT);
    uint4 in[NP];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int p = j * BS + i * TPP + tid / LPT;
        in[i] = make_uint4(0, 0, 0, 0);
        if (p >= lo && p < hi) in[i] = *reinterpret_cast<const uint4*>(x + (long)(p - p0) * a.x[kv].l + c0);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const uint32_t w[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) top = max(top, max(w[q] & 0x7fffu, (w[q] >> 16) & 0x7fffu));
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if (tid % 64 == 0) wave_max[tid / 64] = top;
    float* sp = a.scales[kv] + ((size_t)b * a.H + h) * a.n + j;
    const bool goes_on = lo > j * BS;
    const float s_old = goes_on ? *sp : 0.0f;
    __syncthreads();                         // also: everyone has read the old scale
    top = max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3]));
    float s = scale_for<FMT>(top);
    if (goes_on && !(s_old <= s) && s == s) s = s_old;   // keeps a NaN of either
    if (tid == 0) *sp = s;
    const bool usable = s > 0.0f;            // neither 0 nor NaN
    const float inv = usable ? __fdiv_rn(1.0f, s) : 0.0f;

    uint8_t* codes = a.codes[kv] + ((size_t)b * a.H + h) * (size_t)a.cap * D;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int p = j * BS + i * TPP + tid / LPT;
        if (p < lo || p >= hi) continue;
        const uint32_t w[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
        uint2 out = make_uint2(0, 0);
        if (usable) {
            float f[4], g[4];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                f[2 * q] = __uint_as_float(w[q] << 16);
                f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
                g[2 * q] = __uint_as_float(w[q + 2] << 16);
                g[2 * q + 1] = __uint_as_float(w[q + 2] & 0xffff0000u);
            }
            out = make_uint2(encode4<FMT>(f, s, inv), encode4<FMT>(g, s, inv));
        }
        *reinterpret_cast<uint2*>(codes + (size_t)p * D + c0) = out;
    }
    // the block's earlier tokens under a scale that grew
    if (goes_on && usable && s != s_old)
        for (int p = j * BS + tid / LPT; p < lo; p += TPP) {
            uint2* c = reinterpret_cast<uint2*>(codes + (size_t)p * D + c0);
            const uint2 w = *c;
            *c = make_uint2(requantise4<FMT>(w.x, s_old, s), requantise4<FMT>(w.y, s_old, s));
        }
}

template <int D, int BS, int FMT>
__global__ __launch_bounds__(256) void cache_read_kernel(StoreArgs a) {
    constexpr int LPT = D / 8, TPP = 256 / LPT, NP = BS / TPP;
    const int tid = threadIdx.x;
    int wg = blockIdx.x;
    const int kv = wg & 1;
    wg >>= 1;
    const int t = wg % a.groups;
    wg /= a.groups;
    const int h = wg % a.H, b = wg / a.H;
    if (a.x[kv].p == nullptr) return;
    int p0, p1;
    token_range(a, b, p0, p1);
    const int j = p0 / BS + t;
    const int lo = max(p0, j * BS), hi = min(p1, (j + 1) * BS);
    if (lo >= hi) return;
    const uint8_t* codes = a.codes[kv] + ((size_t)b * a.H + h) * (size_t)a.cap * D;
    const float s = a.scales[kv][((size_t)b * a.H + h) * a.n + j];
    uint16_t* x = a.x[kv].p + b * a.x[kv].b + h * a.x[kv].h;
    const int c0 = 8 * (tid % LPT);
    uint2 in[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int p = j * BS + i * TPP + tid / LPT;
        in[i] = make_uint2(0, 0);
        if (p >= lo && p < hi) in[i] = *reinterpret_cast<const uint2*>(codes + (size_t)p * D + c0);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int p = j * BS + i * TPP + tid / LPT;
        if (p < lo || p >= hi) continue;
        float f[4], g[4];
        decode4<FMT>(in[i].x, f);
        decode4<FMT>(in[i].y, g);
        uint32_t out[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float e0 = q < 2 ? f[2 * q] : g[2 * q - 4], e1 = q < 2 ? f[2 * q + 1] : g[2 * q - 3];
            out[q] = (uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(e0 * s)) |
                     ((uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(e1 * s)) << 16);
        }
        *reinterpret_cast<uint4*>(x + (long)(p - p0) * a.x[kv].l + c0) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

StoreArgs store_args(const CacheView& c, const Strided& k, const Strided& v, int L, int first, const int32_t* starts,
                     const int32_t* counts) {
    StoreArgs a{{c.k, c.v}, {c.ks, c.vs}, {k, v}, c.H, c.cap, c.n, L, first, starts, counts, 0};
    // blocks that L tokens can touch from where they start (anywhere, if the device says)
    a.groups = starts ? (L + c.block - 2) / c.block + 1 : (first + L - 1) / c.block - first / c.block + 1;
    return a;
}

// f(D, BS, FMT) with the cache's values as integral constants
template <class F>
void with_form(const CacheView& c, F&& f) {
    auto fmt = [&](auto d, auto bs) {
        if (c.format == MOD_CACHE_INT8) f(d, bs, std::integral_constant<int, MOD_CACHE_INT8>{});
        else f(d, bs, std::integral_constant<int, MOD_CACHE_E4M3>{});
    };
    using I64 = std::integral_constant<int, 64>;
    using I128 = std::integral_constant<int, 128>;
    if (c.d == 128) {
        if (c.block == 128) fmt(I128{}, I128{});
        else fmt(I128{}, I64{});
    } else {
        if (c.block == 128) fmt(I64{}, I128{});
        else fmt(I64{}, I64{});
    }
}

}  // namespace

hipError_t launch_cache_write(const CacheView& c, const Strided& k, const Strided& v, int L, int first,
                              const int32_t* starts, const int32_t* counts, hipStream_t s) {
    const StoreArgs a = store_args(c, k, v, L, first, starts, counts);
    with_form(c, [&](auto d, auto bs, auto fmt) {
        hipLaunchKernelGGL((cache_write_kernel<d.value, bs.value, fmt.value>),
                           dim3((unsigned)((long)c.B * c.H * a.groups * 2)), dim3(256), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheView& c, const Strided& k, const Strided& v, int L, int first,
                             const int32_t* starts, const int32_t* counts, hipStream_t s) {
    const StoreArgs a = store_args(c, k, v, L, first, starts, counts);
    with_form(c, [&](auto d, auto bs, auto fmt) {
        hipLaunchKernelGGL((cache_read_kernel<d.value, bs.value, fmt.value>),
                           dim3((unsigned)((long)c.B * c.H * a.groups * 2)), dim3(256), 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace moddit
