// C ABI of the cached layer: argument validation, the rotary tables, and the
// kernel launches.
#include "../../include/moddit.h"
#include "moddit_internal.h"

#include <cmath>
#include <new>
#include <vector>

using moddit::fail;
using moddit::hip_fail;

struct mod_rope {
    mod_rope_params params{};
    int device = 0;
    float2* table = nullptr;
    moddit::RopeTable view{};
};

namespace {

constexpr int kMaxCapacity = 1 << 24;   // a head's codes stay below 2^31 bytes
constexpr long kMaxHeads = 1L << 22;    // B * H
constexpr long kMaxGroups = 1L << 22;   // work-groups of a launch (their threads stay below 2^32)

mod_status check_aligned(const void* p, const char* what) {
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
        return fail(MOD_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
    return MOD_OK;
}

// The [B, H, L, d] tensor at p with the caller's strides; `written`: of a tensor
// that a call writes, whose rows must not lie on each other.
mod_status make_strided(const void* p, const mod_strides* st, int B, int H, int L, int d, bool written,
                        const char* what, moddit::Strided* out) {
    const mod_status e = check_aligned(p, what);
    if (e != MOD_OK) return e;
    out->p = static_cast<uint16_t*>(const_cast<void*>(p));
    if (st) {
        if (st->b % 8 != 0 || st->h % 8 != 0 || st->l % 8 != 0)
            return fail(MOD_ERR_INVALID_ARG, "%s: strides must be multiples of 8 elements (b=%ld h=%ld l=%ld)", what,
                        (long)st->b, (long)st->h, (long)st->l);
        auto on_itself = [&](int n, int64_t stride) { return n > 1 && stride > -d && stride < d; };
        if (written && (on_itself(B, st->b) || on_itself(H, st->h) || on_itself(L, st->l)))
            return fail(MOD_ERR_INVALID_ARG, "%s is written: its rows must not overlap (b=%ld h=%ld l=%ld)", what,
                        (long)st->b, (long)st->h, (long)st->l);
        out->b = st->b;
        out->h = st->h;
        out->l = st->l;
    } else {
        out->l = d;
        out->h = (long)L * d;
        out->b = (long)H * L * d;
    }
    return MOD_OK;
}

mod_status check_cache_shape(const mod_cache_shape* s) {
    if (!s) return fail(MOD_ERR_INVALID_ARG, "cache shape is NULL");
    if (s->B <= 0 || s->H <= 0 || s->capacity <= 0)
        return fail(MOD_ERR_INVALID_ARG, "cache sizes must be positive (B=%d H=%d capacity=%d)", s->B, s->H,
                    s->capacity);
    if (s->d != 64 && s->d != 128) return fail(MOD_ERR_UNSUPPORTED, "d=%d (supported: 64, 128)", s->d);
    if (s->block != 64 && s->block != 128)
        return fail(MOD_ERR_UNSUPPORTED, "block=%d (supported: 64, 128)", s->block);
    if (s->format != MOD_CACHE_E4M3 && s->format != MOD_CACHE_INT8)
        return fail(MOD_ERR_INVALID_ARG, "unknown cache format %d", s->format);
    if (s->capacity > kMaxCapacity)
        return fail(MOD_ERR_UNSUPPORTED, "capacity=%d exceeds %d", s->capacity, kMaxCapacity);
    if ((long)s->B * s->H > kMaxHeads) return fail(MOD_ERR_UNSUPPORTED, "B*H too large");
    return MOD_OK;
}

mod_status make_view(const mod_cache_shape* s, const mod_cache* c, moddit::CacheView* out) {
    mod_status st = check_cache_shape(s);
    if (st != MOD_OK) return st;
    if (!c) return fail(MOD_ERR_INVALID_ARG, "cache is NULL");
    if (!c->k || !c->v || !c->k_scale || !c->v_scale)
        return fail(MOD_ERR_INVALID_ARG, "the cache's k, v, k_scale and v_scale must not be NULL");
    st = check_aligned(c->k, "the cache's k");
    if (st == MOD_OK) st = check_aligned(c->v, "the cache's v");
    if (st != MOD_OK) return st;
    *out = {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale,
            s->B, s->H, s->capacity, s->d, s->block, (s->capacity + s->block - 1) / s->block, s->format};
    return MOD_OK;
}

mod_status check_range(const mod_cache_shape* s, int L, int first, const int32_t* starts) {
    if (L <= 0) return fail(MOD_ERR_INVALID_ARG, "L=%d must be positive", L);
    if (first < 0) return fail(MOD_ERR_INVALID_ARG, "first=%d must be >= 0", first);
    if (L > s->capacity || (!starts && (long)first + L > s->capacity))
        return fail(MOD_ERR_INVALID_ARG, "%d tokens from position %d exceed the capacity of %d", L, first,
                    s->capacity);
    if ((long)s->B * s->H * ((L + (long)s->block - 1) / s->block + 1) * 2 > kMaxGroups)
        return fail(MOD_ERR_UNSUPPORTED, "B*H*L too large for one call");
    return MOD_OK;
}

mod_status check_attn(const mod_cache_shape* s, int Hq, int Lq, int max_len) {
    const mod_status st = check_cache_shape(s);
    if (st != MOD_OK) return st;
    if (Hq <= 0 || Lq <= 0) return fail(MOD_ERR_INVALID_ARG, "Hq=%d and Lq=%d must be positive", Hq, Lq);
    if (Hq % s->H != 0) return fail(MOD_ERR_INVALID_ARG, "Hq=%d is not a multiple of H=%d", Hq, s->H);
    if (max_len < 0 || max_len > s->capacity)
        return fail(MOD_ERR_INVALID_ARG, "max_len=%d must be in [0, capacity=%d]", max_len, s->capacity);
    if (Lq > kMaxCapacity || (long)s->B * Hq * ((Lq + 15L) / 16) > kMaxGroups)
        return fail(MOD_ERR_UNSUPPORTED, "B*Hq*Lq too large for one call");
    return MOD_OK;
}

// The plans without and with lists; the bytes that both can do with.
size_t plan_attn(const mod_cache_shape* s, int Hq, int Lq, int max_len, moddit::CacheAttnPlan (&plans)[2]) {
    size_t need = 0;
    for (int lists = 0; lists < 2; ++lists) {
        plans[lists] = moddit::plan_cache_attn(s->B, s->H, s->d, s->block, Hq, Lq, max_len, lists != 0);
        const size_t bytes = moddit::cache_attn_plan_bytes(plans[lists], s->d);
        if (bytes > need) need = bytes;
    }
    return need;
}

mod_status rope_call(const mod_rope* rope, const mod_shape* shape, const void* x, const mod_strides* xs, void* y,
                     const mod_strides* ys, int first, const int32_t* starts, bool backward, void* stream) {
    if (!rope) return fail(MOD_ERR_INVALID_ARG, "rope is NULL");
    if (!shape) return fail(MOD_ERR_INVALID_ARG, "shape is NULL");
    if (!x || !y) return fail(MOD_ERR_INVALID_ARG, "x and y must not be NULL");
    const mod_rope_params& p = rope->params;
    if (shape->B <= 0 || shape->H <= 0 || shape->L <= 0)
        return fail(MOD_ERR_INVALID_ARG, "shape sizes must be positive (B=%d H=%d L=%d)", shape->B, shape->H, shape->L);
    if (shape->d != p.d) return fail(MOD_ERR_INVALID_ARG, "d=%d, but the rope has d=%d", shape->d, p.d);
    if (shape->frame_tokens != 0 && shape->frame_tokens != p.height * p.width)
        return fail(MOD_ERR_INVALID_ARG, "frame_tokens=%d, but the rope has frames of %d x %d", shape->frame_tokens,
                    p.height, p.width);
    if (shape->text_tokens < 0 || shape->text_tokens > shape->L)
        return fail(MOD_ERR_INVALID_ARG, "text_tokens=%d must be in [0, L]", shape->text_tokens);
    if (first < 0) return fail(MOD_ERR_INVALID_ARG, "first=%d must be >= 0", first);
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess || device != rope->device)
        return fail(MOD_ERR_INVALID_ARG, "the rope belongs to device %d, but the current device is %d", rope->device,
                    device);
    const long total = (long)p.frames * p.height * p.width;
    if (!starts && (long)first + shape->L - shape->text_tokens > total)
        return fail(MOD_ERR_INVALID_ARG, "%d tokens from position %d exceed the %ld positions of the rope",
                    shape->L - shape->text_tokens, first, total);
    if ((long)shape->B * ((shape->L + 15L) / 16) > kMaxGroups)
        return fail(MOD_ERR_UNSUPPORTED, "B*L too large for one call");
    if ((long)shape->B * shape->H > kMaxHeads) return fail(MOD_ERR_UNSUPPORTED, "B*H too large");
    moddit::Strided in{}, out{};
    mod_status st = make_strided(x, xs, shape->B, shape->H, shape->L, p.d, false, backward ? "dy" : "x", &in);
    if (st != MOD_OK) return st;
    st = make_strided(y, ys, shape->B, shape->H, shape->L, p.d, true, backward ? "dx" : "y", &out);
    if (st != MOD_OK) return st;
    if (in.p == out.p && ((shape->B > 1 && in.b != out.b) || (shape->H > 1 && in.h != out.h) ||
                          (shape->L > 1 && in.l != out.l)))
        return fail(MOD_ERR_INVALID_ARG, "a rotation in place needs the same strides on both sides");
    const hipError_t e = moddit::launch_rope(rope->view, in, out, shape->B, shape->H, shape->L, p.d,
                                             shape->text_tokens, first, starts, backward,
                                             static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rope launch");
    return MOD_OK;
}

}  // namespace

extern "C" {

mod_status mod_rope_create(const mod_rope_params* params, mod_rope** out) {
    if (!out) return fail(MOD_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    if (!params) return fail(MOD_ERR_INVALID_ARG, "params is NULL");
    const mod_rope_params& p = *params;
    if (p.d != 64 && p.d != 128) return fail(MOD_ERR_UNSUPPORTED, "d=%d (supported: 64, 128)", p.d);
    long sum = 0;
    for (int w : p.dims) {
        if (w < 0 || w % 2 != 0 || w > p.d) return fail(MOD_ERR_INVALID_ARG, "dims must be even and in [0, d]");
        sum += w;
    }
    if (sum < 2 || sum > p.d)
        return fail(MOD_ERR_INVALID_ARG, "dims sum to %ld, must be in [2, d=%d]", sum, p.d);
    if (p.frames <= 0 || p.height <= 0 || p.width <= 0)
        return fail(MOD_ERR_INVALID_ARG, "frames, height and width must be positive");
    const long hw = (long)p.height * p.width;
    if (hw >= (1L << 31) || hw * p.frames >= (1L << 31))
        return fail(MOD_ERR_UNSUPPORTED, "frames*height*width must be below 2^31");
    const int sizes[3] = {p.frames, p.height, p.width};
    long entries = 0;
    for (int a = 0; a < 3; ++a) entries += (long)sizes[a] * (p.dims[a] / 2);
    if (entries >= (1L << 28)) return fail(MOD_ERR_UNSUPPORTED, "position tables of %ld entries are too large", entries);
    if (!(p.theta > 1.0) || !std::isfinite(p.theta))
        return fail(MOD_ERR_INVALID_ARG, "theta must be finite and above 1");
    if (p.pairing != MOD_ROPE_ADJACENT && p.pairing != MOD_ROPE_HALVES)
        return fail(MOD_ERR_INVALID_ARG, "unknown pairing %d", p.pairing);

    std::vector<float2> table;
    mod_rope* r = new (std::nothrow) mod_rope();
    if (!r) return fail(MOD_ERR_NOMEM, "host allocation failed");
    r->params = p;
    (void)hipGetDevice(&r->device);
    try {
        table.reserve((size_t)entries);
        for (int a = 0; a < 3; ++a) {
            r->view.tab_off[a] = (int)table.size();
            r->view.half[a] = p.dims[a] / 2;
            std::vector<double> freq((size_t)p.dims[a] / 2);
            for (size_t j = 0; j < freq.size(); ++j) freq[j] = std::pow(p.theta, -2.0 * (double)j / p.dims[a]);
            for (int i = 0; i < sizes[a]; ++i)
                for (double f : freq) table.push_back({(float)std::cos(i * f), (float)std::sin(i * f)});
        }
    } catch (const std::bad_alloc&) {
        delete r;
        return fail(MOD_ERR_NOMEM, "host allocation failed");
    }
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&r->table), table.size() * sizeof(float2));
    if (e != hipSuccess) {
        (void)hipGetLastError();        // kept for the next launch's check otherwise
        delete r;
        return fail(MOD_ERR_NOMEM, "hipMalloc(%zu): %s", table.size() * sizeof(float2), hipGetErrorString(e));
    }
    e = hipMemcpy(r->table, table.data(), table.size() * sizeof(float2), hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        (void)hipFree(r->table);
        delete r;
        return hip_fail(e, "upload of the position tables");
    }
    r->view.table = r->table;
    r->view.frames = p.frames;
    r->view.height = p.height;
    r->view.width = p.width;
    r->view.halves = p.pairing == MOD_ROPE_HALVES;
    *out = r;
    return MOD_OK;
}

mod_status mod_rope_destroy(mod_rope* rope) {
    if (!rope) return MOD_OK;
    int device = rope->device;                       // the current one, where it is another
    (void)hipGetDevice(&device);
    if (device != rope->device) (void)hipSetDevice(rope->device);
    const hipError_t e = hipDeviceSynchronize();
    (void)hipFree(rope->table);
    if (device != rope->device) (void)hipSetDevice(device);
    delete rope;
    if (e != hipSuccess) return hip_fail(e, "synchronise before destroy");
    return MOD_OK;
}

mod_status mod_rope_fwd(const mod_rope* rope, const mod_shape* shape, const void* x, const mod_strides* x_strides,
                        void* y, const mod_strides* y_strides, int first, const int32_t* starts, void* stream) {
    return rope_call(rope, shape, x, x_strides, y, y_strides, first, starts, false, stream);
}

mod_status mod_rope_bwd(const mod_rope* rope, const mod_shape* shape, const void* dy, const mod_strides* dy_strides,
                        void* dx, const mod_strides* dx_strides, int first, const int32_t* starts, void* stream) {
    return rope_call(rope, shape, dy, dy_strides, dx, dx_strides, first, starts, true, stream);
}

int mod_cache_blocks(const mod_cache_shape* shape) {
    if (check_cache_shape(shape) != MOD_OK) return 0;
    return (shape->capacity + shape->block - 1) / shape->block;
}

mod_status mod_cache_write(const mod_cache_shape* shape, const mod_cache* cache, const void* k,
                           const mod_strides* k_strides, const void* v, const mod_strides* v_strides, int L,
                           int first, const int32_t* starts, const int32_t* counts, void* stream) {
    moddit::CacheView view{};
    mod_status st = make_view(shape, cache, &view);
    if (st != MOD_OK) return st;
    if (!k || !v) return fail(MOD_ERR_INVALID_ARG, "k and v must not be NULL");
    st = check_range(shape, L, first, starts);
    if (st != MOD_OK) return st;
    moddit::Strided ks{}, vs{};
    st = make_strided(k, k_strides, shape->B, shape->H, L, shape->d, false, "k", &ks);
    if (st != MOD_OK) return st;
    st = make_strided(v, v_strides, shape->B, shape->H, L, shape->d, false, "v", &vs);
    if (st != MOD_OK) return st;
    const hipError_t e = moddit::launch_cache_write(view, ks, vs, L, first, starts, counts,
                                                    static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "cache write launch");
    return MOD_OK;
}

mod_status mod_cache_read(const mod_cache_shape* shape, const mod_cache* cache, void* k, const mod_strides* k_strides,
                          void* v, const mod_strides* v_strides, int L, int first, const int32_t* starts,
                          const int32_t* counts, void* stream) {
    moddit::CacheView view{};
    mod_status st = make_view(shape, cache, &view);
    if (st != MOD_OK) return st;
    if (!k && !v) return fail(MOD_ERR_INVALID_ARG, "k and v must not both be NULL");
    st = check_range(shape, L, first, starts);
    if (st != MOD_OK) return st;
    moddit::Strided ks{}, vs{};
    st = make_strided(k, k_strides, shape->B, shape->H, L, shape->d, true, "k", &ks);
    if (st != MOD_OK) return st;
    st = make_strided(v, v_strides, shape->B, shape->H, L, shape->d, true, "v", &vs);
    if (st != MOD_OK) return st;
    const hipError_t e = moddit::launch_cache_read(view, ks, vs, L, first, starts, counts,
                                                   static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "cache read launch");
    return MOD_OK;
}

size_t mod_cache_attn_workspace_bytes(const mod_cache_shape* shape, int Hq, int Lq, int max_len) {
    if (check_attn(shape, Hq, Lq, max_len) != MOD_OK) return 0;
    moddit::CacheAttnPlan plans[2];
    return plan_attn(shape, Hq, Lq, max_len, plans);
}

mod_status mod_cache_attn_plan(const mod_cache_shape* shape, int Hq, int Lq, int max_len, int lists, int* rows,
                               int* parts) {
    const mod_status st = check_attn(shape, Hq, Lq, max_len);
    if (st != MOD_OK) return st;
    if (!rows || !parts) return fail(MOD_ERR_INVALID_ARG, "rows and parts must not be NULL");
    moddit::CacheAttnPlan plans[2];
    plan_attn(shape, Hq, Lq, max_len, plans);
    *rows = plans[lists != 0].rows;
    *parts = plans[lists != 0].C;
    return MOD_OK;
}

mod_status mod_cache_attn_fwd(const mod_cache_shape* shape, const mod_cache* cache, const void* q, int Hq, int Lq,
                              int max_len, const int32_t* kv_len, const int32_t* kv_idx, const int32_t* kv_cnt,
                              float scale, void* o, float* lse, void* workspace, size_t ws_bytes, void* stream) {
    moddit::CacheView view{};
    mod_status st = make_view(shape, cache, &view);
    if (st != MOD_OK) return st;
    st = check_attn(shape, Hq, Lq, max_len);
    if (st != MOD_OK) return st;
    if (!q || !o) return fail(MOD_ERR_INVALID_ARG, "q and o must not be NULL");
    st = check_aligned(q, "q");
    if (st == MOD_OK) st = check_aligned(o, "o");
    if (st != MOD_OK) return st;
    if (max_len == 0) kv_idx = kv_cnt = nullptr;      // no blocks, no lists
    if (!kv_idx != !kv_cnt) return fail(MOD_ERR_INVALID_ARG, "kv_idx and kv_cnt must both be given, or neither");
    if (!(scale >= 0.0f) || !std::isfinite(scale))
        return fail(MOD_ERR_INVALID_ARG, "scale must be finite and >= 0");
    moddit::CacheAttnPlan plans[2];
    const size_t need = plan_attn(shape, Hq, Lq, max_len, plans);
    if (need > 0) {
        if (!workspace || ws_bytes < need)
            return fail(MOD_ERR_INVALID_ARG, "workspace of at least %zu bytes needed (got %zu%s)", need, ws_bytes,
                        workspace ? "" : ", NULL");
        st = check_aligned(workspace, "workspace");
        if (st != MOD_OK) return st;
    }
    const float sc = scale == 0.0f ? (float)(1.0 / std::sqrt((double)shape->d)) : scale;
    const hipError_t e = moddit::launch_cache_attn(plans[kv_idx != nullptr], view, static_cast<const uint16_t*>(q),
                                                   Hq, Lq, max_len, kv_len, kv_idx, kv_cnt, sc,
                                                   static_cast<uint16_t*>(o), lse, workspace,
                                                   static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "cache attention launch");
    return MOD_OK;
}

}  // extern "C"
