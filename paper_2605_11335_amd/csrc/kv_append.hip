// New tokens into a paged 8-bit cache: keys turned by their positions on the way, keys and values as e4m3 codes with one power of two per
// group of 16 tokens (kv_cache.h).  Bound by HBM: 2 or 4 bytes per element in, 1 out.
//
// A power of two costs e4m3 no precision (its own exponent takes up what a finer factor would), and codes move to a larger one exactly unless they
// become subnormal; so a group that is filled token by token keeps the codes it has, moved where a later token needs a larger power.
// The power is taken from what goes in, not from what comes out of the rotation: |a| + |b| bounds a pair under any angle and is the
// same number in any arithmetic, so that neither positions nor the last bit of a sine decide over it.
#include <algorithm>
#include <type_traits>

#include "context.h"
#include "kv_cache.h"
#include "rope.h"
#include "rows.h"

namespace {

constexpr int E_LEAST = -100;          // a group's least power: |x| below 2^-110 becomes zero

struct AppendArgs {
    KvView c;
    cf_rope r;
    const void *k, *v;
    int64_t k_row, k_head, v_row, v_head;
    const int32_t *cu, *lens, *pos;
    int32_t n_tokens;
};

// The least e with m <= 224 * 2^e; m is half of what has to fit under 448 * 2^e (|a| + |b| itself could pass the fp32 range).
__device__ __forceinline__ int power_for(float m) {
    if (!(m > 0.0f)) return E_LEAST;
    const int e = __builtin_amdgcn_frexp_expf(m) - 8 + (__builtin_amdgcn_frexp_mantf(m) > 0.875f);
    return max(e, E_LEAST);
}
// The largest of values that are not negative, as bits: an infinity or a NaN among them comes out, as a number of at least NOT_FINITE.
constexpr uint32_t NOT_FINITE = 0x7f800000u;
__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}
// Codes of two values times 2^-e.  Products are exact and at most 448 (1 + 2^-22), which rounds to 448; a NaN keeps its code.
__device__ __forceinline__ uint32_t codes2(float a, float b, float down) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a * down, b * down, 0, false) & 0xffffu;
}
// four codes at a power larger by `up`
__device__ __forceinline__ uint32_t moved(uint32_t w, int up) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(a[0], -up), __builtin_ldexpf(a[1], -up), 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(b[0], -up), __builtin_ldexpf(b[1], -up), r, true);
    return (uint32_t)r;
}
// A pair of dims as it lies in memory: a word of two bf16, or two floats.
typedef float floatx2 __attribute__((ext_vector_type(2)));
template <class T>
using Pair = std::conditional_t<sizeof(T) == 2, uint32_t, floatx2>;
__device__ __forceinline__ void unpack(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack(floatx2 w, float& a, float& b) {
    a = w[0];
    b = w[1];
}

// A wave has one group at a time, all of it: lane = a pair of dims, for 16 tokens (8 with 64-wide heads, whose other half of the lanes has the other 8).
// Groups of a launch: sequence b, whose tokens are rows [cu[b], cu[b+1]), touches at most (n - 1) / 16 + 2 of them and owns the items from
// S(b) = cu[b] / 16 + 2 b on, so that an item finds its sequence by a search of S and no order among items is needed.
template <class T, int HD, bool ROPE>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
    constexpr int PAIRS = HD / 2, TPL = PAIRS / 4, STEP = 16 * 16 + 16;       // tokens per lane; a chunk's place in LDS
    __shared__ __attribute__((aligned(16))) uint8_t stage[4][HD / 16 * STEP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int item = blockIdx.x, B = a.c.n_seqs;
    // the last sequence that begins at or before the item, and its sizes: all that the search needs and finds comes with one access per 64 sequences
    int b = -1, start = 0, end = 0, held = 0;
    for (int base = 0; base < B; base += 64) {
        const int i = min(base + lane, B - 1);
        const int c0 = a.cu[i], c1 = a.cu[i + 1], l = a.lens[i];
        const int before = __popcll(__ballot(base + lane < B && (kv_clamped(c0, 0, a.n_tokens) >> 4) + 2 * i <= item));
        if (before == 0) break;
        b = base + before - 1;
        start = __builtin_amdgcn_readlane(c0, before - 1);
        end = __builtin_amdgcn_readlane(c1, before - 1);
        held = __builtin_amdgcn_readlane(l, before - 1);
        if (before < 64) break;
    }
    if (b < 0) return;
    start = kv_clamped(start, 0, a.n_tokens);
    const int n = kv_clamped(end, start, a.n_tokens) - start, len = kv_clamped(held, 0, a.c.capacity);
    const int nth = item - ((start >> 4) + 2 * b);
    const int64_t first = ((int64_t)(len >> 4) + nth) << 4;
    if (nth < 0 || first >= (int64_t)len + n || first >= a.c.capacity) return;
    const int p0 = (int)first, lo = max(len - p0, 0), hi = (int)min((int64_t)16, min((int64_t)len + n, (int64_t)a.c.capacity) - p0);      // new slots
    if (lo >= hi) return;
    const int page = a.c.table[(int64_t)b * a.c.table_stride + (p0 >> a.c.page_shift)];               // (rows are asked for before it is there)
    const int pair = lane % PAIRS, s0 = lane / PAIRS * TPL;
    const int64_t row0 = start + (p0 - len);                                   // of slot 0; slots in [lo, hi) have a row

    Pair<T> k_raw[TPL], v_raw[TPL];
    const bool full = lo == 0 && hi == 16;
    auto load = [&](const void* from, int64_t stride, int64_t head, int h, Pair<T> (&raw)[TPL]) __attribute__((always_inline)) {
        const T* const at = (const T*)from + row0 * stride + h * head + 2 * pair;
        if (full) {
            const T* p = at + s0 * stride;                                     // (one pointer from row to row: 16 of them would be kept in registers)
            asm volatile("" : "+v"(p));
#pragma unroll
            for (int t = 0; t < TPL; ++t) raw[t] = __builtin_nontemporal_load((const Pair<T>*)(p + t * stride));
        } else {                                                               // slots without a new token repeat one that has
#pragma unroll
            for (int t = 0; t < TPL; ++t) raw[t] = *(const Pair<T>*)(at + kv_clamped(s0 + t, lo, hi - 1) * stride);
        }
    };
    // The power of a group whose new tokens' pairs are x, y: of |x| + |y| if they are turned, of the larger one else; no less than `was`.
    // What is not finite takes no part, and becomes NaN.
    auto power = [&](float (&x)[TPL], float (&y)[TPL], auto turned, int was) __attribute__((always_inline)) {
        constexpr bool SUM = decltype(turned)::value;
        auto bits = [](float v) { return __float_as_uint(v) & 0x7fffffffu; };
        auto of = [&](float u, float v) { return SUM ? bits(0.5f * fabsf(u) + 0.5f * fabsf(v)) : max(bits(u), bits(v)); };
        uint32_t m = 0;
#pragma unroll
        for (int t = 0; t < TPL; ++t) m = max(m, of(x[t], y[t]));
        m = wave_max(m);
        if (m >= NOT_FINITE) {
            m = 0;
#pragma unroll
            for (int t = 0; t < TPL; ++t) {
                const bool fx = bits(x[t]) < NOT_FINITE, fy = bits(y[t]) < NOT_FINITE;
                if (SUM) m = max(m, fx && fy ? of(x[t], y[t]) : 0u);
                else m = max(m, max(fx ? bits(x[t]) : 0u, fy ? bits(y[t]) : 0u));
                x[t] = fx ? x[t] : __uint_as_float(0x7fc00000u);
                y[t] = fy ? y[t] : __uint_as_float(0x7fc00000u);
            }
            m = wave_max(m);
        }
        return max(power_for(SUM ? __uint_as_float(m) : 0.5f * __uint_as_float(m)), was);
    };
    const int step = 4 * gridDim.y;
    int h = blockIdx.y * 4 + wave;
    if (h < a.c.heads) {
        load(a.k, a.k_row, a.k_head, h, k_raw);
        load(a.v, a.v_row, a.v_head, h, v_raw);
    }
    float cs[TPL], sn[TPL];
    if constexpr (ROPE) {
        const uint64_t turn = a.r.turn[pair];
        const int axis = a.r.axis[pair];
#pragma unroll
        for (int t = 0; t < TPL; ++t) {
            const int slot = kv_clamped(s0 + t, lo, hi - 1);
            rope_sincos(turn, a.pos[(row0 + slot) * a.r.n_axes + axis], cs[t], sn[t]);
        }
    }
    if ((uint32_t)page >= (uint32_t)a.c.n_pages) return;
    for (; h < a.c.heads; h += step) {
        const int g = kv_group_of(a.c, page, h, p0);
        uint8_t* const scale = a.c.scales + 2 * (int64_t)g;
        uint8_t* const kg = a.c.k + (int64_t)g * (16 * HD);
        uint8_t* const vg = a.c.v + (int64_t)g * (16 * HD);
        int was_k = E_LEAST, was_v = E_LEAST;
        if (lo > 0) {                                                          // tokens that were there: their power at least
            const uint32_t was = *(const uint16_t*)scale;
            was_k = (int)(was & 255u) - 127;
            was_v = (int)(was >> 8) - 127;
        }
        {
            float x[TPL], y[TPL];
#pragma unroll
            for (int t = 0; t < TPL; ++t) unpack(k_raw[t], x[t], y[t]);
            if (h + step < a.c.heads) load(a.k, a.k_row, a.k_head, h + step, k_raw);        // the next head's, while this one's are worked on
            const int e = power(x, y, std::bool_constant<ROPE>{}, was_k), up = lo > 0 ? e - was_k : 0;
            const float down = __builtin_ldexpf(1.0f, -e);
            // through LDS, from two dims of many tokens to 16 dims of one
            uint8_t* const my = stage[wave];
#pragma unroll
            for (int t = 0; t < TPL; ++t) {
                if constexpr (ROPE) rope_turn(x[t], y[t], cs[t], sn[t]);
                *(uint16_t*)(my + (pair >> 3) * STEP + (s0 + t) * 16 + (pair & 7) * 2) = (uint16_t)codes2(x[t], y[t], down);
            }
            lds_order();
#pragma unroll
            for (int i = 0; i < HD / 64; ++i) {
                const int at = i * 64 + lane, chunk = at >> 4, slot = at & 15;
                uint32x4 w = *(const uint32x4*)(my + chunk * STEP + slot * 16);
                if (slot >= lo && slot < hi) {
                    *(uint32x4*)(kg + at * 16) = w;
                } else if (slot < lo && up > 0) {
                    w = *(const uint32x4*)(kg + at * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = moved(w[j], up);
                    *(uint32x4*)(kg + at * 16) = w;
                }
            }
            lds_order();                                                       // the next head's codes go to the same place
            if (lane == 0) scale[0] = (uint8_t)(e + 127);
        }
        {
            float x[TPL], y[TPL];
#pragma unroll
            for (int t = 0; t < TPL; ++t) unpack(v_raw[t], x[t], y[t]);
            if (h + step < a.c.heads) load(a.v, a.v_row, a.v_head, h + step, v_raw);
            const int e = power(x, y, std::bool_constant<false>{}, was_v), up = lo > 0 ? e - was_v : 0;
            const float down = __builtin_ldexpf(1.0f, -e);
            // a lane's two dims of its tokens as they lie in memory; what a partly filled group holds besides stays
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                uint32_t* const p = (uint32_t*)(vg + (2 * pair + d) * 16 + s0);
                const float* const v = d ? y : x;
                uint32_t w[TPL / 4];
#pragma unroll
                for (int i = 0; i < TPL / 4; ++i) w[i] = codes2(v[4 * i], v[4 * i + 1], down) | codes2(v[4 * i + 2], v[4 * i + 3], down) << 16;
                if (lo > 0 || hi < 16) {
#pragma unroll
                    for (int i = 0; i < TPL / 4; ++i) {
                        const uint32_t old = p[i], low = up > 0 ? moved(old, up) : old;
                        uint32_t r = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int slot = s0 + 4 * i + j;
                            r |= (slot >= hi ? old : slot >= lo ? w[i] : low) & 255u << (8 * j);
                        }
                        w[i] = r;
                    }
                }
                if constexpr (TPL == 16) *(uint32x4*)p = uint32x4{w[0], w[1], w[2], w[3]};
                else *(uint32x2*)p = uint32x2{w[0], w[1]};
            }
            if (lane == 0) scale[1] = (uint8_t)(e + 127);
        }
    }
}

template <class T, int HD>
void launch(const AppendArgs& a, bool rope, dim3 grid, hipStream_t s) {
    if (rope) hipLaunchKernelGGL((kv_append_kernel<T, HD, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv_append_kernel<T, HD, false>), grid, dim3(256), 0, s, a);
}

}  // namespace

extern "C" int cf_kv_append(const cf_kv_cache* cache, const cf_kv_new* x, void* stream) {
    if (const char* bad = kv_bad(cache)) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: %s", bad);
    if (!x) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: null tokens");
    if (x->dtype != CF_BF16 && x->dtype != CF_F32) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: type %d is neither CF_BF16 nor CF_F32", x->dtype);
    if (x->n_tokens < 0) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: %d tokens", x->n_tokens);
    if (x->n_tokens == 0 || cache->n_seqs == 0) return CF_OK;
    if (!x->k || !x->v || !x->cu || !x->lens) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: null operand");
    if (((uintptr_t)x->k | (uintptr_t)x->v) % 16 || ((uintptr_t)x->cu | (uintptr_t)x->lens | (uintptr_t)x->pos) % 4)
        return cf_fail(nullptr, CF_ERR_ARG, "kv_append: k and v must be 16-byte aligned, offsets, lengths and positions 4");
    const int es = x->dtype == CF_BF16 ? 2 : 4;
    for (const int64_t st : {x->k_row, x->k_head, x->v_row, x->v_head})
        if (st < 0 || st > (int64_t)1 << 40 || st * es % 16) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: strides must be multiples of 16 bytes and not negative");
    if (x->rope) {
        if (const char* bad = rope_bad(x->rope)) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: rotation: %s", bad);
        if (x->rope->head_dim != cache->head_dim) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: the plan turns %d-wide heads, the cache has %d", x->rope->head_dim, cache->head_dim);
        if (!x->pos) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: a rotation without positions");
    }
    const int64_t items = x->n_tokens / 16 + 2ll * cache->n_seqs;
    if (items > MOST_WGS) return cf_fail(nullptr, CF_ERR_ARG, "kv_append: too many tokens and sequences");
    AppendArgs a = {};
    a.c = kv_view(*cache);
    if (x->rope) a.r = *x->rope;
    a.k = x->k; a.v = x->v;
    a.k_row = x->k_row; a.k_head = x->k_head; a.v_row = x->v_row; a.v_head = x->v_head;
    a.cu = x->cu; a.lens = x->lens; a.pos = x->pos;
    a.n_tokens = x->n_tokens;
    // Four heads at a time per workgroup.  Where there are groups enough to fill the chip, one workgroup has all heads of its group, and the angles are
    // computed once: 20460 tokens x 12 heads 44.4 us, with three workgroups for the heads of a group 55.0.
    const int64_t quads = (cache->heads + 3) / 4, slices = std::max<int64_t>(1, std::min(quads, 1024 / items));
    const dim3 grid((unsigned)items, (unsigned)slices);
    hipStream_t s = (hipStream_t)stream;
    if (x->dtype == CF_BF16) {
        if (cache->head_dim == 128) launch<bf16, 128>(a, x->rope != nullptr, grid, s);
        else launch<bf16, 64>(a, x->rope != nullptr, grid, s);
    } else {
        if (cache->head_dim == 128) launch<float, 128>(a, x->rope != nullptr, grid, s);
        else launch<float, 64>(a, x->rope != nullptr, grid, s);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf_fail(nullptr, CF_ERR_HIP, "kv_append launch: %s", hipGetErrorString(e));
}
