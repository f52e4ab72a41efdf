// Rotary positions with several axes: tables for the block path, and q and k turned directly.  Both are bound by HBM.
#include <cmath>

#include "context.h"
#include "rope.h"
#include "rows.h"

namespace {

// ---------------------------------------------------------------------------------------------
// tables: a lane has four pairs of a row
template <int HD>
__global__ __launch_bounds__(256) void rope_tables_kernel(cf_rope r, const int32_t* __restrict__ pos, int64_t n, float* __restrict__ cs, float* __restrict__ sn) {
    constexpr int LANES = HD / 8;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int p0 = threadIdx.x % LANES * 4;
    if (row >= n) return;
    floatx4 c, s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float ce, se;
        rope_sincos(r.turn[p0 + e], pos[row * r.n_axes + r.axis[p0 + e]], ce, se);
        c[e] = ce;
        s[e] = se;
    }
    *(floatx4*)(cs + row * (HD / 2) + p0) = c;
    *(floatx4*)(sn + row * (HD / 2) + p0) = s;
}

// ---------------------------------------------------------------------------------------------
// q and k: a lane has the same eight columns (four pairs) of several heads of a row, whose angles it computes once.
struct RopeArgs {
    cf_rope r;
    cf_rope_operand op[2];
    const int32_t* pos;
    int64_t n;
    int heads;               // of both operands
    int rows_per_wg;
    float sign;              // of the sines: -1 turns back
};

// FAR: past the caches, for operands that these cannot hold until somebody reads them again.  (Compiled for itself: of two accesses behind a
// condition that differ in this alone the compiler makes one.)
template <bool FAR, class V>
__device__ __forceinline__ V get(const V* p) {
    if constexpr (FAR) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool FAR, class V>
__device__ __forceinline__ void put(V* p, V v) {
    if constexpr (FAR) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool FAR, class T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        const bf16x8 v = get<FAR>((const bf16x8*)p);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    } else {
        const floatx4 a = get<FAR>((const floatx4*)p), b = get<FAR>((const floatx4*)(p + 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = a[e];
            x[4 + e] = b[e];
        }
    }
}
template <bool FAR, class T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (bf16)x[e];
        put<FAR>((bf16x8*)p, v);
    } else {
        put<FAR>((floatx4*)p, floatx4{x[0], x[1], x[2], x[3]});
        put<FAR>((floatx4*)(p + 4), floatx4{x[4], x[5], x[6], x[7]});
    }
}

template <class T, int HD, bool FAR>
__global__ __launch_bounds__(256) void rope_apply_kernel(RopeArgs a) {
    constexpr int LANES = HD / 8, SLOTS = 256 / LANES;
    const int slot = threadIdx.x / LANES, col = threadIdx.x % LANES * 8;
    const int per_row = a.rows_per_wg > 1 ? a.heads : SLOTS;
    const int64_t row = (int64_t)blockIdx.x * a.rows_per_wg + slot / per_row;
    if (slot / per_row >= a.rows_per_wg || row >= a.n) return;
    float c[4], s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        rope_sincos(a.r.turn[col / 2 + e], a.pos[row * a.r.n_axes + a.r.axis[col / 2 + e]], c[e], s[e]);
        s[e] *= a.sign;
    }
    for (int h = slot % per_row; h < a.heads; h += SLOTS) {
        const bool second = h >= a.op[0].heads;
        const cf_rope_operand& op = a.op[second];
        const int hh = second ? h - a.op[0].heads : h;
        float x[8];
        load8<FAR>((const T*)op.x + row * op.x_row + hh * op.x_head + col, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) rope_turn(x[2 * e], x[2 * e + 1], c[e], s[e]);
        store8<FAR>((T*)op.y + row * op.y_row + hh * op.y_head + col, x);
    }
}

template <class T>
void launch(const RopeArgs& a, bool far, dim3 grid, hipStream_t s) {
    if (a.r.head_dim == 128) {
        if (far) hipLaunchKernelGGL((rope_apply_kernel<T, 128, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((rope_apply_kernel<T, 128, false>), grid, dim3(256), 0, s, a);
    } else {
        if (far) hipLaunchKernelGGL((rope_apply_kernel<T, 64, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((rope_apply_kernel<T, 64, false>), grid, dim3(256), 0, s, a);
    }
}

}  // namespace

extern "C" int cf_rope_plan(int32_t head_dim, int32_t n_axes, const int32_t* axis_pairs, const double* theta, cf_rope* out) {
    if (!axis_pairs || !theta || !out) return cf_fail(nullptr, CF_ERR_ARG, "rope_plan: null argument");
    if (head_dim != 64 && head_dim != 128) return cf_fail(nullptr, CF_ERR_ARG, "rope_plan: head_dim %d is not 64 or 128", head_dim);
    if (n_axes < 1 || n_axes > CF_ROPE_AXES) return cf_fail(nullptr, CF_ERR_ARG, "rope_plan: %d axes, 1 to %d are possible", n_axes, CF_ROPE_AXES);
    cf_rope r = {};
    r.head_dim = head_dim;
    r.n_axes = n_axes;
    for (int a = 0; a < n_axes; ++a) {
        if (axis_pairs[a] < 1 || axis_pairs[a] > head_dim / 2 - r.n_pairs)
            return cf_fail(nullptr, CF_ERR_ARG, "rope_plan: axis %d has %d pairs; every axis has one and all together at most head_dim / 2", a, axis_pairs[a]);
        if (!(theta[a] >= 1.0) || !std::isfinite(theta[a])) return cf_fail(nullptr, CF_ERR_ARG, "rope_plan: theta of axis %d is not a finite number from 1 on", a);
        for (int j = 0; j < axis_pairs[a]; ++j) {
            // 64 bits of mantissa: the rounding to 2^-64 turns is the only one that counts
            const long double turns = powl((long double)theta[a], -(long double)j / axis_pairs[a]) / 6.283185307179586476925286766559L;
            r.axis[r.n_pairs] = (uint8_t)a;
            r.turn[r.n_pairs++] = (uint64_t)(turns * 18446744073709551616.0L + 0.5L);
        }
    }
    *out = r;
    return CF_OK;
}

extern "C" int cf_rope_tables(const cf_rope* rope, const int32_t* pos, int64_t n, float* cos_out, float* sin_out, void* stream) {
    if (const char* bad = rope_bad(rope)) return cf_fail(nullptr, CF_ERR_ARG, "rope_tables: %s", bad);
    const int rows = 2048 / rope->head_dim;
    if (n < 0 || n > MOST_WGS * rows) return cf_fail(nullptr, CF_ERR_ARG, "rope_tables: %lld rows", (long long)n);
    if (n == 0) return CF_OK;
    if (!pos || !cos_out || !sin_out) return cf_fail(nullptr, CF_ERR_ARG, "rope_tables: null operand");
    if (((uintptr_t)cos_out | (uintptr_t)sin_out) % 16 || (uintptr_t)pos % 4) return cf_fail(nullptr, CF_ERR_ARG, "rope_tables: tables must be 16-byte aligned, positions 4");
    const int64_t bytes = n * (rope->head_dim / 2) * 4, pos_bytes = n * rope->n_axes * 4;
    auto meet = [](const void* p, int64_t n, const void* q, int64_t m) { return (const char*)p < (const char*)q + m && (const char*)q < (const char*)p + n; };
    if (meet(cos_out, bytes, sin_out, bytes) || meet(cos_out, bytes, pos, pos_bytes) || meet(sin_out, bytes, pos, pos_bytes)) return cf_fail(nullptr, CF_ERR_ARG, "rope_tables: operands overlap");
    const dim3 grid((unsigned)((n + rows - 1) / rows));
    if (rope->head_dim == 128) hipLaunchKernelGGL(rope_tables_kernel<128>, grid, dim3(256), 0, (hipStream_t)stream, *rope, pos, n, cos_out, sin_out);
    else hipLaunchKernelGGL(rope_tables_kernel<64>, grid, dim3(256), 0, (hipStream_t)stream, *rope, pos, n, cos_out, sin_out);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf_fail(nullptr, CF_ERR_HIP, "rope_tables launch: %s", hipGetErrorString(e));
}

extern "C" int cf_rope_apply(const cf_rope* rope, const int32_t* pos, int64_t n, const cf_rope_operand* ops, int32_t n_ops, int32_t dtype, int32_t inverse,
                             void* stream) {
    if (const char* bad = rope_bad(rope)) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: %s", bad);
    if (dtype != CF_BF16 && dtype != CF_F32) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: type %d is neither CF_BF16 nor CF_F32", dtype);
    if (!ops || n_ops < 1 || n_ops > 2) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: one or two operands");
    if (n < 0 || n > MOST_WGS) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: %lld rows", (long long)n);
    if (n == 0) return CF_OK;
    if (!pos || (uintptr_t)pos % 4) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: null or misaligned positions");
    const int es = dtype == CF_BF16 ? 2 : 4, hd = rope->head_dim;
    RopeArgs a = {};
    Rows in[2], out[2];
    for (int i = 0; i < n_ops; ++i) {
        const cf_rope_operand& o = ops[i];
        if (!o.x || !o.y) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: null operand");
        if (o.heads < 1 || o.heads > 4096) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: %d heads", o.heads);
        for (const int64_t st : {o.x_row, o.x_head, o.y_row, o.y_head})
            if (st < 0 || st > (int64_t)1 << 40 || st * es % 16) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: strides must be multiples of 16 bytes and not negative");
        if (((uintptr_t)o.x | (uintptr_t)o.y) % 16) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: operands must be 16-byte aligned");
        in[i] = {o.x, n, o.x_row, o.heads, o.x_head, hd, es};
        out[i] = {o.y, n, o.y_row, o.heads, o.y_head, hd, es};
        if (!out[i].apart()) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: outputs overlap one another");
        const bool in_place = o.x == o.y && o.x_row == o.y_row && o.x_head == o.y_head;
        if (!in_place && rows_meet(in[i], out[i])) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: an output overlaps its input; in place means the same pointer and strides");
        a.op[i] = o;
        a.heads += o.heads;
    }
    if (n_ops == 2)
        for (int i = 0; i < 2; ++i)
            if (rows_meet(out[i], in[1 - i]) || rows_meet(out[i], out[1 - i])) return cf_fail(nullptr, CF_ERR_ARG, "rope_apply: an output overlaps the other operand");
    a.r = *rope;
    a.pos = pos;
    a.n = n;
    a.sign = inverse ? -1.0f : 1.0f;
    // 13640 rows x 48 heads of 128 in bf16, 335 MB: 68.7 us (4.9 TB/s; a copy 5.1), through the caches 72.6
    const bool far = n * a.heads * hd * es > 64ll << 20;           // (the L2 caches hold 32 MB)
    const int slots = 2048 / hd;
    a.rows_per_wg = a.heads < slots ? slots / a.heads : 1;
    const dim3 grid((unsigned)((n + a.rows_per_wg - 1) / a.rows_per_wg));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == CF_BF16) launch<bf16>(a, far, grid, st);
    else launch<float>(a, far, grid, st);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf_fail(nullptr, CF_ERR_HIP, "rope_apply launch: %s", hipGetErrorString(e));
}
