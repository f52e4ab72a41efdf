// Softmax attention of ragged queries over a paged 8-bit cache (kv_cache.h).  Each group's codes are multiplied by its power of two; keys past a
// sequence's length, of pages that the table does not name and, causal, behind the query take no part, whatever their codes are.
//
// A wave has one query of one head and goes through the keys 64 at a time, a lane to each: scores, running maximum and sum of the softmax, then a
// lane per output dim over the 64 weights.
#include <cmath>

#include "context.h"
#include "kv_cache.h"

namespace {

struct AttendArgs {
    KvView c;
    const bf16* q;
    bf16* o;
    int64_t q_row, q_head, o_row, o_head;
    const int32_t *cu, *lens;
    int32_t n_tokens, heads, times;        // times: query heads per key head
    int32_t causal;
    float c2;                              // scale * log2(e)
};

__device__ __forceinline__ float code_at(uint32_t w, int byte) { return __builtin_amdgcn_cvt_f32_fp8((int)(w >> (8 * byte)), 0); }

template <int HD>
__global__ __launch_bounds__(64) void kv_attend_kernel(AttendArgs a) {
    __shared__ float sq[HD], sp[64];
    const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y, h = head / a.times, B = a.c.n_seqs;
    int b = -1;
    for (int base = 0; base < B; base += 64) {
        const int i = base + lane;
        b += __popcll(__ballot(i < B && a.cu[i] <= row));
    }
    if (b < 0 || row >= a.cu[b + 1]) return;
    const int start = kv_clamped(a.cu[b], 0, a.n_tokens), n = kv_clamped(a.cu[b + 1], start, a.n_tokens) - start;
    const int len = kv_clamped(a.lens[b], 0, a.c.capacity);
    const int end = a.causal ? min(len, len - n + (row - start) + 1) : len;          // keys [0, end) are seen
    for (int d = lane; d < HD; d += 64) sq[d] = (float)a.q[(int64_t)row * a.q_row + head * a.q_head + d];
    __syncthreads();
    float m = -INFINITY, l = 0.0f, o[HD / 64] = {};
    for (int k0 = 0; k0 < end; k0 += 64) {
        const int key = k0 + lane, g = key < end ? kv_group(a.c, b, h, key & ~15) : -1;
        float s = -INFINITY;
        if (g >= 0) {
            const uint8_t* const p = a.c.k + (int64_t)g * (16 * HD) + (key & 15) * 16;
            s = 0.0f;
            for (int c = 0; c < HD / 16; ++c) {
                const uint32x4 w = *(const uint32x4*)(p + c * 256);
                for (int e = 0; e < 16; ++e) s = fmaf(code_at(w[e / 4], e & 3), sq[c * 16 + e], s);
            }
            s = __builtin_ldexpf(s, (int)a.c.scales[2 * (int64_t)g] - 127) * a.c2;
        }
        float hi = s;
        for (int off = 32; off; off >>= 1) hi = fmaxf(hi, __shfl_xor(hi, off));
        const float m_new = fmaxf(m, hi);
        const bool none = m_new == -INFINITY;
        const float f = none ? 1.0f : exp2f(m - m_new), pj = s == -INFINITY ? 0.0f : exp2f(s - (none ? 0.0f : m_new));      // (NaN comes through)
        float sum = pj;
        for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off);
        l = l * f + sum;
        m = m_new;
        sp[lane] = pj;
        __syncthreads();
        for (int i = 0; i < HD / 64; ++i) o[i] *= f;
        for (int t = 0; t < 4; ++t) {
            const int g2 = __shfl(g, t * 16);
            if (g2 < 0) continue;
            const int e2 = (int)a.c.scales[2 * (int64_t)g2 + 1] - 127;
            for (int i = 0; i < HD / 64; ++i) {
                const uint32x4 w = *(const uint32x4*)(a.c.v + (int64_t)g2 * (16 * HD) + (i * 64 + lane) * 16);
                float x = 0.0f;
                for (int e = 0; e < 16; ++e)
                    if (k0 + t * 16 + e < end) x = fmaf(sp[t * 16 + e], code_at(w[e / 4], e & 3), x);
                o[i] += __builtin_ldexpf(x, e2);
            }
        }
        __syncthreads();
    }
    for (int i = 0; i < HD / 64; ++i) a.o[(int64_t)row * a.o_row + head * a.o_head + i * 64 + lane] = (bf16)(l == 0.0f ? 0.0f : o[i] / l);
}

const char* query_bad(const cf_kv_cache* c, const cf_kv_query* x) {
    if (!x) return "null queries";
    if (x->heads < 1 || x->heads > 65535 || x->heads % c->heads) return "query heads must be a multiple of the cache's heads";
    if (x->n_tokens < 0 || x->max_q < 0) return "sizes must not be negative";
    return nullptr;
}

}  // namespace

extern "C" int cf_kv_attention_workspace(const cf_kv_cache* cache, const cf_kv_query* x, uint64_t* bytes) {
    if (const char* bad = kv_bad(cache)) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention_workspace: %s", bad);
    if (const char* bad = query_bad(cache, x)) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention_workspace: %s", bad);
    if (!bytes) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention_workspace: null result");
    *bytes = 0;
    return CF_OK;
}

extern "C" int cf_kv_attention(const cf_kv_cache* cache, const cf_kv_query* x, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (const char* bad = kv_bad(cache)) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention: %s", bad);
    if (const char* bad = query_bad(cache, x)) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention: %s", bad);
    if (!(x->scale > 0.0f) || !std::isfinite(x->scale)) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention: the scale must be positive and finite");
    if (x->n_tokens == 0 || cache->n_seqs == 0) return CF_OK;
    if (!x->q || !x->o || !x->cu || !x->lens) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention: null operand");
    if (((uintptr_t)x->q | (uintptr_t)x->o) % 16 || ((uintptr_t)x->cu | (uintptr_t)x->lens) % 4)
        return cf_fail(nullptr, CF_ERR_ARG, "kv_attention: q and o must be 16-byte aligned, offsets and lengths 4");
    for (const int64_t st : {x->q_row, x->q_head, x->o_row, x->o_head})
        if (st < 0 || st > (int64_t)1 << 40 || st % 8) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention: strides must be multiples of 16 bytes and not negative");
    AttendArgs a = {};
    a.c = kv_view(*cache);
    a.q = (const bf16*)x->q; a.o = (bf16*)x->o;
    a.q_row = x->q_row; a.q_head = x->q_head; a.o_row = x->o_row; a.o_head = x->o_head;
    a.cu = x->cu; a.lens = x->lens;
    a.n_tokens = x->n_tokens; a.heads = x->heads; a.times = x->heads / cache->heads;
    a.causal = x->causal != 0;
    a.c2 = x->scale * 1.4426950408889634f;
    const dim3 grid((unsigned)x->n_tokens, (unsigned)x->heads);
    if (cache->head_dim == 128) hipLaunchKernelGGL(kv_attend_kernel<128>, grid, dim3(64), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(kv_attend_kernel<64>, grid, dim3(64), 0, (hipStream_t)stream, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf_fail(nullptr, CF_ERR_HIP, "kv_attention launch: %s", hipGetErrorString(e));
}
