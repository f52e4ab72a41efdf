// Layout of the paged 8-bit key/value cache, shared by what writes it and what reads it.
//
// The unit is a group: 16 consecutive tokens of one head.  K codes of a group lie as [hd / 16 chunks][16 tokens][16 dims], V codes as [hd dims][16 tokens]
// (16 * hd bytes each, groups of a page's head one after the other): the 32-row operand fragments of the matrix instructions are then runs of 256
// and 512 consecutive bytes of memory, K with 16 dims and V with 16 tokens per lane, and nothing has to be transposed by who reads.
#pragma once
#include "common.h"
#include "../../include/chunkflow.h"

constexpr int KV_GROUP = 16;          // tokens that share a power of two

// What kernels see of a cf_kv_cache.
struct KvView {
    uint8_t* k;
    uint8_t* v;
    uint8_t* scales;
    const int32_t* table;
    int32_t n_pages, heads, table_stride, n_seqs;
    int32_t page_shift;               // log2 of tokens per page
    int32_t capacity;                 // tokens that a row of the table has pages for
};

// Index of a page's group of head h with position p,
__device__ __forceinline__ int kv_group_of(const KvView& c, int page, int h, int p) {
    return ((page * c.heads + h) << (c.page_shift - 4)) + ((p & ((1 << c.page_shift) - 1)) >> 4);
}
// and that of position p (a multiple of KV_GROUP below capacity) of sequence b and head h; -1 where the table names no page.
__device__ __forceinline__ int kv_group(const KvView& c, int b, int h, int p) {
    const int page = c.table[(int64_t)b * c.table_stride + (p >> c.page_shift)];
    if ((uint32_t)page >= (uint32_t)c.n_pages) return -1;
    return kv_group_of(c, page, h, p);
}

// Offsets of a ragged batch are the caller's device memory: whatever they hold, rows stay within [0, n_rows).
__device__ __forceinline__ int kv_clamped(int x, int lo, int hi) { return min(max(x, lo), hi); }

// LDS accesses of this wave before and after it keep their order.
__device__ __forceinline__ void lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Host checks of a cache; NULL if it is in order.
inline const char* kv_bad(const cf_kv_cache* c) {
    if (!c) return "null cache";
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
    if (c->page_tokens < KV_GROUP || c->page_tokens > 4096 || (c->page_tokens & (c->page_tokens - 1))) return "page_tokens must be a power of two from 16 to 4096";
    if (c->heads < 1 || c->heads > 4096 || c->n_pages < 1 || c->n_seqs < 0 || c->table_width < 1) return "sizes must be positive";
    if ((int64_t)c->n_pages * c->heads * (c->page_tokens / KV_GROUP) > 0x7fffffff) return "more than 2^31 groups of 16 tokens";
    if ((int64_t)c->table_width * c->page_tokens > 0x7fffffff - 4096) return "a sequence would pass 2^31 tokens";
    if (!c->k || !c->v || !c->scales || !c->table) return "null pointer";
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16 || (uintptr_t)c->scales % 2 || (uintptr_t)c->table % 4) return "k and v must be 16-byte aligned, scales 2, table 4";
    return nullptr;
}
inline KvView kv_view(const cf_kv_cache& c) {
    int shift = 4;
    while (1 << shift < c.page_tokens) ++shift;
    return {c.k, c.v, c.scales, c.table, c.n_pages, c.heads, c.table_width, c.n_seqs, shift, c.table_width << shift};
}
