// Softmax attention of ragged queries over a paged 8-bit cache (kv_cache.h).  Each group's codes are multiplied by its power of two; keys past a
// sequence's length, of pages that the table does not name and, causal, behind the query take no part, whatever their codes are.
#include <algorithm>
#include <atomic>
#include <chrono>
#include <cmath>

#include "../../include/chunkflow_diag.h"
#include "context.h"
#include "kv_tile.h"
#include "rows.h"

namespace {

// ---------------------------------------------------------------------------------------------
// Few columns: at most 32 for a (sequence, key head), single tokens above all.  Bound by reading the cache once.  Operand fragments come straight from
// memory into registers, each wave its own tiles, K of the next tile on its way while this one's second half is computed and V behind it: up to
// 16 KB in flight per wave.  All key tiles of the batch laid end to end are cut into equal parts, one per workgroup, wherever sequences and heads
// begin and end; a column tile whose keys lie in several parts is joined by kv_join_kernel.
constexpr int FEW_WAVES = 4, FEW_LEAST = 5 * KV_TILE;           // FEW_LEAST: weight that is worth a workgroup

// One column tile of 32 over key tiles [t0, t1), of which each wave takes every FEW_WAVES-th: its own result.  Tiles that every column sees whole
// come first, one after the other without a break in the loads; then those with an end, a hole in the page table or a power that is none, if there are any.
// FAR: codes go past the caches, where each is read once and there are more of them than the caches hold.
template <int HD, bool FAR>
__device__ __forceinline__ void few_sweep(const AttendArgs& a, const KvSeq& q, int h, int c, int t0, int t1, const bf16x8 (*sq)[64], KvState<HD>& st) {
    constexpr int KJ = HD / 32, DT = HD / 32, GB = 16 * HD, STEP = FEW_WAVES;
    const int lane = threadIdx.x & 63, lj = lane & 31, lg = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KvColumn col = kv_column(a, q, h, 32 * c + lj);
    const int end_least = __builtin_amdgcn_readlane(col.end, 0), end_most = __builtin_amdgcn_readlane(col.end, min(32, q.n * a.times - 32 * c) - 1);
    t1 = min(t1, (max(end_most, 0) + KV_TILE - 1) / KV_TILE);
    st.clear();
    // Groups are looked up for 16 tiles at a time, t, t + STEP, ...: lane l has group l & 3 of the (l >> 2)-th.
    auto where = [&](int t) __attribute__((always_inline)) {
        const int64_t p = (int64_t)(t + STEP * (lane >> 2)) * KV_TILE + 16 * (lane & 3);
        return p < q.len ? kv_group(a.c, q.b, h, (int)p) : -1;
    };
    auto powers = [&](int g) __attribute__((always_inline)) { return g < 0 ? 0x7f7fu : (uint32_t)*(const uint16_t*)(a.c.scales + 2 * (int64_t)g); };
    auto tiles = [&](int t) __attribute__((always_inline)) {                     // bit 4 i: there is an i-th one
        const int m = (t1 - t + STEP - 1) / STEP;
        return 0x1111111111111111ull & (m >= 16 ? ~0ull : (1ull << 4 * max(m, 0)) - 1);
    };
    auto odd_ones = [&](int t, int g, uint32_t p) __attribute__((always_inline)) {
        const bool plain = g >= 0 && (p & 255u) != 255u && p >> 8 != 255u && (t + STEP * (lane >> 2)) * KV_TILE + 16 * (lane & 3) + 16 <= end_least;
        uint64_t m = __ballot(!plain);
        m |= m >> 2;
        return (m | m >> 1) & tiles(t);
    };
    const int slot = (lj & 3) + 4 * (lj >> 3), kg = (lj >> 2) & 1;
    uint32x4 kq[2][KJ], vq[2][DT];
    uint32_t ksc[2], vsc[2];
    auto codes = [](const uint8_t* p) __attribute__((always_inline)) {
        if constexpr (FAR) return __builtin_nontemporal_load((const uint32x4*)p);
        else return *(const uint32x4*)p;
    };
    auto load_k = [&](int g, uint32_t p, int nth) __attribute__((always_inline)) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const int from = nth * 4 + 2 * mt + kg;
            ksc[mt] = __shfl(p, from) & 255u;
            const uint8_t* const at = a.c.k + (int64_t)max(__shfl(g, from), 0) * GB + lg * 256 + slot * 16;
#pragma unroll
            for (int j = 0; j < KJ; ++j) kq[mt][j] = codes(at + j * 512);
        }
    };
    auto load_v = [&](int g, uint32_t p, int nth) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int from = nth * 4 + 2 * s + lg;
            vsc[s] = __shfl(p, from) >> 8;
            const uint8_t* const at = a.c.v + (int64_t)max(__shfl(g, from), 0) * GB + lj * 16;
#pragma unroll
            for (int d = 0; d < DT; ++d) vq[s][d] = codes(at + d * 512);
        }
    };
    floatx16 s[2];
    bf16x8 pf[4];
    auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int v = 0; v < 16; ++v) s[mt][v] = 0.0f;
        const float f0 = kv_power(ksc[0]), f1 = kv_power(ksc[1]);
#pragma unroll
        for (int k = 0; k < 2 * KJ; ++k) {
            const bf16x8 qf = sq[k][lane];
            s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_wide(kq[0][k >> 1][2 * (k & 1)], kq[0][k >> 1][2 * (k & 1) + 1], f0), qf, s[0], 0, 0, 0);
            s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_wide(kq[1][k >> 1][2 * (k & 1)], kq[1][k >> 1][2 * (k & 1) + 1], f1), qf, s[1], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);             // (conversions far ahead of their MFMAs would only hold registers)
        }
    };
    auto values = [&]() __attribute__((always_inline)) {
        const float f0 = kv_power(vsc[0]), f1 = kv_power(vsc[1]);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_wide(vq[ks >> 1][d][2 * (ks & 1)], vq[ks >> 1][d][2 * (ks & 1) + 1], ks >> 1 ? f1 : f0), pf[ks], st.o[d], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
    };

    int t = t0 + wave, odd_from = t1, odd_to = 0;          // the groups' 16 tiles begin at t; of those with odd tiles, the first and the last
    if (t < t1) {
        int g = where(t), t_next = t + 16 * STEP, g_next = where(t_next);
        uint32_t p = powers(g), p_next = 0;
        bool looked = false;                               // p_next is that of g_next
        uint64_t odd = odd_ones(t, g, p), todo = tiles(t) & ~odd;
        auto next = [&]() __attribute__((always_inline)) {
            for (;;) {
                if (odd) {
                    odd_from = min(odd_from, t);
                    odd_to = t;
                    odd = 0;
                }
                if (todo) break;
                if (t_next >= t1) return -1;
                p = looked ? p_next : powers(g_next);
                g = g_next;
                t = t_next;
                t_next += 16 * STEP;
                g_next = where(t_next);
                looked = false;
                odd = odd_ones(t, g, p);
                todo = tiles(t) & ~odd;
            }
            const int nth = __builtin_ctzll(todo) >> 2;
            todo &= todo - 1;
            if (!looked && !(todo >> 32)) {                // its first half is done: the table's entries are there by now
                p_next = powers(g_next);
                looked = true;
            }
            return nth;
        };
        int nth = next();
        if (nth >= 0) {
            load_k(g, p, nth);
            load_v(g, p, nth);
        }
        while (nth >= 0) {
            scores();
            nth = next();
            if (nth >= 0) load_k(g, p, nth);
            __builtin_amdgcn_sched_barrier(0);
            kv_softmax<HD>(st, s, a.c2, pf, false);
            __builtin_amdgcn_sched_barrier(0);
            values();
            if (nth >= 0) load_v(g, p, nth);
        }
    }
    for (t = odd_from; t <= odd_to; t += 16 * STEP) {
        const int g = where(t);
        const uint32_t p = powers(g);
        for (uint64_t odd = odd_ones(t, g, p); odd; odd &= odd - 1) {
            const int nth = __builtin_ctzll(odd) >> 2, k0 = (t + STEP * nth) * KV_TILE;
            load_k(g, p, nth);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const bool none = ksc[mt] == 255u;
                ksc[mt] = none ? 127u : ksc[mt];
#pragma unroll
                for (int j = 0; j < KJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) kq[mt][j][e] = none ? 0x7f7f7f7fu : kq[mt][j][e];
            }
            scores();
            __builtin_amdgcn_sched_barrier(0);
            int rel[2], held[2];           // of the lane's 16 keys of a half: how many its column sees, how many there are (S^T's registers and V's tokens are the same group)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool there = __shfl(g, nth * 4 + 2 * i + lg) >= 0;
                const int from = k0 + 32 * i + 16 * lg;
                held[i] = there ? min(max(q.len - from, 0), 16) : 0;
                rel[i] = there ? min(max(col.end - from, 0), 16) : 0;
            }
            kv_mask(s, rel);
            kv_softmax<HD>(st, s, a.c2, pf, false);
            __builtin_amdgcn_sched_barrier(0);
            load_v(g, p, nth);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool none = vsc[i] == 255u;
                vsc[i] = none || held[i] == 0 ? 127u : vsc[i];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int b = min(max(held[i] - 4 * w, 0), 4);
                    const uint32_t keep = b == 4 ? ~0u : (1u << (8 * b)) - 1u;
#pragma unroll
                    for (int d = 0; d < DT; ++d) vq[i][d][w] = (none ? 0x7f7f7f7fu : vq[i][d][w]) & keep;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            uint32_t nans = 0;
#pragma unroll
            for (int i = 0; i < 2 * DT * 4; ++i) nans |= kv_perhaps_nan(vq[i / (DT * 4)][i / 4 % DT][i & 3]);
            if (__any((nans & 0x80808080u) != 0)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    floatx16 hits;
#pragma unroll
                    for (int v = 0; v < 16; ++v) hits[v] = 0.0f;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        const uint32_t lo = vq[ks >> 1][d][2 * (ks & 1)], hi = vq[ks >> 1][d][2 * (ks & 1) + 1];
                        const uint32_t n_lo = kv_nan_codes(lo), n_hi = kv_nan_codes(hi);
                        vq[ks >> 1][d][2 * (ks & 1)] = kv_without_nan(lo, n_lo);
                        vq[ks >> 1][d][2 * (ks & 1) + 1] = kv_without_nan(hi, n_hi);
                        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_wide(kv_ones(n_lo), kv_ones(n_hi), 1.0f), kv_seen(rel[ks >> 1], ks & 1), hits, 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    kv_spread_nan<HD>(st, d, hits);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            values();
        }
    }
}

template <int HD, bool FAR>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void kv_attend_few_kernel(AttendArgs a) {
    constexpr int DT = HD / 32;
    __shared__ __attribute__((aligned(16))) float so[FEW_WAVES][DT * 4][64][4];
    __shared__ float sm[FEW_WAVES][32][2];
    __shared__ bf16x8 sq[HD / 16][64];                      // query fragments, the same for all waves
    const int lane = threadIdx.x & 63, lj = lane & 31, lg = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = blockIdx.x;
    const KvScan<32> scan(a, 0);
    const KvShares shares(kv_total<32>(a, scan), gridDim.x, a.whole ? 1 : FEW_LEAST);
    KvSeq q = {};
    KvPiece p = {};
    const bool any = w < shares.wgs && shares.total > 0;
    int64_t f = any ? shares.begin(w) : 0;
    const int64_t f1 = any ? shares.begin(w + 1) : 0;
    if (f < f1) q = kv_find<32>(a, f, scan);
    while (f < f1) {
        const int64_t q_end = q.first + q.head() * a.c.heads;
        const int64_t to = min(f1, q_end);
        for (KvPiece n = kv_piece<32>(a, q, f, f1); f < to;) {
            p = n;
            if (p.next < to) n = kv_next<32>(a, q, p, f1);
            const int h = p.h, c = p.c;
            const KvColumn col = kv_column(a, q, h, 32 * c + lj);
            for (int k = wave; k < HD / 16; k += FEW_WAVES)
                sq[k][lane] = *(const bf16x8*)(a.q + (int64_t)col.row * a.q_row + (int64_t)col.head * a.q_head + 32 * (k >> 1) + 16 * lg + 8 * (k & 1));
            __syncthreads();
            KvState<HD> st;
            few_sweep<HD, FAR>(a, q, h, c, p.t0, p.t1, sq, st);
            const float l = kv_sum_halves(st.l);
#pragma unroll
            for (int i = 0; i < DT * 4; ++i)
                *(floatx4*)so[wave][i][lane] = floatx4{st.o[i / 4][i % 4 * 4], st.o[i / 4][i % 4 * 4 + 1], st.o[i / 4][i % 4 * 4 + 2], st.o[i / 4][i % 4 * 4 + 3]};
            if (lg == 0) {
                sm[wave][lj][0] = st.mc;
                sm[wave][lj][1] = l;
            }
            __syncthreads();
            float m = kNoRef, sum = 0.0f, k[FEW_WAVES];
#pragma unroll
            for (int x = 0; x < FEW_WAVES; ++x) m = fmaxf(m, sm[x][lj][0]);
#pragma unroll
            for (int x = 0; x < FEW_WAVES; ++x) {
                k[x] = __builtin_amdgcn_exp2f(sm[x][lj][0] - m);
                sum = fmaf(sm[x][lj][1], k[x], sum);
            }
            const int at = 2 * w + p.from_start;            // the share's first piece may begin inside a column tile, its last may end inside one
            const float inv = kv_inverse(sum);
            for (int i = wave; i < DT * 4; i += FEW_WAVES) {
                floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < FEW_WAVES; ++x) {
                    const floatx4 y = *(const floatx4*)so[x][i][lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = fmaf(y[e], k[x], v[e]);
                }
                const int d = 8 * i + 4 * lg;               // i = 4 dt + v / 4
                if (!col.mine) continue;
                if (p.whole) {
                    bf16x4 r;
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] = (bf16)(v[e] * inv);
                    *(bf16x4*)(a.o + (int64_t)col.row * a.o_row + (int64_t)col.head * a.o_head + d) = r;
                } else {
                    *(floatx4*)(a.part_o + ((int64_t)at * 32 + lj) * HD + d) = v;
                }
            }
            if (!p.whole && col.mine && wave == 0 && lg == 0) *(float2*)(a.part_ml + ((int64_t)at * 32 + lj) * 2) = make_float2(m, sum);
            __syncthreads();
            f = p.next;
        }
        if (f < f1) q = kv_find<32>(a, f, KvScan<32>(a, 0));
    }
    if (!a.whole) kv_leave_cut<32>(a, shares, w, q, p);
}

// ---------------------------------------------------------------------------------------------
// Many columns: a workgroup of NW waves has 32 NW columns of a (sequence, key head) and goes through its share of the keys, tiles of 64 that all its
// waves use.  Bound by the matrix cores and, nearly as much, by reading fragments from LDS.  Codes become bf16 once per workgroup, on their way into
// LDS: a lane's 16 bytes are two fragments' worth (kv_tile.h), stored as the fragments lie, so that a fragment read is 1 KiB in order and
// nothing has to be swizzled.  Page t + 3, codes of t + 2 are on their way from memory and t + 1 is converted into the other buffer while tile t is computed.
struct ManyFlags {
    uint32_t held;                                     // tokens of each of the tile's groups, a byte each
    uint32_t nan;                                      // t + 1 where a value of tile t was NaN
};
template <int HD, int NW>
struct ManyShared {
    bf16x8 k[2][2][HD / 16][64], v[2][4][HD / 32][64];
    char rows[NW][64 * HD];                            // a wave's query rows, as many_row has them, on their way to fragments
    // of tiles that not every column sees whole:
    uint16_t nan_of[2][4 * HD];                        // which of a V chunk's 16 tokens were NaN
    ManyFlags flags[2];
};

// A value that the compiler takes for a new one: addresses made from it are computed where they are used, and not kept in registers all along.
__device__ __forceinline__ int anew(int x) {
    asm volatile("" : "+v"(x));
    return x;
}
// Where 16-byte chunk c of a column's row of head_dim values is kept: rows read or written a chunk per lane meet all banks.
template <int HD>
__device__ __forceinline__ int many_row(int col, int c) { return col * (2 * HD) + ((c ^ (col & (HD / 8 - 1))) << 4); }

// The columns whose rows a lane has a chunk of, of a wave's 32: every (512 / HD)-th, from the lane's first one on.  Where a column's query or output lies takes a
// division and products of 64 bits; from one to the next it is one of two steps.
template <int HD, class T>
struct ManyRow {
    int r, head, last, times, step_heads;
    T* row;                                            // of column r, or of one before it if there is no column r
    int64_t step, wrap;
    __device__ __forceinline__ ManyRow(const AttendArgs& a, const KvSeq& q, int h, int col0, int ln, T* base, int64_t row_stride, int64_t head_stride)
        : r(ln / (HD / 8)), last(q.n * a.times - col0 - 1), times(a.times), step_heads(a.step_heads) {
        const KvColumn c = kv_column(a, q, h, col0 + r);
        head = c.head - h * a.times;
        row = base + (int64_t)c.row * row_stride + (int64_t)c.head * head_stride;
        step = a.step_rows * row_stride + a.step_heads * head_stride;
        wrap = step + row_stride - a.times * head_stride;
    }
    __device__ __forceinline__ void next() {
        r += 512 / HD;
        head += step_heads;
        const bool over = head >= times;
        head -= over ? times : 0;
        const int64_t by = over ? wrap : step;
        row += r <= last ? by : 0;
    }
};

// What is on its way for the workgroup's next piece while it finishes one.
template <int HD, int NW>
struct ManyAhead {
    static constexpr int CHUNKS = 4 * HD, NT = 64 * NW;                         // 16-byte chunks of a tile's K or V
    static constexpr int PER = CHUNKS >= NT ? CHUNKS / NT : 1;                  // of those and of V's, a lane has PER
    int page1[PER];                                    // pages of its second tile
    uint32_t pw[PER];                                  // the first tile's powers,
    int held[PER];                                     // how many tokens of its groups there are,
    uint32x4 kr[PER], vr[PER];                         // and its codes
};

constexpr int AGENT = 16;                              // cache policy of a buffer access: sc1, past the XCD's L2
__device__ __forceinline__ __amdgpu_buffer_rsrc_t agent_rsrc(const void* base, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00020000); }

// Piece p of sequence q.  holes: whether a page of the sequence is not there; -1: find out.  ready: its query rows are in LDS, its first codes on their way (x).  more: piece n of the same sequence comes next, and is made ready.
template <int HD, int NW>
__device__ __forceinline__ void many_sweep(const AttendArgs& a, const KvSeq& q, const KvPiece& p, int& holes, bool ready, const KvPiece& n, bool more,
                                           ManyShared<HD, NW>& sh, ManyAhead<HD, NW>& x, KvState<HD>& st) {
    constexpr int KS = HD / 16, DT = HD / 32, NT = 64 * NW, GB = 16 * HD, CHUNKS = 4 * HD, PER = ManyAhead<HD, NW>::PER;
    constexpr bool BOTH = CHUNKS >= NT;                                         // else half of the lanes have K, half V
    static_assert(CHUNKS % NT == 0 || 2 * CHUNKS == NT, "");
    const int tid = threadIdx.x, lane = tid & 63, lj = lane & 31, lg = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = p.t0, t1 = p.t1;
    const int col0 = 32 * NW * p.c + 32 * wave, cols = min(32, q.n * a.times - col0);          // (cols <= 0: a wave without a column only copies)
    const KvColumn col = kv_column(a, q, p.h, col0 + lj);
    const int32_t* const table = a.c.table + (int64_t)q.b * a.c.table_stride;
    // ---- copies.  Chunk x of K or V: group x / HD of the tile, 16 bytes x % HD of it.
    const bool has_k = BOTH || tid < CHUNKS, has_v = BOTH || tid >= CHUNKS;
    const int x0 = BOTH ? tid : tid % CHUNKS;
    const int last = q.len - 1, page_mask = (1 << a.c.page_shift) - 1;
    int page[PER];                                     // of the tile after the one in flight
    auto& pw = x.pw;
    auto& held = x.held;
    auto& kr = x.kr;
    auto& vr = x.vr;
    auto look_up = [&](int t, int (&page)[PER]) __attribute__((always_inline)) {          // (past the end: some page of the sequence's)
#pragma unroll
        for (int i = 0; i < PER; ++i) page[i] = table[min(t * KV_TILE + 16 * ((i * NT + x0) / HD), last) >> a.c.page_shift];
    };
    auto fetch = [&](int h, int t, const int (&page)[PER]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = i * NT + x0, p = t * KV_TILE + 16 * (x / HD);
            const bool there = (uint32_t)page[i] < (uint32_t)a.c.n_pages;
            held[i] = there ? min(max(q.len - p, 0), 16) : 0;
            const int g = there ? ((page[i] * a.c.heads + h) << (a.c.page_shift - 4)) + ((p & page_mask) >> 4) : 0;
            pw[i] = *(const uint16_t*)(a.c.scales + 2 * (int64_t)g);
            const uint32_t r = (x % HD) * 16;
            if (has_k) kr[i] = *(const uint32x4*)(a.c.k + (int64_t)g * GB + r);
            if (has_v) vr[i] = *(const uint32x4*)(a.c.v + (int64_t)g * GB + r);
        }
    };
    // this wave's query rows from memory into LDS, past the registers: a lane fetches the chunk whose place it fills
    auto ask_queries = [&](const KvPiece& p) __attribute__((always_inline)) {
        const int ln = anew(lane), col0 = 32 * NW * p.c + 32 * wave;
        ManyRow<HD, const bf16> at(a, q, p.h, col0, ln, a.q, a.q_row, a.q_head);
#pragma unroll
        for (int i = 0; i < HD / 16; ++i, at.next()) {
            const int ch = ln % (HD / 8) ^ (at.r & (HD / 8 - 1));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(at.row + ch * 8),
                                             (__attribute__((address_space(3))) void*)(sh.rows[wave] + i * 1024), 16, 0, 0);
        }
    };
    auto landed = []() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
    if (tid < 2) sh.flags[tid].nan = 0;
    // tiles [t0, t_plain) are seen whole by every column of the workgroup and have all their pages
    const int least = kv_end(a, q, (int)((uint32_t)(32 * NW * p.c) / (uint32_t)a.times));
    int t_plain = max(t0, min(t1, max(least, 0) / KV_TILE));
    bool hole = false;
    if (!ready) {
        look_up(t0, page);
        look_up(t0 + 1, x.page1);
        ask_queries(p);
        fetch(p.h, t0, page);
        if (holes < 0)
            for (int i = anew(tid); i <= last >> a.c.page_shift; i += NT) hole |= (uint32_t)table[i] >= (uint32_t)a.c.n_pages;
        landed();
    }
    bf16x8 qf[KS];
    {
        const int ln = anew(lane), col_l = ln & 31, half = ln >> 5;
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[k] = *(const bf16x8*)(sh.rows[wave] + many_row<HD>(col_l, 4 * (k >> 1) + 2 * half + (k & 1)));
    }
    if (holes < 0) holes = __syncthreads_or(hole);
    else if (!holes) __syncthreads();                  // (either way:) the flags are cleared, and what the buffers held before has been read
    if (holes) {                                       // somewhere in the sequence: here?
        hole = false;
        for (int i = (t0 * KV_TILE >> a.c.page_shift) + tid; i <= (t_plain * KV_TILE - 1) >> a.c.page_shift; i += NT) hole |= (uint32_t)table[i] >= (uint32_t)a.c.n_pages;
        if (__syncthreads_or(hole)) t_plain = t0;
    }
    auto convert = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = i * NT + x0, grp = x / HD, r = x % HD;
            uint32_t pk = pw[i] & 255u, pv = pw[i] >> 8;
            if (t >= t_plain || __any(pk == 255u || pv == 255u)) {
                const bool nk = pk == 255u, nv = pv == 255u;
                pk = nk || held[i] == 0 ? 127u : pk;
                pv = nv || held[i] == 0 ? 127u : pv;
                uint32_t m = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int b = min(max(held[i] - 4 * w, 0), 4);
                    const uint32_t keep = b == 4 ? ~0u : (1u << (8 * b)) - 1u;
                    if (has_k) kr[i][w] = nk ? 0x7f7f7f7fu : kr[i][w];
                    if (has_v) {
                        uint32_t v = (nv ? 0x7f7f7f7fu : vr[i][w]) & keep;
                        if (t >= t_plain) {
                            const uint32_t nans = kv_nan_codes(v);
                            v = kv_without_nan(v, nans);
                            m |= ((nans >> 7) * 0x10204080u >> 28) << (4 * w);      // four bits side by side
                        }
                        vr[i][w] = v;
                    }
                }
                if (t >= t_plain) {
                    if (has_v) {
                        sh.nan_of[buf][x] = (uint16_t)m;
                        if (m) sh.flags[buf].nan = (uint32_t)t + 1;
                    }
                    if (has_k && r == 0) ((uint8_t*)&sh.flags[buf].held)[grp] = (uint8_t)held[i];
                }
            }
            if (has_k) {
                const int slot = r & 15, ch = r >> 4, row = (slot & 3) | (grp & 1) << 2 | (slot >> 2) << 3;
                bf16x8* const to = &sh.k[0][grp >> 1][ch & ~1][row + 32 * (ch & 1)] + buf * (2 * KS * 64);
                const float f = kv_power(pk);
                to[0] = kv_wide(kr[i][0], kr[i][1], f);
                to[64] = kv_wide(kr[i][2], kr[i][3], f);
            }
            if (has_v) {
                bf16x8* const to = &sh.v[0][grp & ~1][r >> 5][(r & 31) + 32 * (grp & 1)] + buf * (4 * DT * 64);
                const float f = kv_power(pv);
                to[0] = kv_wide(vr[i][0], vr[i][1], f);
                to[DT * 64] = kv_wide(vr[i][2], vr[i][3], f);
            }
        }
    };
    // while a tile is computed: the next one into LDS, the one after on its way
    auto copies = [&](int t, int buf) __attribute__((always_inline)) {
        if (t + 1 < t1) convert(t + 1, 1 - buf);
        if (t + 2 < t1) {
            fetch(p.h, t + 2, page);
            look_up(t + 3, page);
        }
    };
    floatx16 s[2];
    bf16x8 pf[4];
    // S^T = K Q^T: MFMA i has half i & 1 of the keys and k-step i >> 1; fragments run four reads ahead
    auto scores = [&](int buf) __attribute__((always_inline)) {
        bf16x8 kf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) kf[i] = sh.k[buf][i & 1][i >> 1][lane];
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            floatx16 z;
#pragma unroll
            for (int v = 0; v < 16; ++v) z[v] = 0.0f;
            s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i & 3], qf[i >> 1], i < 2 ? z : s[i & 1], 0, 0, 0);
            if (i + 4 < 2 * KS) kf[i & 3] = sh.k[buf][i & 1][(i + 4) >> 1][lane];
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 2 * KS - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    // O^T += V^T P^T: MFMA i has k-step i / DT and dims 32 (i % DT) ...; the first fragments are read before the softmax
    bf16x8 vf[4];
    auto first_values = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) vf[i] = sh.v[buf][i / DT][i % DT][lane];
    };
    auto values = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4 * DT; ++i) {
            st.o[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i & 3], pf[i / DT], st.o[i % DT], 0, 0, 0);
            if (i + 4 < 4 * DT) vf[i & 3] = sh.v[buf][(i + 4) / DT][(i + 4) % DT][lane];
        }
#pragma unroll
        for (int i = 0; i < 4 * DT - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 1);
    };
    convert(t0, 0);
    fetch(p.h, t0 + 1, x.page1);
    look_up(t0 + 2, page);
    st.clear();
    __syncthreads();
    int next_page[PER];
    if (more) {                                        // (every wave has its queries in registers)
        look_up(n.t0, next_page);
        look_up(n.t0 + 1, x.page1);
        ask_queries(n);
    }
    // tile t is in buffer (t - t0) & 1
    auto plain = [&](int t, int buf, bool fresh) __attribute__((always_inline)) {
        copies(t, buf);
        __builtin_amdgcn_sched_barrier(0);
        scores(buf);
        first_values(buf);
        __builtin_amdgcn_sched_barrier(0);
        kv_softmax<HD>(st, s, a.c2, pf, fresh);
        __builtin_amdgcn_sched_barrier(0);
        values(buf);
        __syncthreads();                               // tile t + 1 is in its buffer, that of t is free
    };
    const int end_most = cols > 0 ? __builtin_amdgcn_readlane(col.end, cols - 1) : 0;
    auto any = [&](int t, int buf) __attribute__((always_inline)) {
        copies(t, buf);
        if (t * KV_TILE < end_most) {
            scores(buf);
            int rel[2];
            const uint32_t there = t < t_plain ? 0x10101010u : sh.flags[buf].held;
#pragma unroll
            for (int i = 0; i < 2; ++i) rel[i] = min((int)(there >> (8 * (2 * i + lg)) & 255u), min(max(col.end - (t * KV_TILE + 32 * i + 16 * lg), 0), 16));
            kv_mask(s, rel);
            __builtin_amdgcn_sched_barrier(0);
            kv_softmax<HD>(st, s, a.c2, pf, t == t0);
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_amdgcn_readfirstlane(sh.flags[buf].nan) == (uint32_t)t + 1) {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    floatx16 hits;
#pragma unroll
                    for (int v = 0; v < 16; ++v) hits[v] = 0.0f;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        const uint32_t m = sh.nan_of[buf][(2 * (ks >> 1) + lg) * HD + 32 * d + lj] >> (8 * (ks & 1));
                        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_bits(m), kv_seen(rel[ks >> 1], ks & 1), hits, 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    kv_spread_nan<HD>(st, d, hits);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            first_values(buf);
            values(buf);
        }
        __syncthreads();
    };
    int t = t0;
    if (cols > 0) {
        if (t < t_plain) plain(t++, 0, true);
        for (; t + 2 <= t_plain; t += 2) {             // (buffers known at compile time: addresses are a lane's offset and a constant)
            plain(t, 1, false);
            plain(t + 1, 0, false);
        }
        if (t < t_plain) plain(t++, 1, false);
    }
    for (; t < t1; ++t) any(t, (t - t0) & 1);
    if (more) {
        landed();                                      // the queries
        fetch(n.h, n.t0, next_page);
    }
}

constexpr int MANY_LEAST = 8 * KV_TILE;                // weight that is worth a workgroup
template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_attend_many_kernel(AttendArgs a) {
    constexpr int DT = HD / 32, COLS = 32 * NW;
    __shared__ ManyShared<HD, NW> sh;
    const int lane = threadIdx.x & 63, lj = lane & 31, lg = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KvScan<COLS> scan(a, 0);
    const KvShares shares(kv_total<COLS>(a, scan), gridDim.x, a.whole ? 1 : MANY_LEAST);
    KvSeq q = {};
    KvPiece p = {};
    const bool any = (int)blockIdx.x < shares.wgs && shares.total > 0;
    const int w = any ? (int)xcd_contiguous_id(blockIdx.x, shares.wgs) : (int)blockIdx.x;         // neighbours in the work, which share keys, on one XCD
    int64_t f = any ? shares.begin(w) : 0;
    const int64_t f1 = any ? shares.begin(w + 1) : 0;
    bool joined = false;                               // the last piece, with what follows it
    if (f < f1) q = kv_find<COLS>(a, f, scan);
    while (f < f1) {
        const int64_t q_end = min(f1, q.first + q.head() * a.c.heads);
        int holes = -1;
        ManyAhead<HD, NW> ahead;
        KvPiece n = kv_piece<COLS>(a, q, f, f1);
        for (bool ready = false; f < q_end;) {
            p = n;
            bool more = p.next < q_end;
            if (more) n = kv_next<COLS>(a, q, p, f1);
            more = more && n.t0 < n.t1;
            KvState<HD> st;
            if (p.t0 < p.t1) {
                many_sweep<HD, NW>(a, q, p, holes, ready, n, more, sh, ahead, st);
                ready = more;
            } else {
                st.clear();
                ready = false;
            }
            const int col0 = COLS * p.c + 32 * wave, cols = min(32, q.n * a.times - col0);
            float l = kv_sum_halves(st.l);
            // A column tile of two pieces: the share after this one began with the other, so that it is nearly always there; if so, it is joined here, in the
            // order and with the roundings of kv_join_kernel.
            if (cols > 0 && p.from_start && !p.whole && p.end <= shares.begin(w + 2) &&
                __hip_atomic_load(a.sent + (w + 1) * NW + wave, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.epoch) {
                asm volatile("" ::: "memory");
                const int64_t at = (int64_t)(2 * (w + 1)) * NW + wave;
                const __amdgpu_buffer_rsrc_t part = agent_rsrc(a.part_o + at * (HD / 8) * 256, HD / 8 * 1024), part_ml = agent_rsrc(a.part_ml + at * 64, 256);
                const float2 ml = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(part_ml, (anew(lane) & 31) * 8, 0, AGENT));
                const float m = fmaxf(fmaxf(kNoRef, st.mc), ml.x), k0 = __builtin_amdgcn_exp2f(st.mc - m), k1 = __builtin_amdgcn_exp2f(ml.x - m);
                l = fmaf(ml.y, k1, l * k0);
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) {
                    const floatx4 y = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(part, anew(lane) * 16, i * 1024, AGENT));
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.o[i / 4][i % 4 * 4 + e] = fmaf(y[e], k1, __fmul_rn(st.o[i / 4][i % 4 * 4 + e], k0));
                }
                joined = true;
            }
            if (cols > 0 && (p.whole || joined)) {
                // rows of 2 head_dim bytes, 16 per lane: stored by dims of a lane, an instruction would touch 32 rows.  Past the caches, which have the keys and
                // values that all workgroups share (13640 queries x 512 tokens x 24 heads: 122 us, 129 through them).
                const float inv = kv_inverse(l);
                const int ln = anew(lane), col_l = ln & 31, half = ln >> 5;
                char* const rows = (char*)&sh.k + wave * (64 * HD);            // where tiles were: k and v are as large as the outputs
                static_assert(sizeof(sh.k) + sizeof(sh.v) >= NW * 64 * HD, "");
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) {
                    bf16x4 r;
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] = (bf16)(st.o[i / 4][i % 4 * 4 + e] * inv);
                    *(bf16x4*)(rows + many_row<HD>(col_l, i) + 8 * half) = r;
                }
                lds_order();
                __builtin_amdgcn_sched_barrier(0);
                ManyRow<HD, bf16> to(a, q, p.h, col0, ln, a.o, a.o_row, a.o_head);
#pragma unroll
                for (int i = 0; i < HD / 16; ++i, to.next()) {
                    const int ch = ln % (HD / 8);
                    const bf16x8 x = *(const bf16x8*)(rows + many_row<HD>(to.r, ch));
                    if (to.r < cols) __builtin_nontemporal_store(x, (bf16x8*)(to.row + ch * 8));
                }
                lds_order();
            } else if (cols > 0) {
                const int64_t at = (int64_t)(2 * w + p.from_start) * NW + wave;
                // past this XCD's L2, for the workgroup that may join it within the launch
                const __amdgpu_buffer_rsrc_t part = agent_rsrc(a.part_o + at * (HD / 8) * 256, HD / 8 * 1024), part_ml = agent_rsrc(a.part_ml + at * 64, 256);
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) {
                    const floatx4 v = {st.o[i / 4][i % 4 * 4], st.o[i / 4][i % 4 * 4 + 1], st.o[i / 4][i % 4 * 4 + 2], st.o[i / 4][i % 4 * 4 + 3]};
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint32x4, v), part, anew(lane) * 16, i * 1024, AGENT);
                }
                if (lg == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(uint32x2, make_float2(st.mc, l)), part_ml, lj * 8, 0, AGENT);
                if (!p.from_start) {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // all of it is there
                    if (lane == 0) __hip_atomic_store(a.sent + w * NW + wave, a.epoch, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            }
            f = p.next;
        }
        if (f < f1) q = kv_find<COLS>(a, f, KvScan<COLS>(a, 0));
    }
    if (!a.whole) {
        kv_leave_cut<COLS>(a, shares, w, q, p);
        if (lane == 0) a.joined[w * NW + wave] = joined;
    }
}

// Joins the pieces of the column tiles that shares cut, in order: a workgroup per cut and 32 columns.  Bound by latency: what to join has been left in
// memory by who cut it, and all of a lane's loads are on their way at once.  Few columns of many pieces are read by all lanes, G of them for the same
// four dims of a column, each every G-th piece, and put together in LDS.
template <int HD, int COLS, int LANES>
__global__ __launch_bounds__(LANES) void kv_join_kernel(AttendArgs a) {
    constexpr int QUADS = HD / 4, TIMES = 32 * QUADS / LANES > 1 ? 32 * QUADS / LANES : 1;      // lanes that a column needs; columns x quads per lane
    __shared__ float sm[LANES], part_l[LANES / QUADS * 32];
    __shared__ __attribute__((aligned(16))) floatx4 part[LANES];
    const int tid = threadIdx.x, w0 = blockIdx.x;
    const KvCut cut = a.cuts[w0];
    if (COLS > 32) {                                           // (many columns)
        if (tid == 0) a.sent[(w0 + 1) * (COLS / 32) + blockIdx.y] = 0;
        if (a.joined[w0 * (COLS / 32) + blockIdx.y]) return;
    }
    const int c0 = blockIdx.y * 32, cols = min(32, cut.n * a.times - cut.col0 - c0), pieces = cut.pieces;
    if (pieces == 0 || cols <= 0) return;
    KvSeq q = {};
    q.start = cut.start;
    q.n = cut.n;
    auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * (COLS / 32) + blockIdx.y; };         // of the i-th piece
    auto load = [&](int i, int lj, int quad) {
        return *(const floatx4*)(a.part_o + (COLS == 32 ? (slot(i) * 32 + lj) * HD + 4 * quad : (slot(i) * (HD / 8) + (quad >> 1)) * 256 + (lj + 32 * (quad & 1)) * 4));
    };
    auto store = [&](int lj, int quad, const floatx4& v, float sum) {
        const float inv = kv_inverse(sum);
        const KvColumn col = kv_column(a, q, cut.h, cut.col0 + c0 + lj);
        bf16x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (bf16)(v[e] * inv);
        *(bf16x4*)(a.o + (int64_t)col.row * a.o_row + (int64_t)col.head * a.o_head + 4 * quad) = r;
    };
    // references: 32 columns x LANES / 32
    {
        const int lj = tid & 31;
        float m = kNoRef;
        if (lj < cols)
            for (int i = tid >> 5; i < pieces; i += LANES / 32) m = fmaxf(m, a.part_ml[(slot(i) * 32 + lj) * 2]);
        sm[tid] = m;
        __syncthreads();
        for (int o = LANES / 2; o >= 32; o >>= 1) {
            if (tid < o) sm[tid] = fmaxf(sm[tid], sm[tid + o]);
            __syncthreads();
        }
    }
    int G = 1;                                                 // (two pieces of many columns: as kv_attend_many_kernel joins them, one after the other)
    if (COLS == 32 || pieces > 2)
        while (2 * G * cols * QUADS <= LANES && G < pieces) G *= 2;
    if (G == 1) {
        floatx4 v[TIMES];
        float sum[TIMES];
        int lj[TIMES], quad[TIMES];
#pragma unroll
        for (int k = 0; k < TIMES; ++k) {
            const int x = min(k * LANES + tid, cols * QUADS - 1);           // (past the end: the last one again)
            lj[k] = COLS == 32 ? x / QUADS : x % cols;
            quad[k] = COLS == 32 ? x % QUADS : x / cols;
            v[k] = floatx4{0.f, 0.f, 0.f, 0.f};
            sum[k] = 0.0f;
        }
#pragma unroll 2
        for (int i = 0; i < pieces; ++i) {
            floatx4 y[TIMES];
            float2 ml[TIMES];
#pragma unroll
            for (int k = 0; k < TIMES; ++k) {
                y[k] = load(i, lj[k], quad[k]);
                ml[k] = *(const float2*)(a.part_ml + (slot(i) * 32 + lj[k]) * 2);
            }
#pragma unroll
            for (int k = 0; k < TIMES; ++k) {
                const float f = __builtin_amdgcn_exp2f(ml[k].x - sm[lj[k]]);
                sum[k] = fmaf(ml[k].y, f, sum[k]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k][e] = fmaf(y[k][e], f, v[k][e]);
            }
        }
#pragma unroll
        for (int k = 0; k < TIMES; ++k)
            if (k * LANES + tid < cols * QUADS) store(lj[k], quad[k], v[k], sum[k]);
        return;
    }
    const int lanes = LANES / G, g = tid / lanes, x = tid % lanes;           // lanes: a multiple of 16
    const int lj = COLS == 32 ? x / QUADS : x % cols, quad = COLS == 32 ? x % QUADS : x / cols;
    const bool some = x < cols * QUADS;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.0f;
    if (some) {
#pragma unroll 4
        for (int i = g; i < pieces; i += G) {
            const floatx4 y = load(i, lj, quad);
            const float2 ml = *(const float2*)(a.part_ml + (slot(i) * 32 + lj) * 2);
            const float f = __builtin_amdgcn_exp2f(ml.x - sm[lj]);
            sum = fmaf(ml.y, f, sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(y[e], f, v[e]);
        }
        part[tid] = v;
        if (quad == 0) part_l[g * 32 + lj] = sum;
    }
    __syncthreads();
    if (!some || g > 0) return;
    for (int k = 1; k < G; ++k) {
        const floatx4 y = part[tid + k * lanes];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += y[e];
        sum += part_l[k * 32 + lj];
    }
    store(lj, quad, v, sum);
}

const char* query_bad(const cf_kv_cache* c, const cf_kv_query* x) {
    if (!x) return "null queries";
    if (x->heads < 1 || x->heads > 65535 || x->heads % c->heads) return "query heads must be a multiple of the cache's heads";
    if (x->n_tokens < 0 || x->max_q < 0) return "sizes must not be negative";
    return nullptr;
}

constexpr int FEW_WGS = 512, MANY_WGS = 256;           // two workgroups on each CU, one

// Whether column tiles are left whole, a workgroup to each, and nothing has to be joined.  `tiles`: of the longest sequence the table has room for, which
// is all that the host knows.
// Few columns: as long as all column tiles run at once and their keys, FEW_WAVES tiles at a time, take little longer than shares of them would, and
// nine such steps for the joining.  One query each, 8 key heads, whole / cut: 1 sequence of 2048 tokens 16.1 / 17.0 us, of 2560 18.5 / 17.0; 8 of 2048
// 17.3 / 22.2, of 3584 23.6 / 21.4; 32 of 4096 46.1 / 52.0; 256 of 512 63.4 / 50.5.
bool few_whole(int64_t units, int64_t tiles) {
    const int64_t steps = (tiles + FEW_WAVES - 1) / FEW_WAVES;
    return units <= FEW_WGS && steps <= steps * units / FEW_WGS + 9;
}
// Many: 1.55 us per tile and 9 for the ends of a column tile, in whole rounds of workgroups, against equal shares and 15 us for leaving and joining their
// pieces.  24 heads, whole / cut: 2560 queries x 2048 keys 65 / 75 us, 3584 x 512 43.6 / 46.0, x 1024 67.7 / 62.2, 4608 x 512 43.4 / 50.7, 5461 x 512
// 64 / 55, x 2048 178 / 140, 7168 x 512 64.5 / 66.0, 8448 x 512 85 / 74, 43690 x 512 360 / 333.
bool many_whole(int64_t units, int64_t tiles) {
    const double one = 9.0 + 1.55 * (double)tiles, rounds = (double)((units + MANY_WGS - 1) / MANY_WGS);
    return rounds * one <= (double)units * one / MANY_WGS + 15.0;
}

// Which kernel, by estimates of both (us; us per key tile of a column tile of 32 or 256 columns, all CUs at work, `fill` of the 256 taken).  32 / 8 heads,
// few / many: 1 sequence of 8192 tokens, 64 queries 29 / 39; 8 of 8192, 12 queries each 54 / 53, 24 76 / 54, 64 164 / 82; 32 of 1024, 16 queries 26 / 27,
// 24 38 / 27; 32 of 8192, 8 queries 96 / 142, 16 157 / 145, 64 598 / 271.
bool many_columns(double few_tiles, double many_tiles, double fill) {
    return 10.0 + 2.4e-3 * few_tiles > std::max(32.0, 14.0 + 1e-3 * (3.4 + 4.2 * fill) * many_tiles);
}

struct AttendPlan {
    bool many;                         // kernel with 32 * MANY_WAVES columns per workgroup
    bool whole;                        // a workgroup per column tile
    bool far;                          // few columns: codes past the caches
    int cols, wgs;
    uint64_t ml_offset, cuts_offset, sent_offset, bytes;         // of the workspace
};
constexpr int MANY_WAVES = 8;
const char* attend_plan(const cf_kv_cache* c, const cf_kv_query* x, int form, AttendPlan* p) {
    const int64_t times = x->heads / c->heads, all = (int64_t)x->n_tokens * times, seqs = std::min(c->n_seqs, x->n_tokens);
    const int64_t most = (x->max_q && x->max_q < x->n_tokens ? x->max_q : x->n_tokens) * times;
    if (all > 0x7fffffff - 4096) return "too many queries";
    // column tiles of all sequences and key heads: never more than from_all; as many as from_most if max_q is right
    auto from_all = [&](int64_t cols) { return (all / cols + seqs) * c->heads; };
    auto units = [&](int64_t cols) { return std::min(from_all(cols), (most + cols - 1) / cols * seqs * c->heads); };
    const int64_t tiles = ((int64_t)c->table_width * c->page_tokens + KV_TILE - 1) / KV_TILE, wide = 32 * MANY_WAVES;
    p->many = many_columns((double)units(32) * tiles, (double)units(wide) * tiles, (double)(all * c->heads) / (double)std::max<int64_t>(1, units(wide) * wide));
    if (form >= 0) p->many = form >= 2;
    p->cols = p->many ? (int)wide : 32;
    if (from_all(p->cols) > 0x7fffffff) return "too many queries";
    p->whole = p->many ? many_whole(units(wide), tiles) : few_whole(units(32), tiles);
    if (form >= 0) p->whole = form & 1;
    // One column tile per sequence and key head reads every code once.  32 ragged sequences of up to 8201 tokens x 8 heads 63.7 us, through the caches 72.9; one of
    // 131001 x 12 73.6 / 83.0.  (64 MiB: twice what the L2 caches hold.)
    p->far = !p->many && most <= 32 && seqs * tiles * c->heads > (64ll << 20) / (2 * KV_TILE * c->head_dim);
    p->wgs = p->whole ? (int)std::min<int64_t>(from_all(p->cols), 1 << 20) : p->many ? MANY_WGS : FEW_WGS;         // (one without work ends at once; past 2^20 one has several)
    const uint64_t slots = p->whole ? 0 : 2ull * p->wgs * p->cols;
    p->ml_offset = slots * c->head_dim * 4;
    p->cuts_offset = p->ml_offset + slots * 2 * 4;
    p->sent_offset = p->cuts_offset + p->wgs * sizeof(KvCut);
    p->bytes = p->whole ? 0 : p->sent_offset + (p->many ? p->wgs * MANY_WAVES * (8 + 4) : 0);
    return nullptr;
}

// A number that no earlier call has had and that memory holds by chance no more often than any other of 64 bits.  (Replays of a captured call have
// the same one: they find the words at 0, as the call before left them.)
unsigned long long next_epoch() {
    static std::atomic<unsigned long long> calls{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() << 20};
    unsigned long long z = calls.fetch_add(1, std::memory_order_relaxed) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    z ^= z >> 31;
    return z ? z : 1;
}

template <int HD>
void launch(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    if (p.many) {
        hipLaunchKernelGGL((kv_attend_many_kernel<HD, MANY_WAVES>), dim3(p.wgs), dim3(64 * MANY_WAVES), 0, s, a);
        if (!p.whole) hipLaunchKernelGGL((kv_join_kernel<HD, 32 * MANY_WAVES, 256>), dim3(p.wgs - 1, MANY_WAVES), dim3(256), 0, s, a);
    } else {
        if (p.far) hipLaunchKernelGGL((kv_attend_few_kernel<HD, true>), dim3(p.wgs), dim3(64 * FEW_WAVES), 0, s, a);
        else hipLaunchKernelGGL((kv_attend_few_kernel<HD, false>), dim3(p.wgs), dim3(64 * FEW_WAVES), 0, s, a);
        if (!p.whole) hipLaunchKernelGGL((kv_join_kernel<HD, 32, 1024>), dim3(p.wgs - 1), dim3(1024), 0, s, a);
    }
}

}  // namespace

static int attend(const char* name, const cf_kv_cache* cache, const cf_kv_query* x, int form, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (const char* bad = kv_bad(cache)) return cf_fail(nullptr, CF_ERR_ARG, "%s: %s", name, bad);
    if (const char* bad = query_bad(cache, x)) return cf_fail(nullptr, CF_ERR_ARG, "%s: %s", name, bad);
    if (!(x->scale > 0.0f) || !std::isfinite(x->scale)) return cf_fail(nullptr, CF_ERR_ARG, "%s: the scale must be positive and finite", name);
    if (x->n_tokens == 0 || cache->n_seqs == 0) return CF_OK;
    if (!x->q || !x->o || !x->cu || !x->lens) return cf_fail(nullptr, CF_ERR_ARG, "%s: null operand", name);
    if (((uintptr_t)x->q | (uintptr_t)x->o) % 16 || ((uintptr_t)x->cu | (uintptr_t)x->lens) % 4)
        return cf_fail(nullptr, CF_ERR_ARG, "%s: q and o must be 16-byte aligned, offsets and lengths 4", name);
    for (const int64_t st : {x->q_row, x->q_head, x->o_row, x->o_head})
        if (st < 0 || st > (int64_t)1 << 40 || st % 8) return cf_fail(nullptr, CF_ERR_ARG, "%s: strides must be multiples of 16 bytes and not negative", name);
    // pieces of one column tile may read its queries at any time
    const Rows q = {x->q, x->n_tokens, x->q_row, x->heads, x->q_head, cache->head_dim, 2}, o = {x->o, x->n_tokens, x->o_row, x->heads, x->o_head, cache->head_dim, 2};
    if (!o.apart()) return cf_fail(nullptr, CF_ERR_ARG, "%s: outputs overlap one another", name);
    if (rows_meet(q, o)) return cf_fail(nullptr, CF_ERR_ARG, "%s: o overlaps q", name);
    AttendPlan p;
    if (const char* bad = attend_plan(cache, x, form, &p)) return cf_fail(nullptr, CF_ERR_ARG, "%s: %s", name, bad);
    if (p.bytes && (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < p.bytes))
        return cf_fail(nullptr, CF_ERR_ARG, "%s: a workspace of %llu bytes, 256-byte aligned, is needed", name, (unsigned long long)p.bytes);
    AttendArgs a = {};
    a.c = kv_view(*cache);
    a.q = (const bf16*)x->q; a.o = (bf16*)x->o;
    a.q_row = x->q_row; a.q_head = x->q_head; a.o_row = x->o_row; a.o_head = x->o_head;
    a.cu = x->cu; a.lens = x->lens;
    a.n_tokens = x->n_tokens; a.heads = x->heads; a.times = x->heads / cache->heads;
    a.step_rows = 512 / cache->head_dim / a.times; a.step_heads = 512 / cache->head_dim % a.times;
    a.causal = x->causal != 0;
    a.end_least = x->causal ? INT32_MIN : INT32_MAX;
    a.whole = p.whole;
    a.c2 = x->scale * 1.4426950408889634f;
    if (!p.whole) {
        a.part_o = (float*)workspace;
        a.part_ml = (float*)((char*)workspace + p.ml_offset);
        a.cuts = (KvCut*)((char*)workspace + p.cuts_offset);
        a.sent = (unsigned long long*)((char*)workspace + p.sent_offset);
        a.joined = (uint32_t*)(a.sent + p.wgs * MANY_WAVES);
        a.epoch = next_epoch();
    }
    if (cache->head_dim == 128) launch<128>(a, p, (hipStream_t)stream);
    else launch<64>(a, p, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf_fail(nullptr, CF_ERR_HIP, "%s launch: %s", name, hipGetErrorString(e));
}

static int attend_view(const char* name, const cf_kv_cache* cache, const cf_kv_query* x, int form, AttendPlan* p) {
    if (const char* bad = kv_bad(cache)) return cf_fail(nullptr, CF_ERR_ARG, "%s: %s", name, bad);
    if (const char* bad = query_bad(cache, x)) return cf_fail(nullptr, CF_ERR_ARG, "%s: %s", name, bad);
    if (const char* bad = attend_plan(cache, x, form, p)) return cf_fail(nullptr, CF_ERR_ARG, "%s: %s", name, bad);
    return CF_OK;
}

extern "C" int cf_kv_attention_workspace(const cf_kv_cache* cache, const cf_kv_query* x, uint64_t* bytes) {
    if (!bytes) return cf_fail(nullptr, CF_ERR_ARG, "kv_attention_workspace: null result");
    AttendPlan p;
    CF_TRY(attend_view("kv_attention_workspace", cache, x, -1, &p));
    *bytes = p.bytes;
    return CF_OK;
}

extern "C" int cf_plan_kv_attention(const cf_kv_cache* cache, const cf_kv_query* x, int32_t form, cf_kv_attention_plan* plan) {
    if (!plan || form < -1 || form > 3) return cf_fail(nullptr, CF_ERR_ARG, "plan_kv_attention: form is -1 to 3, the result not NULL");
    AttendPlan p;
    CF_TRY(attend_view("plan_kv_attention", cache, x, form, &p));
    *plan = {p.many ? 2 + p.whole : 0 + p.whole, p.cols, p.wgs, 0, p.bytes};
    return CF_OK;
}

extern "C" int cf_kv_attention(const cf_kv_cache* cache, const cf_kv_query* x, void* workspace, uint64_t workspace_bytes, void* stream) {
    return attend("kv_attention", cache, x, -1, workspace, workspace_bytes, stream);
}

extern "C" int cf_op_kv_attention_form(const cf_kv_cache* cache, const cf_kv_query* x, int32_t form, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (form < 0 || form > 3) return cf_fail(nullptr, CF_ERR_ARG, "op_kv_attention_form: form is 0 to 3");
    return attend("op_kv_attention_form", cache, x, form, workspace, workspace_bytes, stream);
}
