// What the attention kernels over a paged 8-bit cache share: arguments, how a ragged batch is laid end to end, and the arithmetic of a tile of 64
// keys against a wave's 32 columns.
//
// Columns.  The query rows of a sequence times the query heads of a key head, row after row, are the columns of that (sequence, key head); 32 of them
// are a column tile of a wave.  As in attention.hip a wave works on the transposed problem, S^T = K Q^T and O^T = V^T P^T with 32x32x16 MFMAs: a
// lane owns a column (lane & 31) and half of the keys (lane >> 5), softmax reference and row sum are per-lane scalars, and P^T is S^T repacked.
//
// Operands.  The order of the contracted index is free as long as both operands share it, and so is the key that a row of S^T stands for.  Both are
// chosen so that a lane's part of K or V is 16 consecutive bytes of the cache, two k-steps' worth:
//   S^T: lane group lg (0, 1) has dims 16 (2j + lg) + 8u + 0..7 at k-step 2j + u: K chunk 2j + lg of its key's group.
//   Row r of S^T's half mt is key 32 mt + 16 ((r >> 2) & 1) + (r & 3) + 4 (r >> 3), so that register v of lane group lg is key 32 mt + 16 lg + v.
//   O^T: lane group lg has keys 32 s + 16 lg + 8u + 0..7 at k-step 2s + u: V's 16 tokens of group 2s + lg, and S^T's registers 8u .. 8u + 7 of half s.
#pragma once
#include <math.h>

#include "kv_cache.h"

struct AttendArgs {
    KvView c;
    const bf16* q;
    bf16* o;
    int64_t q_row, q_head, o_row, o_head;
    const int32_t *cu, *lens;
    int32_t n_tokens, heads, times;        // times: query heads per key head
    int32_t step_rows, step_heads;         // 512 / head_dim columns further on (many columns: from one row of 16-byte chunks of a lane's to its next)
    int32_t causal;
    int32_t end_least;                     // of the keys that a query sees, before its sequence's length: INT_MAX, causal INT_MIN
    int32_t whole;                         // no column tile is cut: each is a share of its own
    float c2;                              // scale * log2(e)
    float* part_o;                         // results of pieces of a column tile's keys: few columns [column][head_dim], many as they lie in registers,
                                           // [32 columns][head_dim / 8][lane][4]; then
    float* part_ml;                        // [column][2]: reference (base 2) and sum of the weights
    struct KvCut* cuts;                    // [workgroups]
    // Many columns, [workgroups][waves]: whether the first piece of a share is there for all to see (`epoch` says so; whatever else is in memory does not,
    // and the kernel that joins pieces leaves 0), and whether its last one has been joined with what follows.
    unsigned long long* sent;
    uint32_t* joined;
    unsigned long long epoch;
};
// A column tile whose first piece is the last one of a share: query rows of its sequence, key head, first column, how many pieces (0: no such tile).
struct KvCut {
    int32_t start, n, h, col0, pieces, pad[3];
};

constexpr int KV_TILE = 64;                // keys

// Work is laid end to end -- sequences, in each the key heads, in each the column tiles of COLS columns -- and cut into equal shares wherever that is.
// The weight of a column tile is about the number of keys that it goes through, and as many as its beginning and end take the time of: w0 + c dw for
// the c-th of a sequence (dw = 0 unless causal).
struct KvSeq {
    int b, start, n, len, ct;              // ct: column tiles
    int w0, dw;
    int64_t first;                         // where its work begins
    __device__ __forceinline__ int64_t before(int c) const { return (int64_t)c * w0 + (int64_t)dw * ((int64_t)c * (c - 1) / 2); }        // of a head's column tiles before c
    __device__ __forceinline__ int64_t head() const { return before(ct); }
};

// x / y of what is not negative; nearly always both have 32 bits, and the division of 64 takes 5 times as long
__device__ __forceinline__ int64_t kv_div(int64_t x, int64_t y) {
    return (uint64_t)(x | y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}
// values that all lanes agree on, in scalar registers
__device__ __forceinline__ int64_t kv_lane64(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}
template <int COLS>
__device__ __forceinline__ void kv_weigh(const AttendArgs& a, KvSeq& s) {
    s.ct = (s.n * a.times + COLS - 1) / COLS;
    constexpr int ENDS = COLS == 32 ? 4 * KV_TILE : 6 * KV_TILE;           // about 4 us, and 9 with all workgroups at their queries and outputs
    s.w0 = s.len + ENDS;
    s.dw = 0;
    if (a.whole) {
        s.w0 = 1;
    } else if (a.causal && s.ct > 1) {
        s.dw = COLS / a.times;             // query rows from one column tile to the next
        s.w0 = max(0, s.len - s.n) + s.dw + ENDS;
    }
}
// The sequence of each lane, i = base + lane, and the inclusive sum of the work up to it.
template <int COLS>
struct KvScan {
    KvSeq s;
    int64_t upto;
    __device__ __forceinline__ KvScan(const AttendArgs& a, int base) {
        const int lane = threadIdx.x & 63, i = base + lane;
        s.start = s.n = s.len = 0;
        if (i < a.c.n_seqs) {
            s.start = kv_clamped(a.cu[i], 0, a.n_tokens);
            s.n = kv_clamped(a.cu[i + 1], s.start, a.n_tokens) - s.start;
            s.len = kv_clamped(a.lens[i], 0, a.c.capacity);
        }
        kv_weigh<COLS>(a, s);
        upto = s.head() * a.c.heads;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t x = __shfl_up((long long)upto, o);
            upto += lane >= o ? x : 0;
        }
    }
    __device__ __forceinline__ int64_t all() const { return kv_lane64(upto, 63); }
    __device__ __forceinline__ KvSeq pick(const AttendArgs& a, int base, int64_t before, int lane) const {
        KvSeq r;
        r.b = base + lane;
        r.start = __builtin_amdgcn_readlane(s.start, lane);
        r.n = __builtin_amdgcn_readlane(s.n, lane);
        r.len = __builtin_amdgcn_readlane(s.len, lane);
        kv_weigh<COLS>(a, r);
        r.first = before + kv_lane64(upto, lane) - r.head() * a.c.heads;
        return r;
    }
};
// All work; `first` is the scan of the first 64 sequences.
template <int COLS>
__device__ __forceinline__ int64_t kv_total(const AttendArgs& a, const KvScan<COLS>& first) {
    int64_t t = first.all();
    for (int base = 64; base < a.c.n_seqs; base += 64) t += KvScan<COLS>(a, base).all();
    return t;
}
// The sequence with work f, 0 <= f < kv_total: of the first 64 as scanned, or behind them.
template <int COLS>
__device__ __forceinline__ KvSeq kv_find(const AttendArgs& a, int64_t f, const KvScan<COLS>& first) {
    if (const uint64_t m = __ballot(f < first.upto)) return first.pick(a, 0, 0, __builtin_ctzll(m));
    int64_t before = first.all();
    for (int base = 64;; base += 64) {
        const KvScan<COLS> s(a, base);
        const uint64_t m = __ballot(f < before + s.upto);
        if (m) return s.pick(a, base, before, __builtin_ctzll(m));
        before += s.all();
    }
}

// Query row i of sequence s sees keys [0, this).
__device__ __forceinline__ int kv_end(const AttendArgs& a, const KvSeq& s, int i) { return min(s.len, max(s.len - s.n + i + 1, a.end_least)); }

// A column tile and a share of its keys: tiles [t0, t1) of `tiles`.
struct KvPiece {
    int h, c, t0, t1;
    bool from_start, whole;
    int64_t next, end;                     // where the work after it begins, and where that of its column tile ends
};
// The piece of column tile c of head h that begins x of its work behind its beginning, f in all, in a share that ends at f1.
template <int COLS>
__device__ __forceinline__ KvPiece kv_part(const AttendArgs& a, const KvSeq& s, int h, int c, int64_t x, int64_t f, int64_t f1) {
    KvPiece p;
    p.h = h;
    p.c = c;
    const int64_t w = s.w0 + (int64_t)c * s.dw, to = min(w, x + (f1 - f));
    const int cols = min(COLS, s.n * a.times - COLS * c);
    const int last = (int)((uint32_t)(COLS * c + cols - 1) / (uint32_t)a.times);
    const int end = kv_end(a, s, last);              // of the keys that any column sees
    const int tiles = (max(end, 0) + KV_TILE - 1) / KV_TILE;
    p.t0 = x == 0 ? 0 : (int)kv_div(x * tiles, w);
    p.t1 = to == w ? tiles : (int)kv_div(to * tiles, w);
    p.from_start = x == 0;
    p.whole = x == 0 && to == w;
    p.next = f + (to - x);
    p.end = f + (w - x);
    return p;
}
// The piece of sequence s that begins at f,
template <int COLS>
__device__ __forceinline__ KvPiece kv_piece(const AttendArgs& a, const KvSeq& s, int64_t f, int64_t f1) {
    const int64_t per = s.head();
    int64_t x = f - s.first;
    const int h = (int)kv_div(x, per);
    x -= h * per;
    int lo = 0, hi = s.ct - 1;             // the last column tile that begins at or before x
    if (s.dw == 0) {
        lo = (int)kv_div(x, s.w0);
    } else {
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s.before(mid) <= x) lo = mid;
            else hi = mid - 1;
        }
    }
    return kv_part<COLS>(a, s, h, lo, x - s.before(lo), f, f1);
}
// and the one after p, the whole of the next column tile or the beginning of it.
template <int COLS>
__device__ __forceinline__ KvPiece kv_next(const AttendArgs& a, const KvSeq& s, const KvPiece& p, int64_t f1) {
    const bool same = p.c + 1 < s.ct;
    return kv_part<COLS>(a, s, same ? p.h : p.h + 1, same ? p.c + 1 : 0, 0, p.next, f1);
}
// Equal shares of all work for up to `most` workgroups, none of less than `least`.
struct KvShares {
    int64_t total;
    int wgs;
    __device__ __forceinline__ KvShares(int64_t all, int most, int least) : total(all), wgs((int)max((int64_t)1, min((int64_t)most, (all + least - 1) / least))) {}
    // total * w / wgs, without the product, which might not fit
    __device__ __forceinline__ int64_t begin(int w) const { 
        const int64_t each = kv_div(total, wgs);
        return each * w + kv_div((total - each * wgs) * w, wgs);
    }
    __device__ __forceinline__ int of(int64_t f) const {           // the workgroup with work f
        int w = min((int)((double)f * wgs / (double)total), wgs - 1);
        while (begin(w + 1) <= f) ++w;
        while (begin(w) > f) --w;
        return w;
    }
};

// What the last piece of a workgroup's share (without one: KvPiece{}) leaves for the kernel that joins pieces.
template <int COLS>
__device__ __forceinline__ void kv_leave_cut(const AttendArgs& a, const KvShares& shares, int w, const KvSeq& q, const KvPiece& p) {
    KvCut cut = {};
    if (p.from_start && !p.whole) {
        const int64_t unit = q.first + p.h * q.head() + q.before(p.c);
        cut.start = q.start;
        cut.n = q.n;
        cut.h = p.h;
        cut.col0 = COLS * p.c;
        cut.pieces = shares.of(unit + q.w0 + (int64_t)p.c * q.dw - 1) - w + 1;
    }
    if (threadIdx.x == 0) a.cuts[w] = cut;
}

// A lane's column of a column tile.
struct KvColumn {
    int row, head, end;                    // query row, query head, keys [0, end) are seen
    bool mine;                             // a column, not padding (which repeats the last one)
};
__device__ __forceinline__ KvColumn kv_column(const AttendArgs& a, const KvSeq& s, int h, int col) {
    const int cols = s.n * a.times, c = min(col, cols - 1), i = (int)((uint32_t)c / (uint32_t)a.times);
    return {s.start + i, h * a.times + (c - i * a.times), kv_end(a, s, i), col < cols};
}

// ---- a tile
constexpr float kNoRef = -3.402823466e38f;        // reference of a column before its first score
template <int HD>
struct KvState {
    floatx16 o[HD / 32];                   // O^T: register v of dt = dim 32 dt + (v & 3) + 8 (v >> 2) + 4 lg
    float mc, l;                           // reference, base 2; sum of the weights of this lane's keys
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[d][v] = 0.0f;
        mc = kNoRef;
        l = 0.0f;
    }
};

// eight codes times a power of two, exactly (bf16 has the bits)
__device__ __forceinline__ bf16x8 kv_wide(uint32_t lo, uint32_t hi, float scale) {
    uint32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ float kv_power(uint32_t byte) { return __uint_as_float(byte << 23); }

// Scores of keys that a column does not see become -inf: rel[mt] = how many of the lane's 16 keys of half mt it sees.
__device__ __forceinline__ void kv_mask(floatx16 (&s)[2], const int (&rel)[2]) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int v = 0; v < 16; ++v) s[mt][v] = v < rel[mt] ? s[mt][v] : -INFINITY;
}

// What the two lanes of a column have, for both of them.
__device__ __forceinline__ uint32x2 kv_halves(uint32_t x) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return uint32x2{r[0], r[1]};
}
__device__ __forceinline__ float kv_sum_halves(float x) {
    const uint32x2 r = kv_halves(__float_as_uint(x));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Weights of a tile: P^T in bf16 as the second contraction takes it, and the sum of the weights as rounded.  The reference is not the
// running maximum: softmax does not depend on it, and fp32 and bf16 are as exact at 2^19 as at 1.  It stays where it is as long as a lane's 32 weights
// add up to less than 2^20, which the sum, needed anyway, tells; else it moves to the largest score (always in a column's first tile,
// where weights against kNoRef are infinite; `fresh`: they need not be computed), and what has been summed up is brought to it.
template <int HD>
__device__ __forceinline__ void kv_softmax(KvState<HD>& st, const floatx16 (&s)[2], float c2, bf16x8 (&pf)[4], bool fresh) {
    float psum = 0.0f;
    auto weigh = [&]() __attribute__((always_inline)) {
        float ps[4] = {0.f, 0.f, 0.f, 0.f};
        bf16x2 ones;
        ones[0] = ones[1] = (bf16)1.0f;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                bf16x2 pp;
                pp[0] = (bf16)__builtin_amdgcn_exp2f(fmaf(s[ks >> 1][8 * (ks & 1) + e], c2, -st.mc));
                pp[1] = (bf16)__builtin_amdgcn_exp2f(fmaf(s[ks >> 1][8 * (ks & 1) + e + 1], c2, -st.mc));
                pf[ks][e] = pp[0];
                pf[ks][e + 1] = pp[1];
                ps[(e >> 1) & 3] = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, ps[(e >> 1) & 3], false);
            }
        psum = (ps[0] + ps[1]) + (ps[2] + ps[3]);
    };
    if (!fresh) weigh();
    const bool over = fresh || !(psum < 1048576.0f);
    if (__any(over)) {                     // (only the columns that need it move: a column's bits do not depend on those beside it)
        float mx = s[0][0];
#pragma unroll
        for (int v = 1; v < 32; ++v) mx = fmaxf(mx, s[v >> 4][v & 15]);
        const uint32x2 both = kv_halves(__float_as_uint(mx)), either = kv_halves(over);
        mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
        const float mc = either[0] | either[1] ? fmaxf(st.mc, mx * c2) : st.mc, f = __builtin_amdgcn_exp2f(st.mc - mc);
        st.mc = mc;
        st.l *= f;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) st.o[d][v] *= f;
        weigh();
    }
    st.l += psum;
}

// A NaN among values reaches the columns that see its key and no others, though their weight of zero would carry it there: NaN codes are
// taken out before the second contraction, and a contraction of its own, of which codes were NaN with which keys are seen, says which sums they belong to.
__device__ __forceinline__ uint32_t kv_nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }        // bit 7 of each NaN
// A bit 7 where there is a NaN, and perhaps where there is none.  (Another formula on purpose: the compiler would keep the results of the same one in
// 64 registers until they are used again.)
__device__ __forceinline__ uint32_t kv_perhaps_nan(uint32_t w) { return (~w & 0x7f7f7f7fu) - 0x01010101u; }
__device__ __forceinline__ uint32_t kv_without_nan(uint32_t w, uint32_t nans) { return w & ~((nans << 1) - (nans >> 7)); }
__device__ __forceinline__ uint32_t kv_ones(uint32_t nans) { return (nans >> 7) * 0x38u; }                                          // the code of 1
// 1 for each of eight bits
__device__ __forceinline__ bf16x8 kv_bits(uint32_t m) {
    uint32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = ((m >> (2 * i) & 1u) | (m << (15 - 2 * i) & 0x10000u)) * 0x3f80u;
    return __builtin_bit_cast(bf16x8, r);
}
// which of a lane's keys 8u .. 8u + 7 of a half its column sees
__device__ __forceinline__ bf16x8 kv_seen(int rel, int u) { return kv_bits((1u << rel) - 1u >> (8 * u)); }
template <int HD>
__device__ __forceinline__ void kv_spread_nan(KvState<HD>& st, int d, const floatx16& hits) {
#pragma unroll
    for (int v = 0; v < 16; ++v) st.o[d][v] = hits[v] > 0.0f ? __uint_as_float(0x7fc00000u) : st.o[d][v];
}

// What divides: 0 where a column has seen nothing.
__device__ __forceinline__ float kv_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
