// What the attention of a run of rows and the key masses share: which keys a row sees, how a
// logit comes from its dot product, and the tiles both multiply.
#pragma once

#include "socket_internal.h"

namespace sk {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The caller's modifications of the scores, as the kernels take them.  Everything is in units of
// log 2, so that a weight is one exp2.
struct RowMods {
    float c;              // scale log2(e)
    float y_scale, a;     // capped logits: a tanh(y_scale x), a = cap log2(e); a = 0: not capped
    int window;
    const float *slopes;
    const int32_t *prefix_len;
    const int32_t *doc_begin;
};

inline RowMods row_mods(float scale, const socket_attn_mods *m) {
    RowMods r{};
    r.c = scale * kLog2e;
    if (m) {
        if (m->softcap > 0.0f) {
            r.y_scale = scale / m->softcap;
            r.a = m->softcap * kLog2e;
        }
        r.window = m->window;
        r.slopes = m->slopes;
        r.prefix_len = m->prefix_len;
        r.doc_begin = m->doc_begin;
    }
    return r;
}

// A run of rows: token positions begin .. begin + count - 1 of a sequence that is begin + count
// long.  One that goes past max_n is cut to it, one that begins outside [0, max_n) is empty.
struct RowRun {
    int begin, count;
    __device__ __forceinline__ RowRun(const int32_t *row_begin, const int32_t *row_count, int b, int max_rows, int max_n) {
        begin = scalar_load(&row_begin[b]);
        count = min(scalar_load(&row_count[b]), max_rows);
        if (begin < 0 || begin >= max_n) begin = count = 0;
        count = max(0, min(count, max_n - begin));
    }
    __device__ __forceinline__ int len() const { return begin + count; }
};

// keys lo .. hi that the row at position i sees (none where lo > hi)
__device__ __forceinline__ void row_span(const RowMods &m, int b, int i, int len, int max_n, int &lo, int &hi) {
    lo = 0;
    hi = i;
    if (m.window > 0) lo = max(lo, i - m.window + 1);
    if (m.doc_begin) lo = max(lo, m.doc_begin[(int64_t)b * max_n + i]);
    if (m.prefix_len) {
        const int p = m.prefix_len[b];
        if (p > i) hi = p - 1;
    }
    hi = min(hi, len - 1);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh(y) / y up to |y| = 1/4, z = y^2: the power series 1 - z/3 + 2 z^2/15 - 17 z^3/315 + 62 z^4/2835, its
// last term replaced by what is left of z^4 after a Chebyshev polynomial of degree four on [0, 1/16] is taken from it
// (z^4 = z^3/8 - 5 z^2/1024 + z/16384 up to 1.2e-7, times 62/2835).  Off by 1.2e-8 at most, the series' own rest included.
constexpr float kCapSmall = 0.25f;
__device__ __forceinline__ float tanh_ratio(float z) {
    constexpr double c4 = 62.0 / 2835.0;
    constexpr float c3 = (float)(-17.0 / 315.0 + c4 / 8.0), c2 = (float)(2.0 / 15.0 - c4 * 5.0 / 1024.0), c1 = (float)(-1.0 / 3.0 + c4 / 16384.0);
    return fmaf(fmaf(fmaf(c3, z, c2), z, c1), z, 1.0f);
}
// tanh for any y: beyond 1/4, 1 - 2 / (1 + e^2y), whose rounding is absolute and would be felt only near zero
__device__ __forceinline__ float tanh_any(float y) {
    const float far = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + exp2_fast(y * (2.0f * kLog2e))), 1.0f);
    return fabsf(y) <= kCapSmall ? y * tanh_ratio(y * y) : far;
}

// The logit of a dot product less `ref`, in units of log 2, at distance dist = i - j; slope2 = slope log2(e).
__device__ __forceinline__ float logit2(const RowMods &m, float x, float dist, float slope2, float ref) {
    float s = m.a > 0.0f ? fmaf(m.a, tanh_any(x * m.y_scale), -ref) : fmaf(x, m.c, -ref);
    if (m.slopes) s = fmaf(-slope2, fabsf(dist), s);
    return s;
}

// The same for the N dot products of one query that a lane holds of a tile, the key of x[n] being
// key0 + row_of(n): capped logits are mostly far below the cap, so a wavefront whose arguments all are
// small takes the ratio alone.
template <int N, typename F>
__device__ __forceinline__ void logits2(const RowMods &m, float (&x)[N], float i_minus_key0, float slope2, float ref, F row_of) {
    if (m.a > 0.0f) {
        float top = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            x[n] *= m.y_scale;
            top = fmaxf(top, fabsf(x[n]));
        }
        if (__all(top <= kCapSmall)) {
#pragma unroll
            for (int n = 0; n < N; ++n) x[n] = fmaf(x[n] * m.a, tanh_ratio(x[n] * x[n]), -ref);
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) x[n] = fmaf(m.a, tanh_any(x[n]), -ref);
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = fmaf(x[n], m.c, -ref);
    }
    if (m.slopes) {
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = fmaf(-slope2, fabsf(i_minus_key0 - (float)row_of(n)), x[n]);
    }
}

// The same one by one, for a kernel of its own per kind of logit.
template <bool CAP, bool BIAS> struct LogitOf {
    float c, a, ref, slope2, dist0;
    __device__ __forceinline__ LogitOf(const RowMods &m, float i_minus_key0, float slope, float r)
        : c(CAP ? m.y_scale : m.c), a(m.a), ref(r), slope2(slope), dist0(i_minus_key0) {}
    __device__ __forceinline__ float biased(float s, int row) const { return BIAS ? fmaf(-slope2, fabsf(dist0 - (float)row), s) : s; }
    // capped: right where |y| <= 1/4; `most` becomes the largest |y| so far
    __device__ __forceinline__ float small(float x, int row, float &most) const {
        if (!CAP) return biased(fmaf(x, c, -ref), row);
        const float y = x * c;
        most = fmaxf(most, fabsf(y));
        return biased(fmaf(y * a, tanh_ratio(y * y), -ref), row);
    }
    // of an argument y that is scaled already (capped; else the dot product itself)
    __device__ __forceinline__ float scaled(float y, int row, bool small_) const {
        if (!CAP) return biased(fmaf(y, c, -ref), row);
        return biased(small_ ? fmaf(y * a, tanh_ratio(y * y), -ref) : fmaf(a, tanh_any(y), -ref), row);
    }
    __device__ __forceinline__ float any(float x, int row) const {
        return biased(CAP ? fmaf(a, tanh_any(x * c), -ref) : fmaf(x, c, -ref), row);
    }
};

// Longest sequence of a batch, cut to what a window lets its rows see: by one wavefront.
__device__ __forceinline__ int longest_of(const int32_t *row_begin, const int32_t *row_count, int batch, int max_rows, int max_n, int window) {
    int longest = 0;
    for (int y = (int)(threadIdx.x & 63); y < batch; y += 64) {
        const int begin = row_begin[y], count = min(row_count[y], max_rows);
        if (begin >= 0 && begin < max_n && count > 0) {
            int span = min(begin + count, max_n);
            if (window > 0 && window < span) span = min(span, window + count - 1);
            longest = max(longest, span);
        }
    }
    return (int)wave_max((float)longest);            // (exact: positions are below 2^24)
}

// Rows of one (sequence, KV head) by block, without a branch: a contiguous cache is a single block, 0.
struct BlockRows {
    int64_t stride, base;
    int blocks, page;
    uint32_t page_magic;
    __device__ __forceinline__ BlockRows(const RowMap &m, int b, int h) {
        const bool paged = m.block_table != nullptr;
        stride = paged ? (int64_t)m.Hkv * m.page : 0;
        base = paged ? (int64_t)h * m.page : ((int64_t)b * m.Hkv + h) * m.max_n;
        blocks = paged ? m.num_blocks : 1;
        page = paged ? m.page : 0;
        page_magic = paged ? m.page_magic : 0u;
    }
    __device__ __forceinline__ int64_t at(int blk, int t) const {
        return blk * stride + base + (t - (int)__umulhi((uint32_t)t, page_magic) * page);
    }
};

// 16 bytes a lane from memory to LDS, at `to` + 16 lane (`to` is the same for the wavefront)
__device__ __forceinline__ void lds_fill(const char *from, char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// ---- matrix tiles: 32 keys x 32 queries, logits as K Q^T, so that a lane holds one query's
// logits and the softmax runs along its registers
typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8v_t;

// key row of accumulator register r in a 32 x 32 tile, for lane half hf
__device__ __forceinline__ constexpr int tile_row(int r, int hf) { return 8 * (r / 4) + 4 * hf + r % 4; }

// One 16-byte piece of a row in the operand layouts used here.  bf16: 8 channels, one k-step of 16
// takes piece 2 ks + hf.  fp32: 4 channels, two-channel k-steps 4 c .. 4 c + 3 take piece 2 c + hf
// (which channels meet in a step is free as long as both operands agree).
template <typename T> __device__ __forceinline__ void mma_piece(floatx16_t &c, u32x4_t a, u32x4_t b);
template <> __device__ __forceinline__ void mma_piece<uint16_t>(floatx16_t &c, u32x4_t a, u32x4_t b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8v_t, a), __builtin_bit_cast(bf16x8v_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma_piece<float>(floatx16_t &c, u32x4_t a, u32x4_t b) {
    const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
}

// the same for tiles of 16 rows (lane = column lane % 16; sixteenth of the wavefront g = lane / 16): a
// k-step of bf16 takes piece 4 c + g, four k-steps of fp32 do
typedef float floatx4v_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ floatx4v_t mma16(u32x4_t a, u32x4_t b, floatx4v_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v_t, a), __builtin_bit_cast(bf16x8v_t, b), c, 0, 0, 0);
}

// In fp32 the four k-steps of a piece have a sum each, added up at the end: four short chains of
// additions round less than a long one (twelve outputs over 4096 fp32 keys, d = 128: 3.6e-7 off at most, 1.6e-6 with one).
template <typename T> struct Tile16;
template <> struct Tile16<uint16_t> {
    floatx4v_t c = 0.0f;
    __device__ __forceinline__ void add(u32x4_t a, u32x4_t b) {
        c = mma16(a, b, c);
    }
    __device__ __forceinline__ floatx4v_t total() const { return c; }
};
template <> struct Tile16<float> {
    floatx4v_t c0 = 0.0f, c1 = 0.0f, c2 = 0.0f, c3 = 0.0f;
    __device__ __forceinline__ void add(u32x4_t a, u32x4_t b) {
        const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
        c0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[0], y[0], c0, 0, 0, 0);
        c1 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[1], y[1], c1, 0, 0, 0);
        c2 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[2], y[2], c2, 0, 0, 0);
        c3 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[3], y[3], c3, 0, 0, 0);
    }
    __device__ __forceinline__ floatx4v_t total() const {
        floatx4v_t t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = (c0[e] + c1[e]) + (c2[e] + c3[e]);
        return t;
    }
};

// max over the four sixteenths of a wavefront
__device__ __forceinline__ float sixteenths_max(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// sizes and swizzles of the K / V tiles in LDS, in pieces of 16 bytes
template <typename T, int D> struct KvTile {
    static constexpr int KT = sizeof(T) == 2 && D <= 128 ? 64 : 32;          // keys
    static constexpr int ROWB = D * (int)sizeof(T);
    static constexpr int CPR = ROWB / 16;                        // pieces per row
    static constexpr int BYTES = KT * ROWB;
    // K: 32 rows are read at one piece each: the piece is turned by the row
    static __device__ __forceinline__ int k_turned(int row, int c) { return c ^ (row & (CPR < 16 ? CPR - 1 : 15)); }
    static __device__ __forceinline__ int k_piece(int row, int c) { return row * CPR + k_turned(row, c); }
    // V: bf16 rows are read four at a time, 64 bytes each, and transposed on the way; fp32 rows r and
    // r + 4 at once, 128 bytes each
    static __device__ __forceinline__ int v_turned(int row, int c) {
        if (sizeof(T) == 4) return c ^ (((row >> 2) & 1) << 3);
        return c ^ (CPR == 8 ? ((row >> 1) & 1) << 2 : (row & 3) << 2);
    }
    static __device__ __forceinline__ int v_piece(int row, int c) { return row * CPR + v_turned(row, c); }
};

}  // namespace sk
