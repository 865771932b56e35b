// Attention of a run of query rows per sequence over its cache: one new token, a few, a chunk of
// a prompt or a whole one.  Row at position i, query head g, keys j it sees (row_span):
//     s_j = cap tanh(scale q.k_j / cap) - slope |i - j|,   out = sum_j softmax(s)_j v_j,   lse = log sum_j exp(s_j)
//
// One pass over the keys with a running maximum and sum.  The G query heads of a KV head and the
// rows of the run are one axis of queries, m = row * G + g; a workgroup takes 128 of them, 32 per
// wavefront, and all of its wavefronts walk the same tiles of keys through LDS.  A wavefront forms
// K Q^T (32 keys x 32 queries a tile), so that a lane holds logits of one query and the softmax
// needs one exchange between the lane halves; the weights, as they lie in the accumulators, are
// the B operand of V^T P^T once V's rows are taken in the same order (rows 0-3 and 8-11 of 16 for
// the lower lanes, 4-7 and 12-15 for the upper), so they never leave their lanes.
//
// bf16 caches: products of bf16 with fp32 sums.  The weights are rounded once to bf16 where the
// output is bf16 (half a step each, as the output's own rounding; two pieces, 17 bits, would cost the matrix
// units half as much again), except that few rows, which wait for memory, take two pieces for the
// same time; where the output is fp32 they go in as three, which hold all 24 bits.  fp32 caches:
// fp32 matrix instructions.
//
// Few rows: the keys are split over workgroups, whose (maximum, sum, weighted values) a second
// launch joins, split by split in a fixed order.
//
// Bounds and figures (a large copy reaches 4.85 TB/s here, a large matrix product 1.19 PFLOP/s in bf16
// and 0.135 in fp32, all under the card's power limit).  Prompts and chunks are bound by the matrix units and the
// softmax's vector work beside them: 8192 rows of 32 heads, d = 128, 547 to 583 us on several cards = 0.94 to
// 1.0 PFLOP/s; 4096 rows behind 28672, capped, 2370 us = 0.87 (a cap is seven more operations a logit); 4096 fp32
// rows of 8 heads 321 us = 0.107.  One token is bound by memory: 131072 keys of 8 heads 96 us = 5.6 TB/s, 16 ragged
// paged sequences 266 us = 5.05 TB/s.  4096 keys of one head, fp32, 11.7 us: the latency of two launches.
//
// Values at masked keys never count, whatever they are: a masked weight is 0, but 0 times an
// infinity is not, so a wavefront that ends with a value that is not finite goes over its row
// again one key at a time (attend_plain).
#include "attend_device.h"

namespace sk {

constexpr int kRowsThreads = 256;
constexpr int kRowsQueries = 128;                // queries per workgroup

struct RowsArgs {
    const void *q;
    const void *K;
    const void *V;
    void *out;
    float *lse;
    float *partials;
    const int32_t *row_begin;
    const int32_t *row_count;
    RowMap map;
    RowMods mods;
    int batch, BH, Hq, G, g_log2, max_rows, n_tiles, n_split, out_dtype;
};

// where a query's result goes: its index among all (sequence, row, query head)
__device__ __forceinline__ int64_t query_at(const RowsArgs &a, int b, int h, int m) {
    return ((int64_t)b * a.max_rows + (m >> a.g_log2)) * a.Hq + h * a.G + (m & (a.G - 1));
}

// One query over keys j0 .. j1 by a whole wavefront, key by key: lane = key for the logits, lane =
// channels for the values.  Only for rows that meet infinities or NaN.
template <typename T, int D>
__device__ __forceinline__ void attend_plain(const RowsArgs &a, int b, int h, int m, int i, int j0, int j1, int split) {
    constexpr int PER = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t at = query_at(a, b, h, m);
    const T *q = (const T *)a.q + at * D;
    const float slope2 = a.mods.slopes ? a.mods.slopes[h * a.G + (m & (a.G - 1))] * kLog2e : 0.0f;
    const float ninf = -__builtin_inff();
    float top = ninf, sum = 0.0f, acc[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) acc[k] = 0.0f;
    for (int j = j0; j <= j1; j += 64) {
        const int t = j + lane;
        const int64_t row = t <= j1 ? a.map.row(b, h, t) : -1;
        float s = ninf;
        if (row >= 0) {
            float dot = 0.0f;
#pragma clang loop unroll(disable)
            for (int c = 0; c < D; c += 8) {
                Row8<T> kr, qr;
                kr.load((const T *)a.K + row * D + c);
                qr.load(q + c);
                float kf[8], qf[8];
                kr.get(kf);
                qr.get(qf);
#pragma unroll
                for (int e = 0; e < 8; ++e) dot = fmaf(kf[e], qf[e], dot);
            }
            s = logit2(a.mods, dot, (float)(i - t), slope2, 0.0f);
        }
        const float top_new = fmaxf(top, wave_max(s)), use = top_new == ninf ? 0.0f : top_new;
        const float p = row >= 0 ? exp2_fast(s - use) : 0.0f, alpha = exp2_fast(top - use);
        top = top_new;
        sum = sum * alpha + p;
#pragma unroll
        for (int k = 0; k < PER; ++k) acc[k] *= alpha;
        const unsigned long long there = __ballot(row >= 0);
#pragma clang loop unroll(disable)
        for (int o = 0; o < 64; ++o) {
            if (!((there >> o) & 1ull)) continue;
            const float w = __shfl(p, o);
            const int64_t vrow = a.map.row(b, h, j + o);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const T *v = (const T *)a.V + vrow * D + lane + 64 * k;
                const float x = sizeof(T) == 2 ? bf16_to_f32(*(const uint16_t *)v) : *(const float *)v;
                acc[k] = fmaf(w, x, acc[k]);
            }
        }
    }
    sum = row_sum<64>(sum);
    if (a.n_split > 1) {
        float *part = a.partials + (at * a.n_split + split) * (D + 2);
        if (lane == 0) {
            part[0] = top;
            part[1] = sum;
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) part[2 + lane + 64 * k] = acc[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const float y = sum == 0.0f ? 0.0f : acc[k] / sum;
        if (a.out_dtype == SOCKET_F32) ((float *)a.out)[at * D + lane + 64 * k] = y;
        else ((uint16_t *)a.out)[at * D + lane + 64 * k] = f32_to_bf16_rne(y);
    }
    if (a.lse && lane == 0) a.lse[at] = sum == 0.0f ? ninf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

typedef short shortx4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4_t lds_shortx4_t;

// two floats rounded to bf16, to nearest even (one instruction)
typedef float floatx2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2_t{lo, hi}, bf16x2_t));
}

// The value product O^T += V^T P^T of a tile, in stages: what a stage reads of V, and its matrix instructions.
// w: the weights as it takes them, bf16 in PX pieces, or fp32.
template <typename T, int D, int PX> struct ValueStages;
template <int D, int PX> struct ValueStages<uint16_t, D, PX> {
    using Tile = KvTile<uint16_t, D>;
    static constexpr int NU = Tile::KT / 32, COUNT = NU * 2 * (D / 64);      // two blocks of 32 channels each
    struct Part { u32x4_t v[2]; };
    u32x4_t w[NU][2][PX];
    // elements e, e + 1 of the tile's 16 NU (e even)
    __device__ __forceinline__ void set(int e, float p0, float p1) {
        const int u = e / 16, ks = e % 16 / 8;
#pragma unroll
        for (int x = 0; x < PX; ++x) {
            const uint32_t both = pack_bf16(p0, p1);
            w[u][ks][x][e % 8 / 2] = both;
            if (x + 1 < PX) {
                p0 -= __uint_as_float(both << 16);
                p1 -= __uint_as_float(both & 0xffff0000u);
            }
        }
    }
    // rows 16 ks + 4 hf + 0..3 and + 8 of sub-tile u: a sixteenth of the wavefront reads four rows of 16 channels,
    // transposed
    static __device__ __forceinline__ Part read(const char *v, int stage, int lane) {
        const int u = stage / (D / 32), ks = stage / (D / 64) % 2, cb0 = stage % (D / 64) * 2;
        // v_piece with the lane's part apart, which is one of four (two at d = 64): an address of its own for every
        // read took registers that the kernel lacked
        const int r = (lane & 15) >> 2, turn = Tile::CPR == 8 ? r >> 1 : r, last = Tile::CPR == 8 ? 1 : 3;
        const int at = (4 * (lane >> 5) + r) * Tile::ROWB + (((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;
        Part part;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int cb = cb0 + y;
            const char *from = v + at + 64 * ((cb & last) ^ turn) + ((32 * u + 16 * ks) * Tile::ROWB + 256 * (cb / 4));
            union { shortx4_t h[2]; u32x4_t v; } f;
            f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)from);
            f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(from + 8 * Tile::ROWB));
            part.v[y] = f.v;
        }
        return part;
    }
    __device__ __forceinline__ void add(floatx16_t (&o)[D / 32], int stage, const Part &part) const {
        const int u = stage / (D / 32), ks = stage / (D / 64) % 2, cb0 = stage % (D / 64) * 2;
#pragma unroll
        for (int x = 0; x < PX; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) mma_piece<uint16_t>(o[cb0 + y], part.v[y], w[u][ks][x]);
    }
};
template <int D, int PX> struct ValueStages<float, D, PX> {
    using Tile = KvTile<float, D>;
    static constexpr int NU = Tile::KT / 32, COUNT = 16 * NU;                // a register's rows each
    struct Part { float v[D / 32]; };
    float w[16 * NU];
    __device__ __forceinline__ void set(int e, float p0, float p1) {
        w[e] = p0;
        w[e + 1] = p1;
    }
    static __device__ __forceinline__ Part read(const char *v, int stage, int lane) {
        // channel 32 cb + lane % 32 of row tile_row: v_piece, with the lane's part apart, which is one of two (the
        // compiler keeps an address of its own for every read otherwise, 157 registers too many at d = 256)
        const int hf = lane >> 5, at = 4 * hf * Tile::ROWB + 4 * (lane & 31), side[2] = {at + 128 * hf, at + 128 * (1 - hf)};
        const int row = 32 * (stage / 16) + tile_row(stage % 16, 0);
        Part part;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) part.v[cb] = *(const float *)(v + side[cb & 1] + row * Tile::ROWB + 256 * (cb / 2));
        return part;
    }
    __device__ __forceinline__ void add(floatx16_t (&o)[D / 32], int stage, const Part &part) const {
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) o[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(part.v[cb], w[stage], o[cb], 0, 0, 0);
    }
};

template <bool V> struct BoolTag { static constexpr bool value = V; };
constexpr float kTopSlack = 8.0f;
// wavefronts a SIMD: as many as registers and LDS hold (fp32, d = 64, 4096 rows of 8 heads: 178 us with two, 167 with three)
template <typename T, int D> constexpr int kRowsWaves = D > 128 ? 1 : D == 64 && sizeof(T) == 4 ? 3 : 2;

template <typename T, int D, int PX, bool CAP, bool BIAS>
__global__ __launch_bounds__(kRowsThreads) __attribute__((amdgpu_waves_per_eu(kRowsWaves<T, D>, kRowsWaves<T, D>))) void attend_rows_kernel(RowsArgs a) {
    using Tile = KvTile<T, D>;
    constexpr int KT = Tile::KT, CPR = Tile::CPR, NU = KT / 32, NG = KT / 16;
    constexpr int LOADS = KT * CPR / kRowsThreads;               // pieces of K (and of V) a thread brings
    constexpr int NKS = CPR / 2;                                 // pairs of pieces along the channels
    __shared__ __align__(16) char s_k0[Tile::BYTES], s_v0[Tile::BYTES], s_k1[Tile::BYTES], s_v1[Tile::BYTES];
    constexpr int kAhead = 64;                                   // tiles that are looked up together
    __shared__ int s_rows[kAhead * NG];
    __shared__ int s_lo[4], s_hi[4];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    // all workgroups of a KV head on one XCD where there are eight heads or more (its L2 then serves the
    // head's keys), long rows first
    const int bh = (int)blockIdx.x % a.BH, rest = (int)blockIdx.x / a.BH;
    const int split = rest % a.n_split, qt = a.n_tiles - 1 - rest / a.n_split;
    const int b = bh / a.map.Hkv, h = bh - b * a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    if (qt * kRowsQueries >= run.count * a.G) return;

    // ---- this lane's query: the two halves of the wavefront share it
    const int m = qt * kRowsQueries + wave * 32 + (lane & 31);
    const bool valid = (m >> a.g_log2) < run.count;
    const int i = run.begin + (m >> a.g_log2);
    int lo = 0, hi = -1;
    u32x4_t q[NKS];
    if (valid) {
        row_span(a.mods, b, i, run.len(), a.map.max_n, lo, hi);
        const T *src = (const T *)a.q + query_at(a, b, h, m) * D;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) q[ks] = *(const u32x4_t *)((const char *)src + (2 * ks + hf) * 16);
    } else {
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) q[ks] = 0;
    }
    const float slope2 = a.mods.slopes && valid ? a.mods.slopes[h * a.G + (m & (a.G - 1))] * kLog2e : 0.0f;

    // ---- the keys any query of the workgroup sees: without documents, from the first row's first to the last
    //      row's last
    int k_lo, k_hi;
    if (a.mods.doc_begin == nullptr) {
        const int i0 = run.begin + ((qt * kRowsQueries) >> a.g_log2);
        int unused;
        row_span(a.mods, b, i0, run.len(), a.map.max_n, k_lo, unused);
        row_span(a.mods, b, min(i0 + (kRowsQueries >> a.g_log2), run.len()) - 1, run.len(), a.map.max_n, unused, k_hi);
    } else {
        const bool sees = lo <= hi;
        int lo_w = sees ? lo : 0x7fffffff, hi_w = sees ? hi : -1;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            lo_w = min(lo_w, __shfl_xor(lo_w, o));
            hi_w = max(hi_w, __shfl_xor(hi_w, o));
        }
        if (lane == 0) {
            s_lo[wave] = lo_w;
            s_hi[wave] = hi_w;
        }
        __syncthreads();
        k_lo = min(min(s_lo[0], s_lo[1]), min(s_lo[2], s_lo[3]));
        k_hi = max(max(s_hi[0], s_hi[1]), max(s_hi[2], s_hi[3]));
    }
    k_hi = __builtin_amdgcn_readfirstlane(k_hi);
    const int base = __builtin_amdgcn_readfirstlane(k_lo & ~15);
    const int n_tiles = k_hi >= 0 ? (k_hi - base) / KT + 1 : 0;
    const int per = (n_tiles + a.n_split - 1) / a.n_split;
    const int t_begin = split * per, t_end = min(n_tiles, t_begin + per);

    // ---- staging, straight from memory into LDS: a load of a wavefront fills 64 pieces in a row there, so the
    //      turn of the pieces is done in the address it reads.  Its rows lie in one sixteen of the cache (a block
    //      holds whole ones).  A buffer is an array of its own, and the loop goes over both: the compiler then sees
    //      that reads of one need not wait for the other's loads.
    constexpr int RPL = kRowsThreads / CPR;          // rows that all wavefronts' loads of one turn cover
    const bool paged = a.map.block_table != nullptr;
    const int w_row = wave * 64 / CPR, l_row = lane / CPR, l_piece = lane % CPR;      // first row of the wavefront in a turn, row and piece of the lane
    // the lane's byte in its wavefront's rows of a turn, and whether that is the same for every turn
    constexpr bool ONE_TURN = RPL % 16 == 0;
    auto byte_of = [&](int p, bool values) __attribute__((always_inline)) {
        const int row = (p * RPL + w_row) % 16 + l_row;
        return (uint32_t)(l_row * Tile::ROWB + (values ? Tile::v_turned(row, l_piece) : Tile::k_turned(row, l_piece)) * 16);
    };
    const uint32_t k_byte = byte_of(0, false), v_byte = byte_of(0, true);
    const int64_t head_row = paged ? 0 : (int64_t)bh * a.map.max_n + base;
    const char *const k_head = (const char *)a.K + head_row * Tile::ROWB, *const v_head = (const char *)a.V + head_row * Tile::ROWB;
    int looked_up = t_begin;
    // Paged: the first rows of the sixteens of kAhead tiles, looked up together, wait in LDS (one by one, as
    // scalar loads between the reads of the tiles, they held those up: 777 + 333 rows behind 5003 and 2001 107 us).
    auto look_up = [&](int tile) __attribute__((always_inline)) {
        looked_up = tile;
        for (int x = tid; x < kAhead * NG; x += kRowsThreads) {
            const int t = min(base + tile * KT + 16 * x, k_hi & ~15);
            s_rows[x] = (int)a.map.row(b, h, t);     // (rows are numbered in 31 bits; -1: no block)
        }
    };
    int row[LOADS];                                  // paged: where the rows of K begin that were loaded last; V's of that tile are next
#pragma unroll
    for (int p = 0; p < LOADS; ++p) row[p] = 0;
    auto load_rows = [&](int tile, const char *head, uint32_t byte, char *to, auto is_v) __attribute__((always_inline)) {
        constexpr bool VALUES = decltype(is_v)::value;
        const int t0 = base + tile * KT;
        // (one branch per tile for the form of the address: address arithmetic was a third of the instructions)
        if (!paged && t0 + KT - 1 <= k_hi) {
            const char *from = head + (int64_t)(tile * KT + w_row) * Tile::ROWB;
#pragma unroll
            for (int p = 0; p < LOADS; ++p)
                lds_fill(from + p * RPL * Tile::ROWB + (ONE_TURN ? byte : byte_of(p, VALUES)), to + (p * kRowsThreads + wave * 64) * 16);
        } else {
            if (paged && !VALUES) {
#pragma unroll
                for (int p = 0; p < LOADS; ++p) row[p] = s_rows[(tile - looked_up) * NG + (p * RPL + w_row) / 16];
#pragma unroll
                for (int p = 0; p < LOADS; ++p) row[p] = max(__builtin_amdgcn_readfirstlane(row[p]), 0);
            }
#pragma unroll
            for (int p = 0; p < LOADS; ++p) {
                const int in16 = (p * RPL + w_row) % 16;          // the wavefront's first row in its sixteen
                const int first = min(t0 + p * RPL + w_row - in16, k_hi & ~15);
                const int start = paged ? row[p] : first - base;
                const char *from = head + (int64_t)start * Tile::ROWB;
                // (rows behind the last key read it again)
                const int in = min(in16 + l_row, k_hi - first);
                lds_fill(from + (uint32_t)((in - l_row) * Tile::ROWB + (int)(ONE_TURN ? byte : byte_of(p, VALUES))), to + (p * kRowsThreads + wave * 64) * 16);
            }
        }
    };
    auto load_k = [&](int tile, char *to) __attribute__((always_inline)) { load_rows(tile, k_head, k_byte, to, BoolTag<false>()); };
    auto load_v = [&](int tile, char *to) __attribute__((always_inline)) { load_rows(tile, v_head, v_byte, to, BoolTag<true>()); };

    floatx16_t o[D / 32];
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb) o[cb] = 0.0f;
    const float ninf = -__builtin_inff();
    // what the weights are taken against, and this lane's half of their sum.  It need not be the maximum
    // itself: it stays, and the sums with it, until a logit is 2^8 above it.
    float top = ninf, sum = 0.0f;

    constexpr int E = 16 * NU;                       // logits a lane holds of a tile
    // logit e of a lane is that of key 4 hf + key_row(e) of the tile.  (The lane's part apart, so that nothing but
    // constants differs between the logits: their sums with it were kept in registers otherwise, one each.)
    auto key_row = [](int e) __attribute__((always_inline)) { return 32 * (e / 16) + tile_row(e % 16, 0); };
    const int i_lane = i - 4 * hf - base;
    // fp32 tiles go one part after the other: an instruction keeps its matrix unit busy for 64 cycles, next to which
    // the softmax is little, and the registers of two tiles' logits are spared (2011 rows of 8 heads, d = 64, 33.7 us
    // in the order of the bf16 ones, 30.5 in this; 2048 rows, d = 256, 235 and 224).  A scheduling barrier ends each
    // read and its products: reads that all go first take their registers together.
    constexpr bool SERIAL = sizeof(T) == 4;
    auto read_k = [&](const char *kt, int ks, u32x4_t (&f)[NU]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u)                  // (k_piece of row 32 u + lane % 32)
            f[u] = *(const u32x4_t *)(kt + Tile::k_piece(lane & 31, 2 * ks + hf) * 16 + 32 * u * Tile::ROWB);
    };
    auto products = [&](const char *kt, floatx16_t (&s)[NU]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u) s[u] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            u32x4_t f[NU];
            read_k(kt, ks, f);
#pragma unroll
            for (int u = 0; u < NU; ++u) mma_piece<T>(s[u], f[u], q[ks]);
            if (SERIAL) __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto across = [&](float x) __attribute__((always_inline)) {              // the larger of the two halves'
        auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    };
    auto largest = [&](const floatx16_t (&s)[NU]) __attribute__((always_inline)) {
        float mx = s[0][0];
#pragma unroll
        for (int e = 1; e < E; ++e) mx = fmaxf(mx, s[e / 16][e % 16]);
        return across(mx);
    };
    // masks, and `top` raised where a logit asks for it
    auto settle = [&](int tile, floatx16_t (&s)[NU], float mx) __attribute__((always_inline)) {
        const int t0 = base + tile * KT;
        int gone = 0;
        if (paged) {
#pragma unroll
            for (int g = 0; g < NG; ++g) gone |= (s_rows[(tile - looked_up) * NG + g] < 0) << g;
            gone = __builtin_amdgcn_readfirstlane(gone);
        }
        if (__any(valid && (lo > t0 || hi < t0 + KT - 1)) || gone) {
            // (a row that sees nothing: every difference is negative, and so above the span 0)
            const uint32_t span = lo <= hi ? (uint32_t)(hi - lo) : 0u;
            int from = lo <= hi ? t0 + 4 * hf - lo : -0x40000000;
            asm volatile("" : "+v"(from));           // (its sums belong here, not ahead of the branch)
            if (gone == 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) s[e / 16][e % 16] = (uint32_t)(from + key_row(e)) <= span ? s[e / 16][e % 16] : ninf;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) s[e / 16][e % 16] = (((uint32_t)(from + key_row(e)) <= span) & !((gone >> (e / 8)) & 1)) ? s[e / 16][e % 16] : ninf;
            }
            mx = largest(s);
        }
        const bool raise = mx > kTopSlack || (top == ninf && mx > ninf);
        if (__any(raise)) {
            const float by = raise ? mx : 0.0f, alpha = top == ninf ? 1.0f : exp2_fast(-by);   // (nothing yet: nothing to scale)
            if (raise) top = (top == ninf ? 0.0f : top) + by;
            sum *= alpha;
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb) o[cb] *= alpha;
#pragma unroll
            for (int e = 0; e < E; ++e) s[e / 16][e % 16] -= by;
        }
    };
    // One tile, whose logits are there.  The exponentials run beside the products of the next tile's keys, its
    // values beside the next tile's logits; the tile after that is on its way.  In stages of a few matrix instructions,
    // whose operands are read from LDS a stage or two before (the compiler's own order reads each right before its
    // use, and every matrix instruction waits for LDS) and the vector work of the softmax shared out among them.
    auto sees = [&](int tile) __attribute__((always_inline)) {
        const int t0 = base + tile * KT;
        return __any(valid && lo <= t0 + KT - 1 && hi >= t0);
    };
    bool seen = true;                                // whether the wavefront sees the tile at hand
    auto tile_step = [&](int tile, floatx16_t (&s)[NU], const char *k_next, const char *v_now, char *k_to, char *v_to) __attribute__((always_inline)) {
        using Values = ValueStages<T, D, PX>;
        // (stages that operands are read ahead; 4096 rows, 16 heads, d = 256: 223 us with one, 211 with two; d = 128, 8192
        // rows 551 and 547; capped logits lack the registers, 212 and 220 with a bias)
        constexpr int AHEAD = CAP ? 1 : 2, RING = AHEAD + 1;
        u32x4_t fk[RING][NU];
        typename Values::Part fv[RING];
        Values values;
        if (paged && tile + 3 - looked_up > kAhead) {
            look_up(tile + 1);                       // (the barrier behind the last tile: its readers are done)
            __syncthreads();
        }
        if (tile + 1 < t_end) load_v(tile + 1, v_to);
        if (tile + 2 < t_end) load_k(tile + 2, k_to);
        const bool was_seen = seen;
        seen = tile + 1 < t_end && sees(tile + 1);
        if constexpr (SERIAL) {
            if (was_seen) {
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float p0 = exp2_fast(s[e / 16][e % 16]), p1 = exp2_fast(s[e / 16][e % 16 + 1]);
                    part += p0 + p1;
                    values.set(e, p0, p1);
                }
                sum += part;
#pragma unroll
                for (int st = 0; st < Values::COUNT; ++st) {
                    const typename Values::Part part_v = Values::read(v_now, st, lane);
                    values.add(o, st, part_v);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (seen) {
                products(k_next, s);
                const LogitOf<CAP, BIAS> logit(a.mods, (float)(i_lane - (tile + 1) * KT), slope2, top == ninf ? 0.0f : top);
#pragma unroll
                for (int e = 0; e < E; ++e) s[e / 16][e % 16] = logit.any(s[e / 16][e % 16], key_row(e));
                settle(tile + 1, s, largest(s));
            }
        } else
        if (was_seen || seen) {                      // (neither: the logits are -inf, and stay it)
#pragma unroll
        for (int ks = 0; ks < AHEAD; ++ks) read_k(k_next, ks, fk[ks]);
        floatx16_t c[NU];                            // (behind the last tile: products of what the buffer holds, not used)
#pragma unroll
        for (int u = 0; u < NU; ++u) c[u] = 0.0f;
        float part[2] = {0.0f, 0.0f};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            if (ks + AHEAD < NKS) read_k(k_next, ks + AHEAD, fk[(ks + AHEAD) % RING]);
            else fv[(ks + AHEAD - NKS) % RING] = Values::read(v_now, ks + AHEAD - NKS, lane);
#pragma unroll
            for (int u = 0; u < NU; ++u) mma_piece<T>(c[u], fk[ks % RING][u], q[ks]);
#pragma unroll
            for (int e = E * ks / NKS / 2 * 2; e < E * (ks + 1) / NKS / 2 * 2; e += 2) {
                const float p0 = exp2_fast(s[e / 16][e % 16]), p1 = exp2_fast(s[e / 16][e % 16 + 1]);
                part[0] += p0;
                part[1] += p1;
                values.set(e, p0, p1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum += part[0] + part[1];
        const float ref = top == ninf ? 0.0f : top;
        const LogitOf<CAP, BIAS> logit(a.mods, (float)(i_lane - (tile + 1) * KT), slope2, ref);
        float mx = ninf, most = 0.0f;
#pragma unroll
        for (int st = 0; st < Values::COUNT; ++st) {
            if (st + AHEAD < Values::COUNT) fv[(st + AHEAD) % RING] = Values::read(v_now, st + AHEAD, lane);
            values.add(o, st, fv[st % RING]);
#pragma unroll
            for (int e = E * st / Values::COUNT; e < E * (st + 1) / Values::COUNT; ++e) {
                c[e / 16][e % 16] = logit.small(c[e / 16][e % 16], key_row(e), most);
                mx = fmaxf(mx, c[e / 16][e % 16]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (tile + 1 < t_end) {
            mx = across(mx);
            if (CAP && !__all(most <= kCapSmall)) {  // (also a NaN among them is no matter: the logit is one in either form)
                products(k_next, c);
#pragma unroll
                for (int e = 0; e < E; ++e) c[e / 16][e % 16] = logit.any(c[e / 16][e % 16], key_row(e));
                mx = largest(c);
            }
            settle(tile + 1, c, mx);
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) s[u] = c[u];
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): this wavefront's part of what comes next is there
        __syncthreads();
    };
    if (t_begin < t_end) {
        floatx16_t s[NU];
        if (paged) {
            look_up(t_begin);
            __syncthreads();
        }
        load_k(t_begin, s_k0);
        load_v(t_begin, s_v0);
        if (t_begin + 1 < t_end) load_k(t_begin + 1, s_k1);
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
        products(s_k0, s);
        const LogitOf<CAP, BIAS> logit(a.mods, (float)(i_lane - t_begin * KT), slope2, 0.0f);
#pragma unroll
        for (int e = 0; e < E; ++e) s[e / 16][e % 16] = logit.any(s[e / 16][e % 16], key_row(e));
        settle(t_begin, s, largest(s));
        __syncthreads();
        for (int tile = t_begin; tile < t_end; tile += 2) {
            tile_step(tile, s, s_k1, s_v0, s_k0, s_v1);
            if (tile + 1 < t_end) tile_step(tile + 1, s, s_k0, s_v1, s_k1, s_v0);
        }
    }

    // ---- results
    sum = xor32_sum(sum);
    float check = 0.0f * sum;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) check = fmaf(0.0f, o[cb][r], check);
    unsigned long long again = __ballot(valid && !(check == 0.0f));
    again = (again | (again >> 32)) & 0xffffffffull;
    if (valid && !((again >> (lane & 31)) & 1ull)) {
        const int64_t at = query_at(a, b, h, m);
        if (a.n_split > 1) {
            float *part = a.partials + (at * a.n_split + split) * (D + 2);
            if (hf == 0) *(float2 *)part = make_float2(top, sum);
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
                for (int r = 0; r < 16; r += 2) *(float2 *)(part + 2 + 32 * cb + tile_row(r, hf)) = make_float2(o[cb][r], o[cb][r + 1]);
        } else {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int ch = 32 * cb + tile_row(r, hf);
                    const f32x4_t y = {o[cb][r] * inv, o[cb][r + 1] * inv, o[cb][r + 2] * inv, o[cb][r + 3] * inv};
                    if (a.out_dtype == SOCKET_F32) *(f32x4_t *)((float *)a.out + at * D + ch) = y;
                    else *(uint2 *)((uint16_t *)a.out + at * D + ch) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
                }
            }
            if (a.lse && hf == 0) a.lse[at] = sum == 0.0f ? ninf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
    while (again) {
        const int n = __builtin_ctzll(again);
        again &= again - 1;
        const int nlo = max(__builtin_amdgcn_readlane(lo, n), base + t_begin * KT);
        const int nhi = min(__builtin_amdgcn_readlane(hi, n), base + t_end * KT - 1);
        attend_plain<T, D>(a, b, h, __builtin_amdgcn_readlane(m, n), __builtin_amdgcn_readlane(i, n), nlo, nhi, split);
    }
}

// ---- few rows: at most 16 NQ queries (rows times query heads) to a KV head, so K and V are read for
// nothing else and what counts is bytes in flight.  A workgroup is one wavefront with a share of the keys
// of its own: 32 rows of K and V (16 of wide fp32 rows) come into registers, coalesced, while it works
// on the 32 before them, which lie in its LDS; no barriers.  16 x 16 tiles: keys by queries, then
// channels by queries.
template <typename T, int D> struct FewTile {
    static constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16;
    static constexpr int KT = sizeof(T) == 2 || D == 64 ? 32 : 16, NT = KT / 16;
    static constexpr int BYTES = KT * ROWB, LOADS = KT * CPR / 64;
    static __device__ __forceinline__ int k_piece(int row, int c) { return row * CPR + (c ^ (row & (CPR < 16 ? CPR - 1 : 15))); }
    // bf16: four rows of 32 bytes are read at once; fp32: rows 4 g + r of four g, 64 bytes each
    static __device__ __forceinline__ int v_piece(int row, int c) {
        return row * CPR + (c ^ (sizeof(T) == 2 ? (row & 3) << 1 : ((row >> 2) & 3) << 2));
    }
};

template <typename T, int D, int NQ, int PX>
__global__ __launch_bounds__(64) void attend_few_kernel(RowsArgs a) {
    using Tile = FewTile<T, D>;
    constexpr int KT = Tile::KT, NT = Tile::NT, CPR = Tile::CPR, LOADS = Tile::LOADS, NKS = CPR / 4, NCB = D / 16;
    constexpr int RPL = 64 / CPR > 0 ? 64 / CPR : 1;             // rows per load (wide rows: a part of one)
    extern __shared__ __align__(16) char few_tiles[];            // K, V
    char *const kt = few_tiles, *const vt = few_tiles + Tile::BYTES;

    const int lane = threadIdx.x, g = lane >> 4;
    const int bh = (int)blockIdx.x % a.BH, rest = (int)blockIdx.x / a.BH;
    const int m0 = rest % a.n_tiles * 16 * NQ, split = rest / a.n_tiles;     // (column blocks side by side: they read the same keys)
    const int b = bh / a.map.Hkv, h = bh - b * a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    const int n_m = run.count * a.G;
    if (m0 >= n_m) return;

    // ---- queries of column block x: m = m0 + 16 x + lane % 16
    int lo[NQ], hi[NQ], lo_w = 0x7fffffff, hi_w = -1;
    u32x4_t q[NQ][NKS];
    float slope2[NQ];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const int m = m0 + 16 * x + (lane & 15);
        lo[x] = 0x7fffffff;
        hi[x] = -1;
        slope2[x] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) q[x][ks] = 0;
        if (m < n_m) {
            row_span(a.mods, b, run.begin + (m >> a.g_log2), run.len(), a.map.max_n, lo[x], hi[x]);
            const char *src = (const char *)a.q + query_at(a, b, h, m) * Tile::ROWB;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) q[x][ks] = *(const u32x4_t *)(src + (4 * ks + g) * 16);
            if (a.mods.slopes) slope2[x] = a.mods.slopes[h * a.G + (m & (a.G - 1))] * kLog2e;
            if (lo[x] <= hi[x]) {
                lo_w = min(lo_w, lo[x]);
                hi_w = max(hi_w, hi[x]);
            }
        }
    }
    // the longest span of the batch decides how many keys a split takes: the same for all sequences, so that
    // those of a long one are not behind at the end
    int longest = a.mods.window > 0 && a.mods.window < run.len() ? min(run.len(), a.mods.window + run.count - 1) : run.len();
    if (a.batch > 1) longest = longest_of(a.row_begin, a.row_count, a.batch, a.max_rows, a.map.max_n, a.mods.window);
    int k_lo = a.mods.window > 0 ? max(0, run.begin - a.mods.window + 1) : 0, k_hi = run.len() - 1;
    if (a.mods.doc_begin) {
#pragma unroll
        for (int o = 1; o < 16; o *= 2) {
            lo_w = min(lo_w, __shfl_xor(lo_w, o));
            hi_w = max(hi_w, __shfl_xor(hi_w, o));
        }
        k_lo = lo_w;
        k_hi = hi_w;
    }
    k_hi = __builtin_amdgcn_readfirstlane(k_hi);
    const int base = __builtin_amdgcn_readfirstlane(k_lo & ~15);
    const int n_tiles = k_hi >= 0 ? (k_hi - base) / KT + 1 : 0;
    const int share = ((longest + 15 + KT - 1) / KT + a.n_split - 1) / a.n_split;
    const int per = __builtin_amdgcn_readfirstlane(max(share, 1));
    const int t_begin = min(n_tiles, split * per), t_end = min(n_tiles, t_begin + per);

    // ---- rows of a tile, sixteen by sixteen (a block holds whole sixteens)
    const BlockRows rows(a.map, b, h);
    u32x4_t kreg[LOADS], vreg[LOADS];
    int blk[NT], gone = 0, gone_next = 0;            // blocks of the tile that is loaded next; sixteenths without one
    auto look_up = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            blk[y] = 0;
            if (a.map.block_table && tile < t_end)
                blk[y] = scalar_load(&a.map.block_table[(int64_t)b * a.map.max_blocks + a.map.page_slot(min(base + tile * KT + 16 * y, k_hi))]);
        }
    };
    auto load = [&](int tile) __attribute__((always_inline)) {
        gone_next = 0;
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            const int first = min(base + tile * KT + 16 * y, k_hi & ~15);     // of the sixteen
            const bool absent = (unsigned)blk[y] >= (unsigned)rows.blocks;
            gone_next |= absent << y;
            const int64_t at = rows.at(absent ? 0 : blk[y], first);
            const char *ks = (const char *)a.K + at * Tile::ROWB, *vs = (const char *)a.V + at * Tile::ROWB;
            const int last = k_hi - first;           // rows behind the last key read it again
#pragma unroll
            for (int p = 0; p < LOADS / NT; ++p) {
                const int id = p * 64 + lane;
                const uint32_t off = (uint32_t)(min(id / CPR, last) * Tile::ROWB + id % CPR * 16);
                kreg[y * (LOADS / NT) + p] = *(const u32x4_t *)(ks + off);
                vreg[y * (LOADS / NT) + p] = *(const u32x4_t *)(vs + off);
            }
        }
    };
    static_assert(16 % RPL == 0, "a load stays within a sixteen");

    floatx4v_t o[NQ][NCB];
    float top[NQ], sum[NQ];
    const float ninf = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        top[x] = ninf;
        sum[x] = 0.0f;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb) o[x][cb] = 0.0f;
    }
    if (t_begin < t_end) {
        look_up(t_begin);
        load(t_begin);
        look_up(t_begin + 1);
    }
    for (int tile = t_begin; tile < t_end; ++tile) {
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            const int id = p * 64 + lane, row = id / CPR, c = id % CPR;
            *(u32x4_t *)(kt + Tile::k_piece(row, c) * 16) = kreg[p];
            *(u32x4_t *)(vt + Tile::v_piece(row, c) * 16) = vreg[p];
        }
        gone = gone_next;
        if (tile + 1 < t_end) {
            load(tile + 1);
            look_up(tile + 2);
        }
        const int t0 = base + tile * KT;
        // ---- logits
        float s[NQ][4 * NT];
        {
            Tile16<T> c[NQ][NT];
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const u32x4_t kf = *(const u32x4_t *)(kt + Tile::k_piece(16 * t + (lane & 15), 4 * ks + g) * 16);
#pragma unroll
                    for (int x = 0; x < NQ; ++x) c[x][t].add(kf, q[x][ks]);
                }
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const floatx4v_t dots = c[x][t].total();
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[x][4 * t + e] = dots[e];
                }
        }
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            const float ref = top[x] == ninf ? 0.0f : top[x];
            logits2(a.mods, s[x], (float)(run.begin + ((m0 + 16 * x + (lane & 15)) >> a.g_log2) - 4 * g - t0), slope2[x], ref,
                    [](int e) { return 16 * (e / 4) + e % 4; });
            if (__any(lo[x] > t0 || hi[x] < t0 + KT - 1) || gone) {
                const uint32_t span = lo[x] <= hi[x] ? (uint32_t)(hi[x] - lo[x]) : 0u;
                const int from = lo[x] <= hi[x] ? t0 + 4 * g - lo[x] : -0x40000000;
#pragma unroll
                for (int e = 0; e < 4 * NT; ++e)
                    s[x][e] = (((uint32_t)(from + 16 * (e / 4) + e % 4) <= span) & !((gone >> (e / 4)) & 1)) ? s[x][e] : ninf;
            }
            float mx = s[x][0];
#pragma unroll
            for (int e = 1; e < 4 * NT; ++e) mx = fmaxf(mx, s[x][e]);
            mx = sixteenths_max(mx);
            const bool raise = mx > kTopSlack || (top[x] == ninf && mx > ninf);
            if (__any(raise)) {
                const float by = raise ? mx : 0.0f, alpha = top[x] == ninf ? 1.0f : exp2_fast(-by);
                if (raise) top[x] = ref + by;
                sum[x] *= alpha;
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb) o[x][cb] *= alpha;
#pragma unroll
                for (int e = 0; e < 4 * NT; ++e) s[x][e] -= by;
            }
            float part = 0.0f;
#pragma unroll
            for (int e = 0; e < 4 * NT; ++e) {
                s[x][e] = exp2_fast(s[x][e]);
                part += s[x][e];
            }
            sum[x] += part;
        }
        // ---- values
        if constexpr (sizeof(T) == 2) {
            u32x4_t w[NQ][PX];
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int y = 0; y < PX; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[x][y][e] = pack_bf16(s[x][2 * e], s[x][2 * e + 1]);
                        if (y + 1 < PX) {
                            s[x][2 * e] -= __uint_as_float(w[x][y][e] << 16);
                            s[x][2 * e + 1] -= __uint_as_float(w[x][y][e] & 0xffff0000u);
                        }
                    }
            const int row = 4 * g + ((lane & 15) >> 2), c0 = (lane & 3) >> 1, in = (lane & 1) * 8;
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb) {
                union { shortx4_t h[2]; u32x4_t v; } f;
                f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vt + Tile::v_piece(row, c0 + 2 * cb) * 16 + in));
                f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vt + Tile::v_piece(row + 16, c0 + 2 * cb) * 16 + in));
#pragma unroll
                for (int x = 0; x < NQ; ++x)
#pragma unroll
                    for (int y = 0; y < PX; ++y) o[x][cb] = mma16(f.v, w[x][y], o[x][cb]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4 * NT; ++e) {
                const int row = 16 * (e / 4) + 4 * g + e % 4, ch = lane & 15;
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb) {
                    const float v = *(const float *)(vt + Tile::v_piece(row, 4 * cb + (ch >> 2)) * 16 + (ch & 3) * 4);
#pragma unroll
                    for (int x = 0; x < NQ; ++x) o[x][cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[x][e], o[x][cb], 0, 0, 0);
                }
            }
        }
    }

    // ---- results
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const int m = m0 + 16 * x + (lane & 15);
        const float total = xor32_sum(xor16_sum(sum[x]));
        float check = 0.0f * total;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
            for (int r = 0; r < 4; ++r) check = fmaf(0.0f, o[x][cb][r], check);
        unsigned long long again = __ballot(m < n_m && !(check == 0.0f));
        again |= again >> 32;
        again = (again | (again >> 16)) & 0xffffull;
        if (m < n_m && !((again >> (lane & 15)) & 1ull)) {
            const int64_t at = query_at(a, b, h, m);
            if (a.n_split > 1) {
                float *part = a.partials + (at * a.n_split + split) * (D + 2);
                if (g == 0) *(float2 *)part = make_float2(top[x], total);
                if (t_begin < t_end) {
#pragma unroll
                    for (int cb = 0; cb < NCB; ++cb) {
                        *(float2 *)(part + 2 + 16 * cb + 4 * g) = make_float2(o[x][cb][0], o[x][cb][1]);
                        *(float2 *)(part + 4 + 16 * cb + 4 * g) = make_float2(o[x][cb][2], o[x][cb][3]);
                    }
                }
            } else {
                const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb) {
                    const f32x4_t y = {o[x][cb][0] * inv, o[x][cb][1] * inv, o[x][cb][2] * inv, o[x][cb][3] * inv};
                    if (a.out_dtype == SOCKET_F32) *(f32x4_t *)((float *)a.out + at * D + 16 * cb + 4 * g) = y;
                    else *(uint2 *)((uint16_t *)a.out + at * D + 16 * cb + 4 * g) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
                }
                if (a.lse && g == 0) a.lse[at] = total == 0.0f ? ninf : (top[x] + __builtin_amdgcn_logf(total)) * kLn2;
            }
        }
        while (again) {
            const int n = __builtin_ctzll(again);
            again &= again - 1;
            const int mq = m0 + 16 * x + n;
            const int nlo = max(__builtin_amdgcn_readlane(lo[x], n), base + t_begin * KT);
            const int nhi = min(__builtin_amdgcn_readlane(hi[x], n), base + t_end * KT - 1);
            attend_plain<T, D>(a, b, h, mq, run.begin + (mq >> a.g_log2), nlo, nhi, split);
        }
    }
}

// Joins the splits of one query: out = sum_s w_s acc_s / sum_s w_s l_s, w_s = exp2(m_s - max m), by channel
// pairs; a group of threads takes every NG-th split.  Bound by latency: all loads go out before the first is
// used (one after the other, 128 splits of 32 query heads took 17 us).
constexpr int kRowsMergeThreads = 512;
template <int D>
__global__ __launch_bounds__(kRowsMergeThreads) void attend_rows_merge_kernel(RowsArgs a) {
    constexpr int PAIRS = D / 2, NG = kRowsMergeThreads / PAIRS, BATCH = 8, NB = kMaxSplits / (NG * BATCH);
    __shared__ float s_w[kMaxSplits], s_sum, s_top;
    __shared__ float2 s_red[kRowsMergeThreads];
    const int tid = threadIdx.x, c = tid % PAIRS, grp = tid / PAIRS;
    const int hq = blockIdx.x, r = blockIdx.y, b = blockIdx.z;
    const int64_t at = ((int64_t)b * a.max_rows + r) * a.Hq + hq;
    const float *part = a.partials + at * a.n_split * (D + 2);
    const float ninf = -__builtin_inff();
    float m[2], l[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int s = tid + 64 * j;
        const bool live = tid < 64 && s < a.n_split;
        const float2 ml = live ? *(const float2 *)&part[(int64_t)s * (D + 2)] : make_float2(ninf, 0.0f);
        m[j] = ml.x;
        l[j] = ml.y;
    }
    float2 x[NB][BATCH];
#pragma unroll
    for (int y = 0; y < NB; ++y) {
        if (y * BATCH * NG < a.n_split) {
#pragma unroll
            for (int j = 0; j < BATCH; ++j) x[y][j] = *(const float2 *)&part[(int64_t)min((y * BATCH + j) * NG + grp, a.n_split - 1) * (D + 2) + 2 + 2 * c];
        }
    }
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    if (r >= run.count) return;                      // (what was read is not used)
    if (tid < 64) {
        const float top = wave_max(fmaxf(m[0], m[1])), use = top == ninf ? 0.0f : top;
        const float w0 = exp2_fast(m[0] - use), w1 = exp2_fast(m[1] - use);
        const float sum = row_sum<64>(w0 * l[0] + w1 * l[1]);
        s_w[tid] = w0;
        s_w[tid + 64] = w1;
        if (tid == 0) {
            s_sum = sum;
            s_top = top;
        }
    }
    __syncthreads();
    float2 acc = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int y = 0; y < NB; ++y) {
        if (y * BATCH * NG < a.n_split) {
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int s = (y * BATCH + j) * NG + grp;
                const float w = s < a.n_split ? s_w[s] : 0.0f;
                // (a split without keys has written no values)
                acc.x = w != 0.0f ? fmaf(w, x[y][j].x, acc.x) : acc.x;
                acc.y = w != 0.0f ? fmaf(w, x[y][j].y, acc.y) : acc.y;
            }
        }
    }
    s_red[tid] = acc;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
        for (int k = 1; k < NG; ++k) {
            const float2 v = s_red[k * PAIRS + c];
            acc.x += v.x;
            acc.y += v.y;
        }
        const float sum = s_sum, y0 = sum == 0.0f ? 0.0f : acc.x / sum, y1 = sum == 0.0f ? 0.0f : acc.y / sum;
        if (a.out_dtype == SOCKET_F32) *(float2 *)((float *)a.out + at * D + 2 * c) = make_float2(y0, y1);
        else *(uint32_t *)((uint16_t *)a.out + at * D + 2 * c) = pack_bf16(y0, y1);
        if (a.lse && c == 0) a.lse[at] = sum == 0.0f ? ninf : (s_top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

// The same for few splits of many queries: a wavefront each (2011 rows of 8 heads in 4 splits: 34 us with a
// workgroup each).
constexpr int kFewSplits = 16;
template <int D>
__global__ __launch_bounds__(256) void attend_rows_merge_few_kernel(RowsArgs a, int n_items) {
    constexpr int PER = D / 64;
    const int lane = threadIdx.x & 63, item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (item >= n_items) return;
    const int row = item / a.Hq, b = row / a.max_rows, r = row - b * a.max_rows;
    const float *part = a.partials + (int64_t)item * a.n_split * (D + 2);
    const float ninf = -__builtin_inff();
    const float2 ml = lane < a.n_split ? *(const float2 *)&part[lane * (D + 2)] : make_float2(ninf, 0.0f);
    float x[kFewSplits][PER];
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s)
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (s < a.n_split) x[s][k] = part[s * (D + 2) + 2 + lane + 64 * k];
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    if (r >= run.count) return;                      // (what was read is not used)
    const float top = wave_max(ml.x), use = top == ninf ? 0.0f : top, w = exp2_fast(ml.x - use);
    const float sum = row_sum<64>(w * ml.y);
    float acc[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) acc[k] = 0.0f;
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
        if (s < a.n_split) {
            const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
            // (a split without keys has written no values)
#pragma unroll
            for (int k = 0; k < PER; ++k) acc[k] = ws != 0.0f ? fmaf(ws, x[s][k], acc[k]) : acc[k];
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const float y = sum == 0.0f ? 0.0f : acc[k] / sum;
        if (a.out_dtype == SOCKET_F32) ((float *)a.out)[(int64_t)item * D + lane + 64 * k] = y;
        else ((uint16_t *)a.out)[(int64_t)item * D + lane + 64 * k] = f32_to_bf16_rne(y);
    }
    if (a.lse && lane == 0) a.lse[item] = sum == 0.0f ? ninf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int D, bool CAP, bool BIAS> static void launch_rows(const RowsArgs &a, dim3 grid, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (a.out_dtype == SOCKET_F32) {
            hipLaunchKernelGGL((attend_rows_kernel<T, D, 3, CAP, BIAS>), grid, dim3(kRowsThreads), 0, st, a);
            return;
        }
    }
    hipLaunchKernelGGL((attend_rows_kernel<T, D, 1, CAP, BIAS>), grid, dim3(kRowsThreads), 0, st, a);
}
template <typename T, int D> static void launch_rows(const RowsArgs &a, dim3 grid, hipStream_t st) {
    const bool cap = a.mods.a > 0.0f, bias = a.mods.slopes != nullptr;
    if (cap && bias) launch_rows<T, D, true, true>(a, grid, st);
    else if (cap) launch_rows<T, D, true, false>(a, grid, st);
    else if (bias) launch_rows<T, D, false, true>(a, grid, st);
    else launch_rows<T, D, false, false>(a, grid, st);
}

template <typename T, int D, int PX> static void launch_few(const RowsArgs &a, bool wide, dim3 grid, hipStream_t st) {
    constexpr size_t lds = 2 * FewTile<T, D>::BYTES;
    static_assert(lds <= 64 * 1024, "within the default dynamic LDS limit");
    if constexpr (D < 256) {
        if (wide) {
            hipLaunchKernelGGL((attend_few_kernel<T, D, 2, PX>), grid, dim3(64), lds, st, a);
            return;
        }
    }
    hipLaunchKernelGGL((attend_few_kernel<T, D, 1, PX>), grid, dim3(64), lds, st, a);
}
template <typename T, int D> static void launch_few(const RowsArgs &a, bool wide, dim3 grid, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (a.out_dtype == SOCKET_F32) return launch_few<T, D, 3>(a, wide, grid, st);
    }
    launch_few<T, D, sizeof(T) == 2 ? 2 : 1>(a, wide, grid, st);
}

template <int D> static void launch_rows_merge(const RowsArgs &a, bool few, int items, dim3 grid, hipStream_t st) {
    if (few) hipLaunchKernelGGL(attend_rows_merge_few_kernel<D>, grid, dim3(256), 0, st, a, items);
    else hipLaunchKernelGGL(attend_rows_merge_kernel<D>, grid, dim3(kRowsMergeThreads), 0, st, a);
}

static int pick_splits(int64_t wanted, int64_t most, int64_t room) {
    int64_t n = wanted < most ? wanted : most;
    n = n < room ? n : room;
    n = n < kMaxSplits ? n : kMaxSplits;
    return n < 1 ? 1 : (int)n;
}

int launch_attend_rows(socket_ctx *ctx, const void *q, const void *K, const void *V, const int32_t *block_table,
                       const int32_t *row_begin, const int32_t *row_count, int batch, int max_rows, float scale,
                       const socket_attn_mods *mods, int out_dtype, void *out, float *lse, hipStream_t st) {
    const Geometry &g = ctx->g;
    RowsArgs a;
    a.q = q; a.K = K; a.V = V; a.out = out; a.lse = lse; a.partials = ctx->partials;
    a.row_begin = row_begin; a.row_count = row_count;
    a.map = row_map(g, block_table);
    a.mods = row_mods(scale, mods);
    a.BH = batch * g.Hkv; a.Hq = g.Hq; a.G = g.G; a.g_log2 = __builtin_ctz((unsigned)g.G);
    a.max_rows = max_rows; a.out_dtype = out_dtype;
    a.batch = batch;
    const int64_t room = ctx->partial_floats / ((int64_t)batch * max_rows * g.Hq * (g.d + 2));   // splits whose results fit
    const bool f32 = g.kv_dtype == SOCKET_F32;
    if ((int64_t)max_rows * g.G <= 32) {
        // One wavefront a split, 32 keys each at least (64: 4096 fp32 keys of one head 14.5 us, not 11.6; 131072 of 8
        // heads the same): with 16 and more of them to a compute unit the last ones to finish are a small part.
        // More than 16 queries are two column blocks of a wavefront, at d = 256 (whose registers do not hold
        // two: 8 rows of 4 heads behind 32000 151 us) of two wavefronts.
        const bool two = max_rows * g.G > 16, wide = two && g.d < 256;
        a.n_tiles = two && !wide ? 2 : 1;
        a.n_split = pick_splits(8192 / (a.BH * a.n_tiles), (g.max_n + 31) / 32, room);
        const int64_t grid = (int64_t)a.BH * a.n_tiles * a.n_split;
        if (grid * 64 >= (int64_t)1 << 32) return SOCKET_EUNSUPPORTED;       // (threads of a launch)
        const dim3 gr((unsigned)grid);
        switch (g.d) {
            case 64: f32 ? launch_few<float, 64>(a, wide, gr, st) : launch_few<uint16_t, 64>(a, wide, gr, st); break;
            case 128: f32 ? launch_few<float, 128>(a, wide, gr, st) : launch_few<uint16_t, 128>(a, wide, gr, st); break;
            case 256: f32 ? launch_few<float, 256>(a, wide, gr, st) : launch_few<uint16_t, 256>(a, wide, gr, st); break;
            default: return SOCKET_EUNSUPPORTED;
        }
    } else {
        // Two workgroups per compute unit keep it busy (one at d = 256, where one fits); with fewer the keys are split,
        // as far as the partial results fit (half as many splits: 256 rows behind 32000 245 us instead of 180).  Where
        // the run is most of the cache its first rows see few keys and its last ones many, and twice as many even that
        // out (4096 fp32 rows of 8 heads 455 -> 340 us, 8192 bf16 rows of 8 heads 221 -> 200; but 2048 rows behind
        // 16384 179 -> 197; at d = 256 four to a compute unit: 2048 fp32 rows of 8 heads 195 -> 230).
        // A split's products have to be worth the results it leaves: 512 keys and more in bf16 (256: 512 prompt rows
        // of 32 heads 23 us with the launch that joins them, 17 without), 256 or 128 where a tile of queries or two is
        // all there is and the chain of a split's tiles is what the call waits for (34 rows behind 1633, 16 workgroups,
        // 18 us with 512, 14 with 128; 167 rows of 16 heads behind 2436, 24 workgroups, 23 with 512, 22 with 256, 29
        // with 128); in fp32 they take longer the wider the heads (512 at
        // d = 64: 256 there 33 -> 42 us for 2011 rows; 256 at d = 128: 1024 rows 97 -> 59; 128 at d = 256: 300 rows
        // 54 -> 46).
        a.n_tiles = (int)(((int64_t)max_rows * g.G + kRowsQueries - 1) / kRowsQueries);
        const int64_t wgs = (int64_t)a.BH * a.n_tiles;
        const int wanted = (2 * (int64_t)max_rows >= g.max_n ? 1024 : 512) / (g.d == 256 ? 2 : 1), least = f32 ? 32768 / g.d : wgs <= 16 ? 128 : wgs <= 64 ? 256 : 512;
        a.n_split = pick_splits(wanted / wgs, (g.max_n + least - 1) / least, room);
        const int64_t grid = wgs * a.n_split;
        if (grid * kRowsThreads >= (int64_t)1 << 32) return SOCKET_EUNSUPPORTED;
        const dim3 gr((unsigned)grid);
        switch (g.d) {
            case 64: f32 ? launch_rows<float, 64>(a, gr, st) : launch_rows<uint16_t, 64>(a, gr, st); break;
            case 128: f32 ? launch_rows<float, 128>(a, gr, st) : launch_rows<uint16_t, 128>(a, gr, st); break;
            case 256: f32 ? launch_rows<float, 256>(a, gr, st) : launch_rows<uint16_t, 256>(a, gr, st); break;
            default: return SOCKET_EUNSUPPORTED;
        }
    }
    if (a.n_split > 1) {
        // (items fit 32 bits: their partial results do in the scratch)
        const int items = batch * max_rows * g.Hq;
        const bool few = a.n_split <= kFewSplits && items > 1024;
        const dim3 mg = few ? dim3((items + 3) / 4) : dim3(g.Hq, max_rows, batch);
        switch (g.d) {
            case 64: launch_rows_merge<64>(a, few, items, mg, st); break;
            case 128: launch_rows_merge<128>(a, few, items, mg, st); break;
            default: launch_rows_merge<256>(a, few, items, mg, st); break;
        }
    }
    return record_hip(ctx, hipGetLastError());
}

}  // namespace sk
