// How much attention each cached key got from a run of rows:
//     mass[j] = decay mass[j] + sum over rows i that see j, and the group's query heads, of exp(s_ij - lse_i)
// (keys of the run itself start from 0), lse as attention returned it.  Sums of columns of the
// softmax matrix, so a wavefront owns keys, not rows: it keeps their rows of K in registers and takes
// the queries one tile after the other.  The logits' tile is K Q^T as in the attention, so that a
// lane has one query (one lse, one span of keys) and a few keys, whose sums it keeps in registers;
// the queries of a tile are added up once, at the end, in a fixed order.  No atomics: the same
// masses bit for bit on every run.
//
// Bounds and figures: many queries by the matrix units and, as much, by the softmax's vector work, which no second
// product shares: 4096 rows of 32 heads, d = 128, 118 us = 0.58 PFLOP/s, with a cap 160; fp32, 8 heads, 214 us =
// 0.080 (a large product reaches 1.19, and 0.135 in fp32).  One token by memory: 16 ragged paged sequences up to
// 32768 keys 145 us = 4.8 TB/s, what a large copy reaches.
#include "attend_device.h"

namespace sk {

struct MassArgs {
    const void *q;
    const void *K;
    const float *lse;
    float *mass;
    float *partials;          // [BH][n_seg][max_n] where the queries are split
    const int32_t *row_begin;
    const int32_t *row_count;
    RowMap map;
    RowMods mods;
    int batch, BH, Hq, G, g_log2, max_rows, last_rows, n_seg, seg_tiles;
    float decay;
};

// Queries m_lo .. m_hi - 1 (rows times query heads) that may see a key of j0 .. j1: from the first
// whose own position or prefix reaches j0 to the last whose window does.
__device__ __forceinline__ void queries_of(const MassArgs &a, const RowRun &run, int b, int j0, int j1, int &m_lo, int &m_hi) {
    int r_lo = a.last_rows > 0 && a.last_rows < run.count ? run.count - a.last_rows : 0, r_hi = run.count - 1;
    const bool prefixed = a.mods.prefix_len && scalar_load(&a.mods.prefix_len[b]) > j0;
    if (!prefixed) r_lo = max(r_lo, j0 - run.begin);
    if (a.mods.window > 0 && j1 < 0x7fffffff - a.mods.window) r_hi = min(r_hi, j1 + a.mods.window - 1 - run.begin);
    m_lo = r_lo * a.G;
    m_hi = max(m_lo, (r_hi + 1) * a.G);
}

__device__ __forceinline__ float kept_mass(const MassArgs &a, const RowRun &run, int j, float old, float mine) {
    return j < run.begin && a.decay != 0.0f ? fmaf(a.decay, old, mine) : mine;
}

// ---- many queries: a workgroup's four wavefronts own 32 keys each and share the queries, 64 at a time, in
//      two LDS buffers that are filled straight from memory.  (64 keys each read half as much of LDS, but their
//      registers leave room for two wavefronts a SIMD, not three: 4096 rows 128 us against 118.)  Long runs are cut into
//      segments, whose sums a second launch adds up: the first keys of a prompt are seen by all of
//      its rows, the last by few, and with segments no workgroup has more to do than another.
constexpr int kMassThreads = 256, kMassKeys = 128;

template <typename T, int D> struct MassTile {
    static constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16;
    static constexpr int WAVES = ROWB > 512 ? 1 : ROWB > 256 ? 2 : 3;                    // per SIMD
    static constexpr int QT = ROWB <= 512 ? 64 : 32, NU = QT / 32;                       // queries per tile
    static constexpr int BYTES = QT * ROWB, LOADS = QT * CPR / kMassThreads;
    static __device__ __forceinline__ int turned(int row, int c) { return c ^ (row & (CPR < 16 ? CPR - 1 : 15)); }
};
struct MassMeta {             // what a tile's queries bring beside their channels
    int lo[64], hi[64], i[64];
    float lse[64], slope[64];
};

template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(kMassThreads) __attribute__((amdgpu_waves_per_eu(MassTile<T, D>::WAVES, MassTile<T, D>::WAVES))) void key_mass_kernel(MassArgs a) {
    using Tile = MassTile<T, D>;
    constexpr int ROWB = Tile::ROWB, CPR = Tile::CPR, NKS = CPR / 2, QT = Tile::QT, NU = Tile::NU, LOADS = Tile::LOADS;
    __shared__ __align__(16) char s_q0[Tile::BYTES], s_q1[Tile::BYTES];
    __shared__ MassMeta s_meta0, s_meta1;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const int bh = (int)blockIdx.x % a.BH, rest = (int)blockIdx.x / a.BH;
    const int seg = rest % a.n_seg, kb = rest / a.n_seg;
    const int b = bh / a.map.Hkv, h = bh - b * a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    const int j0 = kb * kMassKeys, len = run.len();
    if (run.count == 0 || j0 >= len) return;
    const int j1 = min(j0 + kMassKeys, len) - 1;
    int m_lo, m_hi;
    queries_of(a, run, b, j0, j1, m_lo, m_hi);
    // segment 0 is there for every key, also one that no query sees (its mass still decays)
    const int t_all = (m_hi - m_lo + QT - 1) / QT, t_begin = seg * a.seg_tiles, t_end = min(t_all, t_begin + a.seg_tiles);
    if (seg > 0 && t_begin >= t_all) return;

    // ---- this wavefront's keys, in registers
    const int w0 = j0 + wave * 32, kj = w0 + (lane & 31);
    const int64_t krow = kj <= j1 ? a.map.row(b, h, kj) : -1;
    const uint32_t there = (uint32_t)__ballot(krow >= 0);
    u32x4_t k[NKS];
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
        k[ks] = 0;
        if (krow >= 0) k[ks] = *(const u32x4_t *)((const char *)a.K + krow * ROWB + (2 * ks + hf) * 16);
    }

    // Tiles start at whole rows (m_lo and QT are multiples of G), so a lane's byte in a turn of loads is the
    // same for every tile and turn, but for where it starts.
    constexpr int RPL = kMassThreads / CPR;          // queries that all wavefronts' loads of one turn cover
    constexpr bool ONE_TURN = RPL % 16 == 0;
    const int w_row = wave * 64 / CPR, l_row = lane / CPR, l_piece = lane % CPR;
    const int64_t row_bytes = (int64_t)a.Hq * ROWB;
    const char *const q_head = (const char *)a.q + (int64_t)b * a.max_rows * row_bytes + (int64_t)h * a.G * ROWB;
    auto byte_of = [&](int p, int row) __attribute__((always_inline)) {      // of query `row` of a tile, in turn p
        return (uint32_t)((row >> a.g_log2) * (a.Hq * ROWB) + (row & (a.G - 1)) * ROWB + Tile::turned((p * RPL + w_row) % 16 + l_row, l_piece) * 16);
    };
    const uint32_t q_byte = byte_of(0, w_row + l_row);
    int n_lo = 0, n_hi = -1, n_i = 0;
    float n_lse = 0.0f, n_slope = 0.0f;
    auto load = [&](int tile, char *qn) __attribute__((always_inline)) {
        const int m0 = m_lo + tile * QT;
        const char *from = q_head + (m0 >> a.g_log2) * row_bytes;
        if (ONE_TURN && m0 + QT <= m_hi) {
#pragma unroll
            for (int p = 0; p < LOADS; ++p) lds_fill(from + (p * RPL >> a.g_log2) * row_bytes + q_byte, qn + (p * kMassThreads + wave * 64) * 16);
        } else {
#pragma unroll
            for (int p = 0; p < LOADS; ++p)          // (queries behind the last read it again)
                lds_fill(from + byte_of(p, min(p * RPL + w_row + l_row, m_hi - 1 - m0)), qn + (p * kMassThreads + wave * 64) * 16);
        }
        // what the tile's queries bring beside their channels: the wavefronts in turn
        const int n = lane, m = m0 + n;
        if ((tile & 3) == wave && n < QT) {
            n_lo = 0;
            n_hi = -1;
            if (m < m_hi) {
                const int hq = h * a.G + (m & (a.G - 1));
                n_i = run.begin + (m >> a.g_log2);
                row_span(a.mods, b, n_i, len, a.map.max_n, n_lo, n_hi);
                n_lse = a.lse[((int64_t)b * a.max_rows + (m >> a.g_log2)) * a.Hq + hq] * kLog2e;
                if (n_lse == -__builtin_inff()) n_hi = -1;       // (a row without weights)
                if (a.mods.slopes) n_slope = a.mods.slopes[hq] * kLog2e;
            }
        }
    };
    auto store_meta = [&](int tile, MassMeta &meta) __attribute__((always_inline)) {
        if ((tile & 3) == wave && lane < QT) {
            meta.lo[lane] = n_lo;
            meta.hi[lane] = n_hi;
            meta.i[lane] = n_i;
            meta.lse[lane] = n_lse;
            if (BIAS) meta.slope[lane] = n_slope;
        }
    };

    floatx16_t acc = 0.0f;
    constexpr int AHEAD = 2, RING = AHEAD + 1;
    // products of the 32 queries u of a tile, in stages: operands are read two stages ahead, and `beside` runs
    // between the matrix instructions
    auto products = [&](const char *qt, int u, floatx16_t &c, auto beside) __attribute__((always_inline)) {
        const int n = 32 * u + (lane & 31);
        u32x4_t f[RING];
        auto read = [&](int ks) __attribute__((always_inline)) { return *(const u32x4_t *)(qt + (n * CPR + Tile::turned(n, 2 * ks + hf)) * 16); };
#pragma unroll
        for (int ks = 0; ks < AHEAD; ++ks) f[ks] = read(ks);
        c = 0.0f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            if (ks + AHEAD < NKS) f[(ks + AHEAD) % RING] = read(ks + AHEAD);
            mma_piece<T>(c, k[ks], f[ks % RING]);
            beside(ks);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // what the 32 queries u add to the keys' masses, element by element, all keys seen
    struct Query { int lo, hi; float lse, dist, slope; };
    auto query = [&](const MassMeta &meta, int u) __attribute__((always_inline)) {
        const int n = 32 * u + (lane & 31);
        return Query{meta.lo[n], meta.hi[n], meta.lse[n], BIAS ? (float)(meta.i[n] - 4 * hf - w0) : 0.0f, BIAS ? meta.slope[n] : 0.0f};
    };
    auto key_row = [](int e) __attribute__((always_inline)) { return tile_row(e, 0); };
    // sums of weights of products c (which become the logits): `whole` where every query sees every key of the
    // wavefront
    auto add_all = [&](floatx16_t &c, const Query &x, bool whole) __attribute__((always_inline)) {
        const LogitOf<CAP, BIAS> logit(a.mods, x.dist, x.slope, x.lse);
        bool small = true;
        if (CAP) {                                   // (scaled first: a wavefront whose arguments all are small takes the ratio alone)
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                c[e] *= logit.c;
                most = fmaxf(most, fabsf(c[e]));
            }
            small = __all(most <= kCapSmall);
        }
        if (whole && small) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                acc[e] += exp2_fast(logit.scaled(c[e], key_row(e), true));
                if (e % 8 == 7) __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
        // (four at a time: more of them under way at once do not fit the registers)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            c[e] = logit.scaled(c[e], key_row(e), false);
            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        // (a row that sees nothing: every difference is negative, and so above the span 0)
        const uint32_t span = x.lo <= x.hi ? (uint32_t)(x.hi - x.lo) : 0u;
        int from = x.lo <= x.hi ? w0 + 4 * hf - x.lo : -0x40000000;
        asm volatile("" : "+v"(from));               // (its sums belong here, not ahead of the branch)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float p = exp2_fast(c[e]);
            const bool vis = ((uint32_t)(from + key_row(e)) <= span) & ((there >> (4 * hf) >> tile_row(e, 0)) & 1u);
            acc[e] += vis ? p : 0.0f;
            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto tile_step = [&](int tile, const char *qt, const MassMeta &meta, char *qn, MassMeta &meta_n) __attribute__((always_inline)) {
        const bool more = tile + 1 < t_end;
        if (more) load(tile + 1, qn);
        floatx16_t c, d;
        Query x = query(meta, 0);
        // (whether any query sees any of the wavefront's keys, and all see all)
        auto any_of = [&](const Query &y) { return __any(y.lo <= w0 + 31 && y.hi >= w0 && y.lo <= y.hi); };
        auto all_of = [&](const Query &y) { return __all(y.lo <= w0 && y.hi >= w0 + 31) && there == 0xffffffffu; };
        if constexpr (NU == 2) {
            const Query z = query(meta, 1);
            if (!CAP && all_of(x) && all_of(z)) {
                // the first half's exponentials beside the second's products (capped, the vector work alone is more than
                // both: the other wavefront's products run beside it)
                products(qt, 0, c, [](int) {});
                const LogitOf<CAP, BIAS> first(a.mods, x.dist, x.slope, x.lse), second(a.mods, z.dist, z.slope, z.lse);
                products(qt, 1, d, [&](int ks) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 16 * ks / NKS; e < 16 * (ks + 1) / NKS; ++e) acc[e] += exp2_fast(first.any(c[e], key_row(e)));
                });
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[e] += exp2_fast(second.any(d[e], key_row(e)));
            } else {
                if (any_of(x)) {
                    products(qt, 0, c, [](int) {});
                    add_all(c, x, all_of(x));
                }
                if (any_of(z)) {
                    products(qt, 1, c, [](int) {});
                    add_all(c, z, all_of(z));
                }
            }
        } else if (any_of(x)) {
            products(qt, 0, c, [](int) {});
            add_all(c, x, all_of(x));
        }
        if (more) store_meta(tile + 1, meta_n);
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): this wavefront's part of the next tile is there
        __syncthreads();
    };
    if (t_begin < t_end) {
        load(t_begin, s_q0);
        store_meta(t_begin, s_meta0);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    for (int tile = t_begin; tile < t_end; tile += 2) {
        tile_step(tile, s_q0, s_meta0, s_q1, s_meta1);
        if (tile + 1 < t_end) tile_step(tile + 1, s_q1, s_meta1, s_q0, s_meta0);
    }

    // ---- over the 32 queries of a tile, then lane r of either half writes register r's key
    float *const part = a.partials + ((int64_t)bh * a.n_seg + seg) * a.map.max_n;
    float *const mass = a.mass + (int64_t)bh * a.map.max_n;
    float mine = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const float t = row_sum<32>(acc[r]);
        mine = (lane & 31) == r ? t : mine;
    }
    const int r = lane & 15, j = w0 + 8 * (r / 4) + 4 * hf + r % 4;
    if ((lane & 31) < 16 && j <= j1) {
        if (a.n_seg > 1) part[j] = mine;
        else mass[j] = kept_mass(a, run, j, mass[j], mine);
    }
}

// adds up the segments, in order
template <int QT>
__global__ __launch_bounds__(256) void key_mass_merge_kernel(MassArgs a) {
    const int bh = (int)blockIdx.x % a.BH, j = (int)blockIdx.x / a.BH * 256 + threadIdx.x, b = bh / a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    if (run.count == 0 || j >= run.len()) return;
    const int j0 = j / kMassKeys * kMassKeys;
    int m_lo, m_hi;
    queries_of(a, run, b, j0, min(j0 + kMassKeys, run.len()) - 1, m_lo, m_hi);
    const int tiles = (m_hi - m_lo + QT - 1) / QT, n = max(1, (tiles + a.seg_tiles - 1) / a.seg_tiles);
    const float *part = a.partials + (int64_t)bh * a.n_seg * a.map.max_n + j;
    float sum = 0.0f;
    for (int s = 0; s < n; ++s) sum += part[(int64_t)s * a.map.max_n];
    float *const at = a.mass + (int64_t)bh * a.map.max_n + j;
    *at = kept_mass(a, run, j, *at, sum);
}

// ---- few queries (at most 16 NQ): K is read for them alone, so what counts is bytes in flight.  Every
//      wavefront walks keys of its own, 32 at a time (16 of wide fp32 rows), their pieces straight from
//      memory into the operand's registers, the next ones under way; 16 x 16 tiles.
template <typename T, int D, int NQ>
__global__ __launch_bounds__(64) void key_mass_few_kernel(MassArgs a) {
    constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16, NKS = CPR / 4, KT = ROWB <= 512 ? 32 : 16, NT = KT / 16;
    const int lane = threadIdx.x, g = lane >> 4;
    const int bh = (int)blockIdx.x % a.BH, share_at = (int)blockIdx.x / a.BH;
    const int b = bh / a.map.Hkv, h = bh - b * a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    if (run.count == 0) return;
    const int len = run.len();
    // the same number of keys for every wavefront of the batch
    const int longest = a.batch > 1 ? longest_of(a.row_begin, a.row_count, a.batch, a.max_rows, a.map.max_n, 0) : len;
    const int per = __builtin_amdgcn_readfirstlane(max(((longest + KT - 1) / KT + a.n_seg - 1) / a.n_seg, 64 / KT));
    const int n_tiles = (len + KT - 1) / KT, t_begin = share_at * per, t_end = min(n_tiles, t_begin + per);
    if (t_begin >= t_end) return;

    const BlockRows rows(a.map, b, h);
    u32x4_t kn[NT][NKS];
    int blk[NT], gone_next = 0;
    float old_next = 0.0f;
    const int e_mine = lane & 15;                    // lane e of a sixteenth writes the mass of its register e
    auto key_of = [&](int t0) { return t0 + 16 * (e_mine / 4) + 4 * g + e_mine % 4; };
    auto look_up = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            blk[y] = 0;
            if (a.map.block_table && tile < t_end)
                blk[y] = scalar_load(&a.map.block_table[(int64_t)b * a.map.max_blocks + a.map.page_slot(min(tile * KT + 16 * y, len - 1))]);
        }
    };
    float *const mass = a.mass + (int64_t)bh * a.map.max_n;
    auto load = [&](int tile) __attribute__((always_inline)) {
        gone_next = 0;
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            const int first = min(tile * KT + 16 * y, (len - 1) & ~15);
            const bool absent = (unsigned)blk[y] >= (unsigned)rows.blocks;
            gone_next |= absent << y;
            const char *ks = (const char *)a.K + rows.at(absent ? 0 : blk[y], first) * ROWB;
            const uint32_t off = (uint32_t)(min(lane & 15, len - 1 - first) * ROWB + g * 16);
#pragma unroll
            for (int x = 0; x < NKS; ++x) kn[y][x] = *(const u32x4_t *)(ks + off + 64 * x);
        }
        const int j = key_of(tile * KT);
        old_next = e_mine < 4 * NT && j < run.begin && a.decay != 0.0f ? mass[j] : 0.0f;
    };
    look_up(t_begin);
    load(t_begin);
    look_up(t_begin + 1);

    // ---- queries of column block x: m = first + 16 x + lane % 16
    const int first_m = a.last_rows > 0 && a.last_rows < run.count ? (run.count - a.last_rows) * a.G : 0, n_m = run.count * a.G;
    int lo[NQ], hi[NQ];
    u32x4_t q[NQ][NKS];
    float slope2[NQ], lse[NQ];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const int m = first_m + 16 * x + (lane & 15);
        lo[x] = 0;
        hi[x] = -1;
        slope2[x] = lse[x] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) q[x][ks] = 0;
        if (m < n_m) {
            const int64_t at = ((int64_t)b * a.max_rows + (m >> a.g_log2)) * a.Hq + h * a.G + (m & (a.G - 1));
            row_span(a.mods, b, run.begin + (m >> a.g_log2), len, a.map.max_n, lo[x], hi[x]);
            lse[x] = a.lse[at] * kLog2e;
            if (lse[x] == -__builtin_inff()) hi[x] = -1;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) q[x][ks] = *(const u32x4_t *)((const char *)a.q + at * ROWB + (4 * ks + g) * 16);
            if (a.mods.slopes) slope2[x] = a.mods.slopes[h * a.G + (m & (a.G - 1))] * kLog2e;
        }
    }
    for (int tile = t_begin; tile < t_end; ++tile) {
        const int t0 = tile * KT, gone = gone_next;
        const float old = old_next;
        Tile16<T> c[NQ][NT];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int y = 0; y < NT; ++y)
#pragma unroll
                for (int x = 0; x < NQ; ++x) c[x][y].add(kn[y][ks], q[x][ks]);
        if (tile + 1 < t_end) {
            load(tile + 1);
            look_up(tile + 2);
        }
        float sum[4 * NT];
#pragma unroll
        for (int e = 0; e < 4 * NT; ++e) sum[e] = 0.0f;
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            float s[4 * NT];
#pragma unroll
            for (int y = 0; y < NT; ++y) {
                const floatx4v_t dots = c[x][y].total();
#pragma unroll
                for (int e = 0; e < 4; ++e) s[4 * y + e] = dots[e];
            }
            logits2(a.mods, s, (float)(run.begin + ((first_m + 16 * x + (lane & 15)) >> a.g_log2) - 4 * g - t0), slope2[x], lse[x],
                    [](int e) { return 16 * (e / 4) + e % 4; });
            const uint32_t span = lo[x] <= hi[x] ? (uint32_t)(hi[x] - lo[x]) : 0u;
            const int from = lo[x] <= hi[x] ? t0 + 4 * g - lo[x] : -0x40000000;
#pragma unroll
            for (int e = 0; e < 4 * NT; ++e) {
                const bool vis = ((uint32_t)(from + 16 * (e / 4) + e % 4) <= span) & !((gone >> (e / 4)) & 1);
                const float p = exp2_fast(s[e]);
                sum[e] += vis ? p : 0.0f;
            }
        }
        float mine = 0.0f;
#pragma unroll
        for (int e = 0; e < 4 * NT; ++e) {
            const float t = row_sum<16>(sum[e]);
            mine = e_mine == e ? t : mine;
        }
        const int j = key_of(t0);
        if (e_mine < 4 * NT && j < len) mass[j] = kept_mass(a, run, j, old, mine);
    }
}

template <typename T, int D, bool CAP, bool BIAS> static int launch_mass_tiles(MassArgs a, int64_t room, int max_n, int rows, hipStream_t st) {
    using Tile = MassTile<T, D>;
    const int64_t tiles = ((int64_t)rows * a.G + Tile::QT - 1) / Tile::QT;
    const int64_t keys = (int64_t)a.BH * ((max_n + kMassKeys - 1) / kMassKeys), most = (tiles + 3) / 4;
    // segments of 16 tiles; shorter ones, four tiles at least, where that is fewer than four workgroups to a compute
    // unit, or eight where the run is most of the cache and half of the workgroups see nothing (500 rows of 32 heads
    // 25 -> 13 us, 4096 fp32 rows of 8 heads 273 -> 214; eight everywhere: four runs of 100 rows behind 2000 18 -> 24)
    const int64_t more = (2 * (int64_t)rows >= max_n ? 2048 : 1024) / keys;
    int64_t seg = more < most ? more : most;
    seg = seg > (tiles + 15) / 16 ? seg : (tiles + 15) / 16;
    const int64_t fits = room / ((int64_t)a.BH * max_n);
    seg = seg < fits ? seg : fits;
    a.n_seg = seg < 1 ? 1 : (int)seg;
    a.seg_tiles = (int)((tiles + a.n_seg - 1) / a.n_seg);
    const int64_t grid = keys * a.n_seg;
    // (threads of a launch; a tile's rows lie within 32 bits of each other)
    if (grid * kMassThreads >= (int64_t)1 << 32 || (int64_t)a.Hq * Tile::ROWB * Tile::QT >= (int64_t)1 << 31) return SOCKET_EUNSUPPORTED;
    hipLaunchKernelGGL((key_mass_kernel<T, D, CAP, BIAS>), dim3((unsigned)grid), dim3(kMassThreads), 0, st, a);
    if (a.n_seg > 1) hipLaunchKernelGGL((key_mass_merge_kernel<Tile::QT>), dim3((unsigned)((max_n + 255) / 256) * (unsigned)a.BH), dim3(256), 0, st, a);
    return SOCKET_OK;
}

template <typename T, int D> static int launch_mass(MassArgs a, int64_t room, int max_n, int max_rows, hipStream_t st) {
    const int rows = a.last_rows > 0 && a.last_rows < max_rows ? a.last_rows : max_rows;
    if ((int64_t)rows * a.G <= 32) {
        // as many wavefronts as keep the card busy, 64 keys each at least
        int64_t n = 8192 / a.BH, most = (max_n + 63) / 64;
        n = n < most ? n : most;
        a.n_seg = n < 1 ? 1 : (int)n;
        const int64_t grid = (int64_t)a.BH * a.n_seg;
        if (grid * 64 >= (int64_t)1 << 32) return SOCKET_EUNSUPPORTED;       // (threads of a launch)
        if ((int64_t)rows * a.G > 16) hipLaunchKernelGGL((key_mass_few_kernel<T, D, 2>), dim3((unsigned)grid), dim3(64), 0, st, a);
        else hipLaunchKernelGGL((key_mass_few_kernel<T, D, 1>), dim3((unsigned)grid), dim3(64), 0, st, a);
        return SOCKET_OK;
    }
    const bool cap = a.mods.a > 0.0f, bias = a.mods.slopes != nullptr;
    return cap && bias ? launch_mass_tiles<T, D, true, true>(a, room, max_n, rows, st) : cap ? launch_mass_tiles<T, D, true, false>(a, room, max_n, rows, st)
           : bias ? launch_mass_tiles<T, D, false, true>(a, room, max_n, rows, st) : launch_mass_tiles<T, D, false, false>(a, room, max_n, rows, st);
}

int launch_key_mass(socket_ctx *ctx, const void *q, const void *K, const float *lse, const int32_t *block_table,
                    const int32_t *row_begin, const int32_t *row_count, int batch, int max_rows, float scale,
                    const socket_attn_mods *mods, float decay, int last_rows, float *mass, hipStream_t st) {
    const Geometry &g = ctx->g;
    MassArgs a;
    a.q = q; a.K = K; a.lse = lse; a.mass = mass; a.partials = ctx->partials; a.row_begin = row_begin; a.row_count = row_count;
    a.map = row_map(g, block_table);
    a.mods = row_mods(scale, mods);
    a.batch = batch; a.BH = batch * g.Hkv; a.Hq = g.Hq; a.G = g.G; a.g_log2 = __builtin_ctz((unsigned)g.G);
    a.max_rows = max_rows; a.last_rows = last_rows; a.decay = decay; a.n_seg = 1; a.seg_tiles = 1;
    const bool f32 = g.kv_dtype == SOCKET_F32;
    const int64_t room = ctx->partial_floats;
    int rc = SOCKET_EUNSUPPORTED;
    switch (g.d) {
        case 64: rc = f32 ? launch_mass<float, 64>(a, room, g.max_n, max_rows, st) : launch_mass<uint16_t, 64>(a, room, g.max_n, max_rows, st); break;
        case 128: rc = f32 ? launch_mass<float, 128>(a, room, g.max_n, max_rows, st) : launch_mass<uint16_t, 128>(a, room, g.max_n, max_rows, st); break;
        case 256: rc = f32 ? launch_mass<float, 256>(a, room, g.max_n, max_rows, st) : launch_mass<uint16_t, 256>(a, room, g.max_n, max_rows, st); break;
    }
    if (rc != SOCKET_OK) return rc;
    return record_hip(ctx, hipGetLastError());
}

}  // namespace sk
