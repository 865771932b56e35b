// How much attention each cached key got from a run of rows:
//     mass[j] = decay mass[j] + sum over rows i that see j, and the group's query heads, of exp(s_ij - lse_i)
// (keys of the run itself start from 0), lse as attention returned it.  Sums of columns of the
// softmax matrix, so a wavefront owns keys, not rows: it keeps their rows of K in registers and takes
// the queries one tile after the other.  The logits' tile is K Q^T as in the attention, so that a
// lane has one query (one lse, one span of keys) and a few keys, whose sums it keeps in registers;
// the queries of a tile are added up once, at the end, in a fixed order.  No atomics: the same
// masses bit for bit on every run.
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

// ---- many queries: a workgroup's four wavefronts own KW keys each and share the queries, 64 at a
//      time, in two LDS buffers that are filled straight from memory.  Long runs are cut into segments
//      of seg_tiles tiles, whose sums a second launch adds up: the first keys of a prompt are seen by all of its
//      rows, the last by few, and with segments no workgroup has more to do than another.
constexpr int kMassThreads = 256;

template <typename T, int D> struct MassTile {
    static constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16;
    static constexpr int KW = sizeof(T) == 2 && D <= 128 ? 64 : 32, NK = KW / 32;        // keys per wavefront
    static constexpr int QT = ROWB <= 512 ? 64 : 32, NU = QT / 32;                       // queries per tile
    static constexpr int BYTES = QT * ROWB, LOADS = QT * CPR / kMassThreads;
    static __device__ __forceinline__ int turned(int row, int c) { return c ^ (row & (CPR < 16 ? CPR - 1 : 15)); }
};
struct MassMeta {             // what a tile's queries bring beside their channels
    int lo[64], hi[64], i[64];
    float lse[64], slope[64];
};

template <typename T, int D>
__global__ __launch_bounds__(kMassThreads, D <= 128 ? 2 : 1) void key_mass_kernel(MassArgs a) {
    using Tile = MassTile<T, D>;
    constexpr int ROWB = Tile::ROWB, CPR = Tile::CPR, NKS = CPR / 2, QT = Tile::QT, NU = Tile::NU, LOADS = Tile::LOADS;
    constexpr int KW = Tile::KW, NK = Tile::NK, KEYS = 4 * KW;
    __shared__ __align__(16) char s_q0[Tile::BYTES], s_q1[Tile::BYTES];
    __shared__ MassMeta s_meta0, s_meta1;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const int bh = (int)blockIdx.x % a.BH, rest = (int)blockIdx.x / a.BH;
    const int seg = rest % a.n_seg, kb = rest / a.n_seg;
    const int b = bh / a.map.Hkv, h = bh - b * a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    const int j0 = kb * KEYS, len = run.len();
    if (run.count == 0 || j0 >= len) return;
    const int j1 = min(j0 + KEYS, len) - 1;
    int m_lo, m_hi;
    queries_of(a, run, b, j0, j1, m_lo, m_hi);
    // segment 0 is there for every key, also one that no query sees (its mass still decays)
    const int t_all = (m_hi - m_lo + QT - 1) / QT, t_begin = seg * a.seg_tiles, t_end = min(t_all, t_begin + a.seg_tiles);
    if (seg > 0 && t_begin >= t_all) return;

    // ---- this wavefront's keys, in registers
    const int w0 = j0 + wave * KW;
    uint32_t there[NK];
    u32x4_t k[NK][NKS];
#pragma unroll
    for (int y = 0; y < NK; ++y) {
        const int kj = w0 + 32 * y + (lane & 31);
        const int64_t krow = kj <= j1 ? a.map.row(b, h, kj) : -1;
        there[y] = (uint32_t)__ballot(krow >= 0);
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            k[y][ks] = 0;
            if (krow >= 0) k[y][ks] = *(const u32x4_t *)((const char *)a.K + krow * ROWB + (2 * ks + hf) * 16);
        }
    }

    int n_lo = 0, n_hi = -1, n_i = 0;
    float n_lse = 0.0f, n_slope = 0.0f;
    const char *const q_head = (const char *)a.q + ((int64_t)b * a.max_rows * a.Hq + h * a.G) * ROWB;
    auto load = [&](int tile, char *qn) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            const int slot = p * kMassThreads + wave * 64, row = (slot + lane) / CPR;
            const int m = min(m_lo + tile * QT + row, m_hi - 1);
            const char *src = q_head + ((int64_t)(m >> a.g_log2) * a.Hq + (m & (a.G - 1))) * ROWB + Tile::turned(row, (slot + lane) % CPR) * 16;
            lds_fill(src, qn + slot * 16);
        }
        if (tid < QT) {
            const int m = m_lo + tile * QT + tid;
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
    auto store_meta = [&](MassMeta &meta) __attribute__((always_inline)) {
        if (tid < QT) {
            meta.lo[tid] = n_lo;
            meta.hi[tid] = n_hi;
            meta.i[tid] = n_i;
            meta.lse[tid] = n_lse;
            meta.slope[tid] = n_slope;
        }
    };

    float acc[NK][16];
#pragma unroll
    for (int y = 0; y < NK; ++y)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[y][r] = 0.0f;
    auto tile_step = [&](int tile, const char *qt, const MassMeta &meta, char *qn, MassMeta &meta_n) __attribute__((always_inline)) {
        const bool more = tile + 1 < t_end;
        if (more) load(tile + 1, qn);
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int n = 32 * u + (lane & 31);
            const int lo = meta.lo[n], hi = meta.hi[n];
            if (!__any(lo <= w0 + KW - 1 && hi >= w0 && lo <= hi)) continue;
            floatx16_t c[NK];
#pragma unroll
            for (int y = 0; y < NK; ++y) c[y] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                const u32x4_t qf = *(const u32x4_t *)(qt + (n * CPR + Tile::turned(n, 2 * ks + hf)) * 16);
#pragma unroll
                for (int y = 0; y < NK; ++y) mma_piece<T>(c[y], k[y][ks], qf);
            }
            const float lse = meta.lse[n];
#pragma unroll
            for (int y = 0; y < NK; ++y) {
                const int v0 = w0 + 32 * y;
                float s[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = c[y][r];
                logits2(a.mods, s, (float)(meta.i[n] - 4 * hf - v0), meta.slope[n], lse, [](int r) { return tile_row(r, 0); });
                if (__all(lo <= v0 && hi >= v0 + 31) && there[y] == 0xffffffffu) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[y][r] += exp2_fast(s[r]);
                } else {
                    // (a row that sees nothing: every difference is negative, and so above the span 0)
                    const uint32_t span = lo <= hi ? (uint32_t)(hi - lo) : 0u, have = there[y] >> (4 * hf);
                    const int from = lo <= hi ? v0 + 4 * hf - lo : -0x40000000;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int row = tile_row(r, 0);
                        const float p = exp2_fast(s[r]);
                        acc[y][r] += (((uint32_t)(from + row) <= span) & ((have >> row) & 1u)) ? p : 0.0f;
                    }
                }
            }
        }
        if (more) store_meta(meta_n);
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): this wavefront's part of the next tile is there
        __syncthreads();
    };
    if (t_begin < t_end) {
        load(t_begin, s_q0);
        store_meta(s_meta0);
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
#pragma unroll
    for (int y = 0; y < NK; ++y) {
        float mine = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float t = row_sum<32>(acc[y][r]);
            mine = (lane & 31) == r ? t : mine;
        }
        const int r = lane & 15, j = w0 + 32 * y + 8 * (r / 4) + 4 * hf + r % 4;
        if ((lane & 31) < 16 && j <= j1) {
            if (a.n_seg > 1) part[j] = mine;
            else mass[j] = kept_mass(a, run, j, mass[j], mine);
        }
    }
}

// adds up the segments, in order
template <int KEYS, int QT>
__global__ __launch_bounds__(256) void key_mass_merge_kernel(MassArgs a) {
    const int bh = (int)blockIdx.x % a.BH, j = (int)blockIdx.x / a.BH * 256 + threadIdx.x, b = bh / a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    if (run.count == 0 || j >= run.len()) return;
    const int j0 = j / KEYS * KEYS;
    int m_lo, m_hi;
    queries_of(a, run, b, j0, min(j0 + KEYS, run.len()) - 1, m_lo, m_hi);
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
        floatx4v_t c[NQ][NT];
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
            for (int y = 0; y < NT; ++y) c[x][y] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int y = 0; y < NT; ++y)
#pragma unroll
                for (int x = 0; x < NQ; ++x) mma_piece16<T>(c[x][y], kn[y][ks], q[x][ks]);
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
            for (int e = 0; e < 4 * NT; ++e) s[e] = c[x][e / 4][e % 4];
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

template <typename T, int D> static int launch_mass(MassArgs a, int64_t room, int max_n, int max_rows, hipStream_t st) {
    using Tile = MassTile<T, D>;
    const int rows = a.last_rows > 0 && a.last_rows < max_rows ? a.last_rows : max_rows;
    if ((int64_t)rows * a.G <= 32) {
        // as many wavefronts as keep the card busy, 64 keys each at least
        int64_t n = 8192 / a.BH, most = (max_n + 63) / 64;
        n = n < most ? n : most;
        a.n_seg = n < 1 ? 1 : (int)n;
        const int64_t grid = (int64_t)a.BH * a.n_seg;
        if (grid >= (int64_t)1 << 31) return SOCKET_EUNSUPPORTED;
        if ((int64_t)rows * a.G > 16) hipLaunchKernelGGL((key_mass_few_kernel<T, D, 2>), dim3((unsigned)grid), dim3(64), 0, st, a);
        else hipLaunchKernelGGL((key_mass_few_kernel<T, D, 1>), dim3((unsigned)grid), dim3(64), 0, st, a);
        return SOCKET_OK;
    }
    constexpr int KEYS = 4 * Tile::KW;
    const int64_t tiles = ((int64_t)rows * a.G + Tile::QT - 1) / Tile::QT;
    int64_t seg = (tiles + 31) / 32;
    const int64_t fits = room / ((int64_t)a.BH * max_n);
    seg = seg < fits ? seg : fits;
    a.n_seg = seg < 1 ? 1 : (int)seg;
    a.seg_tiles = (int)((tiles + a.n_seg - 1) / a.n_seg);
    const int64_t grid = (int64_t)a.BH * ((max_n + KEYS - 1) / KEYS) * a.n_seg;
    if (grid >= (int64_t)1 << 31) return SOCKET_EUNSUPPORTED;
    hipLaunchKernelGGL((key_mass_kernel<T, D>), dim3((unsigned)grid), dim3(kMassThreads), 0, st, a);
    if (a.n_seg > 1) hipLaunchKernelGGL((key_mass_merge_kernel<KEYS, Tile::QT>), dim3((unsigned)((max_n + 255) / 256) * (unsigned)a.BH), dim3(256), 0, st, a);
    return SOCKET_OK;
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
