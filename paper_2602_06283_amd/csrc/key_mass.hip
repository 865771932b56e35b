// How much attention each cached key got from a run of rows:
//     mass[j] = decay mass[j] + sum over rows i that see j, and the group's query heads, of exp(s_ij - lse_i)
// (keys of the run itself start from 0), lse as attention returned it.  Sums of columns of the
// softmax matrix, so a workgroup owns keys, not rows: 128 of them, 32 per wavefront with their rows
// of K in registers, while the queries pass through LDS 32 at a time.  The logits' tile is K Q^T as
// in the attention, so that a lane has one query (one lse, one span of keys) and sixteen keys, whose
// sums it keeps in registers; the 32 queries of a tile are added up once, at the end, in a fixed
// order.  No atomics: the same masses bit for bit on every run.
#include "attend_device.h"

namespace sk {

constexpr int kMassThreads = 256;
constexpr int kMassKeys = 128;                   // keys per workgroup
constexpr int kMassQueries = 64;                 // queries per tile

struct MassArgs {
    const void *q;
    const void *K;
    const float *lse;
    float *mass;
    const int32_t *row_begin;
    const int32_t *row_count;
    RowMap map;
    RowMods mods;
    int BH, Hq, G, g_log2, max_rows, last_rows;
    float decay;
};

template <typename T, int D> constexpr int mass_queries() { return kMassQueries * D * (int)sizeof(T) <= 32768 ? kMassQueries : 32; }
template <typename T, int D> constexpr size_t mass_lds() { return (size_t)2 * mass_queries<T, D>() * D * sizeof(T); }

template <typename T, int D>
__global__ __launch_bounds__(kMassThreads, D <= 128 ? 2 : 1) void key_mass_kernel(MassArgs a) {
    constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16, NKS = CPR / 2;
    constexpr int QT = mass_queries<T, D>(), NU = QT / 32, LOADS = QT * CPR / kMassThreads;
    static_assert(LOADS >= 1, "every thread brings a piece");
    using Tile = KvTile<T, D>;                       // (its turn of the pieces: queries are read as K is in the attention)
    extern __shared__ __align__(16) char mass_tiles[];           // [2][QT queries]
    __shared__ int s_lo[2][QT], s_hi[2][QT], s_i[2][QT];
    __shared__ float s_lse[2][QT], s_slope[2][QT];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hf = lane >> 5;
    const int bh = (int)blockIdx.x % a.BH, kt = (int)blockIdx.x / a.BH;
    const int b = bh / a.map.Hkv, h = bh - b * a.map.Hkv;
    const RowRun run(a.row_begin, a.row_count, b, a.max_rows, a.map.max_n);
    const int j0 = kt * kMassKeys, len = run.len();
    if (run.count == 0 || j0 >= len) return;
    const int j1 = min(j0 + kMassKeys, len) - 1;

    // ---- rows that can see a key of j0 .. j1: from the first whose own position or prefix reaches j0 to
    //      the last whose window does
    int r_lo = a.last_rows > 0 && a.last_rows < run.count ? run.count - a.last_rows : 0, r_hi = run.count - 1;
    const bool prefixed = a.mods.prefix_len && scalar_load(&a.mods.prefix_len[b]) > j0;
    if (!prefixed) r_lo = max(r_lo, j0 - run.begin);
    if (a.mods.window > 0 && j1 < 0x7fffffff - a.mods.window) r_hi = min(r_hi, j1 + a.mods.window - 1 - run.begin);
    const int m_lo = r_lo * a.G, m_hi = (r_hi + 1) * a.G;        // queries m_lo .. m_hi - 1
    const int n_tiles = m_hi > m_lo ? (m_hi - m_lo + QT - 1) / QT : 0;

    // ---- this wavefront's keys, in registers
    const int kj = j0 + wave * 32 + (lane & 31);
    const int64_t krow = kj <= j1 ? a.map.row(b, h, kj) : -1;
    const unsigned long long there_all = __ballot(krow >= 0);
    const uint32_t there = (uint32_t)there_all;
    u32x4_t k[NKS];
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
        k[ks] = 0;
        if (krow >= 0) k[ks] = *(const u32x4_t *)((const char *)a.K + krow * ROWB + (2 * ks + hf) * 16);
    }
    const int w0 = j0 + wave * 32, w1 = min(w0 + 31, j1);

    u32x4_t qreg[LOADS];
    int n_lo = 0, n_hi = -1, n_i = 0;
    float n_lse = 0.0f, n_slope = 0.0f;
    auto load = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            const int id = p * kMassThreads + tid, c = id % CPR;
            const int m = min(m_lo + tile * QT + id / CPR, m_hi - 1);
            const int64_t at = ((int64_t)b * a.max_rows + (m >> a.g_log2)) * a.Hq + h * a.G + (m & (a.G - 1));
            qreg[p] = turn_sign<T>(*(const u32x4_t *)((const char *)a.q + at * ROWB + c * 16), a.mods.sign);
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
    auto store = [&](int buf) __attribute__((always_inline)) {
        char *qt = mass_tiles + buf * QT * ROWB;
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            const int id = p * kMassThreads + tid, row = id / CPR, c = id % CPR;
            *(u32x4_t *)(qt + Tile::k_piece(row, c) * 16) = qreg[p];
        }
        if (tid < QT) {
            s_lo[buf][tid] = n_lo;
            s_hi[buf][tid] = n_hi;
            s_i[buf][tid] = n_i;
            s_lse[buf][tid] = n_lse;
            s_slope[buf][tid] = n_slope;
        }
    };

    float acc[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    if (n_tiles > 0) {
        load(0);
        store(0);
    }
    __syncthreads();
    for (int tile = 0; tile < n_tiles; ++tile) {
        const int buf = tile & 1;
        const char *qt = mass_tiles + buf * QT * ROWB;
        const bool more = tile + 1 < n_tiles;
        if (more) load(tile + 1);
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int n = 32 * u + (lane & 31);
            const int lo = s_lo[buf][n], hi = s_hi[buf][n];
            if (!__any(lo <= w1 && hi >= w0 && lo <= hi) || there == 0) continue;
            floatx16_t c = 0.0f;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                mma_piece<T>(c, k[ks], *(const u32x4_t *)(qt + Tile::k_piece(n, 2 * ks + hf) * 16));
            float s[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = c[r];
            float cc = a.mods.c;
            if (a.mods.general) {
                logits2(a.mods, s, (float)(s_i[buf][n] - w0), s_slope[buf][n], [&](int r) { return tile_row(r, hf); });
                cc = 1.0f;
            }
            const float lse = s_lse[buf][n];
            if (__all(lo <= w0 && hi >= w0 + 31) && there == 0xffffffffu) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] += exp2_fast(fmaf(s[r], cc, -lse));
            } else {
                const uint32_t span = (uint32_t)(hi - lo);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = tile_row(r, hf);
                    const bool vis = lo <= hi && (uint32_t)(w0 + row - lo) <= span && ((there >> row) & 1u);
                    const float p = exp2_fast(fmaf(s[r], cc, -lse));
                    acc[r] += vis ? p : 0.0f;
                }
            }
        }
        if (more) store(buf ^ 1);
        __syncthreads();
    }

    // ---- over the 32 queries of a tile, then lane r of either half writes register r's key
    float mine = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const float t = row_sum<32>(acc[r]);
        mine = (lane & 31) == r ? t : mine;
    }
    if ((lane & 31) < 16) {
        const int r = lane & 15, j = w0 + 8 * (r / 4) + 4 * hf + r % 4;
        if (j <= j1) {
            float *at = a.mass + ((int64_t)b * a.map.Hkv + h) * a.map.max_n + j;
            *at = j < run.begin && a.decay != 0.0f ? fmaf(a.decay, *at, mine) : mine;
        }
    }
}

template <typename T, int D> static int mass_allow() {
    constexpr size_t lds = mass_lds<T, D>();
    if (lds <= 64 * 1024) return SOCKET_OK;
    return hipFuncSetAttribute((const void *)key_mass_kernel<T, D>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess
               ? SOCKET_OK : SOCKET_EHIP;
}
int mass_prepare(int d, int kv_dtype) {
    const bool f32 = kv_dtype == SOCKET_F32;
    return d == 64    ? (f32 ? mass_allow<float, 64>() : mass_allow<uint16_t, 64>())
           : d == 128 ? (f32 ? mass_allow<float, 128>() : mass_allow<uint16_t, 128>())
                      : (f32 ? mass_allow<float, 256>() : mass_allow<uint16_t, 256>());
}

template <typename T, int D> static void launch_mass(const MassArgs &a, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((key_mass_kernel<T, D>), grid, dim3(kMassThreads), (mass_lds<T, D>()), st, a);
}

int launch_key_mass(socket_ctx *ctx, const void *q, const void *K, const float *lse, const int32_t *block_table,
                    const int32_t *row_begin, const int32_t *row_count, int batch, int max_rows, float scale,
                    const socket_attn_mods *mods, float decay, int last_rows, float *mass, hipStream_t st) {
    const Geometry &g = ctx->g;
    MassArgs a;
    a.q = q; a.K = K; a.lse = lse; a.mass = mass; a.row_begin = row_begin; a.row_count = row_count;
    a.map = row_map(g, block_table);
    a.mods = row_mods(scale, mods);
    a.BH = batch * g.Hkv; a.Hq = g.Hq; a.G = g.G; a.g_log2 = __builtin_ctz((unsigned)g.G);
    a.max_rows = max_rows; a.last_rows = last_rows; a.decay = decay;
    const int64_t grid = (int64_t)a.BH * ((g.max_n + kMassKeys - 1) / kMassKeys);
    if (grid >= (int64_t)1 << 31) return SOCKET_EUNSUPPORTED;
    const dim3 gr((unsigned)grid);
    const bool f32 = g.kv_dtype == SOCKET_F32;
    switch (g.d) {
        case 64: f32 ? launch_mass<float, 64>(a, gr, st) : launch_mass<uint16_t, 64>(a, gr, st); break;
        case 128: f32 ? launch_mass<float, 128>(a, gr, st) : launch_mass<uint16_t, 128>(a, gr, st); break;
        case 256: f32 ? launch_mass<float, 256>(a, gr, st) : launch_mass<uint16_t, 256>(a, gr, st); break;
        default: return SOCKET_EUNSUPPORTED;
    }
    return record_hip(ctx, hipGetLastError());
}

}  // namespace sk
