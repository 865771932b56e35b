// Eviction: the scores that rank tokens by the attention they gathered, and the move of the kept
// tokens' rows - K, V, bucket ids, value norms, masses - to the front of a cache.
//
// A move is bound by its bytes, once read and once written.  Bucket ids do not move as they are: a
// token's row of ids is stored turned by its position (socket.h), so a string of 16 ids that goes from
// position t to t' is turned by t' - t more ids.
#include "attend_device.h"

namespace sk {

// ---- scores: the mass, pooled over the tokens around (the largest of pool of them); +inf for the
//      tokens that are always kept, -inf behind the sequence and where there is no block
//      Bound by latency on one sequence (32768 tokens of 8 heads, pool 5: 3.8 us), by the 8 bytes a token on many
//      (16 ragged paged sequences 5.4 us; a token a thread 9.4): four tokens a thread.
constexpr int kPoolThreads = 256, kPoolTokens = 4 * kPoolThreads, kPoolMax = 255;

struct EvictScoreArgs {
    const float *mass;
    float *scores;
    const int32_t *seq_len;
    RowMap map;
    int pool, n_sink, n_window;
};

__global__ __launch_bounds__(kPoolThreads) void evict_scores_kernel(EvictScoreArgs a) {
    constexpr int HALO = (kPoolMax / 2 + 3) / 4 * 4;
    __shared__ __align__(16) float s_x[kPoolTokens + 2 * HALO];  // masses from HALO tokens before the first
    __shared__ int s_gone[kPoolTokens / 16];
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z, side = a.pool / 2;
    const int t0 = blockIdx.x * kPoolTokens, t = t0 + 4 * tid;
    const int64_t row = ((int64_t)b * a.map.Hkv + h) * a.map.max_n;
    const int len = min(a.seq_len[b], a.map.max_n);
    const float ninf = -__builtin_inff(), most = 3.4028234663852886e38f;
    // (max_n is a multiple of 16: a thread's four tokens are all inside it or all behind it)
    f32x4_t s = {ninf, ninf, ninf, ninf};
    if (t0 < len) {
        // (NaN and -inf: the last to be kept; +inf: behind the tokens that are always kept)
        auto clean = [&](float x) { return x >= -most ? fminf(x, most) : -most; };
        f32x4_t own = s;
        if (t < len) own = *(const f32x4_t *)&a.mass[row + t];               // (whole: len <= max_n)
#pragma unroll
        for (int e = 0; e < 4; ++e) own[e] = t + e < len ? clean(own[e]) : ninf;
        *(f32x4_t *)&s_x[HALO + 4 * tid] = own;
        if (tid < 2 * side) {
            const int u = tid < side ? t0 - side + tid : t0 + kPoolTokens + tid - side;
            s_x[HALO + u - t0] = u >= 0 && u < len ? clean(a.mass[row + u]) : ninf;
        }
        if (a.map.block_table && tid < kPoolTokens / 16) {
            const int u = t0 + 16 * tid;
            s_gone[tid] = u < len && a.map.row(b, h, u) < 0;
        }
        __syncthreads();
        s = own;
        if (side && side <= 4) {                     // the four tokens before and the four behind, 16 bytes each
            const f32x4_t left = *(const f32x4_t *)&s_x[HALO + 4 * tid - 4], right = *(const f32x4_t *)&s_x[HALO + 4 * tid + 4];
            const float x[12] = {left.x, left.y, left.z, left.w, own.x, own.y, own.z, own.w, right.x, right.y, right.z, right.w};
#pragma unroll
            for (int o = 1; o <= 4; ++o) {
                if (o > side) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = fmaxf(s[e], fmaxf(x[4 + e - o], x[4 + e + o]));
            }
        } else if (side) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float *x = &s_x[HALO + 4 * tid + e - side];
                for (int o = 0; o < a.pool; ++o) s[e] = fmaxf(s[e], x[o]);
            }
        }
        const bool gone = a.map.block_table && s_gone[tid / 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (t + e < a.n_sink || t + e >= len - a.n_window) s[e] = __builtin_inff();
            if (t + e >= len || gone) s[e] = ninf;
        }
    }
    if (t < a.map.max_n) *(f32x4_t *)&a.scores[row + t] = s;
}

// ---- moving rows
struct MoveArgs {
    const int32_t *idx;
    const int32_t *n_selected;
    const void *K;
    const void *V;
    const char *codes;
    const float *vnorm;
    const float *mass;
    void *K_out;
    void *V_out;
    char *codes_out;
    float *vnorm_out;
    float *mass_out;
    RowMap src, dst;
    int max_k, Lpad, GT, strings, cb;            // strings: of 16 ids, in a token's row of ids; cb = 0: packed, 10 bits an id
    // ordered kernel: workgroups of a head, in this order
    int k_slices, v_slices, code_slices, vnorm_slices, mass_slices;
};

// where entry j of the index row comes from and goes to; -1: it does not
__device__ __forceinline__ void move_rows(const MoveArgs &a, int b, int h, int j, int count, int &t, int64_t &from, int64_t &to) {
    t = j < count ? a.idx[((int64_t)b * a.src.Hkv + h) * a.max_k + j] : -1;
    from = t >= 0 && t < a.src.max_n ? a.src.row(b, h, t) : -1;
    to = from >= 0 ? a.dst.row(b, h, j) : -1;
    if (to < 0) from = -1;
}

// bits [n, n + 32 N) of the N words repeated without end
template <int N, int STEP> __device__ __forceinline__ void turn_step(uint32_t (&w)[N], int by) {
    // (by masks: a choice between two words became one between their addresses, and the words memory)
    const uint32_t mask = (by & STEP) ? 0xffffffffu : 0u;
    uint32_t x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = w[i] ^ ((w[i] ^ w[(i + STEP) % N]) & mask);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = x[i];
}
template <int N> __device__ __forceinline__ void turn_words(uint32_t (&w)[N], int n) {
    uint32_t x[N];
    turn_step<N, 1>(w, n >> 5);
    turn_step<N, 2>(w, n >> 5);
    if constexpr (N > 4) turn_step<N, 4>(w, n >> 5);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_alignbit(w[(i + 1) % N], w[i], n & 31);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = x[i];
}

// one string of 16 ids: CB = 1, 2 bytes an id, or 0: 160 bits, 16 bytes in the tile's main rows and 4 in its tail rows
template <int CB> struct IdString {
    static constexpr int N = CB == 2 ? 8 : CB == 1 ? 4 : 5;
    uint32_t w[N];
    __device__ __forceinline__ void load(const MoveArgs &a, int64_t row, int s) {
        if (CB == 0) {
            const int S = a.GT / 16, grp = s / S, sub = s - grp * S;
            const u32x4_t v = *(const u32x4_t *)(a.codes + packed_word(row, grp, sub, 0, a.Lpad, a.GT));
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = v[i];
            w[N - 1] = *(const uint32_t *)(a.codes + packed_word(row, grp, sub, 4, a.Lpad, a.GT));
        } else {
            const u32x4_t *p = (const u32x4_t *)(a.codes + (row * a.Lpad + s * 16) * CB);
#pragma unroll
            for (int k = 0; k < N / 4; ++k) {
                const u32x4_t v = p[k];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[4 * k + i] = v[i];
            }
        }
    }
    // the string of position t as position j keeps it
    __device__ __forceinline__ void turn(int t, int j) { turn_words<N>(w, ((j - t) & 15) * (CB == 0 ? 10 : 8 * CB)); }
    __device__ __forceinline__ void store(const MoveArgs &a, int64_t row, int s) const {
        if (CB == 0) {
            const int S = a.GT / 16, grp = s / S, sub = s - grp * S;
            *(u32x4_t *)(a.codes_out + packed_word(row, grp, sub, 0, a.Lpad, a.GT)) = u32x4_t{w[0], w[1], w[2], w[3]};
            *(uint32_t *)(a.codes_out + packed_word(row, grp, sub, 4, a.Lpad, a.GT)) = w[N - 1];
        } else {
            u32x4_t *p = (u32x4_t *)(a.codes_out + (row * a.Lpad + s * 16) * CB);
#pragma unroll
            for (int k = 0; k < N / 4; ++k) p[k] = u32x4_t{w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]};
        }
    }
};

// To other tensors or blocks: every row by itself, 32 rows a workgroup.  (4096 of 32768 tokens of 8 heads 6.5 us;
// 16 paged sequences, 1001 tokens of each head, ids of 10 bits, 20 us.)
constexpr int kMoveThreads = 256, kMoveRows = 32;

template <int ROWB, int CB>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(MoveArgs a) {
    constexpr int CPR = ROWB / 16, PER = kMoveRows * CPR / kMoveThreads;     // pieces of K (and of V) a thread moves
    __shared__ int64_t s_from[kMoveRows], s_to[kMoveRows];
    __shared__ int s_t[kMoveRows];
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z, j0 = blockIdx.x * kMoveRows;
    const int count = min(a.n_selected[(int64_t)b * a.src.Hkv + h], a.max_k);
    if (j0 >= count) return;
    if (tid < kMoveRows) {
        int t;
        int64_t from, to;
        move_rows(a, b, h, j0 + tid, count, t, from, to);
        s_t[tid] = t;
        s_from[tid] = from;
        s_to[tid] = to;
        const int64_t base = ((int64_t)b * a.src.Hkv + h) * a.src.max_n;
        if (from >= 0 && a.vnorm_slices) a.vnorm_out[base + j0 + tid] = a.vnorm[base + t];
        if (from >= 0 && a.mass_slices) a.mass_out[base + j0 + tid] = a.mass[base + t];
    }
    __syncthreads();
    u32x4_t k[PER], v[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int id = p * kMoveThreads + tid, r = id / CPR, c = id % CPR;
        const int64_t from = s_from[r];
        if (from >= 0) {
            k[p] = *(const u32x4_t *)((const char *)a.K + from * ROWB + c * 16);
            v[p] = *(const u32x4_t *)((const char *)a.V + from * ROWB + c * 16);
        }
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int id = p * kMoveThreads + tid, r = id / CPR, c = id % CPR;
        const int64_t to = s_to[r];
        if (s_from[r] >= 0) {
            *(u32x4_t *)((char *)a.K_out + to * ROWB + c * 16) = k[p];
            *(u32x4_t *)((char *)a.V_out + to * ROWB + c * 16) = v[p];
        }
    }
    if (a.codes) {
        for (int id = tid; id < kMoveRows * a.strings; id += kMoveThreads) {
            const int r = id / a.strings, s = id - r * a.strings;
            if (s_from[r] < 0) continue;
            IdString<CB> x;
            x.load(a, s_from[r], s);
            x.turn(s_t[r], j0 + r);
            x.store(a, s_to[r], s);
        }
    }
}

// In place, or within the same pools.  Entry j of an ascending index row lies at position j or behind it, so rows that are
// moved in order never land on one that is still to be read; a workgroup takes a slice of the row's
// bytes of one head, reads a pass of rows into registers, and writes them once all of the pass are
// there.  Slices of 64 bytes: what one head's move can be shared out in.
constexpr int kOrderedThreads = 1024, kOrderedPer = 4;

template <int CB>
__global__ __launch_bounds__(kOrderedThreads) void evict_ordered_kernel(MoveArgs a, int rowb) {
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int64_t bh = (int64_t)b * a.src.Hkv + h;
    const int count = min(a.n_selected[bh], a.max_k);
    int slice = blockIdx.x;
    auto rows_of_16 = [&](const char *from_base, char *to_base, int at) __attribute__((always_inline)) {
        for (int j0 = 0; j0 < count; j0 += kOrderedThreads / 4 * kOrderedPer) {
            u32x4_t x[kOrderedPer];
            int64_t to[kOrderedPer];
#pragma unroll
            for (int p = 0; p < kOrderedPer; ++p) {
                int t;
                int64_t from;
                move_rows(a, b, h, j0 + p * (kOrderedThreads / 4) + tid / 4, count, t, from, to[p]);
                x[p] = 0;
                if (from >= 0) x[p] = *(const u32x4_t *)(from_base + from * rowb + at + (tid & 3) * 16);
                else to[p] = -1;
            }
#pragma unroll
            for (int p = 0; p < kOrderedPer; ++p) asm volatile("" ::"v"(x[p]));     // (every load has arrived)
            __syncthreads();
#pragma unroll
            for (int p = 0; p < kOrderedPer; ++p)
                if (to[p] >= 0) *(u32x4_t *)(to_base + to[p] * rowb + at + (tid & 3) * 16) = x[p];
        }
    };
    auto floats = [&](const float *from_base, float *to_base) __attribute__((always_inline)) {
        for (int j0 = 0; j0 < count; j0 += kOrderedThreads * kOrderedPer) {
            float x[kOrderedPer];
            int64_t to[kOrderedPer];
#pragma unroll
            for (int p = 0; p < kOrderedPer; ++p) {
                int t;
                int64_t from;
                const int j = j0 + p * kOrderedThreads + tid;
                move_rows(a, b, h, j, count, t, from, to[p]);
                x[p] = from >= 0 ? from_base[bh * a.src.max_n + t] : 0.0f;
                to[p] = from >= 0 ? bh * a.src.max_n + j : -1;
            }
#pragma unroll
            for (int p = 0; p < kOrderedPer; ++p) asm volatile("" ::"v"(x[p]));
            __syncthreads();
#pragma unroll
            for (int p = 0; p < kOrderedPer; ++p)
                if (to[p] >= 0) to_base[to[p]] = x[p];
        }
    };
    if (slice < a.k_slices) return rows_of_16((const char *)a.K, (char *)a.K_out, slice * 64);
    slice -= a.k_slices;
    if (slice < a.v_slices) return rows_of_16((const char *)a.V, (char *)a.V_out, slice * 64);
    slice -= a.v_slices;
    if (slice < a.code_slices) {                     // one string of the row of ids
        for (int j0 = 0; j0 < count; j0 += kOrderedThreads) {
            IdString<CB> x;
            int t;
            int64_t from, to;
            move_rows(a, b, h, j0 + tid, count, t, from, to);
            if (from >= 0) {
                x.load(a, from, slice);
                x.turn(t, j0 + tid);
            } else {
#pragma unroll
                for (int i = 0; i < IdString<CB>::N; ++i) x.w[i] = 0;
            }
#pragma unroll
            for (int i = 0; i < IdString<CB>::N; ++i) asm volatile("" ::"v"(x.w[i]));
            __syncthreads();
            if (from >= 0) x.store(a, to, slice);
        }
        return;
    }
    slice -= a.code_slices;
    if (slice < a.vnorm_slices) return floats(a.vnorm, a.vnorm_out);
    floats(a.mass, a.mass_out);
}

int launch_evict_scores(socket_ctx *ctx, const float *mass, const int32_t *block_table, const int32_t *seq_len, int batch,
                        int pool, float *scores, hipStream_t st) {
    const Geometry &g = ctx->g;
    EvictScoreArgs a;
    a.mass = mass; a.scores = scores; a.seq_len = seq_len;
    a.map = row_map(g, block_table);
    a.pool = pool; a.n_sink = ctx->n_sink; a.n_window = ctx->n_window;
    hipLaunchKernelGGL(evict_scores_kernel, dim3((g.max_n + kPoolTokens - 1) / kPoolTokens, g.Hkv, batch), dim3(kPoolThreads), 0, st, a);
    return record_hip(ctx, hipGetLastError());
}

template <int ROWB> static void launch_move(const MoveArgs &a, dim3 grid, hipStream_t st) {
    if (a.cb == 1) hipLaunchKernelGGL((evict_move_kernel<ROWB, 1>), grid, dim3(kMoveThreads), 0, st, a);
    else if (a.cb == 2) hipLaunchKernelGGL((evict_move_kernel<ROWB, 2>), grid, dim3(kMoveThreads), 0, st, a);
    else hipLaunchKernelGGL((evict_move_kernel<ROWB, 0>), grid, dim3(kMoveThreads), 0, st, a);
}

int launch_evict_rows(socket_ctx *ctx, const int32_t *idx, const int32_t *n_selected, int batch,
                      const void *K, const void *V, const void *codes, const float *vnorm, const float *mass,
                      const int32_t *block_table, void *K_out, void *V_out, void *codes_out, float *vnorm_out,
                      float *mass_out, const int32_t *block_table_out, hipStream_t st) {
    const Geometry &g = ctx->g;
    MoveArgs a;
    a.idx = idx; a.n_selected = n_selected;
    a.K = K; a.V = V; a.codes = (const char *)codes; a.vnorm = vnorm; a.mass = mass;
    a.K_out = K_out; a.V_out = V_out; a.codes_out = (char *)codes_out; a.vnorm_out = vnorm_out; a.mass_out = mass_out;
    a.src = row_map(g, block_table);
    a.dst = row_map(g, block_table_out);
    a.max_k = g.max_k; a.Lpad = g.Lpad; a.GT = g.GT; a.strings = g.Lpad / 16; a.cb = g.cb;
    const int rowb = g.d * (g.kv_dtype == SOCKET_F32 ? 4 : 2);
    // (the same pools under another table may be in place all the same, if the tables say the same: moving in
    // order is right then, and where the blocks are others)
    const bool in_place = K == K_out || V == V_out || (codes && codes == codes_out);
    // (the float arrays are by sequence, not by block: they can be in place where the caches are not)
    const bool vnorm_ordered = vnorm && (in_place || vnorm == vnorm_out), mass_ordered = mass && (in_place || mass == mass_out);
    if (!in_place) {
        a.vnorm_slices = vnorm && !vnorm_ordered;
        a.mass_slices = mass && !mass_ordered;
        const dim3 grid((g.max_k + kMoveRows - 1) / kMoveRows, g.Hkv, batch);
        switch (rowb) {
            case 128: launch_move<128>(a, grid, st); break;
            case 256: launch_move<256>(a, grid, st); break;
            case 512: launch_move<512>(a, grid, st); break;
            case 1024: launch_move<1024>(a, grid, st); break;
            default: return SOCKET_EUNSUPPORTED;
        }
    }
    a.k_slices = a.v_slices = in_place ? rowb / 64 : 0;
    a.code_slices = in_place && codes ? a.strings : 0;
    a.vnorm_slices = vnorm_ordered;
    a.mass_slices = mass_ordered;
    const int slices = a.k_slices + a.v_slices + a.code_slices + a.vnorm_slices + a.mass_slices;
    if (slices) {
        const dim3 grid(slices, g.Hkv, batch);
        if (a.cb == 1) hipLaunchKernelGGL(evict_ordered_kernel<1>, grid, dim3(kOrderedThreads), 0, st, a, rowb);
        else if (a.cb == 2) hipLaunchKernelGGL(evict_ordered_kernel<2>, grid, dim3(kOrderedThreads), 0, st, a, rowb);
        else hipLaunchKernelGGL(evict_ordered_kernel<0>, grid, dim3(kOrderedThreads), 0, st, a, rowb);
    }
    return record_hip(ctx, hipGetLastError());
}

}  // namespace sk
