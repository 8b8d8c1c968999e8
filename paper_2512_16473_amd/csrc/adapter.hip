// Low-rank adapters of many requests beside a projection that all of them share:
//   y_t = y_in_t + W x_t + scale_a B_a (A_a x_t),   a = adapters[t]
//
// Up to 16 tokens (a decode batch) W is streamed once past all of them (row_stream.h); longer
// batches are a tiled matrix product. Kernels, on one stream:
//   1. shrink: v_t = A_a x_t. Per block of tokens the adapters among them, each a few blocks of
//      16 rows, are multiplied with all the block's tokens; a token keeps its own adapter's sums.
//   up to 16 tokens:
//   2. rows: blocks of 16 rows of W against all the tokens, the columns cut into groups of up
//      to 8 units as in the layer's down projection; with one group the expansion B_a v_t, y_in
//      and the rounding follow in the same kernel, else
//   3. finish adds the groups in order, the expansion and y_in.
//   longer:
//   2. parts: v scaled and cut into bf16 parts; the activations too where they are fp32 or their
//      rows do not end with a K step; and the list of adapters in every tile of tokens;
//   3. gemm: tiles of up to 256 tokens by 256 rows of W; after the K steps of W, each adapter
//      in the tile adds a few more: its B rows against the tile's v, rows of other adapters
//      zero. The tiles of a last, partial round of work groups are split over K, and
//   4. tail adds their parts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "moe_internal.h"
#include "row_stream.h"
#include "tile_plan.h"

namespace moe {
namespace {

using namespace row_stream;

constexpr int kStreamTokens = 16;    // tokens that the rows kernel takes
constexpr int kBlockTokens = 64;     // tokens per shrink block, at most

struct AdapterParams {
    const void *x;                // [T][ldx]
    bool bf16;                    // of x, y_in and y; else fp32
    int64_t ldx, ldy, ldyin;      // row strides (elements)
    const uint8_t *w;             // [o][d] or null
    const uint8_t *a, *b;         // [n][r][d], [n][o][r]
    const int32_t *ids;           // [T]
    const float *scale;           // [n] or null
    int T, d, o, n, r;
    int tb;                       // tokens per shrink block
    int vgroups;                  // K groups of v
    float *v;                     // [vgroups][T][r]
    float *partial;               // [groups][T][o]
    int groups;
    const void *y_in;             // or null
    void *y;
};

__device__ __forceinline__ bool has_adapter(const AdapterParams &p, int id) { return id >= 0 && id < p.n; }
__device__ __forceinline__ float scale_of(const AdapterParams &p, int id) { return p.scale ? p.scale[id] : 1.f; }
__device__ __forceinline__ float load_act(const void *x, bool bf16, size_t at)
{
    return bf16 ? static_cast<float>(static_cast<const __bf16 *>(x)[at]) : static_cast<const float *>(x)[at];
}
__device__ __forceinline__ void store_act(void *y, bool bf16, size_t at, float v)
{
    if (bf16) static_cast<__bf16 *>(y)[at] = static_cast<__bf16>(v);
    else static_cast<float *>(y)[at] = v;
}

// The B operand's fragments of this wave's chunks [c0, c0 + cnt): tokens t0 .. of tn, fp32 ones
// as three columns each (part by part).
template <int S, int NB>
__device__ __forceinline__ void load_tokens(const AdapterParams &p, int t0, int tn, int c0, int cnt, bf16x8_t (&bx)[S][2][NB])
{
    const int lane = threadIdx.x & 63, parts = p.bf16 ? 1 : 3;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int c = nb * 16 + (lane & 15), part = c / tn, t = c - part * tn;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int k = (c0 + s) * kChunk + kb * 32 + (lane >> 4) * 8;
                bx[s][kb][nb] = s < cnt && k < p.d && part < parts ? load_part(p.x, p.bf16, (size_t)(t0 + t) * p.ldx + k, part)
                                                                   : no_tokens();
            }
    }
}

// Wave's chunks of group g: eight units of up to S chunks of the d columns.
template <int S>
__device__ __forceinline__ void group_chunks(int d, int g, int wv, int &c0, int &cnt)
{
    const int C = (d + kChunk - 1) / kChunk, units = (C + S - 1) / S, u = g * kWaves + wv;
    c0 = cnt = 0;
    if (u < units) part_chunks(C, u, units, c0, cnt);
}

struct ShrinkSrc {
    const uint8_t *base0, *base1;
    size_t half;
    int c0, cnt;
    const AdapterParams &p;
    const int *list;
    int it, step, total, rbs;
    template <class R>
    __device__ __forceinline__ bool next(R &)
    {
        if (it >= total || cnt == 0) return false;
        const int j = it / rbs, rb = it - j * rbs;
        const size_t K2 = (size_t)p.d * 2;
        base0 = p.a + ((size_t)list[j] * p.r + (size_t)rb * kRows) * K2;
        half = rb * kRows + 8 < p.r ? 8 * K2 : 0;   // the last block may have 8 rows
        it += step;
        return true;
    }
};

// v of the tokens of block x, K group y; of the block's (adapter, 16 rows) items every gridDim.z-th.
template <int S, int NB>
__global__ __launch_bounds__(kThreads) void k_adapter_shrink(AdapterParams p)
{
    constexpr int RS = NB <= 2 ? 8 : 6;
    constexpr int kRing = kWaves * RS * kStageBytes;
    __shared__ __align__(1024) uint8_t lds[kRing + kWaves * NB * 1024];
    __shared__ int list[kBlockTokens], mine[kBlockTokens], njobs;
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = blockIdx.x * p.tb, tn = min(p.tb, p.T - t0), g = blockIdx.y;
    if (tid < kWave) {   // the distinct adapters, in order of first appearance
        int id = tid < tn ? p.ids[t0 + tid] : -1;
        if (!has_adapter(p, id)) id = -1;
        mine[tid] = id;
        uint64_t m = __ballot(id >= 0);
        int n = 0;
        while (m) {
            const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(m));
            if (tid == 0) list[n] = a;
            ++n;
            m &= ~__ballot(id == a);
        }
        if (tid == 0) njobs = n;
    }
    __syncthreads();
    const int rbs = (p.r + kRows - 1) / kRows, total = __builtin_amdgcn_readfirstlane(njobs) * rbs;
    if ((int)blockIdx.z >= total) return;
    ShrinkSrc src{nullptr, nullptr, 0, 0, 0, p, list, (int)blockIdx.z, (int)gridDim.z, total, rbs};
    group_chunks<S>(p.d, g, wv, src.c0, src.cnt);
    Stream<S, 1, NB, RS, ShrinkSrc> st;
    st.ring.row_bytes((int64_t)p.d * 2);
    st.start(src, lds + wv * RS * kStageBytes);
    bf16x8_t bx[S][2][NB];
    load_tokens<S, NB>(p, t0, tn, src.c0, src.cnt, bx);
    float *red = reinterpret_cast<float *>(lds + kRing);
    const int parts = p.bf16 ? 1 : 3;
    for (int it = blockIdx.z; it < total; it += gridDim.z) {
        floatx4_t acc[1][NB];
        st.item(src, bx, src.cnt, acc);
        lds_barrier();
        put_sums(red, wv, acc);
        lds_barrier();
        const int j = it / rbs, row = tid & 15, i = (it - j * rbs) * kRows + row;
        for (int t = tid >> 4; t < tn; t += kThreads / kRows) {
            if (i >= p.r || mine[t] != list[j]) continue;
            float v = 0.f;
            for (int q = 0; q < parts; ++q) v += get_sum<1, NB>(red, 0, row, q * tn + t);
            p.v[((size_t)g * p.T + t0 + t) * p.r + i] = v;
        }
    }
}

// scale_a v_t, rank i: the K groups' sums in order.
__device__ __forceinline__ float low_rank(const AdapterParams &p, int id, int t, int i)
{
    float v = 0.f;
    for (int g = 0; g < p.vgroups; ++g) v += p.v[((size_t)g * p.T + t) * p.r + i];
    return v * scale_of(p, id);
}
// (B_a)_i v over the r ranks.
__device__ __forceinline__ float expand(const AdapterParams &p, int id, int i, const float *v)
{
    const uint4 *b = reinterpret_cast<const uint4 *>(p.b + ((size_t)id * p.o + i) * p.r * 2);
    float s = 0.f;
#pragma unroll 4
    for (int c = 0; c < p.r / 8; ++c) {
        const uint4 q = b[c];
        const float *u = v + c * 8;
        s = fmaf(__uint_as_float(q.x << 16), u[0], s);
        s = fmaf(__uint_as_float(q.x & 0xffff0000u), u[1], s);
        s = fmaf(__uint_as_float(q.y << 16), u[2], s);
        s = fmaf(__uint_as_float(q.y & 0xffff0000u), u[3], s);
        s = fmaf(__uint_as_float(q.z << 16), u[4], s);
        s = fmaf(__uint_as_float(q.z & 0xffff0000u), u[5], s);
        s = fmaf(__uint_as_float(q.w << 16), u[6], s);
        s = fmaf(__uint_as_float(q.w & 0xffff0000u), u[7], s);
    }
    return s;
}

struct RowsSrc {
    const uint8_t *base0, *base1;
    size_t half;
    int c0, cnt;
    const AdapterParams &p;
    int it, end, rbs, group, wv;
    int s;   // chunks of a unit
    template <class R>
    __device__ __forceinline__ bool next(R &)
    {
        const int C = (p.d + kChunk - 1) / kChunk, units = (C + s - 1) / s;
        for (;;) {
            if (it >= end) return false;
            const int g = it / rbs;
            if (g != group) {
                group = g;
                const int u = g * kWaves + wv;
                c0 = cnt = 0;
                if (u < units) part_chunks(C, u, units, c0, cnt);
            }
            if (cnt) break;
            it = (g + 1) * rbs;   // nothing for this wave in the group
        }
        const int rb = it - group * rbs;
        const size_t K2 = (size_t)p.d * 2;
        base0 = p.w + (size_t)rb * kRows * K2;
        half = rb * kRows + 8 < p.o ? 8 * K2 : 0;
        ++it;
        return true;
    }
};

// W x for up to 16 tokens. A work group takes an equal, contiguous share of the (group, 16 rows)
// items. kOne: there is one group, and the adapters' part, y_in and the rounding follow here.
template <int S, int NB, bool kOne>
__global__ __launch_bounds__(kThreads) void k_adapter_rows(AdapterParams p)
{
    constexpr int RS = NB <= 2 ? 8 : 6;
    constexpr int kRing = kWaves * RS * kStageBytes;
    __shared__ __align__(1024) uint8_t lds[kRing + kWaves * NB * 1024];
    __shared__ float v[kOne ? kStreamTokens * MOE_ADAPTER_MAX_RANK : 1];
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rbs = (p.o + kRows - 1) / kRows;
    const int64_t total = (int64_t)p.groups * rbs;
    const int it0 = (int)(total * blockIdx.x / gridDim.x), it1 = (int)(total * (blockIdx.x + 1) / gridDim.x);
    RowsSrc src{nullptr, nullptr, 0, 0, 0, p, it0, it1, rbs, -1, wv, S};
    Stream<S, 1, NB, RS, RowsSrc> st;
    st.ring.row_bytes((int64_t)p.d * 2);
    st.start(src, lds + wv * RS * kStageBytes);
    if (kOne) {
        for (int i = tid; i < p.T * p.r; i += kThreads) {
            const int t = i / p.r, id = p.ids[t];
            v[i] = has_adapter(p, id) ? low_rank(p, id, t, i - t * p.r) : 0.f;
        }
        __syncthreads();
    }
    float *red = reinterpret_cast<float *>(lds + kRing);
    const int parts = p.bf16 ? 1 : 3;
    const int row = tid & 15, t = tid >> 4;
    const int id = kOne && t < p.T ? p.ids[t] : -1;
    bf16x8_t bx[S][2][NB];
    int group = -1, c0 = 0, cnt = 0;
    for (int it = it0; it < it1; ++it) {
        const int g = it / rbs, rb = it - g * rbs;
        if (g != group) {
            group = g;
            group_chunks<S>(p.d, g, wv, c0, cnt);
            load_tokens<S, NB>(p, 0, p.T, c0, cnt, bx);
        }
        floatx4_t acc[1][NB];
        st.item(src, bx, cnt, acc);
        lds_barrier();
        put_sums(red, wv, acc);
        lds_barrier();
        const int i = rb * kRows + row;
        if (t < p.T && i < p.o) {
            float s = 0.f;
            for (int q = 0; q < parts; ++q) s += get_sum<1, NB>(red, 0, row, q * p.T + t);
            if (kOne) {
                if (p.y_in) s += load_act(p.y_in, p.bf16, (size_t)t * p.ldyin + i);
                if (has_adapter(p, id)) s += expand(p, id, i, v + t * p.r);
                store_act(p.y, p.bf16, (size_t)t * p.ldy + i, s);
            } else {
                p.partial[((size_t)g * p.T + t) * p.o + i] = s;
            }
        }
    }
}

// y of token blockIdx.y, 256 outputs: the groups' sums in order, y_in, the adapter's part.
__global__ __launch_bounds__(256) void k_adapter_finish(AdapterParams p)
{
    __shared__ float v[MOE_ADAPTER_MAX_RANK];
    const int t = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x, id = p.ids[t];
    const bool has = has_adapter(p, id);
    if (has && (int)threadIdx.x < p.r) v[threadIdx.x] = low_rank(p, id, t, threadIdx.x);
    __syncthreads();
    if (i >= p.o) return;
    float s = 0.f;
#pragma unroll 4
    for (int g = 0; g < p.groups; ++g) s += p.partial[((size_t)g * p.T + t) * p.o + i];
    if (p.y_in) s += load_act(p.y_in, p.bf16, (size_t)t * p.ldyin + i);
    if (has) s += expand(p, id, i, v);
    store_act(p.y, p.bf16, (size_t)t * p.ldy + i, s);
}

// ------------------------------------------------------------------ longer batches
constexpr int kTileN = 256;          // rows of W per tile
constexpr int kBK = 64;              // K per stage
constexpr int kRowBytes = kBK * 2;
constexpr int kLoadRows = 1024 / kRowBytes;         // rows per load instruction of a wave
constexpr int kBBytes = kTileN * kRowBytes;         // rows of W of a stage
constexpr int kBLoads = kTileN / kLoadRows / kWaves;
constexpr int kLdsBytes = 163840;
constexpr int kMaxParts = 64;        // part buffers per XCD
constexpr size_t kPartBytes = (size_t)64 << 20;     // all of them, at most
constexpr int kStagger = 2;          // K steps between the starts of neighbouring N tiles

struct GemmParams {
    AdapterParams p;
    const uint16_t *xk;       // activations in bf16, K steps side by side: [T][ldk]
    int64_t ldk;
    int nk, steps;            // K steps of W; of a tile (times the activations' parts)
    const uint16_t *vk;       // v in bf16, [T][vparts][rq * 64]
    int vparts, rq;           // parts of v, K steps of its ranks
    const uint16_t *zeros;    // kBK zeros
    const int32_t *list;      // [mtiles][1 + kTileM] adapters of a tile: count, ids
    int mtiles, ntiles, slots;
    TilePlan plan[kXcds];
    int maxparts, prows;      // part buffers per XCD and their rows
    float *part;              // [8][maxparts][prows][kTileN]
};

// vk, xk (unless the activations are taken as they are), zeros, and the tiles' lists.
struct PartsParams {
    AdapterParams p;
    uint16_t *vk, *xk, *zeros;
    int vparts, rq, nk;
    bool copy;
    int32_t *list;
    int mtiles;
};
__global__ __launch_bounds__(256) void k_adapter_parts(PartsParams g)
{
    const AdapterParams &p = g.p;
    const int tid = threadIdx.x;
    int b = blockIdx.x;
    if (b < g.mtiles) {   // the distinct adapters of tile b: a thread keeps one token's
        __shared__ int ids[kTileM], n;
        const int r0 = tile_row(p.T, b), r1 = tile_row(p.T, b + 1);
        int id = tid < r1 - r0 ? p.ids[r0 + tid] : -1;
        if (!has_adapter(p, id)) id = -1;
        ids[tid] = id;
        if (tid == 0) n = 0;
        __syncthreads();
        bool first = id >= 0;   // the first token with its adapter
        int rank = 0;           // different adapters before its own
        for (int j = 0; j < tid; ++j) first = first && ids[j] != id;
        __syncthreads();
        ids[tid] = first ? id : -1;
        __syncthreads();
        for (int j = 0; j < kTileM; ++j) rank += ids[j] >= 0 && ids[j] < id;
        int32_t *list = g.list + (size_t)b * (kTileM + 1);
        if (first) {
            list[1 + rank] = id;
            atomicAdd(&n, 1);
        }
        __syncthreads();
        if (tid == 0) list[0] = n;
        if (b == 0 && tid < kBK) g.zeros[tid] = 0;
        return;
    }
    // token by token: v's parts, then the activations' 8 at a time
    b -= g.mtiles;
    const int t = b;
    const int id = p.ids[t];
    const bool has = has_adapter(p, id);
    for (int i = tid; i < g.rq * kBK; i += 256) {
        const float v = has && i < p.r ? low_rank(p, id, t, i) : 0.f;
        for (int q = 0; q < g.vparts; ++q)
            g.vk[((size_t)t * g.vparts + q) * g.rq * kBK + i] = g.vparts == 3 ? part_of<3>(v, q) : part_of<2>(v, q);
    }
    if (!g.copy) return;
    const int parts = p.bf16 ? 1 : 3, per = g.nk * kBK / 8;
    for (int i = tid; i < parts * per; i += 256) {
        const int q = i / per, k = (i - q * per) * 8;
        const bf16x8_t v = k < p.d ? load_part(p.x, p.bf16, (size_t)t * p.ldx + k, q) : no_tokens();
        *reinterpret_cast<bf16x8_t *>(g.xk + ((size_t)t * parts + q) * g.nk * kBK + k) = v;
    }
}

// Rings of a tile of HB * 32 tokens: as many stages as LDS holds.
template <int HB>
struct TileCfg {
    static constexpr int kABytes = HB * 32 * kRowBytes;           // token rows of a stage
    static constexpr int kAStages = HB <= 2 ? 4 : HB <= 5 ? 3 : 2;
    static constexpr int kBStages = HB <= 2 ? 4 : 3;
    static constexpr int kBBase = kAStages * kABytes;
    static constexpr int kALoads = (HB + 1) / 2;                  // load instructions per wave and stage
    static constexpr int kLoads = kALoads + kBLoads;
    static constexpr int kRing = HB == 8 || HB == 6 || HB == 4 ? 4 : HB;   // divides 2 HB
    static constexpr int kAhead = kRing < 4 ? kRing : 4;
    static constexpr int kKeep = kAStages == kBStages ? (kAStages - 2) * kLoads : kBLoads;
    static_assert(kBBase + kBStages * kBBytes <= kLdsBytes, "the rings fit LDS");
    static_assert(kAStages == kBStages || (kAStages == 2 && kBStages == 3), "kKeep");
};

// The LDS reads so far are done and at most N of this wave's loads are still in flight; then
// every wave of the work group is at this point.
template <int N>
__device__ __forceinline__ void wait_and_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// A tile of tokens row0 .. row0 + rows (up to HB * 32) by W rows nt * 256 ..: K steps k0 .. k0 +
// nsteps, the adapters' steps too if `ext`. Two waves split the tokens and four the rows of W; both
// operands go straight to LDS in rings of K steps, swizzled so that the operand reads touch all
// banks evenly; one barrier per step (the same scheme as the experts' grouped products).
template <bool kOnce, int HB>
__device__ __forceinline__ void project_tile(const GemmParams &g, uint8_t *lds, int row0, int rows, int nt, int mt, int k0,
                                             int nsteps, int start, bool ext, float *part)
{
    using C = TileCfg<HB>;
    constexpr int NA = C::kAStages, NB = C::kBStages, P = C::kAhead, R = C::kRing, kItems = 2 * HB;
    const AdapterParams &p = g.p;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // keeps the addresses of all tile heights from being computed up front
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wv & 1, wn = wv >> 1;
    const int lr = lane >> 3, lc = ((lane & 7) ^ lr) * 16;   // row of a load instruction, byte of its K step
    const int K2 = p.d * 2;

    auto token_row = [&](int i) {   // rows past the tile read its first
        const int r = min(i * 8 + wv, HB * 4 - 1) * kLoadRows + lr;
        return row0 + (r < rows ? r : 0);
    };
    auto w_block = [&](int i) { return min(nt * kTileN + i * 64 + wv * kLoadRows, p.o - kLoadRows); };   // o % 8 == 0
    auto put_a = [&](int i, const uint8_t *src, int buf) {
        __builtin_amdgcn_global_load_lds((global_cvoid *)src,
                                         (lds_void *)(lds + buf * C::kABytes + min(i * 8 + wv, HB * 4 - 1) * 1024), 16, 0, 0);
    };
    auto put_b = [&](int i, const uint8_t *src, int buf) {
        __builtin_amdgcn_global_load_lds((global_cvoid *)src, (lds_void *)(lds + C::kBBase + buf * kBBytes + (i * 8 + wv) * 1024),
                                         16, 0, kOnce ? 2 : 0);   // 2: nontemporal
    };
    const uint8_t *asrc[C::kALoads];
#pragma unroll
    for (int j = 0; j < C::kALoads; ++j) asrc[j] = reinterpret_cast<const uint8_t *>(g.xk + token_row(j) * g.ldk) + lc;
    const uint32_t wlane = (uint32_t)lr * K2;
    auto step_of = [&](int stage) {   // steps go round from `start`
        const int ks = stage + start;
        return k0 + (ks >= nsteps ? ks - nsteps : ks);
    };
    auto load_a = [&](int i, int stage, int buf) { put_a(i, asrc[i] + (size_t)step_of(stage) * kRowBytes, buf); };
    auto load_b = [&](int i, int stage, int buf) {
        int ks = step_of(stage);
        while (ks >= g.nk) ks -= g.nk;   // the parts of the activations meet the same rows of W
        // past a row's end its last 16 bytes are read; the activations are zero there
        put_b(i, p.w + (size_t)w_block(i) * K2 + (wlane + (uint32_t)min(ks * kRowBytes + lc, K2 - 16)), buf);
    };

    floatx4_t acc[HB][4];
#pragma unroll
    for (int m = 0; m < HB; ++m)
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) acc[m][nb] = floatx4_t{0.f, 0.f, 0.f, 0.f};

    // Operand reads: row lane % 16 of a block, chunk 4 kb + lane / 16. The items of a step are
    // (kb, m) in order; item j's token block is read P items before its MFMAs.
    const int rd = (lane & 15) * kRowBytes + ((lane >> 4) ^ (lane & 7)) * 16;
    const uint8_t *const ra = lds + wm * HB * 16 * kRowBytes;
    const uint8_t *const rb = lds + C::kBBase + wn * 64 * kRowBytes;
    bf16x8_t wf[2][4], tf[R];
    auto read_item = [&](int j, int ba, int bb) {
        const int kb = j / HB, sl = rd ^ (kb * 64);
        if (j % HB == 0) {
#pragma unroll
            for (int nb = 0; nb < 4; ++nb)
                wf[kb][nb] = *reinterpret_cast<const bf16x8_t *>(rb + bb * kBBytes + nb * 16 * kRowBytes + sl);
        }
        tf[j % R] = *reinterpret_cast<const bf16x8_t *>(ra + ba * C::kABytes + (j % HB) * 16 * kRowBytes + sl);
    };
    auto mma = [&](int j, const bf16x8_t t) {
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
            acc[j % HB][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j / HB][nb], t, acc[j % HB][nb], 0, 0, 0);
    };
    if (nsteps > 0) {
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            if (q >= nsteps) continue;
            if (q < NA)
#pragma unroll
                for (int i = 0; i < C::kALoads; ++i) load_a(i, q, q);
#pragma unroll
            for (int i = 0; i < kBLoads; ++i) load_b(i, q, q);
        }
        if (nsteps >= NB) wait_and_barrier<(NA - 1) * C::kALoads + (NB - 1) * kBLoads>();
        else wait_and_barrier<0>();
#pragma unroll
        for (int j = 0; j < P; ++j) read_item(j, 0, 0);
        int s = 0, ba = 0, bb = 0;
        enum { kSteady, kDrain, kFinal };
        auto step = [&](auto mode) {
            constexpr bool kLast = decltype(mode)::value == kFinal, kFull = decltype(mode)::value == kSteady;
            const int na = ba + 1 == NA ? 0 : ba + 1, nb = bb + 1 == NB ? 0 : bb + 1;
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const int at = j - (kItems - P);   // items since the hand-over
                if (at == 0 && !kLast) {
                    if (kFull || s + NB - 1 < nsteps) wait_and_barrier<C::kKeep>();
                    else wait_and_barrier<0>();
                }
                if (at >= 0 && !kLast) {
                    constexpr int kEach = (C::kLoads + P - 1) / P;
#pragma unroll
                    for (int i = at * kEach; i < (at + 1) * kEach && i < C::kLoads; ++i) {
                        if (i < C::kALoads) {
                            if (kFull || s + NA < nsteps) load_a(i, s + NA, ba);
                        } else if (kFull || s + NB < nsteps) {
                            load_b(i - C::kALoads, s + NB, bb);
                        }
                    }
                }
                const bf16x8_t t = tf[j % R];
                if (at < 0) read_item(j + P, ba, bb);
                else if (!kLast) read_item(j + P - kItems, na, nb);
                mma(j, t);
                __builtin_amdgcn_sched_barrier(0);
            }
            ++s;
            ba = na;
            bb = nb;
        };
        while (s + NB < nsteps) step(std::integral_constant<int, kSteady>{});
        while (s + 1 < nsteps) step(std::integral_constant<int, kDrain>{});
        step(std::integral_constant<int, kFinal>{});
    }

    if (ext) {
        // The adapters' steps, two at a time: rows of another adapter (or none) read zeros.
        const int32_t *list = g.list + (size_t)mt * (kTileM + 1);
        const int per = g.vparts * g.rq, r2 = p.r * 2;
        const int total = __builtin_amdgcn_readfirstlane(list[0]) * per;
        int own[C::kALoads];
#pragma unroll
        for (int j = 0; j < C::kALoads; ++j) own[j] = p.ids[token_row(j)];
        for (int e = 0; e < total; e += 2) {
            wait_and_barrier<0>();   // what LDS holds is read
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (e + u >= total) break;
                const int a = __builtin_amdgcn_readfirstlane(list[1 + (e + u) / per]), q = (e + u) % per, rc = q % g.rq;
#pragma unroll
                for (int i = 0; i < C::kALoads; ++i) {
                    const uint16_t *v = g.vk + ((size_t)token_row(i) * per + q) * kBK;
                    put_a(i, reinterpret_cast<const uint8_t *>(own[i] == a ? v : g.zeros) + lc, u);
                }
#pragma unroll
                for (int i = 0; i < kBLoads; ++i)
                    put_b(i, p.b + ((size_t)a * p.o + w_block(i)) * r2 + (uint32_t)(lr * r2 + min(rc * kRowBytes + lc, r2 - 16)), u);
            }
            wait_and_barrier<0>();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (e + u >= total) break;
#pragma unroll
                for (int j = 0; j < kItems; ++j) {
                    read_item(j, u, u);
                    mma(j, tf[j % R]);
                }
            }
        }
    }

    // result r of a 16x16 block: row 4 (lane / 16) + r of W, token lane % 16
    const int c4 = 4 * (lane >> 4);
#pragma unroll
    for (int m = 0; m < HB; ++m) {
        const int tr = (wm * HB + m) * 16 + (lane & 15);
        if (tr >= rows) continue;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) {
            const int col = wn * 64 + nb * 16 + c4, i = nt * kTileN + col;
            floatx4_t s = acc[m][nb];
            if (part) {
                *reinterpret_cast<floatx4_t *>(part + (size_t)tr * kTileN + col) = s;
            } else if (i < p.o) {
                typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
                const size_t t = row0 + tr;
                if (p.bf16) {
                    if (p.y_in) {
                        const bf16x4_t b = *reinterpret_cast<const bf16x4_t *>(static_cast<const __bf16 *>(p.y_in) + t * p.ldyin + i);
                        for (int c = 0; c < 4; ++c) s[c] += static_cast<float>(b[c]);
                    }
                    bf16x4_t o;
                    for (int c = 0; c < 4; ++c) o[c] = static_cast<__bf16>(s[c]);
                    *reinterpret_cast<bf16x4_t *>(static_cast<__bf16 *>(p.y) + t * p.ldy + i) = o;
                } else {
                    if (p.y_in) s += *reinterpret_cast<const floatx4_t *>(static_cast<const float *>(p.y_in) + t * p.ldyin + i);
                    *reinterpret_cast<floatx4_t *>(static_cast<float *>(p.y) + t * p.ldy + i) = s;
                }
            }
        }
    }
}

// One work group per CU, looping over its tiles; the M tile fastest, eight contiguous runs of
// tiles for the eight XCDs. kOnce: W is read once (one tile of tokens).
template <bool kOnce>
__global__ __launch_bounds__(kThreads) void k_adapter_gemm(GemmParams g)
{
    __shared__ __align__(1024) uint8_t lds[kLdsBytes];
    const int xcd = blockIdx.x % kXcds;
    const TilePlan pl = g.plan[xcd];
    const int nunits = pl.full + (pl.units - pl.full) * pl.s;
    for (int u = blockIdx.x / kXcds; u < nunits; u += g.slots) {
        int t = u, ks = 0, parts = 1;
        float *part = nullptr;
        if (u >= pl.full) {
            const int v = u - pl.full;
            t = pl.full + v / pl.s;
            ks = v % pl.s;
            parts = pl.s;
            if (parts > 1) part = g.part + ((size_t)xcd * g.maxparts + v) * g.prows * kTileN;
        }
        t += pl.u0;
        const int mt = t % g.mtiles, nt = t / g.mtiles;
        const int row0 = tile_row(g.p.T, mt), rows = tile_row(g.p.T, mt + 1) - row0;
        const int k0 = (int)((int64_t)g.steps * ks / parts), kn = (int)((int64_t)g.steps * (ks + 1) / parts) - k0;
        const int start = g.mtiles == 1 && kn > 0 ? (int)((unsigned)(nt * kStagger) % (unsigned)kn) : 0;
        const bool ext = ks == parts - 1;
        switch ((rows + 31) >> 5) {
#define MOE_HB_CASE(N) \
    case N: project_tile<kOnce, N>(g, lds, row0, rows, nt, mt, k0, kn, start, ext, part); break;
            MOE_HB_CASE(1) MOE_HB_CASE(2) MOE_HB_CASE(3) MOE_HB_CASE(4)
            MOE_HB_CASE(5) MOE_HB_CASE(6) MOE_HB_CASE(7) MOE_HB_CASE(8)
#undef MOE_HB_CASE
        default: break;
        }
        wait_and_barrier<0>();   // the last stage is read before the next tile's loads overwrite it
    }
}

// y of the tiles split over K: the parts in order, and y_in. Work group b: XCD b mod 8, split tile
// i of that XCD, a block of 16 of its rows.
constexpr int kTailRows = 16;
__global__ __launch_bounds__(256) void k_adapter_tail(GemmParams g)
{
    const AdapterParams &p = g.p;
    const int xcd = blockIdx.x % kXcds, i = (blockIdx.x / kXcds) % g.slots, rb = blockIdx.x / kXcds / g.slots;
    const TilePlan pl = g.plan[xcd];
    if (pl.s < 2 || i >= pl.units - pl.full) return;
    const int t = pl.u0 + pl.full + i, mt = t % g.mtiles, nt = t / g.mtiles;
    const int row0 = tile_row(p.T, mt), rows = tile_row(p.T, mt + 1) - row0;
    const float *part = g.part + ((size_t)xcd * g.maxparts + (size_t)i * pl.s) * g.prows * kTileN;
    for (int c = threadIdx.x; c < kTailRows * kTileN; c += 256) {
        const int tr = rb * kTailRows + c / kTileN, col = c % kTileN, o = nt * kTileN + col;
        if (tr >= rows || o >= p.o) continue;
        float s = 0.f;
        for (int j = 0; j < pl.s; ++j) s += part[((size_t)j * g.prows + tr) * kTileN + col];
        const size_t tok = row0 + tr;
        if (p.y_in) s += load_act(p.y_in, p.bf16, tok * p.ldyin + o);
        store_act(p.y, p.bf16, tok * p.ldy + o, s);
    }
}

// ------------------------------------------------------------------ host side
size_t a256(size_t v) { return (v + 255) & ~(size_t)255; }
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// A token-block product's shape: column blocks and chunks of a unit (row_stream.h), groups of the
// d columns. The fragments take 8 NB S registers.
struct StreamPlan {
    int nb, s, groups;
};
StreamPlan stream_plan(int d, int cols)
{
    StreamPlan q{};
    q.nb = ceil_div(cols, 16);
    q.s = q.nb <= 2 ? 8 : 4;
    const int chunks = ceil_div(d, kChunk);
    while (q.s > 1 && chunks <= q.s / 2 * kWaves) q.s /= 2;
    q.groups = ceil_div(ceil_div(chunks, q.s), kWaves);
    return q;
}

struct AdapterPlan {
    int tb;                    // tokens of a shrink block
    StreamPlan shrink, rows;
    bool gemm;
    int vparts, rq, nk, mtiles, prows, maxparts;
    size_t v, partial, vk, xk, zeros, list, part, bytes;
};

AdapterPlan plan_adapter(int T, int d, int o, int r, bool bf16)
{
    AdapterPlan L{};
    const int parts = bf16 ? 1 : 3;
    L.gemm = T > kStreamTokens;
    // 64 columns of bf16 tokens, 48 of fp32 ones: an adapter's rows are read once per block
    L.tb = std::min(T, bf16 ? kBlockTokens : kStreamTokens);
    L.shrink = stream_plan(d, L.tb * parts);
    L.rows = stream_plan(d, std::min(T, kStreamTokens) * parts);
    // v meets B in three exact parts; beside bf16 activations in two (2^-17 relative)
    L.vparts = bf16 ? 2 : 3;
    L.rq = ceil_div(r, kBK);
    L.nk = ceil_div(d, kBK);
    L.mtiles = tiles_of(T);
    L.prows = std::min(T, kTileM);
    L.maxparts = (int)std::min<size_t>(kMaxParts, kPartBytes / ((size_t)kXcds * L.prows * kTileN * 4));
    size_t at = 0;
    auto take = [&](size_t b) {
        const size_t was = at;
        at += a256(b);
        return was;
    };
    L.v = take((size_t)L.shrink.groups * T * r * 4);
    if (!L.gemm) {
        L.partial = take(L.rows.groups > 1 ? (size_t)L.rows.groups * T * o * 4 : 0);
    } else {
        L.vk = take((size_t)T * L.vparts * L.rq * kBK * 2);
        L.xk = take((size_t)T * parts * L.nk * kBK * 2);
        L.zeros = take(kRowBytes);
        L.list = take((size_t)L.mtiles * (kTileM + 1) * 4);
        L.part = take((size_t)kXcds * L.maxparts * L.prows * kTileN * 4);
    }
    L.bytes = at;
    return L;
}

template <int S, int NB>
hipError_t launch_shrink(const AdapterParams &p, hipStream_t s, dim3 grid)
{
    hipLaunchKernelGGL((k_adapter_shrink<S, NB>), grid, dim3(kThreads), 0, s, p);
    return hipGetLastError();
}
template <int S, int NB>
hipError_t launch_rows(const AdapterParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)std::min<int64_t>(device_cu_count(), (int64_t)p.groups * ceil_div(p.o, kRows)));
    if (p.groups == 1) hipLaunchKernelGGL((k_adapter_rows<S, NB, true>), grid, dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((k_adapter_rows<S, NB, false>), grid, dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

#define MOE_STREAM_CASES(F)                                                                                   \
    F(1, 1) F(1, 2) F(1, 4) F(1, 8) F(2, 1) F(2, 2) F(2, 4) F(2, 8) F(3, 1) F(3, 2) F(3, 4)

hipError_t launch_adapter(AdapterParams p, const AdapterPlan &L, uint8_t *ws, hipStream_t s)
{
    (void)hipGetLastError();
    hipError_t e = hipSuccess;
    p.tb = L.tb;
    p.v = reinterpret_cast<float *>(ws + L.v);
    p.vgroups = L.shrink.groups;
    if (p.n > 0) {
        const int blocks = ceil_div(p.T, L.tb), items = std::min(L.tb, p.n) * ceil_div(p.r, kRows);
        // enough work groups for the chip; a block's items are shared out among them
        const int split = std::max(1, std::min(items, 2 * device_cu_count() / (blocks * L.shrink.groups)));
        const dim3 grid(blocks, L.shrink.groups, split);
        switch (L.shrink.nb * 100 + L.shrink.s) {
#define MOE_CASE(NB, S) \
    case NB * 100 + S: e = launch_shrink<S, NB>(p, s, grid); break;
            MOE_STREAM_CASES(MOE_CASE) MOE_CASE(4, 1) MOE_CASE(4, 2) MOE_CASE(4, 4)
#undef MOE_CASE
        default: return hipErrorInvalidValue;
        }
        if (e != hipSuccess) return e;
    }
    if (!L.gemm) {
        p.groups = p.w ? L.rows.groups : 0;
        p.partial = reinterpret_cast<float *>(ws + L.partial);
        if (p.w) {
            switch (L.rows.nb * 100 + L.rows.s) {
#define MOE_CASE(NB, S) \
    case NB * 100 + S: e = launch_rows<S, NB>(p, s); break;
                MOE_STREAM_CASES(MOE_CASE)
#undef MOE_CASE
            default: return hipErrorInvalidValue;
            }
            if (e != hipSuccess || p.groups == 1) return e;
        }
        hipLaunchKernelGGL(k_adapter_finish, dim3((unsigned)ceil_div(p.o, 256), (unsigned)p.T), dim3(256), 0, s, p);
        return hipGetLastError();
    }
    PartsParams q{};
    q.p = p;
    q.vk = reinterpret_cast<uint16_t *>(ws + L.vk);
    q.xk = reinterpret_cast<uint16_t *>(ws + L.xk);
    q.zeros = reinterpret_cast<uint16_t *>(ws + L.zeros);
    q.list = reinterpret_cast<int32_t *>(ws + L.list);
    q.vparts = L.vparts;
    q.rq = L.rq;
    q.nk = L.nk;
    q.mtiles = L.mtiles;
    // bf16 rows that end with a K step are read where they are
    q.copy = p.w && (!p.bf16 || p.d % kBK != 0);
    hipLaunchKernelGGL(k_adapter_parts, dim3((unsigned)(L.mtiles + p.T)), dim3(256), 0, s, q);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    GemmParams g{};
    const int parts = p.bf16 ? 1 : 3;
    g.p = p;
    g.xk = q.copy ? q.xk : static_cast<const uint16_t *>(p.x);
    g.ldk = q.copy ? (int64_t)parts * L.nk * kBK : p.ldx;
    g.nk = L.nk;
    g.steps = p.w ? parts * L.nk : 0;
    g.vk = q.vk;
    g.vparts = L.vparts;
    g.rq = L.rq;
    g.zeros = q.zeros;
    g.list = q.list;
    g.mtiles = L.mtiles;
    g.ntiles = ceil_div(p.o, kTileN);
    g.slots = std::max(1, device_cu_count() / kXcds);
    g.maxparts = L.maxparts;
    g.prows = L.prows;
    g.part = reinterpret_cast<float *>(ws + L.part);
    const int U = g.mtiles * g.ntiles;
    bool tail = false;
    for (int x = 0; x < kXcds; ++x) {
        const int left = tile_plan(U, g.slots, x, 1).units % g.slots;
        int best = 0x7fffffff;
        for (int k = 1; k <= kMaxSplit; ++k) best = std::min(best, split_key(left, g.steps, g.slots, 0, g.maxparts, 0, k));
        g.plan[x] = tile_plan(U, g.slots, x, best % kMaxSplit + 1);
        tail = tail || (g.plan[x].s > 1 && g.plan[x].units > g.plan[x].full);
    }
    const dim3 grid(kXcds * g.slots);
    if (g.mtiles == 1) hipLaunchKernelGGL(k_adapter_gemm<true>, grid, dim3(kThreads), 0, s, g);
    else hipLaunchKernelGGL(k_adapter_gemm<false>, grid, dim3(kThreads), 0, s, g);
    if ((e = hipGetLastError()) != hipSuccess || !tail) return e;
    hipLaunchKernelGGL(k_adapter_tail, dim3((unsigned)(kXcds * g.slots * ceil_div(g.prows, kTailRows))), dim3(256), 0, s, g);
    return hipGetLastError();
}

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_adapter_workspace_bytes(int T, int d_in, int d_out, int rank, int act_type)
{
    if (T < 1 || T > MOE_ADAPTER_MAX_TOKENS || d_in <= 0 || d_out <= 0 || rank < 1 || rank > MOE_ADAPTER_MAX_RANK ||
        (act_type != MOE_F32 && act_type != MOE_BF16))
        return 0;
    return moe::plan_adapter(T, d_in, d_out, rank, act_type == MOE_BF16).bytes;
}

int moe_adapter_project(const moe_adapter_desc *P, const void *x, int64_t x_stride, int T, const int32_t *adapters,
                        const void *y_in, int64_t y_in_stride, void *y, int64_t y_stride, int act_type, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    MOE_GUARD_BEGIN
    MOE_REQUIRE(P, "moe_adapter_project: null descriptor");
    MOE_REQUIRE(act_type == MOE_F32 || act_type == MOE_BF16,
                "moe_adapter_project: act_type=%d is neither MOE_F32 nor MOE_BF16", act_type);
    MOE_REQUIRE(T >= 0 && T <= MOE_ADAPTER_MAX_TOKENS, "moe_adapter_project: T=%d out of [0,%d]", T, MOE_ADAPTER_MAX_TOKENS);
    MOE_REQUIRE(P->d_in > 0 && P->d_in % 8 == 0 && P->d_in <= MOE_ADAPTER_MAX_D,
                "moe_adapter_project: d_in=%d must be a multiple of 8 in [8,%d]", P->d_in, MOE_ADAPTER_MAX_D);
    MOE_REQUIRE(P->d_out > 0 && P->d_out % 8 == 0 && P->d_out <= MOE_ADAPTER_MAX_D,
                "moe_adapter_project: d_out=%d must be a multiple of 8 in [8,%d]", P->d_out, MOE_ADAPTER_MAX_D);
    MOE_REQUIRE(P->n_adapters >= 0, "moe_adapter_project: n_adapters=%d < 0", P->n_adapters);
    MOE_REQUIRE(P->rank > 0 && P->rank % 8 == 0 && P->rank <= MOE_ADAPTER_MAX_RANK,
                "moe_adapter_project: rank=%d must be a multiple of 8 in [8,%d]", P->rank, MOE_ADAPTER_MAX_RANK);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(x && y && adapters && workspace && (P->n_adapters == 0 || (P->a && P->b)), "moe_adapter_project: null pointer");
    MOE_REQUIRE(x_stride >= P->d_in && x_stride % 8 == 0, "moe_adapter_project: x_stride=%lld must be a multiple of 8 >= d_in=%d",
                (long long)x_stride, P->d_in);
    MOE_REQUIRE(y_stride >= P->d_out && y_stride % 8 == 0,
                "moe_adapter_project: y_stride=%lld must be a multiple of 8 >= d_out=%d", (long long)y_stride, P->d_out);
    MOE_REQUIRE(!y_in || (y_in_stride >= P->d_out && y_in_stride % 8 == 0),
                "moe_adapter_project: y_in_stride=%lld must be a multiple of 8 >= d_out=%d", (long long)y_in_stride, P->d_out);
    MOE_REQUIRE(y_in != y || y_in_stride == y_stride, "moe_adapter_project: y over y_in with another stride");
    MOE_REQUIRE(moe::aligned16(x) && moe::aligned16(y) && moe::aligned16(y_in) && moe::aligned16(P->w) && moe::aligned16(P->a) &&
                    moe::aligned16(P->b),
                "moe_adapter_project: device pointers must be 16-byte aligned");
    MOE_REQUIRE(((uintptr_t)workspace & 255u) == 0, "moe_adapter_project: workspace not 256-byte aligned");
    const bool bf16 = act_type == MOE_BF16;
    const moe::AdapterPlan L = moe::plan_adapter(T, P->d_in, P->d_out, P->rank, bf16);
    MOE_REQUIRE(workspace_bytes >= L.bytes, "moe_adapter_project: workspace %zu < %zu bytes", workspace_bytes, L.bytes);
    moe::AdapterParams p{};
    p.x = x;
    p.bf16 = bf16;
    p.ldx = x_stride;
    p.ldy = y_stride;
    p.ldyin = y_in_stride;
    p.w = static_cast<const uint8_t *>(P->w);
    p.a = static_cast<const uint8_t *>(P->a);
    p.b = static_cast<const uint8_t *>(P->b);
    p.ids = adapters;
    p.scale = P->scale;
    p.T = T;
    p.d = P->d_in;
    p.o = P->d_out;
    p.n = P->n_adapters;
    p.r = P->rank;
    p.y_in = y_in;
    p.y = y;
    MOE_HIP(moe::launch_adapter(p, L, static_cast<uint8_t *>(workspace), (hipStream_t)stream));
    return MOE_OK;
    MOE_GUARD_END
}

}  // extern "C"
