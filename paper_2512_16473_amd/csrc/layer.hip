// One MoE layer for a few tokens (T <= 16), routed on the device:
//   l = Wr x, S_t = the k largest of l_t, g = softmax of l_t over S_t
//   y_t = y_in_t + sum_{e in S_t} g_te FFN_e(x_t) + FFN_shared(x_t),
//   FFN(x) = W2 (SiLU(W1 x) * W3 x)
//
// Every selected expert's weights are read once for all the tokens. Kernels, on one stream:
//   1. logits: fp64 sums, one wave per (token, expert);
//   2. gate/up: each work group selects the top k from the logits and then takes blocks of 16
//      rows of W1 and W3 of the selected experts and of the shared one. All the tokens are
//      multiplied with every expert's rows (the matrix cores have room for 16 columns whether
//      they are used or not), so the tokens' fragments are loaded once per work group. The
//      hidden values of a token that did not select the expert are zero, the others are scaled
//      by the gate weight, so that
//   3. down is one sum over all the experts' hidden columns, y_t = W2_all h_t: the columns are
//      cut into units of up to 512, a work group takes eight units (a group) of 16 rows of W2,
//      and, where there is more than one group,
//   4. the groups' sums are added in order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "common.h"
#include "moe_internal.h"
#include "row_stream.h"

namespace moe {
namespace {

using namespace row_stream;

constexpr int kMaxTok = MOE_LAYER_MAX_TOKENS;
constexpr int kMaxSel = kMaxTok * MOE_MAX_TOPK_INTERNAL;

struct LayerParams {
    const void *x;                // [T][d]
    bool bf16;                    // of x, y_in and y; else fp32
    const float *wr;              // [n][d]
    const uint8_t *pool;
    uint64_t slab_stride;
    const uint8_t *shared;        // shared expert's slab or null
    const int32_t *slotmap;       // [n] or null (expert e in slot e)
    int T, d, f, fs, n, k, nslots;
    double *logits;               // [T][n]
    int32_t *idx;                 // [T][k]
    float *w;                     // [T][k]
    uint8_t *h;                   // hidden values as operand fragments (h_offset)
    int cols;                     // columns of h: T times its parts
    float *partial;               // [groups][T][d]
    const void *y_in;             // or null
    void *y;
};

// Part counts: fp32 activations and hidden values in three parts (exact); for a bf16 layer x is
// exact in one, and the hidden values are kept in two (2^-17 relative: far below the rounding
// of y, at the cost of columns that are there anyway).
__host__ __device__ inline int h_parts(bool bf16) { return bf16 ? 2 : 3; }

// The selected experts that have a slot, in ascending order.
struct Jobs {
    int n;
    int expert[MOE_MAX_EXPERTS];
    int slot[MOE_MAX_EXPERTS];
    int count[MOE_MAX_EXPERTS / kWave];
    int chosen[MOE_MAX_EXPERTS];
};

// From J.chosen (nonzero: selected by some token). Ends with a barrier.
__device__ __forceinline__ void build_jobs(const LayerParams &p, Jobs &J)
{
    const int e = threadIdx.x, lane = e & 63;
    int slot = -1;
    uint64_t m = 0;
    if (e < MOE_MAX_EXPERTS) {
        if (e < p.n && J.chosen[e]) {
            slot = p.slotmap ? p.slotmap[e] : e;
            if (slot >= p.nslots) slot = -1;
        }
        m = __ballot(slot >= 0);
        if (lane == 0) J.count[e >> 6] = __popcll(m);
    }
    __syncthreads();
    if (e < MOE_MAX_EXPERTS) {
        int at = __popcll(m & ((1ull << lane) - 1));
        for (int i = 0; i < e >> 6; ++i) at += J.count[i];
        if (slot >= 0) {
            J.expert[at] = e;
            J.slot[at] = slot;
        }
        if (e == MOE_MAX_EXPERTS - 1) J.n = at + (slot >= 0);
    }
    __syncthreads();
}

// Logits: wave i of the grid takes expert i / T and token i % T.
__global__ __launch_bounds__(256) void k_layer_logits(LayerParams p)
{
    const int lane = threadIdx.x & 63;
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= p.n * p.T) return;
    const int e = i / p.T, t = i - e * p.T;
    const float4 *w = reinterpret_cast<const float4 *>(p.wr + (size_t)e * p.d);
    double acc = 0.0;
    const int nq = p.d >> 2;
    auto dot = [&](const float4 a, const float4 b) {
        acc = fma((double)a.x, (double)b.x, acc);
        acc = fma((double)a.y, (double)b.y, acc);
        acc = fma((double)a.z, (double)b.z, acc);
        acc = fma((double)a.w, (double)b.w, acc);
    };
    if (p.bf16) {
        const uint2 *x = reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p.x) + (size_t)t * p.d);
#pragma unroll 4
        for (int c = lane; c < nq; c += kWave) {
            const uint2 v = x[c];
            dot(w[c], make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                                  __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)));
        }
    } else {
        const float4 *x = reinterpret_cast<const float4 *>(static_cast<const float *>(p.x) + (size_t)t * p.d);
#pragma unroll 4
        for (int c = lane; c < nq; c += kWave) dot(w[c], x[c]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, kWave);
    if (lane == 0) p.logits[(size_t)t * p.n + e] = acc;
}

// The top k of every token: sel[t * k + r] = expert of rank r, w its gate weight, J the jobs.
// An expert's rank is the number of logits before its own (larger, or equal with a lower id; NaN
// counts as -infinity). lg: room for T * n + T * k doubles.
__device__ __forceinline__ void select(const LayerParams &p, double *lg, int *sel, float *w, Jobs &J)
{
    const int tid = threadIdx.x, nl = p.T * p.n, ns = p.T * p.k;
    double *top = lg + nl;
    for (int i = tid; i < nl; i += kThreads) {
        const double v = p.logits[i];
        lg[i] = v != v ? -INFINITY : v;
    }
    if (tid < MOE_MAX_EXPERTS) J.chosen[tid] = 0;
    __syncthreads();
    for (int i = tid; i < nl; i += kThreads) {
        const int t = i / p.n, e = i - t * p.n;
        const double *row = lg + t * p.n, v = row[e];
        int rank = 0;
        for (int j = 0; j < p.n; ++j) {
            const double o = row[j];
            rank += (o > v || (o == v && j < e)) ? 1 : 0;
        }
        if (rank < p.k) {
            sel[t * p.k + rank] = e;
            top[t * p.k + rank] = v;
            J.chosen[e] = 1;
        }
    }
    __syncthreads();
    double ex = 0.0;
    if (tid < ns) ex = exp(top[tid] - top[tid / p.k * p.k]);
    __syncthreads();
    if (tid < ns) top[tid] = ex;
    __syncthreads();
    if (tid < ns) {
        const double *row = top + tid / p.k * p.k;
        double z = 0.0;
        for (int r = 0; r < p.k; ++r) z += row[r];
        w[tid] = (float)(ex / z);
    }
    build_jobs(p, J);
}

// Fragments of the hidden values: of a job's K step (32 values), column block by column block,
// lane by lane, the 8 values of the lane. The shared expert's come first.
__host__ __device__ inline int k_steps(int f) { return (f + kChunk - 1) / kChunk * 2; }
__device__ __forceinline__ size_t h_steps(const LayerParams &p, int job)   // K steps before the job's; -1: shared
{
    return job < 0 ? 0 : (size_t)(p.shared ? k_steps(p.fs) : 0) + (size_t)job * k_steps(p.f);
}

struct GateUpSrc {
    const uint8_t *base0, *base1;
    size_t half;
    int c0, cnt;
    const LayerParams &p;
    const Jobs &J;
    int it, step, total, rbs, rbf;   // next item, items of the layer, row blocks of the shared and of a routed expert
    template <class R>
    __device__ __forceinline__ bool next(R &)
    {
        if (it >= total || cnt == 0) return false;
        const bool sh = it < rbs;
        const int job = sh ? 0 : (it - rbs) / rbf, rb = sh ? it : it - rbs - job * rbf;
        const int f = sh ? p.fs : p.f;
        const uint8_t *slab = sh ? p.shared : p.pool + (uint64_t)J.slot[job] * p.slab_stride;
        const size_t K2 = (size_t)p.d * 2;
        base0 = slab + (size_t)rb * kRows * K2;
        base1 = base0 + (size_t)f * K2;
        half = rb * kRows + 8 < f ? 8 * K2 : 0;   // the last block may have 8 rows
        it += step;
        return true;
    }
};

// Gate/up: h = g * SiLU(W1 x) * (W3 x), for every job, row and token. NB = column blocks of x.
template <int S, int NB>
__global__ __launch_bounds__(kThreads) void k_layer_gate_up(LayerParams p)
{
    constexpr int RS = NB == 1 ? 8 : 6;
    constexpr int kRing = kWaves * RS * kStageBytes;
    __shared__ __align__(1024) uint8_t lds[kRing + kWaves * 2 * NB * 1024];
    __shared__ Jobs J;
    __shared__ int sel[kMaxSel];
    __shared__ float gate[kMaxSel];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    static_assert((kMaxTok * MOE_MAX_EXPERTS + kMaxSel) * sizeof(double) <= kRing, "the logits fit the ring");
    select(p, reinterpret_cast<double *>(lds), sel, gate, J);
    if (blockIdx.x == 0 && tid < p.T * p.k) {
        p.idx[tid] = sel[tid];
        p.w[tid] = gate[tid];
    }
    const int rbs = p.shared ? (p.fs + kRows - 1) / kRows : 0, rbf = (p.f + kRows - 1) / kRows;
    const int total = rbs + __builtin_amdgcn_readfirstlane(J.n) * rbf;
    GateUpSrc src{nullptr, nullptr, 0, 0, 0, p, J, (int)blockIdx.x, (int)gridDim.x, total, rbs, rbf};
    part_chunks((p.d + kChunk - 1) / kChunk, wv, kWaves, src.c0, src.cnt);
    Stream<S, 2, NB, RS, GateUpSrc> st;
    st.ring.row_bytes((int64_t)p.d * 2);
    st.start(src, lds + wv * RS * kStageBytes);
    bf16x8_t bx[S][2][NB];
    const int parts = p.bf16 ? 1 : 3;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int c = nb * 16 + (lane & 15), part = c / p.T, t = c - part * p.T;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int k = (src.c0 + s) * kChunk + kb * 32 + (lane >> 4) * 8;
                bx[s][kb][nb] = s < src.cnt && k < p.d && part < parts ? load_part(p.x, p.bf16, (size_t)t * p.d + k, part)
                                                                       : no_tokens();
            }
    }
    float *red = reinterpret_cast<float *>(lds + kRing);
    const int nb2 = (p.cols + 15) >> 4, hp = h_parts(p.bf16);
    for (int it = blockIdx.x; it < total; it += gridDim.x) {
        floatx4_t acc[2][NB];
        st.item(src, bx, src.cnt, acc);
        lds_barrier();                             // the sums before are read
        put_sums(red, wv, acc);
        lds_barrier();
        const bool sh = it < rbs;
        const int job = sh ? -1 : (it - rbs) / rbf, rb = sh ? it : it - rbs - job * rbf;
        const int row = tid & 15, t = tid >> 4, i = rb * kRows + row;
        if (t < p.T && i < (sh ? p.fs : p.f)) {
            float wt = sh ? 1.f : 0.f;
            bool mine = sh;
            if (!sh) {
                const int e = J.expert[job];
                for (int r = 0; r < p.k; ++r)
                    if (sel[t * p.k + r] == e) {
                        wt = gate[t * p.k + r];
                        mine = true;
                    }
            }
            float g = 0.f, u = 0.f;
            for (int q = 0; q < parts; ++q) {
                g += get_sum<2, NB>(red, 0, row, q * p.T + t);
                u += get_sum<2, NB>(red, 1, row, q * p.T + t);
            }
            const float hv = mine ? wt * (g / (1.0f + expf(-g)) * u) : 0.f;
            const size_t step = h_steps(p, job) + (i >> 5);
            for (int q = 0; q < hp; ++q) {
                const int c = q * p.T + t;
                uint8_t *dst = p.h + ((step * nb2 + (c >> 4)) * kWave + ((i & 31) >> 3) * 16 + (c & 15)) * 16 + (i & 7) * 2;
                *reinterpret_cast<uint16_t *>(dst) = hp == 3 ? part_of<3>(hv, q) : part_of<2>(hv, q);
            }
        }
    }
}

// A wave's unit of the hidden columns: unit u of the layer (the shared expert's first).
struct Unit {
    int job, f, c0, cnt;   // job -1: the shared expert; cnt 0: none
};
__device__ __forceinline__ Unit unit_of(const LayerParams &p, int u, int us, int uf, int units)
{
    Unit r{-1, p.fs, 0, 0};
    if (u >= units) return r;
    if (u < us) {
        part_chunks((p.fs + kChunk - 1) / kChunk, u, us, r.c0, r.cnt);
    } else {
        r.job = (u - us) / uf;
        r.f = p.f;
        part_chunks((p.f + kChunk - 1) / kChunk, u - us - r.job * uf, uf, r.c0, r.cnt);
    }
    return r;
}

struct DownSrc {
    const uint8_t *base0, *base1;
    size_t half;
    int c0, cnt;
    const LayerParams &p;
    const Jobs &J;
    int wv, it, end, rbs, us, uf, units, group;
    const uint8_t *w2;
    size_t K2;
    template <class R>
    __device__ __forceinline__ bool next(R &ring)
    {
        for (;;) {
            if (it >= end) return false;
            const int g = it / rbs;
            if (g != group) {
                group = g;
                const Unit u = unit_of(p, g * kWaves + wv, us, uf, units);
                c0 = u.c0;
                cnt = u.cnt;
                K2 = (size_t)u.f * 2;
                const uint8_t *slab = u.job < 0 ? p.shared : p.pool + (uint64_t)J.slot[u.job] * p.slab_stride;
                w2 = slab + (size_t)2 * u.f * p.d * 2;
                ring.row_bytes((int64_t)K2);
            }
            if (cnt) break;
            it = (g + 1) * rbs;   // nothing for this wave in the group
        }
        const int rb = it - group * rbs;
        base0 = w2 + (size_t)rb * kRows * K2;
        half = rb * kRows + 8 < p.d ? 8 * K2 : 0;
        ++it;
        return true;
    }
};

// Down: the sums of group g (eight units of hidden columns) for 16 rows of W2 and all tokens. A
// work group takes an equal, contiguous share of the (group, row block) items. kOne: there is
// one group, whose sums are the layer's output.
template <int S, int NB, bool kOne>
__global__ __launch_bounds__(kThreads) void k_layer_down(LayerParams p)
{
    constexpr int RS = 8;
    constexpr int kRing = kWaves * RS * kStageBytes;
    __shared__ __align__(1024) uint8_t lds[kRing + kWaves * NB * 1024];
    __shared__ Jobs J;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < MOE_MAX_EXPERTS) J.chosen[tid] = 0;
    __syncthreads();
    if (tid < p.T * p.k) J.chosen[p.idx[tid]] = 1;
    __syncthreads();
    build_jobs(p, J);
    const int chunks_s = p.shared ? (p.fs + kChunk - 1) / kChunk : 0, chunks_f = (p.f + kChunk - 1) / kChunk;
    const int us = (chunks_s + S - 1) / S, uf = (chunks_f + S - 1) / S;
    const int units = us + __builtin_amdgcn_readfirstlane(J.n) * uf;
    const int rbs = (p.d + kRows - 1) / kRows;
    const int groups = kOne ? 1 : (units + kWaves - 1) / kWaves;
    const int64_t total = (int64_t)groups * rbs;
    const int it0 = (int)(total * blockIdx.x / gridDim.x), it1 = (int)(total * (blockIdx.x + 1) / gridDim.x);
    DownSrc src{nullptr, nullptr, 0, 0, 0, p, J, wv, it0, it1, rbs, us, uf, units, -1, nullptr, 0};
    Stream<S, 1, NB, RS, DownSrc> st;
    st.start(src, lds + wv * RS * kStageBytes);
    float *red = reinterpret_cast<float *>(lds + kRing);
    const int parts = h_parts(p.bf16);
    bf16x8_t bx[S][2][NB];
    int group = -1;
    Unit u{};
    for (int it = it0; it < it1; ++it) {
        const int g = it / rbs, rb = it - g * rbs;
        if (g != group) {
            group = g;
            u = unit_of(p, g * kWaves + wv, us, uf, units);
            const size_t step0 = h_steps(p, u.job) + 2 * u.c0;
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const int k = (u.c0 + s) * kChunk + kb * 32 + (lane >> 4) * 8;
                        const bool live = s < u.cnt && k < u.f && nb * 16 + (lane & 15) < p.cols;
                        bx[s][kb][nb] = live ? *reinterpret_cast<const bf16x8_t *>(
                                                   p.h + (((step0 + 2 * s + kb) * NB + nb) * kWave + lane) * 16)
                                             : no_tokens();
                    }
        }
        floatx4_t acc[1][NB];
        st.item(src, bx, u.cnt, acc);
        lds_barrier();
        put_sums(red, wv, acc);
        lds_barrier();
        const int row = tid & 15, t = tid >> 4, i = rb * kRows + row;
        if (t < p.T && i < p.d) {
            float v = 0.f;
            for (int q = 0; q < parts; ++q) v += get_sum<1, NB>(red, 0, row, q * p.T + t);
            const size_t at = (size_t)t * p.d + i;
            if (kOne) {
                if (p.bf16) {
                    if (p.y_in) v += static_cast<float>(static_cast<const __bf16 *>(p.y_in)[at]);
                    static_cast<__bf16 *>(p.y)[at] = static_cast<__bf16>(v);
                } else {
                    if (p.y_in) v += static_cast<const float *>(p.y_in)[at];
                    static_cast<float *>(p.y)[at] = v;
                }
            } else {
                p.partial[(size_t)g * p.T * p.d + at] = v;
            }
        }
    }
}

// y = y_in + the groups' sums, in order.
template <int S>
__global__ __launch_bounds__(256) void k_layer_sum(LayerParams p)
{
    __shared__ Jobs J;
    const int tid = threadIdx.x;
    J.chosen[tid] = 0;
    __syncthreads();
    if (tid < p.T * p.k) J.chosen[p.idx[tid]] = 1;
    __syncthreads();
    build_jobs(p, J);
    const int chunks_s = p.shared ? (p.fs + kChunk - 1) / kChunk : 0, chunks_f = (p.f + kChunk - 1) / kChunk;
    const int units = (chunks_s + S - 1) / S + J.n * ((chunks_f + S - 1) / S);
    const int groups = (units + kWaves - 1) / kWaves;
    const int at = blockIdx.x * 256 + tid, n = p.T * p.d;
    if (at >= n) return;
    float v = 0.f;
#pragma unroll 8
    for (int g = 0; g < groups; ++g) v += p.partial[(size_t)g * n + at];
    if (p.bf16) {
        if (p.y_in) v += static_cast<float>(static_cast<const __bf16 *>(p.y_in)[at]);
        static_cast<__bf16 *>(p.y)[at] = static_cast<__bf16>(v);
    } else {
        if (p.y_in) v += static_cast<const float *>(p.y_in)[at];
        static_cast<float *>(p.y)[at] = v;
    }
}

size_t a256(size_t v) { return (v + 255) & ~(size_t)255; }
int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Sizes that follow from the call's.
struct LayerPlan {
    int cols, nb, s, groups;   // of h: columns and their blocks; chunks of a unit; groups at most
    size_t logits, idx, w, h, partial, bytes;
};

LayerPlan plan_layer(int T, int d, int f, int n, int k, int fs, bool bf16)
{
    LayerPlan L{};
    L.cols = T * h_parts(bf16);
    L.nb = ceil_div(L.cols, 16);
    const int jobs = std::min(n, T * k);
    // Units of 512 columns (256 with three column blocks, whose fragments fill the registers),
    // shorter where eight of them would hold all the columns.
    const int64_t chunks = (int64_t)jobs * ceil_div(f, kChunk) + ceil_div(fs, kChunk);
    L.s = L.nb == 3 ? 4 : 8;
    while (L.s > 1 && chunks <= (int64_t)L.s / 2 * kWaves) L.s /= 2;
    const int64_t units = (int64_t)jobs * ceil_div(ceil_div(f, kChunk), L.s) + ceil_div(ceil_div(fs, kChunk), L.s);
    L.groups = (int)((units + kWaves - 1) / kWaves);
    size_t o = 0;
    auto take = [&](size_t b) {
        const size_t at = o;
        o += a256(b);
        return at;
    };
    L.logits = take((size_t)T * n * 8);
    L.idx = take((size_t)T * k * 4);
    L.w = take((size_t)T * k * 4);
    L.h = take(((size_t)jobs * k_steps(f) + (fs ? k_steps(fs) : 0)) * L.nb * kWave * 16);
    L.partial = take(L.groups > 1 ? (size_t)L.groups * T * d * 4 : 0);
    L.bytes = o;
    return L;
}

template <int S, int NB>
hipError_t launch_gate_up(const LayerParams &p, hipStream_t s)
{
    hipLaunchKernelGGL((k_layer_gate_up<S, NB>), dim3(device_cu_count()), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <int S, int NB>
hipError_t launch_down(const LayerParams &p, int groups, hipStream_t s)
{
    const int rbs = ceil_div(p.d, kRows);
    const dim3 grid((unsigned)std::min<int64_t>(device_cu_count(), (int64_t)groups * rbs));
    if (groups == 1) hipLaunchKernelGGL((k_layer_down<S, NB, true>), grid, dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((k_layer_down<S, NB, false>), grid, dim3(kThreads), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || groups == 1) return e;
    hipLaunchKernelGGL(k_layer_sum<S>, dim3((unsigned)ceil_div(p.T * p.d, 256)), dim3(256), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_layer(const LayerParams &p, const LayerPlan &L, hipStream_t s)
{
    (void)hipGetLastError();
    hipError_t e;
    hipLaunchKernelGGL(k_layer_logits, dim3((unsigned)ceil_div(p.n * p.T, 4)), dim3(256), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int nb1 = ceil_div(p.T * (p.bf16 ? 1 : 3), 16), s1 = ceil_div(ceil_div(p.d, kChunk), kWaves);
    // T * d <= MOE_LAYER_MAX_VALUES: 16 chunks a wave with one column block, 11 with two, 6 with three
    switch (nb1 * 100 + s1) {
#define MOE_GU(NB, S) \
    case NB * 100 + S: e = launch_gate_up<S, NB>(p, s); break;
        MOE_GU(1, 1) MOE_GU(1, 2) MOE_GU(1, 3) MOE_GU(1, 4) MOE_GU(1, 5) MOE_GU(1, 6) MOE_GU(1, 7) MOE_GU(1, 8)
        MOE_GU(1, 9) MOE_GU(1, 10) MOE_GU(1, 11) MOE_GU(1, 12) MOE_GU(1, 13) MOE_GU(1, 14) MOE_GU(1, 15) MOE_GU(1, 16)
        MOE_GU(2, 1) MOE_GU(2, 2) MOE_GU(2, 3) MOE_GU(2, 4) MOE_GU(2, 5) MOE_GU(2, 6) MOE_GU(2, 7) MOE_GU(2, 8)
        MOE_GU(2, 9) MOE_GU(2, 10) MOE_GU(2, 11)
        MOE_GU(3, 1) MOE_GU(3, 2) MOE_GU(3, 3) MOE_GU(3, 4) MOE_GU(3, 5) MOE_GU(3, 6)
#undef MOE_GU
    default: return hipErrorInvalidValue;
    }
    if (e != hipSuccess) return e;
    switch (L.nb * 100 + L.s) {
#define MOE_DN(NB, S) \
    case NB * 100 + S: return launch_down<S, NB>(p, L.groups, s);
        MOE_DN(1, 1) MOE_DN(1, 2) MOE_DN(1, 4) MOE_DN(1, 8)
        MOE_DN(2, 1) MOE_DN(2, 2) MOE_DN(2, 4) MOE_DN(2, 8)
        MOE_DN(3, 1) MOE_DN(3, 2) MOE_DN(3, 4)
#undef MOE_DN
    default: return hipErrorInvalidValue;
    }
}

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_layer_tokens_workspace_bytes(int T, int d, int f, int n, int k, int f_shared)
{
    if (T < 1 || T > MOE_LAYER_MAX_TOKENS || d <= 0 || f <= 0 || n < 1 || k < 1 || k > MOE_MAX_TOPK || f_shared < 0) return 0;
    const size_t a = moe::plan_layer(T, d, f, n, k, f_shared, false).bytes, b = moe::plan_layer(T, d, f, n, k, f_shared, true).bytes;
    return a > b ? a : b;   // the same for both types of activations
}

int moe_layer_tokens(const moe_tokens_desc *P, const void *x, int T, const void *y_in, void *y, int32_t *idx, float *w,
                     int act_type, void *workspace, size_t workspace_bytes, void *stream)
{
    MOE_GUARD_BEGIN
    MOE_REQUIRE(P, "moe_layer_tokens: null descriptor");
    MOE_REQUIRE(act_type == MOE_F32 || act_type == MOE_BF16, "moe_layer_tokens: act_type=%d is neither MOE_F32 nor MOE_BF16",
                act_type);
    MOE_REQUIRE(T >= 0 && T <= MOE_LAYER_MAX_TOKENS, "moe_layer_tokens: T=%d out of [0,%d]", T, MOE_LAYER_MAX_TOKENS);
    MOE_REQUIRE(P->d > 0 && P->d % 8 == 0 && P->d <= MOE_MAX_D, "moe_layer_tokens: d=%d must be a multiple of 8 in [8,%d]",
                P->d, MOE_MAX_D);
    MOE_REQUIRE((int64_t)T * P->d <= MOE_LAYER_MAX_VALUES, "moe_layer_tokens: T*d=%lld exceeds %d", (long long)T * P->d,
                MOE_LAYER_MAX_VALUES);
    MOE_REQUIRE(P->f > 0 && P->f % 8 == 0 && P->f <= MOE_LAYER_MAX_F, "moe_layer_tokens: f=%d must be a multiple of 8 in [8,%d]",
                P->f, MOE_LAYER_MAX_F);
    MOE_REQUIRE(P->f_shared >= 0 && P->f_shared % 8 == 0 && P->f_shared <= MOE_LAYER_MAX_F,
                "moe_layer_tokens: f_shared=%d must be a multiple of 8 in [0,%d]", P->f_shared, MOE_LAYER_MAX_F);
    MOE_REQUIRE(P->n >= 1 && P->n <= MOE_MAX_EXPERTS, "moe_layer_tokens: n=%d out of [1,%d]", P->n, MOE_MAX_EXPERTS);
    MOE_REQUIRE(P->k >= 1 && P->k <= P->n && P->k <= MOE_MAX_TOPK, "moe_layer_tokens: k=%d out of [1,min(n,%d)]", P->k,
                MOE_MAX_TOPK);
    MOE_REQUIRE(P->n_slots >= 0, "moe_layer_tokens: n_slots=%d < 0", P->n_slots);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(x && y && workspace && P->w_router && (P->slot_pool || P->n_slots == 0) && (P->shared || P->f_shared == 0),
                "moe_layer_tokens: null pointer");
    MOE_REQUIRE(moe::aligned16(x) && moe::aligned16(y) && moe::aligned16(y_in) && moe::aligned16(P->w_router) &&
                    moe::aligned16(P->slot_pool) && moe::aligned16(P->shared),
                "moe_layer_tokens: device pointers must be 16-byte aligned");
    MOE_REQUIRE(((uintptr_t)workspace & 255u) == 0, "moe_layer_tokens: workspace not 256-byte aligned");
    const bool bf16 = act_type == MOE_BF16;
    const moe::LayerPlan L = moe::plan_layer(T, P->d, P->f, P->n, P->k, P->f_shared, bf16);
    MOE_REQUIRE(workspace_bytes >= L.bytes, "moe_layer_tokens: workspace %zu < %zu bytes", workspace_bytes, L.bytes);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    moe::LayerParams p{};
    p.x = x;
    p.bf16 = bf16;
    p.wr = P->w_router;
    p.pool = static_cast<const uint8_t *>(P->slot_pool);
    p.slab_stride = moe_slab_bytes(P->d, P->f);
    p.shared = P->f_shared ? static_cast<const uint8_t *>(P->shared) : nullptr;
    p.slotmap = P->slotmap;
    p.T = T;
    p.d = P->d;
    p.f = P->f;
    p.fs = P->f_shared;
    p.n = P->n;
    p.k = P->k;
    p.nslots = P->n_slots;
    p.logits = reinterpret_cast<double *>(ws + L.logits);
    p.idx = idx ? idx : reinterpret_cast<int32_t *>(ws + L.idx);
    p.w = w ? w : reinterpret_cast<float *>(ws + L.w);
    p.h = ws + L.h;
    p.cols = L.cols;
    p.partial = reinterpret_cast<float *>(ws + L.partial);
    p.y_in = y_in;
    p.y = y;
    MOE_HIP(moe::launch_layer(p, L, (hipStream_t)stream));
    return MOE_OK;
    MOE_GUARD_END
}

}  // extern "C"
