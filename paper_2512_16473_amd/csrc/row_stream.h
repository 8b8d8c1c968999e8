// A few tokens against long weight rows: the device code that moe_layer_tokens and
// moe_adapter_project share (HIP device code only).
//
// A work group has 8 waves. It takes weight rows 16 at a time; each wave owns a slice of the
// reduction (a unit: up to S chunks of 64 columns) and multiplies its slice of the 16 rows
// with the tokens by v_mfma_f32_16x16x32_bf16, the weights as the A operand and the tokens
// as the B operand, so the matrix cores do per 1 KiB of weights one or a few instructions
// and the kernel is bound by reading the weights. The tokens' fragments stay in registers
// for all the rows; the weights go from memory straight to LDS (8 rows by 128 bytes per
// load instruction) in a ring of stages that belongs to one wave, so that a wave waits for
// its own loads only and no barrier stands in the stream. The waves' sums of a row block
// meet in LDS.
//
// Reading 2 GiB this way (rows of 8 KiB, nothing multiplied) runs at 6.80 TB/s, and at 6.94
// where 8 KiB are read of each 28 KiB row; loading the same fragments into registers (16
// rows by 64 bytes per instruction) gives 6.0 and 5.2, one contiguous KiB per instruction
// 7.0, and loads that keep the lines in the caches 6.1.
//
// fp32 activations are cut into three bf16 parts of 8 bits each, v = hi + mid + lo exactly,
// which take three columns of the B operand: the products with bf16 weights are then exact
// and the sums fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moe {
namespace row_stream {

constexpr int kWave = 64;
constexpr int kWaves = 8;
constexpr int kThreads = kWave * kWaves;
constexpr int kRows = 16;           // weight rows of an item
constexpr int kChunk = 64;          // columns of a stage
constexpr int kStageBytes = kRows * kChunk * 2;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const void global_cvoid;
typedef __attribute__((address_space(3))) void lds_void;

template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// This wave's LDS accesses are done; then every wave is here. The weight loads stay in flight.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Part p of P (1 to 3) of v in bf16: the parts but the last are cut off, the last is rounded to
// nearest; three hold all 24 bits. Infinities and NaN have no further parts.
template <int P>
__device__ __forceinline__ uint16_t part_of(float v, int p)
{
    const uint32_t u = __float_as_uint(v);
    const float r1 = v - __uint_as_float(u & 0xffff0000u);
    const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
    const float part = p == 0 ? v : p == 1 ? r1 : r2;
    uint32_t bits = __float_as_uint(part) >> 16;
    if (p == P - 1) bits = __builtin_bit_cast(uint16_t, static_cast<__bf16>(part));
    if ((u & 0x7f800000u) == 0x7f800000u) bits = p ? 0 : (u >> 16) | ((u & 0xffffu) ? 0x40u : 0u);
    return (uint16_t)bits;
}

// 8 consecutive activations from element `at` of `x` (bf16 or fp32), part p of each.
__device__ __forceinline__ bf16x8_t load_part(const void *x, bool bf16, size_t at, int p)
{
    if (bf16) return *reinterpret_cast<const bf16x8_t *>(static_cast<const uint16_t *>(x) + at);
    const float4 *src = reinterpret_cast<const float4 *>(static_cast<const float *>(x) + at);
    const float4 a = src[0], b = src[1];
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = part_of<3>(v[2 * i], p) | ((uint32_t)part_of<3>(v[2 * i + 1], p) << 16);
    return __builtin_bit_cast(bf16x8_t, make_uint4(o[0], o[1], o[2], o[3]));
}
__device__ __forceinline__ bf16x8_t no_tokens() { return __builtin_bit_cast(bf16x8_t, make_uint4(0, 0, 0, 0)); }

// The ring of one wave: weights of its items in order, stage by stage.
template <int NM, int RS>
struct Ring {
    static_assert(RS % NM == 0, "a chunk of NM matrices is NM stages");
    uint8_t *lds;              // RS stages
    int slot, rslot;           // next to read, next to fill
    int lane_row;              // byte offset of this lane's row within 8 rows
    int piece, lim;            // byte offset of this lane's 16 bytes in a chunk; the last in a row

    __device__ __forceinline__ void init(uint8_t *mine)
    {
        const int lane = threadIdx.x & 63;
        lds = mine;
        slot = rslot = 0;
        // lane l's 16 bytes land at slot l % 8 of row l / 8: chunk c of row r sits at c ^ r, so
        // that the operand reads (16 rows, one chunk per quarter wave) touch all banks evenly
        piece = ((lane & 7) ^ (lane >> 3)) * 16;
    }
    __device__ __forceinline__ void row_bytes(int64_t K2)
    {
        lane_row = (int)(((threadIdx.x & 63) >> 3) * K2);
        lim = (int)K2 - 16;
    }
    // Stage of 16 rows from `base` (rows 8 .. 15 from base + half), chunk `c` of the rows.
    __device__ __forceinline__ void fill(const uint8_t *base, size_t half, int c)
    {
        // past a row's end its last piece is read; the token operand is zero there
        const int o = min(c * (kChunk * 2) + piece, lim);
        const uint8_t *p = base + (uint32_t)(lane_row + o);
        uint8_t *to = lds + rslot * kStageBytes;
        __builtin_amdgcn_global_load_lds((global_cvoid *)p, (lds_void *)to, 16, 0, 2);   // 2: nontemporal
        __builtin_amdgcn_global_load_lds((global_cvoid *)(p + half), (lds_void *)(to + kStageBytes / 2), 16, 0, 2);
        rslot = rslot + 1 == RS ? 0 : rslot + 1;
    }
    // A operands of the next stage: its two K steps of 32.
    __device__ __forceinline__ void read(bf16x8_t (&w)[2])
    {
        const int lane = threadIdx.x & 63, row = lane & 15;
        const uint8_t *p = lds + slot * kStageBytes + row * (kChunk * 2);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) w[kb] = *reinterpret_cast<const bf16x8_t *>(p + ((kb * 4 + (lane >> 4)) ^ (row & 7)) * 16);
        slot = slot + 1 == RS ? 0 : slot + 1;
    }
};

// A wave's way through its items: the ring is kept full from `src`, which runs ahead of the
// sums by the ring's length. Src has base0 (and base1, the second matrix), half, c0, cnt of the item whose stages come
// next, and next(), which moves on to the wave's next item with cnt > 0 (false: none is left)
// and sets the ring's row length.
template <int S, int NM, int NB, int RS, class Src>
struct Stream {
    Ring<NM, RS> ring;
    bool left;                  // another stage is to be filled; then RS stages are on their way
    int q;                      // of the item in src: chunks times NM matrices

    __device__ __forceinline__ void issue(Src &src)
    {
        if (!left) return;
        ring.fill(NM == 1 || !(q & 1) ? src.base0 : src.base1, src.half, src.c0 + (NM == 1 ? q : q >> 1));
        if (++q == NM * src.cnt) {
            q = 0;
            left = src.next(ring);
        }
    }
    __device__ __forceinline__ void start(Src &src, uint8_t *lds)
    {
        ring.init(lds);
        q = 0;
        left = src.next(ring);
        for (int i = 0; i < RS; ++i) issue(src);
    }
    // acc[m][nb] = the sums of one item over this wave's cnt chunks
    __device__ __forceinline__ void item(Src &src, const bf16x8_t (&bx)[S][2][NB], int cnt, floatx4_t (&acc)[NM][NB])
    {
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[m][nb] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (s < cnt) {
                if (left) wait_loads<2 * (RS - NM)>();
                else wait_loads<0>();
                bf16x8_t w[NM][2];
#pragma unroll
                for (int m = 0; m < NM; ++m) ring.read(w[m]);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the slots are filled again
#pragma unroll
                for (int m = 0; m < NM; ++m) issue(src);
#pragma unroll
                for (int m = 0; m < NM; ++m)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
                            acc[m][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[m][kb], bx[s][kb][nb], acc[m][nb], 0, 0, 0);
            }
        }
    }
};

// The sums of a wave in LDS, [m][nb][256]: a lane's four rows of a column side by side.
template <int NM, int NB>
__device__ __forceinline__ void put_sums(float *red, int wv, const floatx4_t (&acc)[NM][NB])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            *reinterpret_cast<floatx4_t *>(red + ((wv * NM + m) * NB + nb) * 256 + lane * 4) = acc[m][nb];
}
// Sum over the waves, in order, of matrix m's (row, column c).
template <int NM, int NB>
__device__ __forceinline__ float get_sum(const float *red, int m, int row, int c)
{
    const float *p = red + (m * NB + (c >> 4)) * 256 + ((row >> 2) * 16 + (c & 15)) * 4 + (row & 3);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += p[w * NM * NB * 256];
    return v;
}

// Chunk range [c0, c0 + cnt) of part i of n equal parts of C chunks.
__device__ __forceinline__ void part_chunks(int C, int i, int n, int &c0, int &cnt)
{
    c0 = (int)((int64_t)C * i / n);
    cnt = (int)((int64_t)C * (i + 1) / n) - c0;
}

}  // namespace row_stream
}  // namespace moe
