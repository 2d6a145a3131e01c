// Products of bf16 or fp32 matrices on the matrix cores, tile by tile, for the loss over a vocabulary (include/tahq_loss.h).
#pragma once
#include <type_traits>

#include "tahq_mx4_common.hpp"
#include "tahq_tiles.hpp"

namespace tahq {

// Columns of a stage: 64 bytes of every row.
template <bool BF16>
constexpr int kStageCols = BF16 ? 32 : 16;

// How an operand of a product, C[m, n] = sum over k of A[m, k] B[n, k], lies in memory.
//   kBlocks, kBlocksTurned: blocks of 64 bytes of every row, [block][row][64 bytes], so that whatever a tile takes at a time is whole cache lines;
//     k along the blocks (m the rows), or, turned, k the rows (m along the blocks).  What a call makes itself lies like this.
//   kRows: row-major, k along a row, rows of whole 64 bytes.  Lines are 128 bytes: two stages are loaded at a time, or each line would be
//     fetched twice (logits of 8192 x 4096 x 131072 6.57 ms, stage by stage 6.79; of 5 x 1600 x 50257 out of the last cache 25.4 us, 27.1).
//   kTurned: row-major, k the rows.
enum Lies { kBlocks, kBlocksTurned, kRows, kTurned };

struct Operand {
    const uint8_t *base;
    uint64_t ld;               // bytes: row-major from row to row, blocks from block to block
    uint32_t rows;             // that may be read in memory
    uint32_t blocks;           // kBlocksTurned: that may be read
    uint64_t plane;            // bytes from plane to plane
};

// fp32 in planes: x = x1 + x2 + x3, bf16 each, every one what is left rounded to nearest; exact, as 8 bits, and twice 8 bits and a sign, are 24 and more.
// Of the nine products of two such sums six are taken, x1 y1, x1 y2, x1 y3, x2 y1, x2 y2, x3 y1; the others are up to 2^-24 of |x y| together (|x2| reaches
// 2^-8 |x|, |x3| 2^-17 |x|).  They are summed in fp32 like the columns of one product six times as long: stage 6 k + i has columns 32 k on of the i-th of
// these.  Numbers from 3.39e38 on, which bf16 rounds to infinity, begin with its largest one; infinity and NaN are the first plane alone, and products of
// an infinite number's planes are NaN where those of the number need not be (as_fp32).
__device__ __forceinline__ uint32_t plane_of_a(uint32_t i) { return i < 3 ? 0 : i < 5 ? 1 : 2; }
__device__ __forceinline__ uint32_t plane_of_b(uint32_t i) { return i < 3 ? i : i < 5 ? i - 3 : 0; }
__device__ __forceinline__ void split_planes(const float (&x)[8], uint4 (&planes)[3])
{
    constexpr float MOST = 3.3895313892515355e38f;           // of bf16
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = __builtin_isfinite(x[i]) ? __builtin_fminf(__builtin_fmaxf(x[i], -MOST), MOST) : x[i];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        const uint32_t w[4] = {two_bf16(left[0], left[1]), two_bf16(left[2], left[3]), two_bf16(left[4], left[5]), two_bf16(left[6], left[7])};
        planes[p] = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
        for (int i = 0; i < 8; ++i) left[i] = __builtin_isfinite(x[i]) ? (p ? left[i] : x[i]) - __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16) : 0.0f;
    }
}

// The tile of a workgroup: WM * MF units of 32 rows of A by WN * NF units of B; its four wavefronts take MF x NF units each.  A stage is 64 bytes of every
// row (32 columns of bf16, 16 of fp32); four of them are in LDS, one in use, three on their way (loads straight to LDS), of kRows three pairs.
//   What lies in LDS: a unit's 32 rows of 64 bytes (pairs: 128) in chunks of 16; turned, blocks' rows of k, or whole rows of k of the tile.  Loads write
//   LDS in a row; which 16 bytes a lane loads is chosen so that the operands' reads meet no bank twice, among eight lanes and among sixteen:
//   chunk c of row r is at place c ^ swap(r)
//   turned, bf16: 32 bytes (16 rows) number c of k are at place c ^ swap(k): four rows of k are read at a time, transposed on the way
//   to registers (ds_read_b64_tr_b16: sixteen lanes address 4 x 16 elements and each gets a column).  fp32: one number at a time.
//   Tiles of 256 x 256 take all of a compute unit's LDS and four wavefronts with 128 x 128 results each: an operand read from LDS goes into four products.
//   A stage takes 0.75 us, the products alone 0.55; a tile's start and end 11 us.  Workgroups that go on to further tiles, whose loads begin before the
//   results are stored, were 8 % slower.
//   Order of work as in the mx4 products: operands of a step (two to a stage) are read while the step before is multiplied; at the last step of a stage all
//   wavefronts have the operands in registers, the next stage's loads are waited for, and the stage just read is loaded over.
template <bool BF16, int WM_, int WN_, int MF_, int NF_>
struct TileKind {
    static constexpr int WM = WM_, WN = WN_, MF = MF_, NF = NF_, W = WM * WN, UM = WM * MF, UN = WN * NF;
    static constexpr int LOADS_A = 2 * UM, LOADS_B = 2 * UN, EACH_A = (LOADS_A + W - 1) / W, EACH_B = (LOADS_B + W - 1) / W, EACH = EACH_A + EACH_B, PRODUCTS = MF * NF;
    static constexpr int COLS = kStageCols<BF16>, ES = BF16 ? 2 : 4, STAGE_A = UM * 2048, STAGE_B = UN * 2048;
    static_assert(W == 4, "four wavefronts");
    // whether multiply_tile takes sums in parts: of fp32, where registers hold results twice
    template <int PLANES>
    static constexpr bool parts() { return (!BF16 || PLANES == 3) && PRODUCTS <= 4; }
    // and whether a kernel takes them run after run instead
    template <int PLANES>
    static constexpr bool runs() { return PLANES == 3 && !parts<PLANES>(); }
};
// What a workgroup has of LDS: a variable for each stage (kRows: of B for each pair), as the compiler then knows which loads a read has to wait for.
struct Stages {
    uint8_t *a[4], *b[4];
};
template <class T, Lies LIES_B>
__device__ __forceinline__ Stages stages_of()
{
    constexpr int BYTES = T::STAGE_B * (LIES_B == kRows ? 2 : 1);
    __shared__ __attribute__((aligned(1024))) uint8_t a0[T::STAGE_A], a1[T::STAGE_A], a2[T::STAGE_A], a3[T::STAGE_A], b0[BYTES], b1[BYTES], b2[BYTES];
    if constexpr (LIES_B == kRows) {
        return {{a0, a1, a2, a3}, {b0, b1, b2, b0}};
    } else {
        __shared__ __attribute__((aligned(1024))) uint8_t b3[BYTES];
        return {{a0, a1, a2, a3}, {b0, b1, b2, b3}};
    }
}

__device__ __forceinline__ uint32_t swap_of(uint32_t row) { return (row >> 2 & 1) << 1 | ((row >> 1 ^ row >> 3) & 1); }      // of four chunks
__device__ __forceinline__ uint32_t swap_of_pair(uint32_t row) { return (row & 7) ^ (row >> 3 & 1); }                        // of eight
__device__ __forceinline__ uint32_t swap_of_k(uint32_t k) { return (k & 3) | (k & 1) << 2; }                                 // of rows of k of a tile
__device__ __forceinline__ uint32_t swap_of_block(uint32_t k) { return k >> 1 & 1; }                                         // of rows of k of a block

// 32 rows of each operand and, of bf16, 16 columns (8 of fp32, four instructions).  Layout as the mx4 products': B goes first, a lane holds row
// lane % 32 and of the result row lane % 32 of A, rows 8 * (i / 4) + 4 * (lane / 32) + i % 4 of B.
template <bool BF16>
__device__ __forceinline__ float16v multiply32(const uint4 &b, const uint4 &a, float16v c)
{
    if constexpr (BF16) {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.x), __uint_as_float(a.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.y), __uint_as_float(a.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.z), __uint_as_float(a.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.w), __uint_as_float(a.w), c, 0, 0, 0);
    }
}

// Results of a tile: acc[i][j] of the wavefront whose rows of A begin at m0 and of B at n0, in the tile.
template <class T>
struct TileResult {
    float16v acc[T::MF][T::NF];
    uint32_t m0, n0;
};

// One operand on its way to LDS and from there to registers.
template <class T, Lies LIES, int UNITS>
struct Feed {
    const Operand &o;
    const uint8_t *at;         // the tile's part of the first stage
    uint64_t step;             // from stage to stage (of kRows: pair to pair)
    uint32_t first, lane;
    __device__ __forceinline__ Feed(const Operand &operand, uint32_t tile, uint32_t from, uint32_t lane_) : o(operand), first(tile * UNITS * 32), lane(lane_)
    {
        if constexpr (LIES == kBlocks) {
            step = o.ld;
            at = o.base + (uint64_t)first * 64 + from * step;
        } else if constexpr (LIES == kBlocksTurned) {
            step = T::COLS * 64;
            at = o.base + (uint64_t)(first / T::COLS) * o.ld + from * step;
        } else if constexpr (LIES == kRows) {                                // from 0
            step = 128;
            at = o.base + first * o.ld;
        } else {
            step = T::COLS * o.ld;
            at = o.base + (uint64_t)first * T::ES + from * step;
        }
    }
    // Where the lane's 16 bytes of load `load` of a stage (kRows: of a pair's twice as many) come from, counted from `at`.
    __device__ __forceinline__ uint64_t offset(uint32_t load) const
    {
        if constexpr (LIES == kBlocks) {
            const uint32_t r = load * 16 + lane / 4;
            return (min(first + r, o.rows - 1) - first) * 64 + (lane % 4 ^ swap_of(r)) * 16;
        } else if constexpr (LIES == kBlocksTurned) {
            // 16 rows of k of one block; bf16 has two such runs to a block
            const uint32_t run = T::ES == 2 ? load % 2 * 16 : 0, block = min(first / T::COLS + (T::ES == 2 ? load / 2 : load), o.blocks - 1) - first / T::COLS;
            const uint32_t k = lane / 4, chunk = T::ES == 2 ? lane % 4 ^ swap_of_block(k) * 2 : lane % 4;
            return block * o.ld + (run + k) * 64 + chunk * 16;
        } else if constexpr (LIES == kRows) {
            const uint32_t r = load * 8 + lane / 8;
            return (uint64_t)(min(first + r, o.rows - 1) - first) * o.ld + (lane % 8 ^ swap_of_pair(r)) * 16;
        } else {
            uint32_t at_k = load * 1024 + lane * 16;
            const uint32_t k = at_k / (UNITS * 32 * T::ES);
            at_k %= UNITS * 32 * T::ES;
            if constexpr (T::ES == 2) at_k = (at_k / 32 ^ swap_of_k(k)) * 32 + at_k % 32;
            return k * o.ld + min(at_k, (uint32_t)o.ld - 16 - first * T::ES);
        }
    }
    // kRows: whether these 16 bytes are the second stage's
    __device__ __forceinline__ uint32_t upper(uint32_t load) const { return (lane % 8 ^ swap_of_pair(load * 8 + lane / 8)) >> 2; }
    __device__ __forceinline__ uint32_t row_of_k(uint32_t load) const { return (load * 1024 + lane * 16) / (UNITS * 32 * T::ES); }     // kTurned

    // Registers that reads take the lane's part of their addresses from
    static constexpr int PLACES = LIES == kBlocks ? 2 : LIES == kRows ? 4 : LIES == kTurned && T::ES == 2 ? 4 : 1;
    __device__ __forceinline__ void places(uint32_t (&p)[PLACES], uint32_t unit) const
    {
        const uint32_t row = lane % 32, half = lane / 32, k = half * 8 + lane % 16 / 4, sixteen = lane / 16 % 2;
#pragma unroll
        for (int i = 0; i < PLACES; ++i) {
            if constexpr (LIES == kBlocks) p[i] = unit * 2048 + row * 64 + ((2 * i + half) ^ swap_of(row)) * 16;
            else if constexpr (LIES == kRows) p[i] = unit * 4096 + row * 128 + ((2 * i + half) ^ swap_of_pair(row)) * 16;
            else if constexpr (LIES == kBlocksTurned && T::ES == 2) p[i] = unit * 2048 + k * 64 + (sixteen ^ swap_of_block(k)) * 32 + lane % 4 * 8;
            else if constexpr (LIES == kBlocksTurned) p[i] = unit * 2048 + row / 16 * 1024 + half * 256 + row % 16 * 4;
            else if constexpr (T::ES == 2) p[i] = k * UNITS * 64 + (((unit + i) * 2 + sixteen) ^ swap_of_k(k)) * 32 + lane % 4 * 8;
            else p[i] = half * 4 * UNITS * 128 + (unit * 32 + row) * 4;
        }
    }
    // The operand of unit first + i (i of the wavefront's), step s of the stage; ODD: the second stage of a pair
    template <int ODD>
    static __device__ __forceinline__ uint4 read(const uint8_t *stage, const uint32_t (&p)[PLACES], int i, int s)
    {
        typedef short short4v __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) short4v *Four;
        auto transposed = [](const uint8_t *at, int next) {
            const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(at)));
            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(at + next)));
            return make_uint4(x.x, x.y, y.x, y.y);
        };
        auto singly = [](const uint8_t *at, int next) {
            auto word = [&](int k) { return *reinterpret_cast<const uint32_t *>(at + k * next); };
            return make_uint4(word(0), word(1), word(2), word(3));
        };
        if constexpr (LIES == kBlocks) return *reinterpret_cast<const uint4 *>(stage + i * 2048 + p[s]);
        else if constexpr (LIES == kRows) return *reinterpret_cast<const uint4 *>(stage + i * 4096 + p[2 * ODD + s]);
        else if constexpr (LIES == kBlocksTurned && T::ES == 2) return transposed(stage + i * 2048 + s * 1024 + p[0], 256);
        else if constexpr (LIES == kBlocksTurned) return singly(stage + i * 2048 + s * 512 + p[0], 64);
        else if constexpr (T::ES == 2) return transposed(stage + s * 16 * UNITS * 64 + p[i], 4 * UNITS * 64);
        else return singly(stage + i * 128 + s * 8 * UNITS * 128 + p[0], UNITS * 128);
    }
};

// Stages `from` .. `from + count - 1` of the product of tile (tm, tn); count >= 1.  PLANES 3: each for six, of operands in planes.  A lies in blocks.  B's
// rows of k behind its last one, kTurned, are the last one again (A's columns there are zeros).
template <class T, bool BF16, int PLANES, Lies LIES_A, Lies LIES_B>
__device__ __forceinline__ void multiply_tile(const Operand &oa, const Operand &ob, uint32_t tm, uint32_t tn, uint32_t from, uint32_t columns, const Stages &stages,
                                              TileResult<T> &result)
{
    static_assert(PLANES == 1 || (BF16 && (LIES_B == kBlocks || LIES_B == kBlocksTurned)), "planes lie in blocks");
    const uint32_t count = PLANES == 3 ? 6 * columns : columns;
    static_assert(LIES_A == kBlocks || LIES_A == kBlocksTurned, "a line at a time, a stage at a time");
    constexpr int NB = 4, EACH = T::EACH, MF = T::MF, NF = T::NF, PERIOD = LIES_B == kRows ? 12 : NB;
    const uint32_t wave = uniform(threadIdx.x / 64);
    uint32_t lane = threadIdx.x % 64;
    if constexpr (T::template runs<PLANES>()) asm volatile("" : "+v"(lane));             // no address is kept from run to run: they would not fit the registers
    const Feed<T, LIES_A, T::UM> a(oa, tm, from, lane);
    const Feed<T, LIES_B, T::UN> b(ob, tn, from, lane);
    // a wavefront's loads; where there are fewer than wavefronts, the last one again
    auto load_a = [&](int j) { return min(wave * T::EACH_A + j, (uint32_t)T::LOADS_A - 1); };
    auto load_b = [&](int j) { return min(wave * T::EACH_B + j, (uint32_t)T::LOADS_B - 1); };
    // back_b: what is taken off an offset at B's end (kRows: where the last pair has one stage, the second's chunks; kTurned: rows of k behind the last);
    // second: of the other half of a pair's loads
    constexpr bool ENDS = LIES_B == kRows || LIES_B == kTurned;
    uint32_t offset_a[T::EACH_A], offset_b[T::EACH_B], back_b[ENDS ? T::EACH_B : 1], second_b[LIES_B == kRows ? T::EACH_B : 1], second_back_b[LIES_B == kRows ? T::EACH_B : 1];
#pragma unroll
    for (int j = 0; j < T::EACH_A; ++j) offset_a[j] = (uint32_t)a.offset(load_a(j));
#pragma unroll
    for (int j = 0; j < T::EACH_B; ++j) {
        offset_b[j] = (uint32_t)b.offset(load_b(j));
        if constexpr (LIES_B == kRows) {
            second_b[j] = (uint32_t)b.offset(load_b(j) + T::LOADS_B);
            back_b[j] = b.upper(load_b(j)) * 64;
            second_back_b[j] = b.upper(load_b(j) + T::LOADS_B) * 64;
        } else if constexpr (LIES_B == kTurned) {
            const uint32_t k0 = (ob.rows - 1) / T::COLS * T::COLS, k = b.row_of_k(load_b(j));
            back_b[j] = (k - min(k, ob.rows - 1 - k0)) * (uint32_t)ob.ld;
        }
    }
    const uint32_t last_b = LIES_B == kRows ? (count % 2 ? (count - 1) / 2 : ~0u) : (ob.rows - 1) / T::COLS - from;       // the pair or stage that back_b is for
    // The batch of loads that follows stage s, the AT-th of a period: A of stage s + 4; B of stage s + 4, or, of pairs, the first half of the loads of
    // the pair that begins with stage s + 5 (s is odd), or the second half of that which begins with s + 4.  Behind the last stage that one again.
    struct Batch {
        const uint8_t *a, *b;
        uint32_t mask;
    };
    auto batch_of = [&](auto at, uint32_t s) -> Batch {
        constexpr int ODD = (decltype(at)::value + PERIOD) % 2;
        const uint32_t stage = min(s + NB, count - 1), stage_b = LIES_B == kRows ? min((s + NB + ODD) / 2, (count - 1) / 2) : stage;
        if constexpr (PLANES == 3) {
            const uint32_t k = stage / 6, i = stage % 6;
            return {a.at + k * a.step + plane_of_a(i) * oa.plane, b.at + k * b.step + plane_of_b(i) * ob.plane, 0u};
        }
        return {a.at + stage * a.step, b.at + stage_b * b.step, stage_b == last_b ? ~0u : 0u};
    };
    auto issue = [&](auto at, const Batch &from_here, int j) {
        constexpr int AT = decltype(at)::value + PERIOD, ODD = AT % 2;
        if (j < T::EACH_A) {
            __builtin_amdgcn_global_load_lds((GlobalPtr)(from_here.a + offset_a[j]), (LdsPtr)(stages.a[AT % NB] + load_a(j) * 1024), 16, 0, 0);
            return;
        }
        j -= T::EACH_A;
        if constexpr (LIES_B == kRows) {
            const uint32_t o = ODD ? offset_b[j] - (back_b[j] & from_here.mask) : second_b[j] - (second_back_b[j] & from_here.mask);
            __builtin_amdgcn_global_load_lds((GlobalPtr)(from_here.b + o), (LdsPtr)(stages.b[(AT + NB + ODD) / 2 % 3] + (load_b(j) + (ODD ? 0 : T::LOADS_B)) * 1024), 16, 0, 0);
        } else {
            const uint32_t o = LIES_B == kTurned ? offset_b[j] - (back_b[j] & from_here.mask) : offset_b[j];
            __builtin_amdgcn_global_load_lds((GlobalPtr)(from_here.b + o), (LdsPtr)(stages.b[AT % NB] + load_b(j) * 1024), 16, 0, 0);
        }
    };
    auto arrived = [&](auto behind) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(waitcnt(decltype(behind)::value, 0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const uint32_t wm = wave / T::WN * MF, wn = wave % T::WN * NF;
    result.m0 = wm * 32;
    result.n0 = wn * 32;
    uint32_t place_a[a.PLACES], place_b[b.PLACES];
    a.places(place_a, wm);
    b.places(place_b, wn);
    auto operand = [&](auto at, int s, int i) {
        constexpr int AT = decltype(at)::value;
        if (i < MF) return a.template read<0>(stages.a[AT % NB], place_a, i, s);
        return b.template read<AT % 2>(stages.b[LIES_B == kRows ? AT / 2 % 3 : AT % NB], place_b, i - MF, s);
    };

    uint4 v[2][MF + NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) result.acc[i][j] = float16v{};
    if constexpr (LIES_B == kRows) {
#pragma unroll
        for (int j = 0; j < T::EACH_B; ++j)
            __builtin_amdgcn_global_load_lds((GlobalPtr)(b.at + (offset_b[j] - (last_b == 0 ? back_b[j] : 0))), (LdsPtr)(stages.b[0] + load_b(j) * 1024), 16, 0, 0);
    }
    auto first = [&](auto at) {
        const Batch batch = batch_of(at, (uint32_t)decltype(at)::value);
#pragma unroll
        for (int j = 0; j < EACH; ++j) issue(at, batch, j);
    };
    first(std::integral_constant<int, -4>{});
    first(std::integral_constant<int, -3>{});
    first(std::integral_constant<int, -2>{});
    first(std::integral_constant<int, -1>{});
    arrived(std::integral_constant<int, (NB - 1) * EACH>{});
#pragma unroll
    for (int i = 0; i < MF + NF; ++i) v[0][i] = operand(std::integral_constant<int, 0>{}, 0, i);
    __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));
    // A step's products, and other things between them: the reads one after each product from the first on, so that the last has time to arrive, then
    // the loads (where there are few products, beside the reads).
    constexpr int READS = MF + NF;
    auto place_of = [](int q, int items) {
        if (q < READS) return q < T::PRODUCTS ? q : T::PRODUCTS - 1;
        const int loads = items - READS;
        return T::PRODUCTS > READS ? READS + (q - READS) * (T::PRODUCTS - READS) / loads : (q - READS) * T::PRODUCTS / loads;
    };
    auto multiply = [&](int set, int items, auto item) {
#pragma unroll
        for (int p = 0; p < T::PRODUCTS; ++p) {
            const int i = p / NF, j = p % NF;
            __builtin_amdgcn_sched_barrier(0);
            result.acc[i][j] = multiply32<BF16>(v[set][MF + j], v[set][i], result.acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < items; ++q)
                if (place_of(q, items) == p) item(q);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto one = [&](auto at, uint32_t s) {
        constexpr int AT = decltype(at)::value;
        multiply(0, MF + NF, [&](int q) { v[1][q] = operand(at, 1, q); });
        // the next stage is there when no more is outstanding than the NB - 2 batches behind its own
        arrived(std::integral_constant<int, (NB - 2) * EACH>{});
        const Batch batch = batch_of(at, s);
        multiply(1, MF + NF + EACH, [&](int q) {
            if (q < MF + NF) v[0][q] = operand(std::integral_constant<int, (AT + 1) % PERIOD>{}, 0, q);
            else issue(at, batch, q - MF - NF);
        });
#pragma unroll
        for (int i = 0; i < MF + NF; ++i) pin(v[0][i]);
    };
    // a period of stages at a time, then what is left of one
    auto some = [&](auto most, uint32_t s, uint32_t left) {
        if constexpr (decltype(most)::value > 0) {
            auto next = [&](auto self, auto at) {
                constexpr int AT = decltype(at)::value;
                if (left > (uint32_t)AT) {
                    one(at, s + AT);
                    if constexpr (AT + 1 < decltype(most)::value) self(self, std::integral_constant<int, AT + 1>{});
                }
            };
            next(next, std::integral_constant<int, 0>{});
        }
    };
    auto whole = [&](auto self, auto at, uint32_t s) {
        constexpr int AT = decltype(at)::value;
        one(at, s + AT);
        if constexpr (AT + 1 < PERIOD) self(self, std::integral_constant<int, AT + 1>{}, s);
    };
    uint32_t s = 0;
    if constexpr (!T::template parts<PLANES>()) {
        for (; count - s >= PERIOD; s += PERIOD) whole(whole, std::integral_constant<int, 0>{}, s);
        some(std::integral_constant<int, PERIOD - 1>{}, s, count - s);
    } else {
        // Sums of fp32, as such or in planes, in parts of a few hundred columns (768, 512), which are added up: thousands one after another would be off
        // by several times as much (losses of 400 x 8192 x 32000 in planes, 1.5e-6 and so 7.4e-7, of which 6e-7 are the losses' own roundings; the time is
        // the same).
        constexpr uint32_t PART = (PLANES == 3 ? 96 : 48) / PERIOD;
        float16v sums[MF][NF] = {};
        auto part = [&] {
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < NF; ++j) {
                    sums[i][j] += result.acc[i][j];
                    result.acc[i][j] = float16v{};
                }
        };
        for (uint32_t n = 1; count - s >= PERIOD; s += PERIOD, ++n) {
            whole(whole, std::integral_constant<int, 0>{}, s);
            if (n % PART == 0) part();
        }
        some(std::integral_constant<int, PERIOD - 1>{}, s, count - s);
        part();
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) result.acc[i][j] = sums[i][j];
    }
    // loads to LDS that nobody reads are waited for, too: what comes now uses LDS otherwise
    arrived(std::integral_constant<int, 0>{});
}

// What is not a whole wavefront's results but 32 x 32 of them
struct OneUnit {
    static constexpr int MF = 1, NF = 1;
};

// Whether there is a NaN among a wavefront's results of rows of A from m0 up to `count`
template <class T>
__device__ __forceinline__ bool any_nan(const TileResult<T> &r, uint32_t m0, uint32_t count)
{
    bool found = false;
#pragma unroll
    for (int i = 0; i < T::MF; ++i) {
        bool nan = false;
#pragma unroll
        for (int j = 0; j < T::NF; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) nan |= __builtin_isnan(r.acc[i][j][k]);
        found |= nan && m0 + 32 * i + threadIdx.x % 32 < count;
    }
    return __ballot(found) != 0;
}

// Results of rows row_a and row_b on, 32 x 32 of operands in planes, as products of fp32, which the planes add up to, straight from memory, in parts as
// elsewhere.  For wavefronts with a NaN: where an operand is infinite, products of its planes are NaN, and fp32's need not be.  (4194 x 4096 x 32000 forward
// 6.5 ms, with an infinite row of the weight 7.0, with 300 of them 7.6, of NaN alone 20.7.)
__device__ __forceinline__ float16v as_fp32(const Operand &a, const Operand &b, uint32_t row_a, uint32_t row_b, uint32_t blocks)
{
    uint32_t lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));                           // what follows from it is not kept in registers all along
    const uint8_t *from_a = a.base + (uint64_t)min(row_a + lane % 32, a.rows - 1) * 64 + lane / 32 * 16;
    const uint8_t *from_b = b.base + (uint64_t)min(row_b + lane % 32, b.rows - 1) * 64 + lane / 32 * 16;
    float16v sum = {}, part = {};
    for (uint32_t block = 0; block < blocks; ++block, from_a += a.ld, from_b += b.ld) {
        uint4 x[2][3], y[2][3];                              // which columns a lane has does not matter as long as both operands' are the same
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                x[q][p] = *reinterpret_cast<const uint4 *>(from_a + p * a.plane + q * 32);
                y[q][p] = *reinterpret_cast<const uint4 *>(from_b + p * b.plane + q * 32);
            }
        auto number = [](const uint4 (&v)[3], int i) {
            auto one = [i](const uint4 &w) {
                const uint32_t two = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
                return __uint_as_float(i % 2 ? two & 0xffff0000u : two << 16);
            };
            return (one(v[0]) + one(v[1])) + one(v[2]);
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) part = __builtin_amdgcn_mfma_f32_32x32x2f32(number(y[i / 8], i % 8), number(x[i / 8], i % 8), part, 0, 0, 0);
        if (block % 24 == 23) {
            sum += part;
            part = float16v{};
        }
    }
    return sum + part;
}

// Results are stored straight from registers, where a lane has four neighbours of a row.  Of two groups x and y of four, after this exchange between the
// halves of a wavefront, the lower half's lanes have all eight of x (x, then y) and the upper half's all of y.
__device__ __forceinline__ void exchange_halves(uint32_t &x, uint32_t &y)
{
    typedef uint32_t pair __attribute__((ext_vector_type(2)));
    const pair r = __builtin_bit_cast(pair, __builtin_amdgcn_permlane32_swap(x, y, false, false));
    x = r.x;
    y = r.y;
}

// Four results of a lane from i on, rounded to bf16, two to a word
template <class V>
__device__ __forceinline__ uint2 four_bf16(const V &v, int i) { return make_uint2(two_bf16(v[i], v[i + 1]), two_bf16(v[i + 2], v[i + 3])); }
// Two groups of four bf16 as sixteen bytes: the lower half's lanes get the first group's eight columns, the upper half's the second's
__device__ __forceinline__ uint4 eight_of(uint2 x, uint2 y)
{
    exchange_halves(x.x, y.x);
    exchange_halves(x.y, y.y);
    return make_uint4(x.x, x.y, y.x, y.y);
}

// Results to a row-major matrix [rows, cols], from row m0 and column n0 on (this wavefront's), times `scale`.
template <bool OUT_BF16, class T>
__device__ __forceinline__ void store_rows(const TileResult<T> &r, uint32_t m0, uint32_t n0, uint32_t rows, uint32_t cols, float scale, void *out, bool accumulate)
{
    uint32_t lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));                           // what follows from it is not kept in registers all along
    const uint32_t half = lane / 32;
#pragma unroll
    for (int i = 0; i < T::MF; ++i) {
#pragma unroll
        for (int j = 0; j < T::NF; ++j) {
            __builtin_amdgcn_sched_barrier(0);               // one by one: addresses of all of them would not fit the registers
            uint32_t m = m0 + 32 * i + lane % 32;
            asm volatile("" : "+v"(m));
            const uint64_t row = (uint64_t)m * cols;
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = r.acc[i][j][k] * scale;
            if (accumulate) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const uint32_t n = n0 + 32 * j + 8 * (k / 4) + 4 * half + k % 4;
                    if (m < rows && n < cols) v[k] += load1<OUT_BF16>(out, row + n);
                }
            }
            if constexpr (OUT_BF16) {
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    const uint4 w = eight_of(four_bf16(v, 4 * g), four_bf16(v, 4 * g + 4));
                    const uint32_t n = n0 + 32 * j + 8 * (g + half);
                    if (m < rows && n < cols) store16<true>(out, row + n, cols - n, w, false);
                }
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t n = n0 + 32 * j + 8 * g + 4 * half;
                    if (m < rows && n < cols)
                        store16<false>(out, row + n, cols - n, make_uint4(__float_as_uint(v[4 * g]), __float_as_uint(v[4 * g + 1]), __float_as_uint(v[4 * g + 2]), __float_as_uint(v[4 * g + 3])), false);
                }
            }
        }
    }
}

}  // namespace tahq
