// Products of bf16 or fp32 matrices on the matrix cores, tile by tile, for the loss over a vocabulary (include/tahq_loss.h).
#pragma once
#include <type_traits>

#include "tahq_mx4_common.hpp"
#include "tahq_tiles.hpp"

namespace tahq {

// Columns of a stage: 64 bytes of every row.
template <bool BF16>
constexpr int kStageCols = BF16 ? 32 : 16;

// One operand of a product, C[m, n] = sum over k of A[m, k] B[n, k], as a workgroup's tile takes it from memory.
//   TURNED 0: rows of k are contiguous, [m][k].  1: the matrix lies the other way, [k][m].
struct Operand {
    const uint8_t *base;       // the matrix
    uint64_t ld;               // bytes from one row in memory to the next
    uint32_t rows;             // of the operand, m
    uint32_t depth;            // TURNED: rows in memory, k, that may be read
};

// The tile of a workgroup: WM * MF units of 32 rows of A by WN * NF units of B; its four wavefronts take MF x NF units each.  A stage is
// 64 bytes of every row (32 columns of bf16, 16 of fp32); four of them are in LDS, one in use, three on their way (loads straight to LDS).
//   What lies in LDS: a row's 64 bytes as four chunks of 16, or, turned, a row of k with the tile's rows side by side.  Loads write LDS in a
// row; which 16 bytes a lane loads is chosen so that the operands' reads meet no bank twice:
//   rows       chunk c of row r is at place c ^ swap(r): eight neighbouring rows' equal chunks fill the 32 banks, sixteen all 64
//   turned     bf16: 32 bytes (16 rows) number c of k are at place c ^ swap_k(k): four rows of k are read at a time, transposed on the way
//   to registers (ds_read_b64_tr_b16: sixteen lanes address 4 x 16 elements and each gets a column).  fp32: one number at a time.
//   Order of work as in the mx4 products: operands of a step (two to a stage) are read while the step before is multiplied; at the last step of
// a stage all wavefronts have the operands in registers, the next stage's loads are waited for, and the stage just read is loaded over.
template <bool BF16, int WM_, int WN_, int MF_, int NF_>
struct TileKind_ {
    static constexpr int WM = WM_, WN = WN_, MF = MF_, NF = NF_, W = WM * WN, UM = WM * MF, UN = WN * NF, ROWS = UM + UN;
    static constexpr int STAGE = ROWS * 2048, LOADS = 2 * ROWS, EACH = (LOADS + W - 1) / W, PRODUCTS = MF * NF;
    static constexpr int COLS = kStageCols<BF16>, ES = BF16 ? 2 : 4;
    static_assert(W == 4, "four wavefronts");
};

__device__ __forceinline__ uint32_t swap_of(uint32_t row) { return (row >> 2 & 1) << 1 | ((row >> 1 ^ row >> 3) & 1); }
__device__ __forceinline__ uint32_t swap_of_k(uint32_t k) { return (k & 3) | (k & 1) << 2; }

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

// Results of a tile: acc[i][j] of wavefront (wm, wn), its units of A from wm on and of B from wn on.
template <class T>
struct TileResult {
    float16v acc[T::MF][T::NF];
    uint32_t m0, n0;           // first row of A and of B that this wavefront has, in the tile
};

// Where 16 bytes of an operand's stage come from: the lane's offset from the tile's first row (or, turned, column) at the stage's first column
template <class T, bool TURNED>
__device__ __forceinline__ uint32_t lane_offset(const Operand &o, uint32_t first, uint32_t units, uint32_t load, uint32_t &k)
{
    const uint32_t lane = threadIdx.x % 64;
    k = 0;
    if constexpr (!TURNED) {
        const uint32_t r = load * 16 + lane / 4, row = min(first + r, o.rows - 1) - first;
        return row * (uint32_t)o.ld + ((lane % 4) ^ swap_of(r)) * 16;
    } else {
        const uint32_t wide = units * 32 * T::ES, byte = load * 1024 + lane * 16;
        k = byte / wide;
        uint32_t at = byte % wide;
        if constexpr (T::ES == 2) at = ((at / 32) ^ swap_of_k(k)) * 32 + at % 32;
        return k * (uint32_t)o.ld + min(at, (uint32_t)o.ld - 16 - first * T::ES);
    }
}

// Stages `from` .. `from + count - 1` of the product of tile (tm, tn); count >= 1.  `stages`: LDS.
// CLAMP: B's rows of k behind its depth are the last one again (A's columns there are zeros).
template <class T, bool BF16, bool TA, bool TB, bool CLAMP>
__device__ __forceinline__ void multiply_tile(const Operand &a, const Operand &b, uint32_t tm, uint32_t tn, uint32_t from, uint32_t count,
                                              uint8_t *const (&stages)[4], TileResult<T> &result)
{
    constexpr int NB = 4, EACH = T::EACH, MF = T::MF, NF = T::NF;
    static_assert(!CLAMP || TB, "rows of k in memory");
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
    const uint32_t first_a = tm * T::UM * 32, first_b = tn * T::UN * 32;
    const uint64_t step_a = TA ? T::COLS * a.ld : 64, step_b = TB ? T::COLS * b.ld : 64;
    const uint8_t *const at_a = a.base + (TA ? (uint64_t)first_a * T::ES : first_a * a.ld) + from * step_a;
    const uint8_t *const at_b = b.base + (TB ? (uint64_t)first_b * T::ES : first_b * b.ld) + from * step_b;
    uint32_t offset[EACH], row_k[EACH];
    auto is_a = [&](int j) { return wave * EACH + j < 2 * T::UM; };
    auto load_of = [&](int j) { return min(wave * EACH + j, (uint32_t)T::LOADS - 1); };
#pragma unroll
    for (int j = 0; j < EACH; ++j)
        offset[j] = is_a(j) ? lane_offset<T, TA>(a, first_a, T::UM, load_of(j), row_k[j]) : lane_offset<T, TB>(b, first_b, T::UN, load_of(j) - 2 * T::UM, row_k[j]);
    // load j of stage s, into the `at`-th of the stages in LDS; behind the last stage that one again
    auto issue = [&](int at, uint32_t s, int j) {
        const uint32_t stage = min(s, count - 1);
        const uint8_t *p = is_a(j) ? at_a + stage * step_a : at_b + stage * step_b;
        uint32_t o = offset[j];
        if constexpr (CLAMP) {
            const uint32_t k0 = (from + stage) * T::COLS;                    // below the depth, as every stage has a row at least
            if (!is_a(j) && k0 + T::COLS > b.depth) o -= (row_k[j] - min(row_k[j], b.depth - 1 - k0)) * (uint32_t)b.ld;
        }
        __builtin_amdgcn_global_load_lds((GlobalPtr)(p + o), (LdsPtr)(stages[at % NB] + load_of(j) * 1024), 16, 0, 0);
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
    // this lane's part of an operand's address
    uint32_t plain[2], turned_a[MF], turned_b[NF];
#pragma unroll
    for (int s = 0; s < 2; ++s) plain[s] = lane % 32 * 64 + ((2 * s + lane / 32) ^ swap_of(lane % 32)) * 16;
    auto turned_offset = [&](uint32_t unit, uint32_t units) -> uint32_t {
        if constexpr (BF16) {
            const uint32_t k = lane / 32 * 8 + lane % 16 / 4;
            return k * units * 64 + ((unit * 2 + lane / 16 % 2) ^ swap_of_k(k)) * 32 + lane % 4 * 8;
        } else {
            return lane / 32 * 4 * units * 128 + (unit * 32 + lane % 32) * 4;
        }
    };
#pragma unroll
    for (int i = 0; i < MF; ++i) turned_a[i] = TA ? turned_offset(wm + i, T::UM) : 0;
#pragma unroll
    for (int i = 0; i < NF; ++i) turned_b[i] = TB ? turned_offset(wn + i, T::UN) : 0;
    auto read = [&](auto turned, const uint8_t *image, uint32_t unit, uint32_t offset_turned, uint32_t units, int s) {
        uint4 v;
        if constexpr (!decltype(turned)::value) {
            v = *reinterpret_cast<const uint4 *>(image + unit * 2048 + plain[s]);
        } else if constexpr (BF16) {
            typedef short short4v __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) short4v *Four;
            const uint8_t *p = image + offset_turned + s * 16 * units * 64;
            const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(p)));
            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(p + 4 * units * 64)));
            v = make_uint4(x.x, x.y, y.x, y.y);
        } else {
            const uint8_t *p = image + offset_turned + s * 8 * units * 128;
            v.x = *reinterpret_cast<const uint32_t *>(p);
            v.y = *reinterpret_cast<const uint32_t *>(p + units * 128);
            v.z = *reinterpret_cast<const uint32_t *>(p + 2 * units * 128);
            v.w = *reinterpret_cast<const uint32_t *>(p + 3 * units * 128);
        }
        return v;
    };
    auto operand = [&](const uint8_t *stage, int s, int i) {
        if (i < MF) return read(std::bool_constant<TA>{}, stage, wm + i, turned_a[i < MF ? i : 0], T::UM, s);
        return read(std::bool_constant<TB>{}, stage + T::UM * 2048, wn + i - MF, turned_b[i < MF ? 0 : i - MF], T::UN, s);
    };

    uint4 v[2][MF + NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) result.acc[i][j] = float16v{};
#pragma unroll
    for (int at = 0; at < NB; ++at)
#pragma unroll
        for (int j = 0; j < EACH; ++j) issue(at, at, j);
    arrived(std::integral_constant<int, (NB - 1) * EACH>{});
#pragma unroll
    for (int i = 0; i < MF + NF; ++i) v[0][i] = operand(stages[0], 0, i);
    __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));
    auto multiply = [&](int set, int items, auto item) {
#pragma unroll
        for (int p = 0; p < T::PRODUCTS; ++p) {
            const int i = p / NF, j = p % NF;
            __builtin_amdgcn_sched_barrier(0);
            result.acc[i][j] = multiply32<BF16>(v[set][MF + j], v[set][i], result.acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < items; ++q)
                if (q * T::PRODUCTS / items == p) item(q);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto one = [&](auto at, uint32_t s) {
        constexpr int AT = decltype(at)::value;
        multiply(0, MF + NF, [&](int q) { v[1][q] = operand(stages[AT % NB], 1, q); });
        // the next stage is there when no more is outstanding than the NB - 2 stages behind it
        arrived(std::integral_constant<int, (NB - 2) * EACH>{});
        multiply(1, MF + NF + EACH, [&](int q) {
            if (q < MF + NF) v[0][q] = operand(stages[(AT + 1) % NB], 0, q);
            else issue(AT, s + NB, q - MF - NF);
        });
#pragma unroll
        for (int i = 0; i < MF + NF; ++i) pin(v[0][i]);
    };
    uint32_t s = 0, left = count;
    for (; left >= NB; left -= NB, s += NB) {
        one(std::integral_constant<int, 0>{}, s);
        one(std::integral_constant<int, 1>{}, s + 1);
        one(std::integral_constant<int, 2>{}, s + 2);
        one(std::integral_constant<int, 3>{}, s + 3);
    }
    if (left > 0) one(std::integral_constant<int, 0>{}, s);
    if (left > 1) one(std::integral_constant<int, 1>{}, s + 1);
    if (left > 2) one(std::integral_constant<int, 2>{}, s + 2);
    // loads to LDS that nobody reads are waited for, too: what comes now uses LDS otherwise
    arrived(std::integral_constant<int, 0>{});
}

// A wavefront's results to rows in memory, through LDS of its own, so that they are written a line at a time.  value(i, j, k): unit of A, of B, and
// which of the lane's sixteen numbers; put(m, n, valid, x[4]): four neighbours, n .. n + 3 of row m, counted in the tile.
template <class T, class Value, class Put>
__device__ __forceinline__ void store_tile(const TileResult<T> &r, uint8_t *const (&stages)[4], Value value, Put put)
{
    constexpr int WIDE = T::NF * 32 * 4, STRIDE = WIDE + 16, LANES = WIDE / 16;          // 16 bytes more: rows start in other banks
    static_assert(32 * STRIDE <= T::STAGE, "a wavefront's rows fit");
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
    uint8_t *const mine = wave == 0 ? stages[0] : wave == 1 ? stages[1] : wave == 2 ? stages[2] : stages[3];
#pragma unroll
    for (int i = 0; i < T::MF; ++i) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < T::NF; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float4 x;
                x.x = value(i, j, 4 * g);
                x.y = value(i, j, 4 * g + 1);
                x.z = value(i, j, 4 * g + 2);
                x.w = value(i, j, 4 * g + 3);
                *reinterpret_cast<float4 *>(mine + lane % 32 * STRIDE + (32 * j + 8 * g + lane / 32 * 4) * 4) = x;
            }
        asm volatile("" ::: "memory");                       // this wavefront's own rows: LDS keeps its accesses in order
#pragma unroll
        for (int k = 0; k < LANES / 2; ++k) {
            const uint32_t row = k * (64 / LANES) + lane / LANES;
            const float4 x = *reinterpret_cast<const float4 *>(mine + row * STRIDE + lane % LANES * 16);
            const float y[4] = {x.x, x.y, x.z, x.w};
            put(r.m0 + i * 32 + row, r.n0 + lane % LANES * 4, y);
        }
        asm volatile("" ::: "memory");
    }
}

}  // namespace tahq
