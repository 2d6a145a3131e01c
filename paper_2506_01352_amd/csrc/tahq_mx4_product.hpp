// C = A B^T of two packed mx4 matrices on the matrix cores (v_mfma_scale_f32_32x32x64_f8f6f4, 4-bit operands, fp32 sums).
#pragma once
#include <type_traits>

#include "tahq_mx4_common.hpp"

namespace tahq {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

// One instruction: 32 rows of each operand, 64 columns.  A lane holds row lane % 32 of both operands, columns 32 * (lane / 32) on,
// and of D column lane % 32 (second operand's row), rows 8 * (i / 4) + 4 * (lane / 32) + i % 4 (first operand's).  B goes first, so that a lane's
// results are four neighbours of a row of C.  BYTE: which of the four scale bytes.
template <int BYTE>
__device__ __forceinline__ float16v mfma(const uint4 &b, const uint4 &a, const float16v &c, uint32_t sb, uint32_t sa)
{
    const int8v vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    const int8v va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vb, va, c, 4, 4, BYTE, (int)sb, BYTE, (int)sa);
}

// Four neighbours of a row of C: row m, columns n .. n + 3
template <bool BF16>
__device__ __forceinline__ void store4(void *c, uint64_t ldc, uint32_t m, uint32_t n, uint32_t N, float (&v)[4], bool accumulate)
{
    const uint64_t at = (uint64_t)m * ldc + n;
    const bool whole = n + 4 <= N;
    if (accumulate) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (whole || n + i < N) v[i] += load1<BF16>(c, at + i);
    }
    if (whole) {
        if constexpr (BF16) {
            const uint32_t w[2] = {two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
            __builtin_memcpy(static_cast<uint16_t *>(c) + at, w, 8);
        } else {
            __builtin_memcpy(static_cast<float *>(c) + at, v, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) store1<BF16>(c, at + i, v[i]);
    }
}

// ---------------------------------------------------------------- tiles through LDS

// Workgroups go around the eight dies, each with a cache of its own: a die gets neighbouring tiles, in strips of eight rows of tiles.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn)
{
    const uint32_t total = tiles_m * tiles_n, die = id % 8, extra = total % 8;
    id = die * (total / 8) + min(die, extra) + id / 8;
    const uint32_t strip = id / (8 * tiles_n), at = id % (8 * tiles_n), height = min(tiles_m - strip * 8, 8u);
    tm = strip * 8 + at % height;
    tn = at / height;
}

// s_waitcnt's operand: at most `vm` loads and `lgkm` LDS accesses outstanding (no exports are)
constexpr int waitcnt(int vm, int lgkm) { return (vm & 15) | 7 << 4 | lgkm << 8 | (vm >> 4) << 14; }

// what was read is used here: the reads are not moved behind this place
__device__ __forceinline__ void pin(uint4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

// Eight bf16 or four fp32 neighbours of a row of C, of which `valid` are there; fp32 may be added to what is there
template <bool BF16>
__device__ __forceinline__ void store16(void *c, uint64_t at, uint32_t valid, uint4 x, bool accumulate)
{
    constexpr uint32_t COUNT = BF16 ? 8 : 4;
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    if constexpr (!BF16) {
        if (accumulate)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < valid) w[i] = __float_as_uint(__uint_as_float(w[i]) + static_cast<const float *>(c)[at + i]);
    }
    if (valid >= COUNT) {
        __builtin_memcpy(static_cast<uint8_t *>(c) + at * (16 / COUNT), w, 16);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < COUNT; ++i)
            if (i < valid) {
                if constexpr (BF16) static_cast<uint16_t *>(c)[at + i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
                else static_cast<uint32_t *>(c)[at + i] = w[i];
            }
    }
}

// A workgroup's tile is WM * MF units of A's rows by WN * NF of B's; its WM * WN wavefronts take MF x NF units each.  A stage is 128
// columns; four of them are in LDS: one in use, three on their way (loads straight to LDS).  Units keep the order that they have in memory, which
// is the operand's, so that a wavefront reads 1 KB in a row: no bank conflicts, no address arithmetic.  Scales come once in two stages.
//   Operands of a step of 64 columns are read while the step before is multiplied.  At the last step of a stage all wavefronts have the
// operands in registers: there the next stage's loads are waited for (by each wavefront for its own, then the barrier), and the stage just
// read is loaded over.  Reads and loads are spread between the matrix instructions.
//   Columns behind the last unit: the last unit's codes again, with the scales that fill up a group of 256, which are 2^-127 on both sides: the
// products are nothing beside 2^-149, the smallest fp32 number.
//   KS: teams of WM * WN wavefronts that share the tile's columns, each with stages of its own, where there are too few tiles for two to a compute
// unit: one wavefront to a vector unit waits more than it multiplies.
//   OUT: 0 fp32, 1 bf16, 2 fp32 parts of a sum over k in gridDim.y runs of `run` groups of 256 columns.
//   Measured, 256 x 256 tiles: 8192 x 8192 x 8192 257 to 295 us, 4.2 PFLOP/s of the 8.7 that the instruction alone reaches.  Two things are
// lost.  Of 445 k cycles the matrix cores work in 262 k; the others go to starts and ends of four rounds of tiles, about 10 us a round, with nothing
// beside them on a compute unit, and to waits between stages.  And the clock gives way to power: matrices of zeros take as many cycles, but 186
// to 192 us, at 2.35 GHz instead of 1.72.
// Small products wait: 2048 x 1600 x 1600 8.0 us (1.3 PFLOP/s), launch, first loads and last stores being about 4 of them.
template <int WM, int WN, int MF, int NF, int NB, int KS, int PER_CU, int OUT>
__global__ __launch_bounds__(64 * WM * WN * KS, PER_CU * KS)
void k_mx4_tiles(const uint8_t *a, const uint8_t *b, void *c, uint32_t M, uint32_t N, uint32_t K, uint64_t ldc, uint32_t accumulate,
                 uint32_t tiles_m, uint32_t tiles_n, uint32_t run)
{
    constexpr int UM = WM * MF, ROWS = UM + WN * NF, W = WM * WN;        // units of rows of A, of both, in a stage
    constexpr int CODES = ROWS * 2048, SCALES = ROWS * 256;
    constexpr int EACH = ROWS * 2 / W, EACH_S = (ROWS + W - 1) / W, PRODUCTS = MF * NF;
    static_assert(KS == 1 || NB == 4, "teams' scales lie side by side");
    static_assert(ROWS * 2 % W == 0, "the same number of loads in every wavefront");
    // a variable for each stage: the compiler then knows which loads a read has to wait for
    __shared__ __attribute__((aligned(1024))) uint8_t s0[KS * CODES], s1[KS * CODES], s2[KS * CODES], s3[NB == 4 ? KS * CODES : 16];
    __shared__ __attribute__((aligned(256))) uint8_t t0[KS * (NB == 4 ? SCALES : 2 * SCALES)], t1[NB == 4 ? KS * SCALES : 16];
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64 % W), team = KS == 1 ? 0 : uniform(threadIdx.x / 64 / W);
    uint8_t *const codes[4] = {s0, s1, s2, s3};
    // where the scales of the group of 256 columns with stage s are; s is `at` and a multiple of the unrolled stages
    auto scale_words = [&](int at, uint32_t s) { return NB == 4 ? (at / 2 % 2 ? t1 : t0) : t0 + s / 2 % 2 * SCALES; };
    constexpr int TURN = NB == 3 ? 3 : 2;                    // groups of 256 columns that bring the buffers round

    const Mx4Layout LA(M, K), LB(N, K);
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    // groups of 256 columns: a team's first one, how many it has, and how many all of them take their turn for
    const uint32_t in_run = min(run, LA.kc - blockIdx.y * run), groups = (in_run + KS - 1) / KS;
    const uint32_t first = blockIdx.y * run + team * groups, own = in_run > team * groups ? min(groups, in_run - team * groups) : 0;

    // this wavefront's share of a stage; units behind the last row are not there: the last one again, whose results are not stored
    const uint8_t *from[EACH], *from_s[EACH_S];
    auto row_unit = [&](uint32_t i) { return i < UM ? min(tm * UM + i, LA.rb - 1) : min(tn * (WN * NF) + i - UM, LB.rb - 1); };
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const uint32_t i = (wave * EACH + j) / 2;
        from[j] = (i < UM ? a : b) + (uint64_t)row_unit(i) * LA.kb * 1024;
    }
#pragma unroll
    for (int j = 0; j < EACH_S; ++j) {
        const uint32_t i = min(wave * EACH_S + j, (uint32_t)ROWS - 1);
        from_s[j] = (i < UM ? a + LA.scales() : b + LB.scales()) + (uint64_t)row_unit(i) * LA.kc * 256;
    }
    // load j of stage `stage`, the `at`-th of the unrolled ones: codes, then with the first of two stages the scales
    auto issue = [&](int at, uint32_t stage, int j) {
        if (j < EACH) {
            const uint32_t unit = wave * EACH + j, kb = uniform(min(4 * first + 2 * stage + unit % 2, LA.kb - 1));
            __builtin_amdgcn_global_load_lds((GlobalPtr)(from[j] + (uint64_t)kb * 1024 + lane * 16), (LdsPtr)(codes[at % NB] + (team * CODES + unit * 1024)), 16, 0, 0);
        } else {
            const uint32_t unit = min(wave * EACH_S + j - EACH, (uint32_t)ROWS - 1), group = uniform(min(first + stage / 2, LA.kc - 1));
            __builtin_amdgcn_global_load_lds((GlobalPtr)(from_s[j - EACH] + (uint64_t)group * 256 + lane * 4),
                                             (LdsPtr)(scale_words(at, stage) + (team * SCALES + unit * 256)), 4, 0, 0);
        }
    };
    // all wavefronts have the operands that they asked for, and their loads but the last `behind`
    auto arrived = [&](auto behind) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(waitcnt(decltype(behind)::value, 0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    float16v acc[MF][NF] = {};
    uint4 v[2][MF + NF];                                     // operands: A's, then B's
    uint32_t sc[MF + NF], next_sc[MF + NF];
    const uint32_t wm = wave / WN * MF, wn = UM + wave % WN * NF;        // this wavefront's units in a stage
    auto unit_at = [&](int i) { return i < MF ? wm + i : wn + i - MF; };
    auto operand = [&](const uint8_t *s, int kb, int i) { return *reinterpret_cast<const uint4 *>(s + (team * CODES + unit_at(i) * 2048 + kb * 1024 + lane * 16)); };
    auto scale = [&](const uint8_t *s, int i) { return *reinterpret_cast<const uint32_t *>(s + (team * SCALES + unit_at(i) * 256 + lane * 4)); };

#pragma unroll
    for (int at = 0; at < NB; ++at)
#pragma unroll
        for (int j = 0; j < EACH + (at % 2 ? 0 : EACH_S); ++j) issue(at, at, j);
    arrived(std::integral_constant<int, (NB - 1) * EACH + (NB - 1) / 2 * EACH_S>{});
#pragma unroll
    for (int i = 0; i < MF + NF; ++i) {
        sc[i] = KS == 1 || own ? scale(scale_words(0, 0), i) : 0;
        v[0][i] = operand(codes[0], 0, i);
    }
    __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));

    // a step's products, and `items` other things spread between them, in this order
    auto multiply = [&](int set, auto byte, int items, auto item) {
#pragma unroll
        for (int p = 0; p < PRODUCTS; ++p) {
            const int i = p / NF, j = p % NF;
            __builtin_amdgcn_sched_barrier(0);
            acc[i][j] = mfma<decltype(byte)::value>(v[set][MF + j], v[set][i], acc[i][j], sc[MF + j], sc[i]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < items; ++q)
                if (q * PRODUCTS / items == p) item(q);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // stage s, the AT-th of the unrolled ones; ODD: the second of a group of 256 columns
    auto one = [&](auto at, uint32_t s) {
        constexpr int AT = decltype(at)::value, ODD = AT % 2;
        multiply(0, std::integral_constant<int, 2 * ODD>{}, MF + NF, [&](int q) { v[1][q] = operand(codes[AT % NB], 1, q); });
        // the next stage is there when no more is outstanding than the NB - 2 stages behind it, every other one with scales
        arrived(std::integral_constant<int, (NB - 2) * EACH + (NB == 4 || !ODD ? EACH_S : 0)>{});
        constexpr int READS = MF + NF + (ODD ? MF + NF : 0), LOADS = EACH + ((AT + NB) % 2 ? 0 : EACH_S);
        multiply(1, std::integral_constant<int, 2 * ODD + 1>{}, READS + LOADS, [&](int q) {
            if (q < MF + NF) v[0][q] = operand(codes[(AT + 1) % NB], 0, q);
            else if (q < READS) next_sc[q - MF - NF] = scale(scale_words(AT + 1, s + 1), q - MF - NF);
            else issue(AT + NB, s + NB, q - READS);
        });
#pragma unroll
        for (int i = 0; i < MF + NF; ++i) {
            pin(v[0][i]);
            if (ODD) sc[i] = KS == 1 || (s + 1) / 2 < own ? next_sc[i] : 0;
        }
    };
    auto group = [&](auto at, uint32_t s) {
        one(at, s);
        one(std::integral_constant<int, decltype(at)::value + 1>{}, s + 1);
    };
    const std::integral_constant<int, 0> first_group;
    const std::integral_constant<int, 2> second_group;
    // groups of 256 columns; the last one's last stage may be one of zeros
    uint32_t s = 0, left = groups;
    for (; left >= TURN; left -= TURN, s += 2 * TURN) {
        group(first_group, s);
        group(second_group, s + 2);
        if constexpr (TURN == 3) group(std::integral_constant<int, 4>{}, s + 4);
    }
    if (left > 0) group(first_group, s);
    if constexpr (TURN == 3) {
        if (left > 1) group(second_group, s + 2);
    }
    // loads to LDS that nobody reads are waited for, too: the results pass through LDS, so that rows of C are written a line at a time
    arrived(std::integral_constant<int, 0>{});
    if constexpr (KS > 1) {
        // the teams' sums to the first one, which adds them in order: a piece is 16 numbers of every lane of a team
        constexpr int PIECE = W * 4096, EACH_STAGE = KS * CODES / PIECE;
        static_assert(NB == 4 && (KS - 1) * PRODUCTS <= NB * EACH_STAGE, "all pieces fit");
        uint8_t *const stages[4] = {s0, s1, s2, s3};
        auto piece = [&](int from, int p) {
            const int at = (from - 1) * PRODUCTS + p;
            return reinterpret_cast<float4 *>(stages[at / EACH_STAGE] + at % EACH_STAGE * PIECE + wave * 4096) + lane;
        };
#pragma unroll
        for (int from = 1; from < KS; ++from)
            if (team == (uint32_t)from)
#pragma unroll
                for (int p = 0; p < PRODUCTS; ++p)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float16v &x = acc[p / NF][p % NF];
                        piece(from, p)[q * 64] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                    }
        __syncthreads();
        if (team == 0)
#pragma unroll
            for (int from = 1; from < KS; ++from)
#pragma unroll
                for (int p = 0; p < PRODUCTS; ++p)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float4 x = piece(from, p)[q * 64];
                        float16v &to = acc[p / NF][p % NF];
                        to[4 * q] += x.x;
                        to[4 * q + 1] += x.y;
                        to[4 * q + 2] += x.z;
                        to[4 * q + 3] += x.w;
                    }
        __syncthreads();
        if (team != 0) return;
    }
    if constexpr (OUT == 2) c = static_cast<float *>(c) + (uint64_t)blockIdx.y * M * N;
    if (OUT == 1 && accumulate) {                            // sums are added in fp32, which the rows in LDS are not
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                __builtin_amdgcn_sched_barrier(0);           // one by one: addresses of all of them would not fit the registers
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t m = (tm * UM + wm + i) * 32 + lane % 32;
                    const uint32_t n = (tn * (WN * NF) + wn - UM + j) * 32 + 8 * g + 4 * (lane / 32);
                    float x[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                    if (m < M && n < N) store4<true>(c, ldc, m, n, N, x, true);
                }
            }
        return;
    }
    uint8_t *const mine = wave == 0 ? s0 : wave == 1 ? s1 : wave == 2 ? s2 : NB == 4 ? s3 : s0 + CODES / 2;
    constexpr int ES = OUT == 1 ? 2 : 4, WIDE = NF * 32 * ES, STRIDE = WIDE + 16, LANES = WIDE / 16;   // 16 bytes more: rows start in other banks
    static_assert(W == 4 && 32 * STRIDE <= (NB == 4 ? CODES : CODES / 2), "a wavefront's rows fit");
    const uint32_t n0 = (tn * (WN * NF) + wn - UM) * 32;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint8_t *to = mine + lane % 32 * STRIDE + (32 * j + 8 * g + lane / 32 * 4) * ES;
                if constexpr (OUT == 1) {
                    *reinterpret_cast<uint2 *>(to) = make_uint2(two_bf16(acc[i][j][4 * g], acc[i][j][4 * g + 1]),
                                                                two_bf16(acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]));
                } else {
                    *reinterpret_cast<float4 *>(to) = make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
                }
            }
        asm volatile("" ::: "memory");                       // this wavefront's own rows: LDS keeps its accesses in order
        const uint32_t n = n0 + lane % LANES * (16 / ES);
#pragma unroll
        for (int k = 0; k < LANES / 2; ++k) {
            const uint32_t r = k * (64 / LANES) + lane / LANES, m = (tm * UM + wm + i) * 32 + r;
            const uint4 x = *reinterpret_cast<const uint4 *>(mine + r * STRIDE + lane % LANES * 16);
            if (m < M && n < N) store16<OUT == 1>(c, (uint64_t)m * (OUT == 2 ? N : ldc) + n, N - n, x, OUT != 2 && accumulate != 0);
        }
        asm volatile("" ::: "memory");
    }
}

// C from `parts` sums over runs of k, [parts][M][N], added in order
template <bool BF16>
__global__ __launch_bounds__(256)
void k_mx4_sum_parts(const float *from, void *c, uint32_t M, uint32_t N, uint64_t ldc, uint32_t accumulate, uint32_t parts)
{
    const uint64_t total = (uint64_t)M * N, at = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    float v[4] = {};
    const bool whole = at + 4 <= total;
    for (uint32_t p = 0; p < parts; ++p) {
        const float *src = from + p * total + at;
        if (whole) {
            float x[4];
            __builtin_memcpy(x, src, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += x[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < total) v[i] += src[i];
        }
    }
    if (whole && N % 4 == 0) {
        store4<BF16>(c, ldc, (uint32_t)(at / N), (uint32_t)(at % N), N, v, accumulate != 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at + i >= total) continue;
            const uint64_t to = (at + i) / N * ldc + (at + i) % N;
            store1<BF16>(c, to, accumulate ? v[i] + load1<BF16>(c, to) : v[i]);
        }
    }
}

// ---------------------------------------------------------------- few rows of A

typedef float float4v __attribute__((ext_vector_type(4)));

// 16 rows of each operand, 128 columns: a lane holds row lane % 16, columns 32 * (lane / 16) on, of D column lane % 16 and rows
// 4 * (lane / 16) + i.  BYTE as above.
template <int BYTE>
__device__ __forceinline__ float4v mfma16(const uint4 &b, const uint4 &a, const float4v &c, uint32_t sb, uint32_t sa)
{
    const int8v vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    const int8v va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vb, va, c, 4, 4, BYTE, (int)sb, BYTE, (int)sa);
}

// Up to 16 * MT rows of A: what counts is how fast B streams in.  A workgroup takes 16 * NT rows of B (half a unit, or whole ones); its
// wavefronts share the columns by groups of 256, ask for several groups before they use the first, and add their sums in LDS.  Bound by
// memory: 5 x 8192 x 8192 10.8 us out of HBM (after a copy of 1 GiB), 3.3 TB/s, of which a launch's start is 2; 7.8 where the last
// cache still holds the matrix, 4.6 TB/s.  One token of 1600 x 1600, with its quantization, 5.0 and 2.9 us, a launch's time and one
// round trip to memory.
//   QUANT 0: A is packed.  1, 2: A is a tensor of bf16, fp32 with up to 2 * PAIRS <= 16 rows, of which every wavefront quantizes its
// own columns, 32 lanes to a row of a group, and turns them into operands through LDS that no other wavefront uses.
constexpr int kFewWaves = 8, kFewAhead = 4;

struct FewInput {
    const void *a;                       // packed, or a tensor of row stride ld
    uint64_t ld;
    uint32_t cover;
};

template <int MT, int NT, int QUANT, bool ROTATE, int PAIRS>
__global__ __launch_bounds__(64 * kFewWaves)
void k_mx4_few(const uint8_t *b, FewInput in, void *c, uint32_t M, uint32_t N, uint32_t K, uint64_t ldc, uint32_t accumulate, uint32_t out_bf16)
{
    static_assert(QUANT == 0 || MT == 1, "a tile of rows");
    __shared__ __attribute__((aligned(16))) uint8_t turned[QUANT ? kFewWaves : 1][QUANT ? 2048 + 256 : 16];
    __shared__ __attribute__((aligned(16))) float4v sums[kFewWaves][MT * NT][64];
    const Mx4Layout LA(M, K), LB(N, K);
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), row = lane % 16, quarter = lane / 16;
    const uint32_t n0 = blockIdx.x * 16 * NT;
    // 128 columns from column 32 * block: this lane's 32, of row r
    auto codes_of = [&](const uint8_t *p, uint32_t r, uint32_t unit) {
        return *reinterpret_cast<const uint4 *>(p + ((uint64_t)(r / 32) * LB.kb + min(unit + quarter / 2, LB.kb - 1)) * 1024 + quarter % 2 * 512 + r % 32 * 16);
    };
    // the bytes of this lane's blocks of a group of 256 columns, at places 0 and 2
    auto scales_of = [&](const uint8_t *p, uint32_t r, uint32_t group) {
        return reinterpret_cast<const uint32_t *>(p)[((uint64_t)(r / 32) * LB.kc + group) * 64 + quarter % 2 * 32 + r % 32] >> (quarter / 2 * 8);
    };
    const uint8_t *const a = static_cast<const uint8_t *>(in.a);
    float4v acc[MT][NT] = {};
    for (uint32_t g0 = wave; g0 < LB.kc; g0 += kFewWaves * kFewAhead) {
        uint4 vb[kFewAhead][NT][2], va[QUANT ? 1 : kFewAhead][MT][2];
        uint32_t sb[kFewAhead][NT], sa[QUANT ? 1 : kFewAhead][MT];
        Eight<QUANT == 1> x[QUANT ? kFewAhead : 1][PAIRS] = {};
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
            const uint32_t g = g0 + u * kFewWaves;
            if (g >= LB.kc) continue;
            if constexpr (QUANT != 0) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const uint32_t r = 2 * i + lane / 32, c = lane % 32 * 8, wide = K - g * 256;
                    if (r < M && c < wide) x[u][i] = fetch<QUANT == 1, false>(a + ((uint64_t)r * in.ld + g * 256) * (QUANT == 1 ? 2 : 4), c, wide, more_behind(r, M, in.ld));
                }
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t r = min(n0 + 16 * j + row, 32 * LB.rb - 1);
                sb[u][j] = scales_of(b + LB.scales(), r, g);
                vb[u][j][0] = codes_of(b, r, 4 * g);
                vb[u][j][1] = codes_of(b, r, 4 * g + 2);
            }
            if constexpr (QUANT == 0) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint32_t r = min(16 * i + row, M - 1);
                    sa[u][i] = scales_of(a + LA.scales(), r, g);
                    va[u][i][0] = codes_of(a, r, 4 * g);
                    va[u][i][1] = codes_of(a, r, 4 * g + 2);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
            if (g0 + u * kFewWaves >= LB.kc) continue;
            if constexpr (QUANT != 0) {
                // block t = 32 columns; operands [t][row: 16][16 bytes], scales [t % 4][row][4] at byte t / 4 * 2
                uint8_t *const mine = turned[wave];
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    uint32_t s;
                    const uint32_t w = quantize_quad<QUANT == 1, ROTATE>(x[u][i], in.cover, s), t = lane % 32 / 4, r = 2 * i + lane / 32;
                    *reinterpret_cast<uint32_t *>(mine + (t * 16 + r) * 16 + lane % 4 * 4) = w;
                    if (lane % 4 == 0) mine[2048 + (t % 4 * 16 + r) * 4 + t / 4 * 2] = (uint8_t)s;
                }
                asm volatile("" ::: "memory");               // this wavefront's own: LDS keeps its accesses in order
                __builtin_amdgcn_wave_barrier();
                va[0][0][0] = *reinterpret_cast<const uint4 *>(mine + lane * 16);
                va[0][0][1] = *reinterpret_cast<const uint4 *>(mine + 1024 + lane * 16);
                sa[0][0] = *reinterpret_cast<const uint32_t *>(mine + 2048 + lane * 4);
                __builtin_amdgcn_wave_barrier();
                asm volatile("" ::: "memory");
            }
            constexpr int OWN = QUANT ? 0 : 1;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    acc[i][j] = mfma16<0>(vb[u][j][0], va[OWN * u][i][0], acc[i][j], sb[u][j], sa[OWN * u][i]);
                    acc[i][j] = mfma16<2>(vb[u][j][1], va[OWN * u][i][1], acc[i][j], sb[u][j], sa[OWN * u][i]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    if (wave < MT * NT) {
        float4v t = sums[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) t += sums[w][wave][lane];
        const uint32_t m = wave / NT * 16 + row, n = n0 + wave % NT * 16 + quarter * 4;
        float v[4] = {t[0], t[1], t[2], t[3]};
        if (m < M && n < N) {
            if (out_bf16) store4<true>(c, ldc, m, n, N, v, accumulate != 0);
            else store4<false>(c, ldc, m, n, N, v, accumulate != 0);
        }
    }
}

}  // namespace tahq
