// Products C[j, i] = sum_k A[i, k] B[j, k] on the 16-bit and 8-bit matrix instructions, for operands that lie packed in memory.
//
// A packed operand has rows of `pitch` bytes, a row being a series of steps of 128 bytes, which hold
//   kHalf     64 columns of 16-bit floating point;
//   kHalfTwo  32 columns of two terms: 64 bytes of the rounded numbers, then 64 bytes of what rounding left over. The product
//             of a pair of numbers is lo*hi + hi*lo + hi*hi, accumulated in 32 bits in this order (lo*lo is below 2^-22 of it);
//   kInt8     128 columns of 8-bit integers, accumulated exactly in 32 bits.
// Columns beyond the operands' are zero in one of the two at least (kInt8) or in both. These ways move the same bytes from
// memory through LDS into registers and differ in the matrix instructions alone: a lane's 16 bytes are 8 or 16 consecutive columns of one row.
//   kHalfByTwo  A as in kHalf, half a step of it at a time, B as in kHalfTwo: lo*x + hi*x of 32 columns.
//
// Tile TM x TN, WM x WN wavefronts, blocks of 32 x 32. A step of the tile goes from memory straight into LDS (16 bytes a
// lane), into the buffer that the step before last used, while the step that arrived before is multiplied: one barrier a
// step. LDS: row r's 128 bytes are 8 chunks of 16, chunk c at place c ^ (r & 7), so that 8 lanes that read the same chunk of 8
// rows meet all banks once (and the permutation is made by the loads' addresses, at no cost). Rows of 64 bytes: chunk c at place c ^ (r / 2 & 3).
//
// What bounds it (counters of the cycles in which a CU holds a tile): with tiles of 256 and two terms the matrix instructions, busy 76 to 80 % of them at a
// clock of 1.7 GHz, which is what the power allows; with one term or 8 bits, whose steps are shorter, they are busy 42 to 59 %, and the
// wavefronts wait for the next step 35 to 44 % of their time. 32768 x 2048 x 8192 of 16-bit numbers 877 us (1250 TFLOP/s); the same
// without the loads 710, the loads alone 560 to 730, the matrix instructions alone 490 to 540. 50000 x 5000 x 10241 of 8-bit ones 2.43 to 2.56
// ms (2000 to 2110 TOP/s). With the smaller tiles, waiting for the steps (matrix instructions 20 to 39 %), and CUs without a tile.
#pragma once

#include "rfsf_internal.h"

#include <type_traits>

namespace rfsf {

enum PlaneMode { kHalf = 0, kHalfTwo = 1, kInt8 = 2, kHalfByTwo = 3 };
constexpr int kStepBytes = 128;
constexpr int step_bytes_a(PlaneMode mode) { return mode == kHalfByTwo ? kStepBytes / 2 : kStepBytes; }

struct Planes {
    const char *data;
    int64_t pitch;          // bytes from row to row
    int64_t rows;           // >= 1; rows beyond are read as the last one, and what they give is not stored
};

namespace plane {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

template <PlaneMode MODE> struct Acc { typedef floatx16 type; };
template <> struct Acc<kInt8> { typedef intx16 type; };

__device__ __forceinline__ floatx16 mfma(const intx4 &a, const intx4 &b, const floatx16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}
__device__ __forceinline__ intx16 mfma(const intx4 &a, const intx4 &b, const intx16 &c)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

// 16 bytes a lane from base + off to LDS at dst + 16 * lane. Written out because the compiler, which cannot tell the buffers
// apart, would wait for the loads in flight before every read of LDS; the caller waits (m0 is the compiler's own register,
// that it is written has to be said, and is warned about).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void direct_load16(const char *base, uint32_t off, uint32_t dst)
{
    const uint32_t to = __builtin_amdgcn_readfirstlane(dst);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Tiles in the order that the XCDs' L2s see them: eight contiguous pieces of an order that goes through strips of kStrip tiles of A.
constexpr int kStrip = 8;
__device__ __forceinline__ bool tile_of_block(unsigned block, int64_t tiles_i, int64_t tiles_j, int cuts, int64_t *ti, int64_t *tj, int *cut)
{
    const int64_t tiles = tiles_i * tiles_j, all = tiles * cuts, per = (all + 7) / 8;
    int64_t rank = (int64_t)(block % 8) * per + block / 8;
    if (rank >= all) return false;
    *cut = cuts > 1 ? (int)(rank / tiles) : 0;          // (an XCD's tiles are of few cuts, whose columns no other one reads)
    rank -= *cut * tiles;
    const int64_t strip = rank / (kStrip * tiles_j), at = rank - strip * kStrip * tiles_j;
    const int64_t left = tiles_i - strip * kStrip, width = left < kStrip ? left : kStrip;
    *tj = at / width;
    *ti = strip * kStrip + (at - *tj * width);
    return true;
}
inline unsigned blocks_of(int64_t tiles) { return (unsigned)((tiles + 7) / 8 * 8); }

// What an epilogue is given: the wavefront's accumulators and where they belong. Element e of acc[a][b] of a lane is row
// i0 + 32 a + 8 (e / 4) + 4 (lane / 32) + e % 4 and column j0 + 32 b + lane % 32.
//
// A tile of EXTRA has another 32 rows, from extra_i on: one block for each wavefront, that of its columns 32 wave_i .. + 31. Operands
// with one more row than whole tiles (features have 1 + M*D columns) then need no further tiles for it.
template <PlaneMode MODE, int TM, int TN, int WM, int WN, bool EXTRA>
struct Tile {
    static constexpr int BM = TM / WM / 32, BN = TN / WN / 32, ROWS = TM, COLUMNS = TN, WAVES_I = WM;
    static constexpr bool HAS_EXTRA = EXTRA;
    typename Acc<MODE>::type acc[BM][BN], extra;
    int64_t i0, j0, tile_i, tile_j, extra_i;
    int wave_i, wave_j, cut;
    char *lds;                  // free for the epilogue after a barrier
    // f(block, first row, number of the block of columns), for every block
    template <typename F>
    __device__ __forceinline__ void each_block(const F &f)
    {
#pragma unroll
        for (int a = 0; a < BM; ++a)
#pragma unroll
            for (int b = 0; b < BN; ++b) f(acc[a][b], i0 + 32 * a, b);
        if constexpr (EXTRA) {
#pragma unroll
            for (int b = 0; b < BN; ++b)
                if (b == wave_i) f(extra, extra_i, b);
        }
    }
};

template <PlaneMode MODE, int TM, int TN, int WM, int WN, int STAGES, bool EXTRA, typename Epilogue>
__device__ __forceinline__ void run_tile(char *buffers, const Planes &A, const Planes &B, int64_t steps, int64_t tile_i, int64_t tile_j, int cut, const Epilogue &epilogue)
{
    typedef Tile<MODE, TM, TN, WM, WN, EXTRA> T;
    constexpr int BM = T::BM, BN = T::BN, kStepA = step_bytes_a(MODE), kLoadRows = 1024 / kStepA;           // rows of A that a load of a wavefront brings
    constexpr int kLoadsA = TM / kLoadRows, kStartB = TM * kStepA, kStartX = kStartB + TN * kStepBytes, kBuffer = kStartX + (EXTRA ? 32 * kStepA : 0);
    constexpr int NL = (kLoadsA + TN / 8) / (WM * WN);
    static_assert((kLoadsA + TN / 8) % (WM * WN) == 0 && TM % kLoadRows == 0, "every wavefront makes as many loads, of whole groups of rows");
    static_assert(!EXTRA || (WM == BN && WM * WN >= 4 && STAGES == 2), "a block for every wavefront, one load of its rows for each of a few");
    static_assert(STAGES >= 2 && (STAGES - 1) * NL < 64, "loads in flight can be counted");
    T t;
    t.tile_i = tile_i;
    t.tile_j = tile_j;
    t.cut = cut;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int half = lane >> 5, col = lane & 31;
    const int64_t first_i = t.tile_i * TM, first_j = t.tile_j * TN;
    t.wave_i = wave / WN;
    t.wave_j = wave % WN;
    t.i0 = first_i + t.wave_i * (TM / WM);
    t.j0 = first_j + t.wave_j * (TN / WN);
    t.extra_i = first_i + TM;
    t.lds = buffers;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)buffers;

    // LDS: the rows of A, those of B, the extra ones of A
    const char *base_a = A.data + first_i * A.pitch, *base_b = B.data + first_j * B.pitch;
    uint32_t off[NL + 1];       // from the tile's first row: at most 287 rows on, checked by the callers to stay below 2^32
#pragma unroll
    for (int l = 0; l <= NL; ++l) {
        const int at = l < NL ? wave * NL + l : wave;
        const bool is_b = l < NL && at >= kLoadsA;
        const int row = is_b ? 8 * (at - kLoadsA) + (lane >> 3) : (l < NL ? 0 : TM) + kLoadRows * at + lane / (kStepA / 16);
        const int chunk = is_b || kStepA == kStepBytes ? (lane & 7) ^ (lane >> 3) : (lane & 3) ^ (lane >> 3 & 3);
        const int64_t last = is_b ? B.rows - 1 - first_j : A.rows - 1 - first_i;
        off[l] = (uint32_t)((row < last ? row : last) * (is_b ? B.pitch : A.pitch)) + 16u * (uint32_t)chunk;
    }
    auto load = [&](int64_t step, int buffer) {
#pragma unroll
        for (int l = 0; l < NL; ++l) {
            const int at = wave * NL + l;
            direct_load16(at >= kLoadsA ? base_b + step * kStepBytes : base_a + step * kStepA, off[l], lds + (uint32_t)(buffer * kBuffer + 1024 * at));
        }
        if (EXTRA && wave < 32 / kLoadRows)
            direct_load16(base_a + step * kStepA, off[NL], lds + (uint32_t)(buffer * kBuffer + kStartX + 1024 * wave));
    };
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        t.extra[e] = 0;
#pragma unroll
        for (int a = 0; a < BM; ++a)
#pragma unroll
            for (int b = 0; b < BN; ++b) t.acc[a][b][e] = 0;
    }

    // Software pipeline. A step is cut into phases of BM x BN matrix instructions, whose operands have been read from LDS during the phase before,
    // so that a wavefront's matrix instructions follow one another. Before the last phases of a step, when all of it has been read, the
    // wavefront waits for its loads of the next step (those of the steps after it stay in flight) and then for everybody: the
    // next step can be read, and this step's buffer takes the loads of the step STAGES ahead.
    const int row_a = t.wave_i * (TM / WM) + col, row_b = t.wave_j * (TN / WN) + col, turn_a = kStepA == kStepBytes ? col & 7 : col >> 1 & 3;
    const char *buf = buffers;
    int slot = 0;
    auto read_a = [&](intx4 (&f)[BM], const char *from, int c) {
#pragma unroll
        for (int a = 0; a < BM; ++a) f[a] = *reinterpret_cast<const intx4 *>(from + (row_a + 32 * a) * kStepA + 16 * ((c + half) ^ turn_a));
    };
    auto read_b = [&](intx4 (&f)[BN], const char *from, int c) {
#pragma unroll
        for (int b = 0; b < BN; ++b) f[b] = *reinterpret_cast<const intx4 *>(from + kStartB + (row_b + 32 * b) * kStepBytes + 16 * ((c + half) ^ (col & 7)));
    };
    auto read_x = [&](const char *from, int c) {
        if constexpr (!EXTRA) return intx4{0, 0, 0, 0};
        return *reinterpret_cast<const intx4 *>(from + kStartX + col * kStepA + 16 * ((c + half) ^ turn_a));
    };
    auto multiply = [&](const intx4 (&fa)[BM], const intx4 (&fb)[BN], const intx4 &fx) {
#pragma unroll
        for (int a = 0; a < BM; ++a)
#pragma unroll
            for (int b = 0; b < BN; ++b) t.acc[a][b] = mfma(fa[a], fb[b], t.acc[a][b]);
        if constexpr (EXTRA) t.extra = mfma(fx, t.wave_i == 0 ? fb[0] : fb[BN - 1], t.extra);
    };
    // READS reads spread over the phase's matrix instructions
    auto interleave = [&](auto reads) {
        constexpr int R = decltype(reads)::value, PRODUCTS = BM * BN;
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            const int now = (i + 1) * R / PRODUCTS - i * R / PRODUCTS;
            if (now == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (now == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            if (now > 2) __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        }
    };
    // the step after s has landed, for everybody
    auto landed = [&](int64_t s) {
        if (STAGES > 2 && s + STAGES <= steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * NL) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto next_buffer = [&] { return buffers + (slot + 1 == STAGES ? 0 : slot + 1) * kBuffer; };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (s < steps) load(s, s);
    landed(-1);
    if (STAGES - 1 < steps) load(STAGES - 1, STAGES - 1);
    if constexpr (MODE == kHalfTwo) {
        intx4 ah[BM], al[BM], bh[BN], bl[BN], next[BN], xh, xl = read_x(buf, 4);
        read_a(al, buf, 4);
        read_b(bh, buf, 0);
        for (int64_t s = 0; s < steps; ++s) {
            const char *other = next_buffer();
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const bool last = ks == 1;
                read_a(ah, buf, 2 * ks);
                xh = read_x(buf, 2 * ks);
                read_b(bl, buf, 4 + 2 * ks);
                multiply(al, bh, xl);
                interleave(std::integral_constant<int, BM + BN>{});
                if (last) {
                    landed(s);
                    if (s + STAGES < steps) load(s + STAGES, slot);
                }
                read_a(al, last ? other : buf, last ? 4 : 6);
                xl = read_x(last ? other : buf, last ? 4 : 6);
                multiply(ah, bl, xh);
                interleave(std::integral_constant<int, BM>{});
                read_b(next, last ? other : buf, last ? 0 : 2);
                multiply(ah, bh, xh);
                interleave(std::integral_constant<int, BN>{});
#pragma unroll
                for (int b = 0; b < BN; ++b) bh[b] = next[b];
            }
            buf = other;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
    } else if constexpr (MODE == kHalfByTwo) {
        // phases: the rest of columns 0 to 15, their rounded numbers, and the same of 16 to 31; A's fragments serve two of them
        constexpr int CHUNK[5] = {4, 0, 6, 2, 4};
        intx4 fa[2][BM], fb[2][BN], fx[2];
        fx[0] = read_x(buf, 0);
        read_a(fa[0], buf, 0);
        read_b(fb[0], buf, CHUNK[0]);
        for (int64_t s = 0; s < steps; ++s) {
            const char *other = next_buffer();
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const bool last = ks == 3;
                if (last) {
                    landed(s);
                    if (s + STAGES < steps) load(s + STAGES, slot);
                }
                read_b(fb[(ks + 1) & 1], last ? other : buf, CHUNK[ks + 1]);
                if (ks & 1) {
                    read_a(fa[last ? 0 : 1], last ? other : buf, last ? 0 : 2);
                    fx[last ? 0 : 1] = read_x(last ? other : buf, last ? 0 : 2);
                }
                multiply(fa[ks >> 1], fb[ks & 1], fx[ks >> 1]);
                if (ks & 1) interleave(std::integral_constant<int, BM + BN>{});
                else interleave(std::integral_constant<int, BN>{});
            }
            buf = other;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
    } else {
        intx4 fa[2][BM], fb[2][BN], fx[2];
        fx[0] = read_x(buf, 0);
        read_a(fa[0], buf, 0);
        read_b(fb[0], buf, 0);
        for (int64_t s = 0; s < steps; ++s) {
            const char *other = next_buffer();
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const bool last = ks == 3;
                if (last) {
                    landed(s);
                    if (s + STAGES < steps) load(s + STAGES, slot);
                }
                read_a(fa[(ks + 1) & 1], last ? other : buf, last ? 0 : 2 * ks + 2);
                read_b(fb[(ks + 1) & 1], last ? other : buf, last ? 0 : 2 * ks + 2);
                fx[(ks + 1) & 1] = read_x(last ? other : buf, last ? 0 : 2 * ks + 2);
                multiply(fa[ks & 1], fb[ks & 1], fx[ks & 1]);
                interleave(std::integral_constant<int, BM + BN>{});
            }
            buf = other;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
    }
    epilogue(t);
}

}  // namespace plane

// Products of one launch: the second one's tiles follow the first one's and share the GPU with their rest. The sum of a product may be cut into
// parts of per_cut steps, each of which gives tiles of its own (Tile::cut) for the epilogue to keep apart.
template <typename Epilogue>
struct Product {
    Planes A, B;
    int64_t steps;
    Epilogue epilogue;
    int64_t per_cut = 0;        // 0: not cut
    int cuts() const { return per_cut > 0 ? (int)((steps + per_cut - 1) / per_cut) : 1; }
};

namespace plane {

template <typename Epilogue>
struct Products {
    Product<Epilogue> product[2];
    int64_t tiles_i[2], tiles_j[2];
    int cuts[2];
    unsigned blocks_of_first;
};

template <PlaneMode MODE, int TM, int TN, int WM, int WN, int STAGES, bool EXTRA, typename Epilogue>
__global__ __launch_bounds__(64 * WM * WN, 2)
void plane_product(Products<Epilogue> all)
{
    extern __shared__ __attribute__((aligned(1024))) char buffers[];
    const int which = blockIdx.x < all.blocks_of_first ? 0 : 1;
    const Product<Epilogue> &p = all.product[which];
    const int64_t tiles_i = all.tiles_i[which];
    int64_t tile_i, tile_j, steps = p.steps;
    int cut;
    if (!tile_of_block(blockIdx.x - (which ? all.blocks_of_first : 0), tiles_i, all.tiles_j[which], all.cuts[which], &tile_i, &tile_j, &cut)) return;
    Planes A = p.A, B = p.B;
    if (p.per_cut > 0) {
        A.data += cut * p.per_cut * step_bytes_a(MODE);
        B.data += cut * p.per_cut * kStepBytes;
        steps = steps - cut * p.per_cut < p.per_cut ? steps - cut * p.per_cut : p.per_cut;
    }
    if (EXTRA && tile_i == tiles_i - 1 && p.A.rows > tiles_i * TM)
        run_tile<MODE, TM, TN, WM, WN, STAGES, EXTRA>(buffers, A, B, steps, tile_i, tile_j, cut, p.epilogue);
    else
        run_tile<MODE, TM, TN, WM, WN, STAGES, false>(buffers, A, B, steps, tile_i, tile_j, cut, p.epilogue);
}

}  // namespace plane

// Tiles along A, which an epilogue may number its parts by. A last tile of up to 32 rows of 256 is joined to the one before.
inline bool plane_extra(int64_t rows_a, int tile) { return tile == 256 && rows_a > 256 && rows_a % 256 > 0 && rows_a % 256 <= 32; }
inline int64_t plane_tiles_a(int64_t rows_a, int tile) { return plane_extra(rows_a, tile) ? rows_a / tile : (rows_a + tile - 1) / tile; }
inline int64_t plane_tiles(int64_t rows_a, int64_t rows_b, int tile) { return plane_tiles_a(rows_a, tile) * ((rows_b + tile - 1) / tile); }

// The edge of a launch's tiles: the one of which the steps take the least time, from the number of tiles that each edge makes (of the longest
// product's steps). A CU holds one tile of 256 or 128, or two of 64; a step of a tile takes 1.2, 0.48 and 0.22 us where few CUs have any and
// up to 2.1, 0.88 and 0.57 where all do, as the L2s deliver about 9.5 TB/s. (us a step over all tiles, edges 64, 128, 256, 8-bit
// products of 81 steps but the last: 128 x 16384 rows 0.36, 0.62, 1.29; 128 x 24576 0.96, 0.67, 1.42; 128 x 65536 2.55, 1.91, 1.98; 256 x 32768 2.22,
// 1.52, 1.74, where 256 is chosen; 256 x 65536 4.51, 3.10, 2.45; 333 x 10000, 41 steps 0.80, 0.65, 1.73.)
struct PlaneWay { int edge; double slots, alone, beside; };
constexpr PlaneWay kPlaneWays[] = {{256, 256, 1.2, 0.9}, {128, 256, 0.48, 0.4}, {64, 512, 0.22, 0.35}};
inline double plane_step_time(const PlaneWay &way, double tiles)
{
    const double full = (double)(int64_t)(tiles / way.slots), rest = tiles - full * way.slots;
    return full * (way.alone + way.beside) + (rest > 0 ? way.alone + way.beside * rest / way.slots : 0.0);
}
template <typename Tiles>
int plane_tile_of(const Tiles &tiles)
{
    int best = 0;
    double least = 0.0;
    for (const PlaneWay &way : kPlaneWays) {
        const double time = plane_step_time(way, tiles(way.edge));
        if (best == 0 || time < least) {
            best = way.edge;
            least = time;
        }
    }
    return best;
}
inline int plane_tile(int64_t rows_a, int64_t rows_b)
{
    return plane_tile_of([&](int edge) { return (double)plane_tiles(rows_a, rows_b, edge); });
}

namespace plane {

template <PlaneMode MODE, int TM, int TN, int WM, int WN, int STAGES, bool EXTRA, typename Epilogue>
hipError_t launch_tiles(const Product<Epilogue> *p, int count, hipStream_t stream)
{
    constexpr size_t lds = STAGES * (size_t)((TM + (EXTRA ? 32 : 0)) * step_bytes_a(MODE) + TN * kStepBytes);
    static LdsLimit limit;
    auto kernel = plane_product<MODE, TM, TN, WM, WN, STAGES, EXTRA, Epilogue>;
    const hipError_t e = allow_lds(limit, reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    Products<Epilogue> all;
    unsigned blocks[2] = {0, 0};
    for (int k = 0; k < 2; ++k) {
        all.product[k] = p[k < count ? k : 0];
        all.tiles_i[k] = plane_tiles_a(all.product[k].A.rows, TM);
        all.tiles_j[k] = (all.product[k].B.rows + TN - 1) / TN;
        all.cuts[k] = all.product[k].cuts();
        if (k < count) blocks[k] = blocks_of(all.tiles_i[k] * all.tiles_j[k] * all.cuts[k]);
    }
    all.blocks_of_first = blocks[0];
    kernel<<<dim3(blocks[0] + blocks[1]), dim3(64 * WM * WN), lds, stream>>>(all);
    return hipGetLastError();
}

}  // namespace plane

// One product, or two in one launch, in tiles of edge `tile`.
template <PlaneMode MODE, typename Epilogue>
hipError_t launch_plane_products(const Product<Epilogue> *p, int count, int tile, hipStream_t stream)
{
    if (plane_extra(p[0].A.rows, tile) || (count > 1 && plane_extra(p[1].A.rows, tile)))
        return plane::launch_tiles<MODE, 256, 256, 2, 4, 2, true>(p, count, stream);
    if (tile == 256) return plane::launch_tiles<MODE, 256, 256, 2, 4, 2, false>(p, count, stream);
    if (tile == 128) return plane::launch_tiles<MODE, 128, 128, 2, 2, 4, false>(p, count, stream);
    return plane::launch_tiles<MODE, 64, 64, 2, 2, 4, false>(p, count, stream);
}
template <PlaneMode MODE, typename Epilogue>
hipError_t launch_plane_product(const Planes &A, const Planes &B, int64_t steps, int tile, const Epilogue &epilogue, hipStream_t stream)
{
    const Product<Epilogue> p = {A, B, steps, epilogue, 0};
    return launch_plane_products<MODE>(&p, 1, tile, stream);
}

}  // namespace rfsf
