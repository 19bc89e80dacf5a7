// Device code of the head's matrix products: one tiled product on the matrix cores, whose operands may be stored either
// way round and whose epilogue is a functor.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace cgx {
namespace gemm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;      // bytes of the summed axis that one step of the main loop takes per row
constexpr int kMnUnit = 64;          // elements that a tile side must be a multiple of

// What a lane feeds the matrix cores at once: 16 bytes of consecutive elements of the summed axis.  Four groups of 16 lanes
// make 64 bytes of it; one or (binary32) four instructions consume them.
template <typename T>
struct Element;
template <>
struct Element<__bf16> {
    using Frag = bf16x8;
    static constexpr int kProducts = 1;
    static __device__ __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Element<_Float16> {
    using Frag = f16x8;
    static constexpr int kProducts = 1;
    static __device__ __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Element<float> {
    using Frag = f32x4;
    static constexpr int kProducts = 4;
    static __device__ __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// An operand of the product C[m][n] = sum_k A(m, k) B(n, k).
enum Layout {
    kSumContiguous,      // element (row, k) at row * pitch + k
    kSumStrips,          // the same, read in strips of 64 rows: fragment j holds rows 4 j .. 4 j + 3 of each 16 of the strip
    kRowContiguous       // element (row, k) at k * pitch + row
};

// 16 bytes per lane from base + offset (base uniform) to LDS, lane l's at address dst + 16 l (dst uniform).  Written out because the compiler,
// which cannot tell apart the stage that such a load fills and the one that a transposing LDS read takes, makes every such read wait for all
// loads that the builtin has issued; the waits that are needed are in Tile.  (The compiler keeps m0 for itself, so no clobber may name it; it sets it
// just ahead of what needs it, and nothing else in these kernels does.)
__device__ __forceinline__ void to_lds(const void *base, uint32_t offset, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(dst) : "memory");
}
// A barrier that no LDS access moves across (what it is a barrier for has been waited for by then: unlike __syncthreads, it adds no waits).
__device__ __forceinline__ void barrier()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return uint32_t(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void *)p));
}

// One side (ROWS rows) of a tile in LDS, kStepBytes of the summed axis deep, filled straight from memory by THREADS threads.
// The 16-byte pieces of a row are permuted within it (each thread fetches the piece that belongs where its lane writes), so that
// the lanes of a fragment read fall on different banks.
template <typename T, Layout LAYOUT, int ROWS, int THREADS>
struct Side {
    static constexpr int kPer = 16 / int(sizeof(T));                       // elements of a piece
    static constexpr int kDepth = kStepBytes / int(sizeof(T));             // of the summed axis per step
    static constexpr int kPieces = ROWS * kStepBytes / 16;
    static constexpr int kLoads = kPieces / THREADS;
    static constexpr int kBytes = ROWS * kStepBytes;
    static_assert(kPieces % THREADS == 0 && ROWS % kMnUnit == 0, "a tile side is filled by whole instructions");
    static constexpr int kUnits = ROWS / 16 - 1 < 7 ? ROWS / 16 - 1 : 7;   // of 32 bytes, that the rows of 16-bit elements are permuted among
    static constexpr int kReadsPerFragment = LAYOUT != kRowContiguous ? 1 : sizeof(T) == 2 ? 2 : 4;
    static constexpr int kPiecesPerRow = LAYOUT != kRowContiguous ? kStepBytes / 16 : ROWS / kPer;

    const T *base;            // of the current step, uniform
    int64_t pitch;
    int64_t step;             // elements from a step to the next
    uint32_t offset[kLoads];  // of this thread's pieces, in bytes

    // Row of LDS piece q, and the piece of memory that belongs there.
    static __device__ __forceinline__ int stored_row(int q) { return q / kPiecesPerRow; }
    static __device__ __forceinline__ int source_piece(int q)
    {
        const int row = stored_row(q), piece = q % kPiecesPerRow;
        if constexpr (LAYOUT == kSumContiguous) return piece ^ ((row >> 1) & 7);
        else if constexpr (LAYOUT == kSumStrips) return piece ^ (((row >> 1) & 1) | ((row >> 3) & 6));
        else if constexpr (sizeof(T) == 2) return piece ^ ((((row & 3) | ((row >> 1) & 4)) & kUnits) << 1);
        else return piece ^ (((row >> 2) & 3) << 2);
    }

    // rows: how many rows exist from row0 on; those past the end are read from the last ones, and their results are not used.
    // depth: how much of the summed axis exists; a kRowContiguous side re-reads its last row past it (the other side holds
    // zeros there), the others have to be readable up to a whole step.
    __device__ __forceinline__ void start(const T *all, int64_t pitch_, int64_t row0, int64_t rows, int64_t k0, int tid)
    {
        pitch = pitch_;
        if constexpr (LAYOUT != kRowContiguous) {
            base = all + row0 * pitch + k0;
            step = kDepth;
        } else {
            base = all + k0 * pitch + row0;
            step = int64_t(kDepth) * pitch;
        }
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int q = i * THREADS + tid;
            int row = stored_row(q), piece = source_piece(q);
            if constexpr (LAYOUT != kRowContiguous) row = row < rows ? row : int(rows) - 1;
            else piece = (piece + 1) * kPer <= rows ? piece : int(rows) / kPer - 1;
            offset[i] = uint32_t((uint32_t(row) * uint32_t(pitch) + uint32_t(piece) * kPer) * sizeof(T));
        }
    }
    __device__ __forceinline__ void clamp_depth(int64_t depth, int tid)
    {
        if constexpr (LAYOUT == kRowContiguous) {
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                const int row = stored_row(i * THREADS + tid);
                if (row >= depth) offset[i] -= uint32_t(row - int(depth) + 1) * uint32_t(pitch) * uint32_t(sizeof(T));
            }
        }
    }
    __device__ __forceinline__ void load(uint32_t lds, int wave)
    {
        const unsigned char *b = reinterpret_cast<const unsigned char *>(base);
#pragma unroll
        for (int i = 0; i < kLoads; i++) to_lds(b, offset[i], lds + uint32_t(i * THREADS + wave * 64) * 16);
        base += step;
    }
    // Fragment j of the rows from `first` on (a multiple of 64 for strips, of 16 otherwise): 16 rows, the half-th 64 bytes of the step.
    static __device__ __forceinline__ typename Element<T>::Frag fragment(const unsigned char *lds, int first, int j, int half, int lane)
    {
        using Frag = typename Element<T>::Frag;
        const int g = lane >> 4, r = lane & 15, row0 = first + 16 * j;
        if constexpr (LAYOUT == kSumStrips) {
            const int row = first + 16 * (r >> 2) + 4 * j + (r & 3);
            return *reinterpret_cast<const Frag *>(lds + row * kStepBytes + (((half * 4 + g) ^ (((r >> 1) & 1) | ((r >> 1) & 6))) << 4));
        } else if constexpr (LAYOUT == kSumContiguous) {
            return *reinterpret_cast<const Frag *>(lds + (row0 + r) * kStepBytes + (((half * 4 + g) ^ (r >> 1)) << 4));
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read a 4 x 16 block of 16-bit elements and get it transposed: four elements of the summed axis each
            const int unit = (row0 >> 4) ^ (((r >> 2) | ((g & 1) << 2)) & kUnits);
            const unsigned char *p = lds + (half * 32 + g * 8 + (r >> 2)) * (ROWS * 2) + unit * 32 + (r & 3) * 8;
            using Lds4 = __attribute__((address_space(3))) s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4 *)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4 *)(p + 4 * ROWS * 2));
            const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(Frag, both);
        } else {
            const int m = row0 + r;
            const unsigned char *p = lds + (half * 16 + g * 4) * (ROWS * 4) + (((m >> 2) ^ (g << 2)) << 4) + (m & 3) * 4;
            Frag f;
#pragma unroll
            for (int i = 0; i < 4; i++) f[i] = *reinterpret_cast<const float *>(p + i * (ROWS * 4));
            return f;
        }
    }
};

// A tile of C of BM x BN elements by WM x WN waves.  A lane ends with acc[i][j][e] = C[m][n] for
//   m = 16 i + lane % 16 (+ the wave's first row), n = 16 j + 4 (lane / 16) + e (+ the wave's first column):
// four neighbouring columns of a row (the side of the columns is the instruction's first operand).  With kSumStrips columns
// n = 16 (lane / 16) + 4 j + e: sixteen neighbouring ones, which an epilogue of 16-bit elements stores 16 bytes at a time.
template <typename T_, int BM_, int BN_, int WM_, int WN_, Layout LA, Layout LB, int STAGES = 2>
struct Tile {
    using T = T_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * 64;
    using A = Side<T, LA, BM, kThreads>;
    using B = Side<T, LB, BN, kThreads>;
    static constexpr int kDepth = A::kDepth;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    static_assert(LB != kSumStrips || TN == 4, "strips are as wide as a wave's columns");
    static constexpr int kStage = A::kBytes + B::kBytes;
    static constexpr int kLds = STAGES * kStage;

    f32x4 acc[TM][TN];
    int wave, lane, wm, wn;

    using Frag = typename Element<T>::Frag;
    struct Frags {
        Frag a[TM], b[TN];
    };
    __device__ __forceinline__ void fetch(Frags &f, const unsigned char *stage, int half) const
    {
#pragma unroll
        for (int j = 0; j < TN; j++) f.b[j] = B::fragment(stage + A::kBytes, wn, j, half, lane);
#pragma unroll
        for (int i = 0; i < TM; i++) f.a[i] = A::fragment(stage, wm, i, half, lane);
    }
    __device__ __forceinline__ void multiply(const Frags &f)
    {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) acc[i][j] = Element<T>::mfma(f.b[j], f.a[i], acc[i][j]);
    }
    // Spreads LDS reads and loads from memory between the matrix instructions of a half step.
    template <int READS, int LOADS>
    static __device__ __forceinline__ void interleave()
    {
        constexpr int kProducts = TM * TN * Element<T>::kProducts;
        constexpr int kSlots = kProducts < 16 ? kProducts : 16;      // (every one has a product)
#pragma unroll
        for (int k = 0; k < kSlots; k++) {
            if (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, (READS + kSlots - 1) / kSlots, 0);
            if (LOADS > 0) __builtin_amdgcn_sched_group_barrier(0x20, (LOADS + kSlots - 1) / kSlots, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, kProducts / kSlots, 0);
        }
    }
    static constexpr int kReads = TM * A::kReadsPerFragment + TN * B::kReadsPerFragment;

    // Waits for the oldest stage that is on its way (MORE: others are, and may stay so) and for LDS reads.
    template <bool MORE>
    static __device__ __forceinline__ void wait()
    {
        constexpr int kLater = MORE ? (STAGES - 2) * (A::kLoads + B::kLoads) : 0;
        static_assert(kLater < 16, "a count of four bits");
        __builtin_amdgcn_s_waitcnt(0x0070 | kLater);
    }
    static __device__ __forceinline__ uint32_t next(uint32_t now) { return STAGES == 2 ? kStage - now : now == (STAGES - 1) * kStage ? 0 : now + kStage; }

    // One step: the products of the stage at `now`, whose first half is in f0 already.  LOAD: the step STAGES steps on exists and
    // is loaded into the same place; NEXT: another step follows, its first half is fetched into f0.
    template <bool LOAD, bool NEXT>
    __device__ __forceinline__ void step(A &a, B &b, Frags &f0, Frags &f1, const unsigned char *lds, uint32_t at, uint32_t now)
    {
        __builtin_amdgcn_sched_barrier(0);
        fetch(f1, lds + now, 1);
        multiply(f0);
        interleave<kReads, 0>();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (NEXT) {
            // the next stage is here, and everybody is done reading this one
            wait<LOAD>();
            barrier();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (LOAD) {
                a.load(at + now, wave);
                b.load(at + now + A::kBytes, wave);
            }
            fetch(f0, lds + next(now), 0);
        }
        multiply(f1);
        interleave<NEXT ? kReads : 0, LOAD ? A::kLoads + B::kLoads : 0>();
        __builtin_amdgcn_sched_barrier(0);
    }

    // steps: of kDepth each; the last one has `last` elements of the summed axis (kRowContiguous sides).
    // Stages in LDS: the loads that fill one are issued half a step after its last read, STAGES - 1 steps before they are waited for.
    __device__ __forceinline__ void run(A &a, B &b, int steps, int last, unsigned char *lds)
    {
        const int tid = int(threadIdx.x);
        wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        lane = tid & 63;
        wm = (wave / WN) * (BM / WM);
        wn = (wave % WN) * (BN / WN);
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (steps <= 0) return;
        const auto shorten = [&] {
            if (last < kDepth) {
                a.clamp_depth(last, tid);
                b.clamp_depth(last, tid);
            }
        };
        const uint32_t at = lds_address(lds);
        uint32_t now = 0;
        const auto first = [&](int s) {
            if (s >= steps) return;
            if (s == steps - 1) shorten();
            a.load(at + s * kStage, wave);
            b.load(at + s * kStage + A::kBytes, wave);
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; s++) first(s);
        if (steps >= STAGES - 1) wait<true>();
        else wait<false>();
        barrier();
        first(STAGES - 1);
        Frags f0, f1;
        fetch(f0, lds, 0);
        int s = 0;
        for (; s + STAGES + 1 < steps; s++) {
            step<true, true>(a, b, f0, f1, lds, at, now);
            now = next(now);
        }
        if (s + STAGES < steps) {
            shorten();
            step<true, true>(a, b, f0, f1, lds, at, now);
            now = next(now);
            s++;
        }
#pragma unroll
        for (int k = 1; k < STAGES; k++) {
            if (s + 1 < steps) {
                step<false, true>(a, b, f0, f1, lds, at, now);
                now = next(now);
                s++;
            }
        }
        step<false, false>(a, b, f0, f1, lds, at, now);
    }
};

// Tiles are handed out so that the blocks of one XCD (block % 8) work on neighbouring ones: within a run of tiles, bands of
// kBand tile rows are walked column by column.  Of the first `whole` blocks, that is (all of them, if there are more); any others
// take the tiles that follow, in order.
constexpr int kXcds = 8, kBand = 4;
__device__ __forceinline__ bool tile_of_block(uint32_t block, uint32_t whole, uint32_t tiles_m, uint32_t tiles_n, int &m, int &n)
{
    const uint32_t all = tiles_m * tiles_n, total = whole < all ? whole : all;
    if (block >= all) return false;
    uint32_t at = block;
    if (block < total) {
        const uint32_t each = total / kXcds, more = total % kXcds, x = block % kXcds;
        at = x * each + (x < more ? x : more) + block / kXcds;
    }
    const uint32_t band = at / (kBand * tiles_n), in = at % (kBand * tiles_n);
    const uint32_t high = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    m = __builtin_amdgcn_readfirstlane(int(band * kBand + in % high));
    n = __builtin_amdgcn_readfirstlane(int(in / high));
    return true;
}

}  // namespace gemm
}  // namespace cgx
