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
constexpr int kMnUnit = 128;         // elements that a tile side must be a multiple of

// What a lane feeds the matrix cores at once: 16 bytes of consecutive elements of the summed axis.  Four groups of 16 lanes
// make 64 bytes of it; one or (binary32) four instructions consume them.
template <typename T>
struct Element;
template <>
struct Element<__bf16> {
    using Frag = bf16x8;
    static __device__ __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Element<_Float16> {
    using Frag = f16x8;
    static __device__ __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Element<float> {
    using Frag = f32x4;
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
    kRowContiguous       // element (row, k) at k * pitch + row
};

__device__ __forceinline__ void to_lds(const void *src, void *dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                     (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
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
    static constexpr int kPiecesPerRow = LAYOUT == kSumContiguous ? kStepBytes / 16 : ROWS / kPer;

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
        else if constexpr (sizeof(T) == 2) return piece ^ (((row & 3) | ((row >> 1) & 4)) << 1);
        else return piece ^ (((row >> 2) & 3) << 2);
    }

    // rows: how many rows exist from row0 on; those past the end are read from the last ones, and their results are not used.
    // depth: how much of the summed axis exists; a kRowContiguous side re-reads its last row past it (the other side holds
    // zeros there), a kSumContiguous one has to be readable up to a whole step.
    __device__ __forceinline__ void start(const T *all, int64_t pitch_, int64_t row0, int64_t rows, int64_t k0, int tid)
    {
        pitch = pitch_;
        if constexpr (LAYOUT == kSumContiguous) {
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
            if constexpr (LAYOUT == kSumContiguous) row = row < rows ? row : int(rows) - 1;
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
    __device__ __forceinline__ void load(unsigned char *lds, int wave)
    {
        const unsigned char *b = reinterpret_cast<const unsigned char *>(base);
#pragma unroll
        for (int i = 0; i < kLoads; i++) to_lds(b + offset[i], lds + (i * THREADS + wave * 64) * 16);
        base += step;
    }
    // The fragment of rows row0 .. row0 + 15 (row0 a multiple of 16) and the half-th 64 bytes of the step.
    static __device__ __forceinline__ typename Element<T>::Frag fragment(const unsigned char *lds, int row0, int half, int lane)
    {
        using Frag = typename Element<T>::Frag;
        const int g = lane >> 4, r = lane & 15;
        if constexpr (LAYOUT == kSumContiguous) {
            return *reinterpret_cast<const Frag *>(lds + (row0 + r) * kStepBytes + (((half * 4 + g) ^ (r >> 1)) << 4));
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read a 4 x 16 block of 16-bit elements and get it transposed: four elements of the summed axis each
            const int unit = (row0 >> 4) ^ ((r >> 2) | ((g & 1) << 2));
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
// four neighbouring columns of a row (the side of the columns is the instruction's first operand).
template <typename T_, int BM_, int BN_, int WM_, int WN_, Layout LA, Layout LB>
struct Tile {
    using T = T_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * 64;
    using A = Side<T, LA, BM, kThreads>;
    using B = Side<T, LB, BN, kThreads>;
    static constexpr int kDepth = A::kDepth;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    static constexpr int kStage = A::kBytes + B::kBytes;
    static constexpr int kLds = 2 * kStage;

    f32x4 acc[TM][TN];
    int wave, lane, wm, wn;

    __device__ __forceinline__ void multiply(const unsigned char *stage)
    {
        using Frag = typename Element<T>::Frag;
#pragma unroll
        for (int half = 0; half < 2; half++) {
            Frag a[TM], b[TN];
#pragma unroll
            for (int j = 0; j < TN; j++) b[j] = B::fragment(stage + A::kBytes, wn + 16 * j, half, lane);
#pragma unroll
            for (int i = 0; i < TM; i++) a[i] = A::fragment(stage, wm + 16 * i, half, lane);
#pragma unroll
            for (int i = 0; i < TM; i++)
#pragma unroll
                for (int j = 0; j < TN; j++) acc[i][j] = Element<T>::mfma(b[j], a[i], acc[i][j]);
        }
    }

    // steps: of kDepth each; the last one has `last` elements of the summed axis (kRowContiguous sides).
    __device__ __forceinline__ void run(A &a, B &b, int64_t steps, int last, unsigned char *lds)
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
        if (steps == 1 && last < kDepth) {
            a.clamp_depth(last, tid);
            b.clamp_depth(last, tid);
        }
        a.load(lds, wave);
        b.load(lds + A::kBytes, wave);
        unsigned char *now = lds, *next = lds + kStage;
        for (int64_t s = 0; s < steps; s++) {
            // the stage is here, and everybody is done with the other one
            __builtin_amdgcn_s_waitcnt(0x0f70);
            __syncthreads();
            if (s + 1 < steps) {
                if (s + 2 == steps && last < kDepth) {
                    a.clamp_depth(last, tid);
                    b.clamp_depth(last, tid);
                }
                a.load(next, wave);
                b.load(next + A::kBytes, wave);
            }
            multiply(now);
            unsigned char *t = now;
            now = next;
            next = t;
        }
    }
};

// Tiles are handed out so that the blocks of one XCD (block % 8) work on neighbouring ones: within a run of tiles, bands of
// kBand tile rows are walked column by column.
constexpr int kXcds = 8, kBand = 4;
__device__ __forceinline__ bool tile_of_block(int64_t block, int64_t tiles_m, int64_t tiles_n, int64_t &m, int64_t &n)
{
    const int64_t total = tiles_m * tiles_n;
    if (block >= total) return false;
    const int64_t each = total / kXcds, more = total % kXcds, x = block % kXcds;
    const int64_t at = x * each + (x < more ? x : more) + block / kXcds;
    const int64_t band = at / (kBand * tiles_n), in = at % (kBand * tiles_n);
    const int64_t high = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    m = band * kBand + in % high;
    n = in / high;
    return true;
}

}  // namespace gemm
}  // namespace cgx
