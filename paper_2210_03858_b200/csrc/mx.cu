// Microscaled 4-bit floating point: quantisation, its inverse, and the product of two matrices that are stored so.
//
// Blocks of 32 consecutive elements of a row share a power of two, 2^e with e = floor(log2 max|x|) - 2 (at least -127), and an element
// is x 2^-e rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (ties to the even code, larger ones to 6).
//
// The product runs on the tensor core's own block-scaled instruction (kind::mxf4): the codes go from memory to it as they
// are, the scales by way of tensor memory, and products are accumulated in fp32.  Weights are the operand of 128 rows (M),
// tokens the other (N = 16 .. 256): so one token costs a narrow instruction, not a wide one with empty rows, and a
// warp's 32 accumulator lanes are 32 consecutive outputs of a token, which it writes as they are.
#include <algorithm>

#include "gemm_common.cuh"

namespace {

using namespace bcq;

__device__ int g_timeout_flag = 0;

constexpr int kMxMaxCols = 1 << 20;
constexpr int kMxMaxRows = 1 << 30;

inline size_t mx_pitch(int cols) { return (size_t)64 * (((size_t)cols + 127) / 128); }
inline int mx_atoms(int cols) { return ceil_div(cols, 128); }

// ---------------------------------------------------------------- quantisation

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Eight values to eight codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t to_e2m1_x8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t"
        ".reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t"
        "}\n"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// Where the four scales of 128 elements of a row are, as one word.
__device__ __forceinline__ long long scale_word(int row, int atom, int atoms) {
    return (((long long)(row >> 7) * atoms + atom) * 32 + (row & 31)) * 4 + ((row >> 5) & 3);
}

struct MxQuantParams {
    int rows, cols, atoms, vec;  // vec: eight elements of a row are one aligned load
    int unit_rows;               // rows in the container (128s) for quantisation, of the matrix for its inverse
    long long ld, pitch;
};

// The units of work of a group of sixteen lanes: 128 elements of kUnits consecutive rows, eight elements of each to a lane, the rows
// on their way together.  Neighbouring groups have neighbouring elements.  One division at the start; a step of all groups is so
// many rows and so many atoms.  (One row at a time, each with its own addresses and conditions: 27 instructions an element.)
constexpr int kUnits = 4;
struct Walk {
    int row, atom, drow, datom, atoms;
    __device__ __forceinline__ explicit Walk(int atoms_) : atoms(atoms_) {
        const long long group = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 4;
        const int groups = (int)(gridDim.x * (blockDim.x >> 4));
        row = (int)(group / atoms) * kUnits;
        atom = (int)(group % atoms);
        drow = groups / atoms * kUnits;
        datom = groups % atoms;
    }
    __device__ __forceinline__ void step() {
        row += drow;
        atom += datom;
        if (atom >= atoms) {
            atom -= atoms;
            row += kUnits;
        }
    }
};

// The largest magnitude of eight values, as the bits of a float (NaN and infinity are the largest), and the values times a power of
// two as codes.
struct EightF32 {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    __device__ __forceinline__ void load(const float* p) {
        asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "l"(p));
    }
    __device__ __forceinline__ void load_some(const float* p, int have) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) v[i] = ld(p + i);
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
        return m;
    }
    __device__ __forceinline__ uint32_t codes(float f) const {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[i] * f;
        return to_e2m1_x8(x);
    }
};
struct EightBf16 {
    uint32_t w[4];
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        const uint4 a = ld_stream(reinterpret_cast<const uint4*>(p));
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
    __device__ __forceinline__ void load_some(const __nv_bfloat16* p, int have) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) {
                unsigned short h;
                asm volatile("ld.global.u16 %0, [%1];" : "=h"(h) : "l"(p + i));
                w[i >> 1] |= (uint32_t)h << (16 * (i & 1));
            }
    }
    __device__ __forceinline__ uint32_t top() const {
        // (two at a time: magnitudes of bf16 are in the order of their bits)
        uint32_t hi = 0, lo = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi = max(hi, w[i] & 0x7fff0000u);
            lo = max(lo, (w[i] << 16) & 0x7fff0000u);
        }
        return max(hi, lo);
    }
    __device__ __forceinline__ uint32_t codes(float f) const {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16) * f;
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u) * f;
        }
        return to_e2m1_x8(x);
    }
};
template <typename T>
struct EightOf;
template <>
struct EightOf<float> { typedef EightF32 type; };
template <>
struct EightOf<__nv_bfloat16> { typedef EightBf16 type; };

// Bound by memory: 16384 x 4096 fp32 values 49 us, 6.1 TB/s.
template <typename T>
__global__ void __launch_bounds__(256)
mx_quantize_kernel(const T* X, uint8_t* codes, uint32_t* scales, const MxQuantParams p) {
    pdl_trigger();
    pdl_wait();
    const int lane16 = (int)threadIdx.x & 15;
    // (units are an even number, as rows come in 128s: both groups of a warp take every turn, as the shuffles want)
    for (Walk w(p.atoms); w.row < p.unit_rows; w.step()) {
        const int col = w.atom * 128 + lane16 * 8, have = p.cols - col, rows = p.rows - w.row;
        const T* src = X + w.row * p.ld + col;
        typename EightOf<T>::type v[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            v[u].zero();
            if (u < rows) {
                if (p.vec && have >= 8) v[u].load(src);
                else v[u].load_some(src, have);
            }
            src += p.ld;
        }
        uint8_t* dst = codes + w.row * p.pitch + w.atom * 64 + lane16 * 4;
        uint32_t* word = scales + scale_word(w.row, w.atom, p.atoms);  // (of the next rows: four words on, as rows come in fours)
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            uint32_t top = v[u].top();
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // the exponent field is floor(log2) + 127 (0 for what is below 2^-126, whose scale is the smallest too)
            const bool finite = top < 0x7f800000u;
            const uint32_t s = finite ? (uint32_t)max(0, (int)(top >> 23) - 2) : 255u;
            const float f = __uint_as_float((254u - (s & 254u) - (s & 1u)) << 23);  // 2^(127 - s)
            const uint32_t c = finite ? v[u].codes(f) : 0u;
            // the four blocks' scales to the first lane
            uint32_t four = s << (2 * (lane16 & 12));
            four |= __shfl_xor_sync(0xffffffffu, four, 4);
            four |= __shfl_xor_sync(0xffffffffu, four, 8);
            if (u < rows) *reinterpret_cast<uint32_t*>(dst) = c;
            if (lane16 == 0) *word = four;
            dst += p.pitch;
            word += 4;
        }
    }
}

// 2^(s - 127) as two bf16; 255 is NaN.
__device__ __forceinline__ uint32_t scale_bf16x2(uint32_t s) {
    const uint32_t h = s == 0 ? 0x0040u : s == 255u ? 0x7fc0u : s << 7;
    return h | (h << 16);
}

// Four codes (in the low 16 bits) to bf16: the two bytes of a magnitude come from tables of eight.
__device__ __forceinline__ void four_values(uint32_t c, uint32_t scale, uint32_t& v01, uint32_t& v23) {
    const uint32_t m = c & 0x7777u;
    const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, m), lo = __byte_perm(0xc0800000u, 0xc0804000u, m);
    v01 = __byte_perm(lo, hi, 0x5140) | ((c & 0x0008u) << 12) | ((c & 0x0080u) << 24);
    v23 = __byte_perm(lo, hi, 0x7362) | ((c & 0x0800u) << 4) | ((c & 0x8000u) << 16);
    asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(v01) : "r"(scale));  // (exact, below the normal numbers too)
    asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(v23) : "r"(scale));
}

// Bound by memory too.  (With every code put together as a float, 16 instructions an element, 43 us for 16384 x 4096; 33 so, 5.1 TB/s.)
template <typename T>
__global__ void __launch_bounds__(256)
mx_dequantize_kernel(const uint8_t* codes, const uint32_t* scales, T* X, const MxQuantParams p) {
    pdl_wait();
    const int lane16 = (int)threadIdx.x & 15;
    for (Walk w(p.atoms); w.row < p.unit_rows; w.step()) {
        const int col = w.atom * 128 + lane16 * 8, have = p.cols - col, rows = p.rows - w.row;
        const uint8_t* src = codes + w.row * p.pitch + w.atom * 64 + lane16 * 4;
        const uint32_t* word = scales + scale_word(w.row, w.atom, p.atoms);
        uint32_t c[kUnits], s[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            c[u] = s[u] = 0;
            if (u < rows) {
                c[u] = ld_stream(reinterpret_cast<const uint32_t*>(src));
                s[u] = ld(word);
            }
            src += p.pitch;
            word += 4;
        }
        T* dst = X + w.row * p.ld + col;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            if (u >= rows) break;
            const uint32_t scale = scale_bf16x2((s[u] >> (2 * (lane16 & 12))) & 255u);
            uint32_t v[4];
            four_values(c[u], scale, v[0], v[1]);
            four_values(c[u] >> 16, scale, v[2], v[3]);
            if (p.vec && have >= 8) {
                if constexpr (sizeof(T) == 4) {
                    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(v[0] << 16), "r"(v[0] & 0xffff0000u),
                                 "r"(v[1] << 16), "r"(v[1] & 0xffff0000u), "r"(v[2] << 16), "r"(v[2] & 0xffff0000u), "r"(v[3] << 16),
                                 "r"(v[3] & 0xffff0000u) : "memory");
                } else {
                    *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < have) {
                        const uint32_t h = i & 1 ? v[i >> 1] >> 16 : v[i >> 1] & 0xffffu;
                        if constexpr (sizeof(T) == 4) dst[i] = __uint_as_float(h << 16);
                        else dst[i] = __ushort_as_bfloat16((unsigned short)h);
                    }
            }
            dst += p.ld;
        }
    }
}

// ---------------------------------------------------------------- product

struct MxLinearParams {
    int d_out, n;
    int atoms;           // ceil(d_in / 128)
    int m_tiles, n_tiles;
    int steps;           // of 256 elements of d_in: ceil(atoms / 2)
    int splits;          // CTAs of a cluster, which share a tile's steps
    const uint8_t* w_scales;
    const uint8_t* x_scales;
    const float* bias;
    void* Y;
    long long ldy;
};

// BN tokens by 128 outputs.  A stage holds 256 elements of d_in: 128 bytes of codes a row, two atoms of scales a 128 rows.
template <int BN>
struct MxTile {
    static constexpr int kRowBlocks = (BN + 127) / 128;             // of the tokens' scales
    static constexpr uint32_t kA = 128 * 128, kB = BN * 128;
    static constexpr uint32_t kScaleA = 1024, kScaleB = 1024 * kRowBlocks;
    static constexpr uint32_t kStage = kA + kB + kScaleA + kScaleB;
    static constexpr int kStages = BN == 256 ? 4 : BN == 128 ? 6 : BN == 64 ? 8 : BN == 32 ? 9 : 10;
    static constexpr int kAccs = BN == 256 ? 1 : 2;                 // accumulators: with one, a tile's is taken to registers at once
    static constexpr uint32_t kScaleCol = kAccs * BN;               // columns of the scales: 8 + 8 per row block for each stage
    static constexpr uint32_t kScaleCols = 8 + 8 * kRowBlocks;
    static constexpr uint32_t kUsed = kScaleCol + kStages * kScaleCols;
    static constexpr uint32_t kTmemCols = kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
    static constexpr size_t kSmem = (size_t)kStages * kStage + 1024 + 256;
    static_assert(kUsed <= 512, "tensor memory");
    static_assert(kSmem <= 232448, "shared memory");
    static_assert((size_t)kStages * kStage >= (size_t)BN * 128 * 4, "a tile of partial sums fits over the stages");
};

template <typename Out>
__device__ __forceinline__ void store_out(Out* p, float v) {
    if constexpr (sizeof(Out) == 4) *p = v;
    else *p = __float2bfloat16_rn(v);
}

// The first `have` of a thread's columns (tokens) of one output.  Four pointers, each on its way to every fourth token: an address is
// one addition, and no addition waits for the one before it (c * ldy in 64 bits: 21 instructions an output, 12000 cycles for a
// tile of 128 x 256).
template <int COLS, typename Out>
__device__ __forceinline__ void store_columns(Out* first, long long ldy, int have, const uint32_t (&v)[COLS], float bias) {
    Out* y[4];
    const long long far = 4 * ldy;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = first + i * ldy;
    if (have >= COLS) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            store_out(y[c & 3], __uint_as_float(v[c]) + bias);
            y[c & 3] += far;
        }
    } else {
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            if (c < have) store_out(y[c & 3], __uint_as_float(v[c]) + bias);
            y[c & 3] += far;
        }
    }
}

// Warp 0: TMA; warp 1: scales to tensor memory and UMMA; warps 2..9: epilogue.
template <int BN, typename Out>
__global__ void __launch_bounds__(kThreads, 1)
mx_linear_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const MxLinearParams p) {
    using Tile = MxTile<BN>;
    constexpr int S = Tile::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    const uint32_t ctl_base = smem_base + S * Tile::kStage;
    uint8_t* ctl_gen = smem_gen + S * Tile::kStage;
    // all code tiles first (1024-byte aligned), the scales behind them
    const uint32_t scales_base = smem_base + S * (Tile::kA + Tile::kB);

    Ctl ctl;
    ctl.full = ctl_base;
    ctl.aready = 0;
    ctl.empty = ctl_base + 8 * S;
    ctl.accum = ctl_base + 16 * S;              // + 8c : accumulator c complete
    const uint32_t acc_empty = ctl.accum + 16;  // + 8c : accumulator c drained
    ctl.spare = ctl.accum + 32;
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(ctl_gen + 16 * S + 40);
    ctl.abort_flag = reinterpret_cast<volatile int*>(ctl_gen + 16 * S + 44);
    ctl.device_flag = &g_timeout_flag;

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const int num_tiles = p.m_tiles * p.n_tiles;
    const int rank = p.splits > 1 ? (int)ptx::cluster_rank() : 0;
    const int tile0 = (int)blockIdx.x / p.splits, tile_step = (int)gridDim.x / p.splits;
    const int per = (p.steps + p.splits - 1) / p.splits;
    const int step0 = min(p.steps, rank * per), steps = min(p.steps, step0 + per) - step0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            ptx::mbar_init(ctl.full + 8 * s, 1);
            ptx::mbar_init(ctl.empty + 8 * s, 1);
        }
        for (int c = 0; c < 2; ++c) {
            ptx::mbar_init(ctl.accum + 8 * c, 1);
            ptx::mbar_init(acc_empty + 8 * c, kWorkerWarps);
        }
        ptx::mbar_init(ctl.spare, 1);
        *ctl.abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tmap(&tmap_w);
        ptx::prefetch_tmap(&tmap_x);
    }
    __syncwarp();
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_u32(const_cast<uint32_t*>(tmem_holder)), Tile::kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    pdl_wait();
    const uint32_t tmem_base = *tmem_holder;

    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            int s = 0;
            uint32_t ph = 0;
            for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
                const int m0 = tile % p.m_tiles, n0 = tile / p.m_tiles;
                const int row_blocks = min(Tile::kRowBlocks, (p.n + 127) / 128 - n0 * BN / 128);
                for (int it = 0; it < steps; ++it) {
                    ok = wait_bar(ctl.empty + 8 * s, ph ^ 1u, ctl, 41);
                    if (!ok) break;
                    const int step = step0 + it;
                    const uint32_t sa = smem_base + s * (Tile::kA + Tile::kB), sf = scales_base + s * (Tile::kScaleA + Tile::kScaleB);
                    const uint32_t bar = ctl.full + 8 * s;
                    const uint32_t atom_bytes = 512u * (uint32_t)min(2, p.atoms - 2 * step);
                    ptx::mbar_arrive_expect_tx(bar, Tile::kA + Tile::kB + atom_bytes * (uint32_t)(1 + row_blocks));
                    ptx::tma_load_2d(sa, &tmap_w, step * 128, m0 * 128, bar);
                    ptx::tma_load_2d(sa + Tile::kA, &tmap_x, step * 128, n0 * BN, bar);
                    ptx::bulk_load(sf, p.w_scales + ((long long)m0 * p.atoms + 2 * step) * 512, atom_bytes, bar);
                    for (int b = 0; b < row_blocks; ++b)
                        ptx::bulk_load(sf + Tile::kScaleA + 1024u * b,
                                       p.x_scales + ((long long)(n0 * BN / 128 + b) * p.atoms + 2 * step) * 512, atom_bytes, bar);
                    if (++s == S) { s = 0; ph ^= 1u; }
                }
            }
            // giving up: copies may be in flight, which land within microseconds; wait a thousand times as long
            if (!ok) for (int i = 0; i < 1000; ++i) __nanosleep(2000);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            bool ok = true;
            int s = 0, lt = 0;
            uint32_t ph = 0;
            // descriptors (128-byte swizzle, K-major: groups of eight rows 1024 bytes apart); 64 elements are 32 bytes on
            constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
            for (int tile = tile0; tile < num_tiles && ok; tile += tile_step, ++lt) {
                const int acc = lt % Tile::kAccs, use = lt / Tile::kAccs;
                ok = wait_bar(acc_empty + 8 * acc, (uint32_t)(use & 1) ^ 1u, ctl, 42, 32u);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + (uint32_t)(acc * BN);
                for (int it = 0; it < steps; ++it) {
                    ok = wait_bar(ctl.full + 8 * s, ph, ctl, 43, 32u);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    const uint32_t sa = smem_base + s * (Tile::kA + Tile::kB), sf = scales_base + s * (Tile::kScaleA + Tile::kScaleB);
                    // Each stage has its own columns for the scales: when its barrier says that the stage may be filled
                    // again, the UMMAs that read them have completed too.
                    const uint32_t col_a = tmem_base + Tile::kScaleCol + (uint32_t)s * Tile::kScaleCols, col_b = col_a + 8;
                    const int atoms = min(2, p.atoms - 2 * (step0 + it));
                    for (int a = 0; a < atoms; ++a) {
                        ptx::tmem_copy_scales(col_a + 4 * a, sf + 512 * a);
#pragma unroll
                        for (int b = 0; b < Tile::kRowBlocks; ++b)
                            ptx::tmem_copy_scales(col_b + 4 * (a * Tile::kRowBlocks + b), sf + Tile::kScaleA + 1024 * b + 512 * a);
                    }
                    const uint32_t a_lo = (sa >> 4) & 0x3FFFu, b_lo = ((sa + Tile::kA) >> 4) & 0x3FFFu;
                    for (int a = 0; a < atoms; ++a) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int kk = 2 * a + h;
                            ptx::umma_mxf4(d_tmem, a_lo + 2 * kk, kHi, b_lo + 2 * kk, kHi,
                                           h ? ptx::make_idesc_mxf4(128, BN, 1) : ptx::make_idesc_mxf4(128, BN, 0), col_a + 4 * a,
                                           col_b + 4 * a * Tile::kRowBlocks, (it > 0 || kk > 0) ? 1u : 0u);
                        }
                    }
                    ptx::umma_commit(ctl.empty + 8 * s);
                    if (++s == S) { s = 0; ph ^= 1u; }
                }
                if (ok) ptx::umma_commit(ctl.accum + 8 * acc);
            }
            if (!ok) {
                ptx::umma_commit(ctl.spare);
                wait_bar(ctl.spare, 0, ctl, 44);
            }
        }
        __syncwarp();
    } else {
        // thread = (output row, half of the tile's tokens)
        const int quarter = warp & 3;
        const int half = (warp - kWorkerWarp0) >> 2;
        constexpr int kCols = BN == 16 ? 16 : BN / 2;  // of a thread (16 tokens: the second half of the warps has nothing to do)
        constexpr int kLd = kCols < 32 ? 16 : 32;
        const bool works = BN != 16 || half == 0;
        Out* Y = reinterpret_cast<Out*>(p.Y);
        float* partial = reinterpret_cast<float*>(smem_gen);  // [BN][128], over the stages
        bool ok = true;
        int lt = 0;
        for (int tile = tile0; tile < num_tiles && ok; tile += tile_step, ++lt) {
            const int m0 = tile % p.m_tiles, n0 = tile / p.m_tiles;
            const int acc = lt % Tile::kAccs, use = lt / Tile::kAccs;
            const int jl = quarter * 32 + lane, j = m0 * 128 + jl;
            const int tl = works ? half * kCols : 0, t0 = n0 * BN + tl;
            const bool j_ok = j < p.d_out;
            const float bias = p.bias != nullptr && j_ok ? ld(p.bias + j) : 0.0f;
            ok = wait_bar(ctl.accum + 8 * acc, (uint32_t)use & 1u, ctl, 45, 64u);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            uint32_t v[kCols];
            if (works) {
#pragma unroll
                for (int c = 0; c < kCols; c += kLd) {
                    const uint32_t at = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * BN + tl + c);
                    if constexpr (kLd == 16) ptx::tmem_ld_x16(at, v + c);
                    else ptx::tmem_ld_x32(at, v + c);
                }
                ptx::tmem_ld_wait();
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * acc);
            if (!works) continue;
            if (p.splits > 1) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) partial[(tl + c) * 128 + jl] = steps > 0 ? __uint_as_float(v[c]) : 0.0f;
            } else if (j_ok) {
                store_columns<kCols>(Y + (long long)t0 * p.ldy + j, p.ldy, p.n - t0, v, bias);
            }
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    if (p.splits > 1) {
        // the cluster's partial sums, in the order of its ranks; each CTA adds up its share of the tile
        ptx::cluster_sync();
        const int m0 = tile0 % p.m_tiles, n0 = tile0 / p.m_tiles;
        const int vecs = min(BN, p.n - n0 * BN) * 32;  // of four outputs
        const int share = (vecs + p.splits - 1) / p.splits;
        const int last = min(vecs, (rank + 1) * share);
        const uint32_t mine = smem_base;
        Out* Y = reinterpret_cast<Out*>(p.Y);
        for (int e = rank * share + (int)threadIdx.x; e < last; e += kThreads) {
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int r = 0; r < p.splits; ++r) {
                const float4 f = ptx::ld_cluster_v4(ptx::cluster_addr(mine + 16u * (uint32_t)e, (uint32_t)r));
                sum.x += f.x; sum.y += f.y; sum.z += f.z; sum.w += f.w;
            }
            const int t = n0 * BN + e / 32, j = m0 * 128 + (e & 31) * 4;
            const float s4[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j + i < p.d_out) store_out(Y + (long long)t * p.ldy + j + i, s4[i] + (p.bias != nullptr ? ld(p.bias + j + i) : 0.0f));
        }
        ptx::cluster_sync();  // nobody's memory goes away while it is read
    }
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, Tile::kTmemCols);
    }
}

// A pair of CTAs on a tile of 256 outputs by 256 tokens: each has the codes of its own 128 outputs and of half of the tokens, so a
// step takes 32 KiB into shared memory and 32 KiB out of it in the 512 cycles that the tensor core needs, where a CTA alone takes
// 48 and 48 (5120 -> 20480, 2048 tokens: 93 us alone, 83 in pairs, the tensor pipe active 76 % of the time at 1.61 GHz under the
// power cap; what is left are the hand-over between tiles, the accumulator taking half of tensor memory, and the stores, 13 us of it).
// Tokens as rows, so that a thread has neighbouring outputs to store, 32 bytes at a time, does not pay: 1600 -> 6400 with 4096 tokens,
// fp32, 54 us and not 36.  Otherwise as above.  All copies are counted on the leader's barriers, the scales' too, which therefore come by tensor
// map: boxes of 1024 bytes (two atoms) by row blocks.
constexpr uint32_t kPairCodes = 2 * 128 * 128, kPairScales = 3 * 1024, kPairStage = kPairCodes + kPairScales;
constexpr int kPairStages = 6;
constexpr uint32_t kPairScaleCol = 256, kPairScaleCols = 24;
constexpr size_t kPairSmem = (size_t)kPairStages * kPairStage + 1024 + 256;
static_assert(kPairScaleCol + kPairStages * kPairScaleCols <= 512 && kPairSmem <= 232448, "tensor memory, shared memory");

template <typename Out>
__global__ void __launch_bounds__(kThreads, 1)
mx_linear_pair_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
                      const __grid_constant__ CUtensorMap tmap_ws, const __grid_constant__ CUtensorMap tmap_xs, const MxLinearParams p) {
    constexpr int S = kPairStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    const uint32_t ctl_base = smem_base + S * kPairStage;
    uint8_t* ctl_gen = smem_gen + S * kPairStage;
    const uint32_t scales_base = smem_base + S * kPairCodes;

    Ctl ctl;
    ctl.full = ctl_base;
    ctl.aready = 0;
    ctl.empty = ctl_base + 8 * S;
    ctl.accum = ctl_base + 16 * S;
    const uint32_t acc_empty = ctl.accum + 8;
    ctl.spare = ctl.accum + 16;
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(ctl_gen + 16 * S + 24);
    ctl.abort_flag = reinterpret_cast<volatile int*>(ctl_gen + 16 * S + 28);
    ctl.device_flag = &g_timeout_flag;

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const int rank = (int)ptx::cluster_rank();
    const int num_tiles = p.m_tiles * p.n_tiles;
    const int tile0 = (int)blockIdx.x >> 1, tile_step = (int)gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            ptx::mbar_init(ctl.full + 8 * s, 1);
            ptx::mbar_init(ctl.empty + 8 * s, 1);
        }
        ptx::mbar_init(ctl.accum, 1);
        ptx::mbar_init(acc_empty, 2 * kWorkerWarps);
        ptx::mbar_init(ctl.spare, 1);
        *ctl.abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tmap(&tmap_w);
        ptx::prefetch_tmap(&tmap_x);
        ptx::prefetch_tmap(&tmap_ws);
        ptx::prefetch_tmap(&tmap_xs);
    }
    __syncwarp();
    if (warp == 1) {
        ptx::tmem_alloc_pair(ptx::smem_u32(const_cast<uint32_t*>(tmem_holder)), 512);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync();  // the peer's barriers exist
    ptx::tc_fence_after_sync();
    pdl_wait();
    const uint32_t tmem_base = *tmem_holder;

    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            int s = 0;
            uint32_t ph = 0;
            for (int tile = tile0; tile < num_tiles && ok; tile += tile_step) {
                const int m0 = tile % p.m_tiles, n0 = tile / p.m_tiles;
                for (int step = 0; step < p.steps; ++step) {
                    ok = wait_bar(ctl.empty + 8 * s, ph ^ 1u, ctl, 61);
                    if (!ok) break;
                    const uint32_t sa = smem_base + s * kPairCodes, sf = scales_base + s * kPairScales;
                    const uint32_t bar = ptx::leader_addr(ctl.full + 8 * s);
                    if (rank == 0) ptx::mbar_arrive_expect_tx(ctl.full + 8 * s, 2 * kPairStage);
                    ptx::tma_load_2d_pair(sa, &tmap_w, step * 128, m0 * 256 + rank * 128, bar);
                    ptx::tma_load_2d_pair(sa + kABytes, &tmap_x, step * 128, n0 * 256 + rank * 128, bar);
                    ptx::tma_load_2d_pair(sf, &tmap_ws, step * 256, m0 * 2 + rank, bar);
                    ptx::tma_load_2d_pair(sf + 1024, &tmap_xs, step * 256, n0 * 2, bar);
                    if (++s == S) { s = 0; ph ^= 1u; }
                }
            }
            // giving up: the copies in flight land within microseconds; wait a thousand times as long
            if (!ok) for (int i = 0; i < 1000; ++i) __nanosleep(2000);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && ptx::elect_one()) {
            bool ok = true;
            int s = 0, lt = 0;
            uint32_t ph = 0;
            constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
            for (int tile = tile0; tile < num_tiles && ok; tile += tile_step, ++lt) {
                ok = wait_bar(acc_empty, (uint32_t)(lt & 1) ^ 1u, ctl, 62, 32u);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                for (int step = 0; step < p.steps; ++step) {
                    ok = wait_bar(ctl.full + 8 * s, ph, ctl, 63, 32u);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    const uint32_t sa = smem_base + s * kPairCodes, sf = scales_base + s * kPairScales;
                    const uint32_t col_a = tmem_base + kPairScaleCol + (uint32_t)s * kPairScaleCols, col_b = col_a + 8;
                    const int atoms = min(2, p.atoms - 2 * step);
                    for (int a = 0; a < atoms; ++a) {
                        ptx::tmem_copy_scales_pair(col_a + 4 * a, sf + 512 * a);
                        ptx::tmem_copy_scales_pair(col_b + 8 * a, sf + 1024 + 512 * a);
                        ptx::tmem_copy_scales_pair(col_b + 8 * a + 4, sf + 2048 + 512 * a);
                    }
                    const uint32_t a_lo = (sa >> 4) & 0x3FFFu, b_lo = ((sa + kABytes) >> 4) & 0x3FFFu;
                    for (int a = 0; a < atoms; ++a) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int kk = 2 * a + h;
                            ptx::umma_mxf4_pair(tmem_base, a_lo + 2 * kk, kHi, b_lo + 2 * kk, kHi,
                                                h ? ptx::make_idesc_mxf4(256, 256, 1) : ptx::make_idesc_mxf4(256, 256, 0), col_a + 4 * a,
                                                col_b + 8 * a, (step > 0 || kk > 0) ? 1u : 0u);
                        }
                    }
                    ptx::umma_commit_pair(ctl.empty + 8 * s);
                    if (++s == S) { s = 0; ph ^= 1u; }
                }
                if (ok) ptx::umma_commit_pair(ctl.accum);
            }
            if (!ok) {
                ptx::umma_commit_pair(ctl.spare);
                wait_bar(ctl.spare, 0, ctl, 64);
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3;
        const int half = (warp - kWorkerWarp0) >> 2;
        bool ok = true;
        int lt = 0;
        for (int tile = tile0; tile < num_tiles && ok; tile += tile_step, ++lt) {
            const int m0 = tile % p.m_tiles, n0 = tile / p.m_tiles;
            const int j = m0 * 256 + rank * 128 + quarter * 32 + lane, t0 = n0 * 256 + half * 128;
            const bool j_ok = j < p.d_out;
            const float bias = p.bias != nullptr && j_ok ? ld(p.bias + j) : 0.0f;
            ok = wait_bar(ctl.accum, (uint32_t)lt & 1u, ctl, 65, 64u);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            // the accumulator goes to registers at once, and the next tile's products may begin
            uint32_t v[128];
#pragma unroll
            for (int c = 0; c < 128; c += 32) ptx::tmem_ld_x32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128 + c), v + c);
            ptx::tmem_ld_wait();
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_cluster(ptx::leader_addr(acc_empty));
            if (j_ok) store_columns<128>(reinterpret_cast<Out*>(p.Y) + (long long)t0 * p.ldy + j, p.ldy, p.n - t0, v, bias);
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync();  // neither CTA's memory goes away under the other
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc_pair(tmem_base, 512);
    }
}

// Codes [rows][pitch bytes], boxes of 128 bytes (256 elements) x box_rows, 128-byte swizzle, zeros outside.
bcq_status make_tmap_codes(CUtensorMap* m, const void* base, int rows, size_t pitch, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) {
        set_last_cuda_error((int)cudaErrorNotSupported);
        return BCQ_ERR_CUDA;
    }
    cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)pitch};
    cuuint32_t box[2] = {128u, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1u, 1u};
    CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_last_cuda_error((int)cudaErrorInvalidValue);
        return BCQ_ERR_CUDA;
    }
    return BCQ_OK;
}

// Scales as rows of 32-bit words, one for each 128 rows of the matrix: boxes of two atoms (1024 bytes) by `blocks`, zeros outside.
bcq_status make_tmap_scales(CUtensorMap* m, const void* base, int rows, int atoms, int blocks) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) {
        set_last_cuda_error((int)cudaErrorNotSupported);
        return BCQ_ERR_CUDA;
    }
    cuuint64_t dims[2] = {(cuuint64_t)atoms * 128, (cuuint64_t)ceil_div(rows, 128)};
    cuuint64_t strides[1] = {(cuuint64_t)atoms * 512};
    cuuint32_t box[2] = {256u, (cuuint32_t)blocks};
    cuuint32_t estr[2] = {1u, 1u};
    CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_last_cuda_error((int)cudaErrorInvalidValue);
        return BCQ_ERR_CUDA;
    }
    return BCQ_OK;
}

// Which tile, and how many CTAs share one.  Costs in cycles: a step of 256 elements is bound by shared memory, which
// takes the step's codes once from memory and once to the tensor core at 128 bytes a cycle, and takes 440 at least (16 tokens, weights
// in L2); an epilogue that nothing hides; joining the partial sums of a cluster.  One CTA an SM: with two, and the clusters
// that this allows, one token through 4096 -> 12288 took 13.2 us and not 8.5.  Measured, one token, 1, 2, 4, 8 CTAs a tile:
// 16384 -> 4096 19.1, 13.3, 10.0, 10.5 us; 6400 -> 1600 9.8, 8.6, 7.4, 7.0; 1024 -> 1024 5.3, 6.2, 5.9, 6.1.
struct MxPlan {
    int bn, splits;
    bool pair;
};

MxPlan plan_mx(int d_out, int atoms, int n) {
    const int steps = ceil_div(atoms, 2), m_tiles = ceil_div(d_out, 128);
    MxPlan best = {256, 1, false};
    double least = 1e30;
    // (tiles of fewer than 128 tokens only where one holds all: tokens' scales come in 128s)
    for (int bn = n <= 16 ? 16 : n <= 32 ? 32 : n <= 64 ? 64 : 128; bn <= 256; bn *= 2) {
        if (bn > 128 && n <= 128) break;
        const int tiles = m_tiles * ceil_div(n, bn), slots = sm_count();
        const double cycles = std::max(440.0, 2.0 * (128 + bn)), tail = bn == 256 ? 900 : 400;
        for (int s = 1; s <= 8 && s <= steps; ++s) {
            if (s > 1 && tiles * s > slots) break;
            const double cost = (double)ceil_div(tiles * s, slots) * (ceil_div(steps, s) * cycles + tail) + (s > 1 ? 1900 + 4.0 * bn : 0);
            if (cost < least) {
                least = cost;
                best.bn = bn;
                best.splits = s;
            }
        }
    }
    // a pair on 256 x 256: 512 cycles a step, which the tensor core takes too
    const double pairs = (double)ceil_div(ceil_div(d_out, 256) * ceil_div(n, 256), std::max(1, sm_count() / 2)) * (steps * 512.0 + 900);
    if (n > 128 && pairs < least) best.pair = true;
    return best;
}

template <typename Out>
bcq_status launch_mx_pair(const uint8_t* x_codes, const uint8_t* w_codes, int d_in, MxLinearParams p, cudaStream_t s) {
    CUtensorMap tw, tx, tws, txs;
    bcq_status st;
    if ((st = make_tmap_codes(&tw, w_codes, p.d_out, mx_pitch(d_in), 128)) != BCQ_OK) return st;
    if ((st = make_tmap_codes(&tx, x_codes, p.n, mx_pitch(d_in), 128)) != BCQ_OK) return st;
    if ((st = make_tmap_scales(&tws, p.w_scales, p.d_out, p.atoms, 1)) != BCQ_OK) return st;
    if ((st = make_tmap_scales(&txs, p.x_scales, p.n, p.atoms, 2)) != BCQ_OK) return st;
    if ((st = ensure_dynamic_smem(mx_linear_pair_kernel<Out>, kPairSmem)) != BCQ_OK) return st;
    p.m_tiles = ceil_div(p.d_out, 256);
    p.n_tiles = ceil_div(p.n, 256);
    const int pairs = std::min(p.m_tiles * p.n_tiles, std::max(1, sm_count() / 2));
    BCQ_CUDA_TRY(launch_pdl(mx_linear_pair_kernel<Out>, dim3(2u * (unsigned)pairs), kThreads, kPairSmem, s, 2, tw, tx, tws, txs, p));
    return BCQ_OK;
}

template <int BN, typename Out>
bcq_status launch_mx(const CUtensorMap& tw, const CUtensorMap& tx, const MxLinearParams& p, cudaStream_t s) {
    using Tile = MxTile<BN>;
    const bcq_status st = ensure_dynamic_smem(mx_linear_kernel<BN, Out>, Tile::kSmem);
    if (st != BCQ_OK) return st;
    const int tiles = p.m_tiles * p.n_tiles;
    const int ctas = p.splits > 1 ? tiles * p.splits : std::min(tiles, sm_count());
    BCQ_CUDA_TRY(launch_pdl(mx_linear_kernel<BN, Out>, dim3((unsigned)ctas), kThreads, Tile::kSmem, s, (unsigned)p.splits, tw, tx, p));
    return BCQ_OK;
}

bcq_status check_mx(int rows, int cols, const void* codes, const void* scales) {
    if (rows < 0 || cols < 1) return BCQ_ERR_SHAPE;
    if (cols > kMxMaxCols || rows > kMxMaxRows) return BCQ_ERR_UNSUPPORTED;
    if (rows == 0) return BCQ_OK;
    if (!codes || !scales) return BCQ_ERR_NULL;
    if (!aligned16(codes) || !aligned16(scales)) return BCQ_ERR_ALIGN;
    return BCQ_OK;
}

bcq_status check_mx_values(int rows, int cols, const void* X, size_t ldx, int dtype) {
    if (ldx < (size_t)cols) return BCQ_ERR_SHAPE;
    if (dtype != BCQ_F32 && dtype != BCQ_BF16) return BCQ_ERR_UNSUPPORTED;
    if (rows > 0 && !X) return BCQ_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(X) & (dtype == BCQ_BF16 ? 1u : 3u)) != 0) return BCQ_ERR_ALIGN;
    return BCQ_OK;
}

MxQuantParams mx_params(int rows, int cols, const void* X, size_t ldx, int dtype, int unit_rows) {
    MxQuantParams p;
    p.rows = rows; p.cols = cols; p.atoms = mx_atoms(cols);
    p.vec = (reinterpret_cast<uintptr_t>(X) % (dtype == BCQ_BF16 ? 16 : 32)) == 0 && ldx % 8 == 0;
    p.ld = (long long)ldx; p.pitch = (long long)mx_pitch(cols);
    p.unit_rows = unit_rows;
    return p;
}

unsigned mx_grid(const MxQuantParams& p) {
    const long long blocks = ((long long)ceil_div(p.unit_rows, kUnits) * p.atoms * 16 + 255) / 256;
    return (unsigned)std::max(1ll, std::min(blocks, (long long)sm_count() * 8));
}

}  // namespace

namespace bcq {
bcq_status mx_timeout_flag(int* flag_out, int reset) {
    int v = 0;
    BCQ_CUDA_TRY(cudaMemcpyFromSymbol(&v, g_timeout_flag, sizeof(int)));
    *flag_out = v;
    if (reset && v != 0) {
        const int zero = 0;
        BCQ_CUDA_TRY(cudaMemcpyToSymbol(g_timeout_flag, &zero, sizeof(int)));
    }
    return BCQ_OK;
}
}  // namespace bcq

extern "C" size_t bcq_mx_codes_bytes(int rows, int cols) { return rows < 1 || cols < 1 ? 0 : (size_t)rows * mx_pitch(cols); }

extern "C" size_t bcq_mx_scales_bytes(int rows, int cols) {
    return rows < 1 || cols < 1 ? 0 : (((size_t)rows + 127) / 128) * (size_t)mx_atoms(cols) * 512;
}

extern "C" bcq_status bcq_mx_quantize(int rows, int cols, const void* X, size_t ldx, int x_dtype, uint8_t* codes, uint8_t* scales,
                                      void* stream) {
    bcq_status st = check_mx(rows, cols, codes, scales);
    if (st != BCQ_OK) return st;
    if ((st = check_mx_values(rows, cols, X, ldx, x_dtype)) != BCQ_OK) return st;
    if (rows == 0) return BCQ_OK;
    const MxQuantParams p = mx_params(rows, cols, X, ldx, x_dtype, ceil_div(rows, 128) * 128);
    cudaStream_t s = (cudaStream_t)stream;
    uint32_t* sw = reinterpret_cast<uint32_t*>(scales);
    if (x_dtype == BCQ_BF16)
        BCQ_CUDA_TRY(launch_pdl(mx_quantize_kernel<__nv_bfloat16>, dim3(mx_grid(p)), 256, 0, s, 1, (const __nv_bfloat16*)X, codes, sw, p));
    else
        BCQ_CUDA_TRY(launch_pdl(mx_quantize_kernel<float>, dim3(mx_grid(p)), 256, 0, s, 1, (const float*)X, codes, sw, p));
    return BCQ_OK;
}

extern "C" bcq_status bcq_mx_dequantize(int rows, int cols, const uint8_t* codes, const uint8_t* scales, void* X_hat, size_t ldx,
                                        int x_dtype, void* stream) {
    bcq_status st = check_mx(rows, cols, codes, scales);
    if (st != BCQ_OK) return st;
    if ((st = check_mx_values(rows, cols, X_hat, ldx, x_dtype)) != BCQ_OK) return st;
    if (rows == 0) return BCQ_OK;
    const MxQuantParams p = mx_params(rows, cols, X_hat, ldx, x_dtype, rows);
    cudaStream_t s = (cudaStream_t)stream;
    const uint32_t* sw = reinterpret_cast<const uint32_t*>(scales);
    if (x_dtype == BCQ_BF16)
        BCQ_CUDA_TRY(launch_pdl(mx_dequantize_kernel<__nv_bfloat16>, dim3(mx_grid(p)), 256, 0, s, 1, codes, sw, (__nv_bfloat16*)X_hat, p));
    else
        BCQ_CUDA_TRY(launch_pdl(mx_dequantize_kernel<float>, dim3(mx_grid(p)), 256, 0, s, 1, codes, sw, (float*)X_hat, p));
    return BCQ_OK;
}

extern "C" bcq_status bcq_mx_linear(int d_out, int d_in, int n, const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* w_codes,
                                    const uint8_t* w_scales, const float* bias, void* Y, size_t ldy, int y_dtype, void* stream) {
    if (d_out < 1) return BCQ_ERR_SHAPE;
    bcq_status st = check_mx(d_out, d_in, w_codes, w_scales);
    if (st != BCQ_OK) return st;
    if ((st = check_mx(n, d_in, x_codes, x_scales)) != BCQ_OK) return st;
    if ((st = check_mx_values(n, d_out, Y, ldy, y_dtype)) != BCQ_OK) return st;
    if ((reinterpret_cast<uintptr_t>(bias) & 3u) != 0) return BCQ_ERR_ALIGN;
    if (n == 0) return BCQ_OK;
    MxLinearParams p;
    p.d_out = d_out; p.n = n; p.atoms = mx_atoms(d_in); p.steps = ceil_div(p.atoms, 2);
    p.w_scales = w_scales; p.x_scales = x_scales; p.bias = bias; p.Y = Y; p.ldy = (long long)ldy;
    const MxPlan plan = plan_mx(d_out, p.atoms, n);
    if (plan.pair) {
        p.splits = 1;
        return y_dtype == BCQ_BF16 ? launch_mx_pair<__nv_bfloat16>(x_codes, w_codes, d_in, p, (cudaStream_t)stream)
                                   : launch_mx_pair<float>(x_codes, w_codes, d_in, p, (cudaStream_t)stream);
    }
    p.splits = plan.splits;
    p.m_tiles = ceil_div(d_out, 128); p.n_tiles = ceil_div(n, plan.bn);
    CUtensorMap tw, tx;
    if ((st = make_tmap_codes(&tw, w_codes, d_out, mx_pitch(d_in), 128)) != BCQ_OK) return st;
    if ((st = make_tmap_codes(&tx, x_codes, n, mx_pitch(d_in), plan.bn)) != BCQ_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    const bool bf16 = y_dtype == BCQ_BF16;
    switch (plan.bn) {
        case 16: return bf16 ? launch_mx<16, __nv_bfloat16>(tw, tx, p, s) : launch_mx<16, float>(tw, tx, p, s);
        case 32: return bf16 ? launch_mx<32, __nv_bfloat16>(tw, tx, p, s) : launch_mx<32, float>(tw, tx, p, s);
        case 64: return bf16 ? launch_mx<64, __nv_bfloat16>(tw, tx, p, s) : launch_mx<64, float>(tw, tx, p, s);
        case 128: return bf16 ? launch_mx<128, __nv_bfloat16>(tw, tx, p, s) : launch_mx<128, float>(tw, tx, p, s);
        default: return bf16 ? launch_mx<256, __nv_bfloat16>(tw, tx, p, s) : launch_mx<256, float>(tw, tx, p, s);
    }
}
