// Operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, and the
// distillation loss against a teacher's top log probabilities with its gradient.
//
// With c = log2(e) / T everything is a sum over a row of 2^(c x - b), b = c max x.  The kernels read a row once
// for its sums (and the gradient's once more, from L2 as far as it is still there): a thread keeps a running maximum and the sums that
// go with it, and rescales them when a batch of its vectors has a larger one, so no second pass is needed for the sums; the sums of
// threads, warps and CTAs are joined in a fixed order.  b is the rounded product and is subtracted everywhere (from a target, from an
// alternative), so its rounding error, which would be that of a probability, drops out (where it would be too large for that,
// |b| > 2^31, exponents are c (x - max x)).  What bounds them is memory: n vocab sizeof(T) bytes read (and written, for the gradient).
// Next to that is the issue of instructions: an element of bf16 costs a conversion, an exponential (16 a cycle and SM: 0.7 of the time
// its bytes take), half a product and half a sum for each result (two at a time, fma.rn.f32x2), a quarter of a maximum and half a
// clamp, and with everything that goes with a row 7.6 instructions (9.1 with products and sums one at a time).
// Measured: 2048 rows of 50304 in fp32, no list, 62 us, the rate of a copy; 4096 rows of 50257 in bf16, no list 66 us (95 %),
// 64 alternatives 103; the loss of 2048 rows of 50272 in fp32 69 us (91 %), of 50257 in bf16 49 us (64 %), with the gradient 93 us
// (68 %), in fp32 169 us (75 %).
//
// Rows start at any element (an odd vocabulary in bf16 leaves rows at odd addresses): the elements before the
// first and after the last whole 16-byte vector of a row belong to single threads.
//
// A row goes to a cluster of 1, 2, 4 or 8 CTAs, more where there are few rows: one row of 50257 elements is 100 KB, which
// one SM alone takes 3 us to bring in.
#include <cuda_bf16.h>

#include <cfloat>

#include <algorithm>
#include <type_traits>

#include "gemm_common.cuh"

namespace {

using namespace bcq;

constexpr int kVocabMax = 393216;
constexpr int kRowsMax = 1 << 30;
constexpr int kTopMax = 128;
constexpr int kBatch = 4;          // 16-byte vectors of a thread between two looks at the running maximum
constexpr float kFloor = -1000.0f; // exponents below are as good as this one (2^-1000 = 0), and 0 * -1000 is 0
constexpr int kCandidates = 2048;  // elements that may be as large as the k-th largest, and batches that hold some
constexpr float kLn2 = 0.693147180559945309f;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float quiet_nan() { return __int_as_float(0x7fc00000); }

// Two floats in a register pair, and the instructions of sm_100 that take them.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// The base of a sum with maximum m is the rounded product b = rn(m c) where it is at most this either way, and m c itself beyond, with
// exponents (x - m) c.  Subtracting b from c x leaves b's rounding error in the exponent, half a step of b: 2^6 at most, the same for
// all terms, so it drops out (sums are below 2^90 with it, and a logit next to m is a step of m away, so the exponents lose nothing).  Of
// a product of 1e10 it would be hundreds, and the sum infinite or 0.  (2^31 and not less, since masks of -1e9 are common: threads that
// see nothing else take 1.2 to 1.7 times as long with the other kind of base.)
constexpr float kNear = 2147483648.0f;
// Logits below this are as good as this one next to a base that is near, and times c it is finite.
constexpr float kLowest = -1.26765060e30f;  // -2^100

__device__ __forceinline__ bool is_near(float b) { return fabsf(b) <= kNear; }  // (not so for an infinite m)

// Exponent of 2 of an element x relative to the base of m, and that of a sum at the base of a when it is taken to the base of m,
// exactly what lies between the two bases.
__device__ __forceinline__ float rel(float x, float m, float c) {
    const float b = __fmul_rn(m, c);
    return is_near(b) ? fmaf(fmaxf(x, kLowest), c, -b) : (x - m) * c;
}
// What a near base leaves of m c (0 for one that is not near).
__device__ __forceinline__ float base_error(float m, float c) {
    const float b = __fmul_rn(m, c), e = fmaf(m, c, -b);
    return is_near(b) ? e : 0.0f;
}
// (without a branch: a row goes through some twenty of these one after the other)
__device__ __forceinline__ float rel_base(float a, float m, float c) {
    return (a - m) * c + (base_error(m, c) - base_error(a, c));
}

// ---------------------------------------------------------------- element types

template <typename T>
struct Elem;
template <>
struct Elem<float> {
    static constexpr int E = 4;  // of a 16-byte vector
    static constexpr uint32_t kMasked = 0xff800000u;
    static __device__ __forceinline__ float get(const float* p) { return ld(p); }
    static __device__ __forceinline__ float at(const uint4& v, int i) {
        return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
    }
    static __device__ __forceinline__ float max_of(const uint4& v) {
        return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float max_of4(const uint4* v) {
        return max_nan(max_nan(max_of(v[0]), max_of(v[1])), max_nan(max_of(v[2]), max_of(v[3])));
    }
    static __device__ __forceinline__ void clamp(uint4& v) {
        v.x = __float_as_uint(fmaxf(__uint_as_float(v.x), kLowest));
        v.y = __float_as_uint(fmaxf(__uint_as_float(v.y), kLowest));
        v.z = __float_as_uint(fmaxf(__uint_as_float(v.z), kLowest));
        v.w = __float_as_uint(fmaxf(__uint_as_float(v.w), kLowest));
    }
    static __device__ __forceinline__ void mask(uint4& v, uint32_t bits) {
        if (bits & 1u) v.x = kMasked;
        if (bits & 2u) v.y = kMasked;
        if (bits & 4u) v.z = kMasked;
        if (bits & 8u) v.w = kMasked;
    }
};
template <>
struct Elem<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t kMasked = 0xff80ff80u;
    static __device__ __forceinline__ float get(const __nv_bfloat16* p) {
        unsigned short h;
        asm volatile("ld.global.u16 %0, [%1];" : "=h"(h) : "l"(p));
        return __uint_as_float((uint32_t)h << 16);
    }
    static __device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    static __device__ __forceinline__ float at(const uint4& v, int i) {
        const uint32_t w = word(v, i >> 1);
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ uint32_t max2_of(const uint4& v) {
        return max_nan_bf16x2(max_nan_bf16x2(v.x, v.y), max_nan_bf16x2(v.z, v.w));
    }
    static __device__ __forceinline__ float max_of4(const uint4* v) {
        const uint32_t m = max_nan_bf16x2(max_nan_bf16x2(max2_of(v[0]), max2_of(v[1])), max_nan_bf16x2(max2_of(v[2]), max2_of(v[3])));
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t clamp2(uint32_t w) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0xf180f180u));  // -2^100
        return r;
    }
    static __device__ __forceinline__ void clamp(uint4& v) {
        v = make_uint4(clamp2(v.x), clamp2(v.y), clamp2(v.z), clamp2(v.w));
    }
    static __device__ __forceinline__ void mask(uint4& v, uint32_t bits) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (bits & (1u << (2 * i))) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
            if (bits & (2u << (2 * i))) w[i] = (w[i] & 0x0000ffffu) | 0xff800000u;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// The elements of a row that a CTA of its cluster has: whole vectors [v0, v1), and single elements at the ends of the row,
// one to a thread (element -1: none).
template <typename T>
struct Share {
    const T* row;
    int head;          // elements before the first whole vector of the row
    int v0, v1, nvec;  // vectors of this CTA, and of the row
    int single;        // this thread's
    int first, last;   // elements [first, last) of this CTA

    // 2^lg CTAs
    __device__ __forceinline__ Share(const T* row_, int vocab, int rank, int lg) : row(row_) {
        constexpr int E = Elem<T>::E;
        head = min(vocab, (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(row_) & 15u)) & 15u) / sizeof(T)));
        nvec = (vocab - head) / E;
        const int ctas = 1 << lg, per = (nvec + ctas - 1) >> lg;
        v0 = min(nvec, rank * per);
        v1 = min(nvec, v0 + per);
        const int tail0 = head + nvec * E, tid = (int)threadIdx.x;  // (a helper warp's threads come last and get none)
        single = -1;
        if (rank == 0 && tid < head) single = tid;
        if (rank == ctas - 1 && tid >= E && tid < E + (vocab - tail0)) single = tail0 + tid - E;  // (head < E)
        first = rank == 0 ? 0 : head + v0 * E;
        last = rank == ctas - 1 ? vocab : head + v1 * E;
    }
    __device__ __forceinline__ const uint4* vec(int v) const { return reinterpret_cast<const uint4*>(row + head) + v; }
};

// Sums of e and e z over a vector where the base is not near, or the thread has found nothing above -inf so far.
template <typename T>
__device__ __noinline__ float2 far_sums(uint4 v, float m, float c) {
    const float base = m == neg_inf() ? 0.0f : m;
    float2 r = make_float2(0.0f, 0.0f);
    for (int i = 0; i < Elem<T>::E; ++i) {
        const float z = fmaxf((Elem<T>::at(v, i) - base) * c, kFloor), e = ex2(z);
        r.x += e;
        r.y = fmaf(e, z, r.y);
    }
    return r;
}

// Running maximum and the sums relative to it.  ENTROPY: sum of e z too, z the exponent of e.
template <typename T, bool ENTROPY>
struct Running {
    float m = neg_inf();
    float s[2] = {0.0f, 0.0f}, t[2] = {0.0f, 0.0f};  // (two partial sums each)
    bool bad = false;                                // a NaN or +inf was seen

    __device__ __forceinline__ void raise(float x, float c) {
        if (x <= m) return;  // (not so with a NaN)
        if (x > m) {
            const float d = fmaxf(rel_base(m, x, c), kFloor), f = ex2(d);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (ENTROPY) t[i] = f * fmaf(d, s[i], t[i]);
                s[i] *= f;
            }
            m = x;
        }
        if (!(x < __int_as_float(0x7f800000))) bad = true;
    }
    __device__ __forceinline__ void add_near(uint4 v, float c, float nb) {
        if (ENTROPY) Elem<T>::clamp(v);  // (what is -inf must not be multiplied with its e = 0)
        f32x2 s2 = pack2(s[0], s[1]), t2 = pack2(t[0], t[1]);
        const f32x2 c2 = pack2(c, c), nb2 = pack2(nb, nb);
#pragma unroll
        for (int i = 0; i < Elem<T>::E; i += 2) {
            const f32x2 z = fma2(pack2(Elem<T>::at(v, i), Elem<T>::at(v, i + 1)), c2, nb2);
            float a, b;
            unpack2(z, a, b);
            const f32x2 e = pack2(ex2(a), ex2(b));
            s2 = add2(s2, e);
            if (ENTROPY) t2 = fma2(e, z, t2);
        }
        unpack2(s2, s[0], s[1]);
        if (ENTROPY) unpack2(t2, t[0], t[1]);
    }
    __device__ __forceinline__ void add_far(uint4 v, float c) {
        const float2 f = far_sums<T>(v, m, c);
        s[0] += f.x;
        if (ENTROPY) t[0] += f.y;
    }
    // Adds the first `have` of the vectors (the others are masked); returns the largest element.
    template <bool WHOLE>
    __device__ __forceinline__ float batch(const uint4 (&v)[kBatch], int have, float c) {
        const float x = Elem<T>::max_of4(v);
        raise(x, c);
        const float nb = -__fmul_rn(m, c);
        if (is_near(nb)) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (WHOLE || u < have) add_near(v[u], c, nb);
        } else {
            for (int u = 0; u < kBatch; ++u)
                if (WHOLE || u < have) add_far(u == 0 ? v[0] : u == 1 ? v[1] : u == 2 ? v[2] : v[3], c);
        }
        return x;
    }
    __device__ __forceinline__ void one(float x, float c) {
        raise(x, c);
        const float z = m == neg_inf() ? kFloor : fmaxf(rel(x, m, c), kFloor), e = ex2(z);
        s[0] += e;
        if (ENTROPY) t[0] = fmaf(e, z, t[0]);
    }
};

// Goes through the vectors of a share, kBatch of a thread at a time, each batch on its way while the one before it is used:
// use(whole, b, v, have) gets batch b, of which this thread has the first `have` vectors.  The last, incomplete batch
// comes first: the loop has whole ones only, without a condition on any load.  start() sends for the first two.
// AGAIN: the share is read a second time, last batches first: the loads leave it in L1 and L2 as far as there is room.
template <typename T, int NT, bool AGAIN = false>
struct Stream {
    const uint4* at;
    int whole, rest;  // whole batches, vectors of this thread in the incomplete one
    bool more;        // there is an incomplete one

    __device__ __forceinline__ explicit Stream(const Share<T>& sh) {
        const int nv = sh.v1 - sh.v0, tid = (int)threadIdx.x;
        at = sh.vec(sh.v0 + tid);
        whole = nv / (kBatch * NT);
        const int left = nv - whole * (kBatch * NT);
        more = left > 0;
        rest = (left - tid + NT - 1) / NT;
    }
    __device__ __forceinline__ int batches() const { return whole + (more ? 1 : 0); }
    __device__ __forceinline__ void load(int b, uint4 (&v)[kBatch]) const {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const uint4* from = at + b * (kBatch * NT) + u * NT;
            v[u] = AGAIN ? ld(from) : ld_stream(from);
        }
    }
    __device__ __forceinline__ void load_rest(uint4 (&v)[kBatch]) const {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            v[u] = make_uint4(Elem<T>::kMasked, Elem<T>::kMasked, Elem<T>::kMasked, Elem<T>::kMasked);
            const uint4* from = at + whole * (kBatch * NT) + u * NT;
            if (u < rest) v[u] = AGAIN ? ld(from) : ld_stream(from);
        }
    }
    __device__ __forceinline__ void start(uint4 (&a)[kBatch], uint4 (&b)[kBatch]) const {
        if (more) load_rest(a);
        if (whole > 0) load(0, b);
    }
    // Backwards: the last whole batch first, the incomplete one last.
    __device__ __forceinline__ void load_back(int i, uint4 (&v)[kBatch]) const {
        if (i < whole) load(whole - 1 - i, v);
        else if (more) load_rest(v);
    }
    __device__ __forceinline__ void start_back(uint4 (&a)[kBatch], uint4 (&b)[kBatch]) const {
        load_back(0, a);
        if (batches() > 1) load_back(1, b);
    }
    template <typename Use>
    __device__ __forceinline__ void run_back(uint4 (&a)[kBatch], uint4 (&b)[kBatch], Use use) const {
        for (int i = 0; i < whole; i += 2) {
            use(std::true_type(), whole - 1 - i, a, kBatch);
            if (i + 2 < batches()) load_back(i + 2, a);
            if (i + 1 < whole) {
                use(std::true_type(), whole - 2 - i, b, kBatch);
                if (i + 3 < batches()) load_back(i + 3, b);
            }
        }
        if (more) {
            if (whole & 1) use(std::false_type(), whole, b, rest);
            else use(std::false_type(), whole, a, rest);
        }
    }
    template <typename Use>
    __device__ __forceinline__ void run(uint4 (&a)[kBatch], uint4 (&b)[kBatch], Use use) const {
        if (more) use(std::false_type(), whole, a, rest);
        for (int i = 0; i < whole; i += 2) {
            if (i + 1 < whole) load(i + 1, a);
            use(std::true_type(), i, b, kBatch);
            if (i + 1 < whole) {
                if (i + 2 < whole) load(i + 2, b);
                use(std::true_type(), i + 1, a, kBatch);
            }
        }
    }
};

struct Stats {
    float m, s, t;
    int bad;
};

// Takes two sums over different elements to the larger of their maxima.
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b, float c) {
    Stats r;
    r.m = fmaxf(a.m, b.m);
    const float base = r.m == neg_inf() ? 0.0f : r.m;
    const float da = fmaxf(rel_base(a.m, base, c), kFloor), db = fmaxf(rel_base(b.m, base, c), kFloor), fa = ex2(da), fb = ex2(db);
    r.s = a.s * fa + b.s * fb;
    r.t = fa * (a.t + da * a.s) + fb * (b.t + db * b.s);
    r.bad = a.bad | b.bad;
    return r;
}

// Order of the top list: larger value first, then the lower index.  Zeros of either sign are equal.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ unsigned long long key_of(float x, int index) {
    return ((unsigned long long)order_of(x) << 32) | (uint32_t)~index;
}

// Barrier of the NT threads that go through a row (a helper warp is not among them), and an or over them.
constexpr uint32_t kRowBarrier = 1;
template <int NT>
__device__ __forceinline__ void row_sync() { ptx::named_bar_sync(kRowBarrier, NT); }
template <int NT>
__device__ __forceinline__ bool row_sync_or(bool v) {
    uint32_t r;
    asm volatile(
        "{\n\t"
        ".reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t"
        "}\n"
        : "=r"(r)
        : "r"((uint32_t)v), "r"(kRowBarrier), "n"(NT)
        : "memory");
    return r != 0;
}

// Everything of the row, in every thread of the cluster.  `part` holds NT / 32 entries; `mine` is read by the other CTAs.
// First the maximum, then every thread's sums relative to it.
template <int NT, typename R>
__device__ __forceinline__ Stats join_row(const R& run, Stats* part, Stats* mine, int ctas, float c) {
    constexpr int NW = NT / 32;
    static_assert(NW <= 16 && (NW & (NW - 1)) == 0, "warps");
    const int lane = (int)threadIdx.x & 31, warp = (int)threadIdx.x >> 5;
    const uint32_t top = __reduce_max_sync(0xffffffffu, order_of(run.m));
    if (lane == 0) part[warp].m = value_of(top);
    Stats v;
    v.bad = row_sync_or<NT>(run.bad);
    v.m = value_of(__reduce_max_sync(0xffffffffu, order_of(part[lane & (NW - 1)].m)));
    const float d = fmaxf(rel_base(run.m, v.m == neg_inf() ? 0.0f : v.m, c), kFloor), f = ex2(d);
    v.s = run.s[0] + run.s[1];
    v.t = f * fmaf(d, v.s, run.t[0] + run.t[1]);
    v.s *= f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
        v.t += __shfl_xor_sync(0xffffffffu, v.t, o);
    }
    if (lane == 0) {
        part[warp].s = v.s;
        part[warp].t = v.t;
    }
    row_sync<NT>();
    v.s = part[lane & (NW - 1)].s;
    v.t = part[lane & (NW - 1)].t;
#pragma unroll
    for (int o = NW / 2; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
        v.t += __shfl_xor_sync(0xffffffffu, v.t, o);
    }
    if (ctas == 1) return v;
    if (threadIdx.x == 0) *mine = v;
    __syncwarp();
    ptx::cluster_sync();
    static_assert(sizeof(Stats) == 16, "one load");
    for (int r = 0; r < ctas; ++r) {
        const float4 q = ptx::ld_cluster_v4(ptx::cluster_addr(ptx::smem_u32(mine), (uint32_t)r));
        const Stats w = {q.x, q.y, q.z, __float_as_int(q.w)};
        v = r == 0 ? w : join(v, w, c);
    }
    return v;
}

// ---------------------------------------------------------------- log probabilities

constexpr int kLpThreads = 256;
// Without a list smaller CTAs, which leave and come more evenly: 2048 rows of 50304, fp32, 64.0 and 61.4 us; 4096 of 50257, bf16, 68.7 and
// 66.1.  (With one, the bound from 128 threads is too low for long lists: 128 alternatives 136 us, 1137 so.)
constexpr int kLpThreadsPlain = 128;

struct TopShared {
    unsigned long long cand[kCandidates];
    unsigned long long best[kTopMax];       // of this CTA, in order; 0: none
    unsigned long long others[8 * kTopMax]; // the lists of the cluster
    int place[kTopMax + 1];                 // in the row's list; the last: how many places are taken
    float largest[kLpThreads];              // of each thread
    int events[kCandidates];
    int num_cand, num_events;
    float threshold;
    unsigned long long sum;
};

template <int NT>
__device__ unsigned long long block_sum(unsigned long long v, unsigned long long* cell) {
    if (threadIdx.x == 0) *cell = 0;
    __syncthreads();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) atomicAdd(cell, v);  // (whole numbers: any order)
    __syncthreads();
    v = *cell;
    __syncthreads();
    return v;
}

// More elements than fit are as large as the lower bound (long runs of equal logits): the k-th largest value by bisection over
// the order of values, then the index up to which elements of that value belong to the list.  Every step reads this
// CTA's share of the row again.
template <typename T>
__device__ __noinline__ void gather_exactly(const Share<T> sh, int k, TopShared* ts) {
    constexpr int E = Elem<T>::E, NT = kLpThreads;
    auto each = [&](auto f) {
        for (int v = sh.v0 + (int)threadIdx.x; v < sh.v1; v += NT) {
            const uint4 x = ld(sh.vec(v));
            for (int i = 0; i < E; ++i) f(order_of(Elem<T>::at(x, i)), sh.head + v * E + i);
        }
        if (sh.single >= 0) f(order_of(Elem<T>::get(sh.row + sh.single)), sh.single);
    };
    auto count = [&](auto f) {
        unsigned long long c = 0;
        each([&](uint32_t o, int i) { c += f(o, i) ? 1 : 0; });
        return block_sum<NT>(c, &ts->sum);
    };
    uint32_t lo = order_of(neg_inf()) + 1, hi = order_of(__int_as_float(0x7f7fffff));  // the k-th largest is in [lo, hi]
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        if (count([&](uint32_t o, int) { return o >= mid; }) >= (unsigned long long)k) lo = mid;
        else hi = mid - 1;
    }
    const uint32_t kth = lo;
    const unsigned long long above = count([&](uint32_t o, int) { return o > kth; });
    int a = 0, b = sh.last - 1;  // the last index that still belongs is in [a, b]
    while (a < b) {
        const int mid = a + (b - a) / 2;
        if (above + count([&](uint32_t o, int i) { return o == kth && i <= mid; }) >= (unsigned long long)k) b = mid;
        else a = mid + 1;
    }
    if (threadIdx.x == 0) ts->num_cand = 0;
    __syncthreads();
    each([&](uint32_t o, int i) {
        if (o > kth || (o == kth && i <= a)) {
            const int at = atomicAdd(&ts->num_cand, 1);
            if (at < kCandidates) ts->cand[at] = ((unsigned long long)o << 32) | (uint32_t)~i;  // (k of them)
        }
    });
    __syncthreads();
}

// The k largest of this CTA's share, in order, to ts->best.  k distinct threads have an element at least as large as the
// k-th largest of the threads' maxima, so that is a lower bound of the k-th largest element, and only batches
// whose maximum reaches it are read again (with 50257 elements and k = 64 about 75 batches and as many elements).
template <typename T>
__device__ __forceinline__ void top_of_share(const Share<T>& sh, int k, float mine, float single, const float* batch_max, int batches,
                                             TopShared* ts) {
    constexpr int E = Elem<T>::E, NT = kLpThreads;
    const int tid = (int)threadIdx.x;
    ts->largest[tid] = mine;
    if (tid == 0) {
        ts->num_cand = 0;
        ts->num_events = 0;
    }
    for (int i = tid; i < k; i += NT) ts->best[i] = 0;
    __syncthreads();
    if (tid < 32) {
        // the k-th largest by bisection over the order of values, to 2^12 steps of fp32 (all of bf16): one warp, eight maxima a
        // lane.  (Every thread counting the larger ones: 2 us of the 6.5 that an SM spent on a row.)
        uint32_t o[NT / 32];
#pragma unroll
        for (int i = 0; i < NT / 32; ++i) o[i] = order_of(ts->largest[32 * i + tid]);
        // (from the first bit on in which the largest and the smallest of them differ)
        uint32_t most = o[0], least = o[0];
#pragma unroll
        for (int i = 1; i < NT / 32; ++i) {
            most = max(most, o[i]);
            least = min(least, o[i]);
        }
        most = __reduce_max_sync(0xffffffffu, most);
        least = __reduce_min_sync(0xffffffffu, least);
        int bit = 31 - __clz((int)(most ^ least));          // -1: all are equal
        uint32_t lo = bit < 0 ? most : most >> 1 >> bit << bit << 1;  // at least k are as large
        constexpr int kLast = sizeof(T) == 2 ? 16 : 12;
#pragma unroll 1
        for (; bit >= kLast; --bit) {
            const uint32_t mid = lo | (1u << bit);
            int c = 0;
#pragma unroll
            for (int i = 0; i < NT / 32; ++i) c += o[i] >= mid;
            if (__reduce_add_sync(0xffffffffu, c) >= k) lo = mid;
        }
        if (tid == 0) ts->threshold = value_of(max(lo, order_of(-FLT_MAX)));  // (-inf never belongs)
    }
    __syncthreads();
    const float bound = ts->threshold;
    auto belongs = [&](float x) { return x >= bound; };
    if (sh.single >= 0 && belongs(single)) {
        const int at = atomicAdd(&ts->num_cand, 1);
        if (at < kCandidates) ts->cand[at] = key_of(single, sh.single);
    }
    if (belongs(mine))
        for (int b = 0; b < batches; ++b)
            if (belongs(batch_max[b * NT + tid])) {
                const int at = atomicAdd(&ts->num_events, 1);
                if (at < kCandidates) ts->events[at] = b * NT + tid;
            }
    __syncthreads();
    const int events = ts->num_events;
    if (events <= kCandidates)
        for (int i = tid; i < events * kBatch; i += NT) {
            const int e = ts->events[i / kBatch];
            const int v = sh.v0 + ((e / NT) * kBatch + i % kBatch) * NT + e % NT;
            if (v < sh.v1) {
                const uint4 x = ld(sh.vec(v));
                int have = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) have += belongs(Elem<T>::at(x, j));
                if (have > 0) {
                    int at = atomicAdd(&ts->num_cand, have);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float y = Elem<T>::at(x, j);
                        if (belongs(y) && at < kCandidates) ts->cand[at++] = key_of(y, sh.head + v * E + j);
                    }
                }
            }
        }
    __syncthreads();
    if (events > kCandidates || ts->num_cand > kCandidates) gather_exactly<T>(sh, k, ts);
    const int n = min(ts->num_cand, kCandidates);
    if (tid == 0 && (n & 1)) ts->cand[n] = 0;  // (two are read at a time)
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
        const unsigned long long key = ts->cand[i];
        int r = 0;
        for (int j = 0; j < n; j += 2) {
            const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&ts->cand[j]);
            r += (o.x > key) + (o.y > key);
        }
        if (r < k) ts->best[r] = key;
    }
    __syncthreads();
}

struct LogprobParams {
    int vocab, ctas, lg, top;  // ctas = 2^lg
    long long ld;
    const long long* targets;
    float c, inv_t;
    float *logprob, *entropy, *top_logprob;
    int* top_index;
};

// Relative to a near base with the exponent that the logit has in the sum; otherwise, and where that exponent may overflow, by the quotient.
__device__ __forceinline__ float log_prob(float x, float m, float log_s, const LogprobParams& p) {
    if (x >= kLowest && is_near(__fmul_rn(m, p.c))) return (rel(x, m, p.c) - log_s) * kLn2;
    return (x - m) * p.inv_t - log_s * kLn2;
}

// LIST 0: none; 1: a short one; 2: a long one, of which more batches are read again, so that the first reading leaves them in L1 as
// far as there is room.  Measured past L1 and so, us, for rows of 16000 to 131072 in bf16 and fp32, 1500 to 4096 of them: 20 alternatives
// 47 to 237 and 52 to 247; 40 48 to 240 and 54 to 250 (past L1 is 1 to 16 % faster everywhere); 64 the one as often as the other (4096 rows of 50257
// in bf16 110 and 103, 2048 of them 54 and 58; fp32 83 and 87); 96 60 to 99 and 62 to 92; 128 75 to 277 and 68 to 279.
constexpr int kLongList = 48;
template <typename T, int LIST>
__global__ void __launch_bounds__(LIST ? kLpThreads : kLpThreadsPlain)
token_logprobs_kernel(const T* logits, const LogprobParams p) {
    constexpr bool TOP = LIST != 0;
    constexpr int NT = TOP ? kLpThreads : kLpThreadsPlain;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Stats part[NT / 32];
    __shared__ Stats mine;
    pdl_wait();
    const int row = (int)blockIdx.x / p.ctas, rank = (int)blockIdx.x % p.ctas;
    const Share<T> sh(logits + (long long)row * p.ld, p.vocab, rank, p.lg);
    const int tid = (int)threadIdx.x;
    TopShared* ts = reinterpret_cast<TopShared*>(smem);
    float* batch_max = reinterpret_cast<float*>(smem + sizeof(TopShared));

    // of the given token (wanted by one thread at the end)
    long long target = -1;
    float given = 0.0f;
    if (rank == 0 && tid == 0 && p.targets != nullptr) {
        target = ld(p.targets + row);
        if (target >= 0 && target < p.vocab) given = Elem<T>::get(sh.row + target);
    }
    const float single = sh.single >= 0 ? Elem<T>::get(sh.row + sh.single) : neg_inf();

    Running<T, true> run;
    const Stream<T, NT, LIST == 2> stream(sh);
    uint4 va[kBatch], vb[kBatch];
    stream.start(va, vb);
    stream.run(va, vb, [&](auto whole, int b, uint4(&v)[kBatch], int have) {
        const float x = run.template batch<decltype(whole)::value>(v, have, p.c);
        if (TOP) batch_max[b * NT + tid] = x;
    });
    if (sh.single >= 0) run.one(single, p.c);

    // (first, so that the cluster meets once for the sums and the lists; of a row that is no distribution it comes to nothing)
    if constexpr (TOP) top_of_share<T>(sh, p.top, run.m, single, batch_max, stream.batches(), ts);
    const Stats st = join_row<NT>(run, part, &mine, p.ctas, p.c);
    const bool none = st.bad || !(st.s > 0.0f);  // no distribution
    const float log_s = log2f(st.s);
    if (rank == 0 && tid == 0) {
        if (p.logprob != nullptr) {
            float lp = log_prob(given, st.m, log_s, p);
            if (none || target >= p.vocab) lp = quiet_nan();
            else if (target < 0) lp = 0.0f;
            p.logprob[row] = lp;
        }
        if (p.entropy != nullptr) p.entropy[row] = none ? quiet_nan() : (log_s - st.t / st.s) * kLn2;
    }
    if (TOP) {
        const int k = p.top;
        float* out = p.top_logprob + (long long)row * k;
        int* out_i = p.top_index + (long long)row * k;
        auto put = [&](int at, unsigned long long key) {
            out[at] = key ? log_prob(value_of((uint32_t)(key >> 32)), st.m, log_s, p) : neg_inf();
            out_i[at] = key ? (int)~(uint32_t)key : -1;
        };
        if (none) {  // the same in all CTAs of the row
            if (rank == 0)
                for (int i = tid; i < k; i += NT) {
                    out[i] = quiet_nan();
                    out_i[i] = -1;
                }
        } else {
            if (p.ctas == 1) {
                for (int i = tid; i < k; i += NT) put(i, ts->best[i]);
            } else {
                // Each CTA finds the places of its own in the row's list: its place here, and how many of each other list come before
                // it, by bisection in copies of them.  Rank 0 also counts how many places are taken.
                for (int i = tid; i < p.ctas * k; i += NT) {
                    unsigned long long key;
                    const uint32_t from = ptx::cluster_addr(ptx::smem_u32(&ts->best[i % k]), (uint32_t)(i / k));
                    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(key) : "r"(from) : "memory");
                    ts->others[i] = key;
                }
                for (int i = tid; i <= k; i += NT) ts->place[i] = 0;
                __syncthreads();
                for (int i = tid; i < p.ctas * (k + 1); i += NT) {
                    const int of = i / p.ctas, r = i % p.ctas;
                    const unsigned long long* list = ts->others + r * k;
                    const unsigned long long key = of < k ? ts->best[of] : 0;
                    int lo = 0, hi = k;  // how many are larger
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (list[mid] > key) lo = mid + 1;
                        else hi = mid;
                    }
                    atomicAdd(&ts->place[of], lo);
                }
                __syncthreads();
                for (int i = tid; i < k; i += NT) {
                    if (ts->best[i] != 0 && ts->place[i] < k) put(ts->place[i], ts->best[i]);
                    if (rank == 0 && i >= ts->place[k]) put(i, 0);
                }
            }
        }
    }
    __syncwarp();
    if (p.ctas > 1) ptx::cluster_sync();  // nobody's memory goes away while it is read
}

// ---------------------------------------------------------------- distillation

// The teacher's tokens of a row, and what a row comes to.
struct Teacher {
    int index[kTopMax];   // -1: left out
    float logp[kTopMax];
    float x[kTopMax];     // the student's logit of the token
    double p[kTopMax];    // relative to the likeliest entry's without a tail
    int word[kTopMax];       // of its mark; -1: not in this CTA's share
    float mass_of[kTopMax];  // p of all entries with this index, normalised without a tail; in the first of them
    int first[kTopMax];      // 1: the first entry with this index
    double total;            // of p
    float log_base;          // logarithm of what p is relative to
    float own_m, own_s;      // largest logit of these tokens, and their sum relative to it
    float mass, r;           // of the teacher's tokens (1 without a tail), of all others
    float w;                 // what the row counts
    int bad;
    // from the whole row
    int none;                // no distribution
    float m, s;              // the largest logit, the sum over all tokens
    float m_rest, s_rest;    // the same of the tokens that the teacher does not name (0 and 0: there is none)
};

struct DistillParams {
    int n, vocab, ctas, lg, k, tail;  // ctas = 2^lg
    int marks_bytes;
    long long ld, ldd;
    const int* index;
    const float* logp;
    const float* dloss;
    float c, inv_t;
    float* loss;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Where element j has its bit in the marks: bit i of byte v - v0 + 1 is element i of vector v, the bytes at both ends stand for the
// single elements before and after the vectors.
template <typename T>
__device__ __forceinline__ int mark_place(const Share<T>& sh, int j) { return j - (sh.head + sh.v0 * Elem<T>::E) + Elem<T>::E; }

// Loads the teacher's list of a row, marks its tokens among this CTA's vectors, and works out what does not need the row's sums.
// marked() is called when
// the marks are there, which are all that the first pass wants.  One warp, ahead of those that go through the row.  te and marks are of the row before the last (`used`).
template <typename T, typename Marked>
__device__ __forceinline__ void prepare_row(const DistillParams& p, const Share<T>& sh, int row, Teacher* te, uint32_t* marks, bool used, Marked marked) {
    constexpr int E = Elem<T>::E;
    const int lane = (int)threadIdx.x & 31;
    if (used)
        for (int i = lane; i < p.k; i += 32)
            if (te->word[i] >= 0) marks[te->word[i]] = 0;
    __syncwarp();
    bool bad = false, again = false;
    int index[kTopMax / 32];
    float logp[kTopMax / 32];
#pragma unroll
    for (int u = 0; u < kTopMax / 32; ++u) {
        const int i = u * 32 + lane;
        index[u] = -1;
        logp[u] = 0.0f;
        if (i < p.k) {
            index[u] = ld(p.index + (long long)row * p.k + i);
            logp[u] = ld(p.logp + (long long)row * p.k + i);
        }
    }
    const float w = p.dloss != nullptr ? ld(p.dloss + row) : 0.0f;
    float x[kTopMax / 32];
#pragma unroll
    for (int u = 0; u < kTopMax / 32; ++u) {
        if (index[u] >= p.vocab) {
            bad = true;
            index[u] = -1;
        }
        index[u] = max(index[u], -1);
        int word = -1;
        if (index[u] >= sh.first && index[u] < sh.last) {
            const int at = mark_place(sh, index[u]);  // >= 0: the elements before the first vector are fewer than E
            const uint32_t bit = 1u << (8 * ((at / E) & 3) + at % E);
            word = at / E >> 2;
            if (atomicOr(&marks[word], bit) & bit) again = true;
        }
        if (u * 32 + lane < p.k) te->word[u * 32 + lane] = word;
    }
    marked();
#pragma unroll
    for (int u = 0; u < kTopMax / 32; ++u) x[u] = index[u] >= 0 ? Elem<T>::get(sh.row + index[u]) : neg_inf();
    // an index that is there twice: of several CTAs each has marked its own share only, so all are compared
    if (p.ctas > 1) {
#pragma unroll
        for (int u = 0; u < kTopMax / 32; ++u) {
            if (u * 32 >= p.k) break;
            const uint32_t same = __match_any_sync(0xffffffffu, index[u] >= 0 ? index[u] : -1 - lane);
            again |= (same & (same - 1)) != 0;
#pragma unroll
            for (int o = 0; o < u; ++o)
#pragma unroll 4
                for (int l = 0; l < 32; ++l) {
                    const int other = __shfl_sync(0xffffffffu, index[o], l);
                    again |= index[u] >= 0 && other == index[u];
                }
        }
    }
    // without a tail only ratios of probabilities count, and these may be too small for 64 bits: they are taken relative to the largest
    float log_base = 0.0f;
    if (!p.tail) {
        float most = neg_inf();
#pragma unroll
        for (int u = 0; u < kTopMax / 32; ++u)
            if (index[u] >= 0) most = fmaxf(most, logp[u]);
        most = value_of(__reduce_max_sync(0xffffffffu, order_of(most)));
        if (most > neg_inf()) log_base = most;
    }
    double total = 0.0;
#pragma unroll
    for (int u = 0; u < kTopMax / 32; ++u) {
        const int i = u * 32 + lane;
        if (i >= p.k) break;
        te->index[i] = index[u];
        te->logp[i] = logp[u];
        te->x[i] = x[u];
        const double q = index[u] >= 0 ? exp((double)logp[u] - (double)log_base) : 0.0;
        te->p[i] = q;
        total += q;
        if (!(x[u] < __int_as_float(0x7f800000))) bad = true;
    }
    total = warp_sum(total);
    const bool repeated = __any_sync(0xffffffffu, again);
    const double keep = p.tail ? 1.0 : (total > 0.0 ? 1.0 / total : 0.0);
    __syncwarp();
    float m = neg_inf();
    for (int i = lane; i < p.k; i += 32) {
        const int j = te->index[i];
        bool first = j >= 0;
        double sum = te->p[i];
        if (repeated && first) {
            for (int o = 0; o < i; ++o) first &= te->index[o] != j;
            for (int o = i + 1; o < p.k; ++o)
                if (te->index[o] == j) sum += te->p[o];
        }
        te->first[i] = first;
        te->mass_of[i] = (float)(sum * keep);
        if (first) m = fmaxf(m, te->x[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = 0.0f;
    for (int i = lane; i < p.k; i += 32)
        if (te->first[i] && m > neg_inf()) s += ex2(fmaxf(rel(te->x[i], m, p.c), kFloor));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) {
        te->total = total;
        te->log_base = log_base;
        te->own_m = m;
        te->own_s = s;
        const double mass = p.tail ? total : (total == 0.0 ? 0.0 : total * keep);
        te->mass = (float)mass;
        te->r = p.tail ? (float)fmax(0.0, 1.0 - mass) : 0.0f;
        te->w = w;
        te->bad = bad;
    }
    __syncwarp();
}

// What a class adds to the divergence, p (d + expm1(-d)) with d = log p - log q: never negative, so near distributions lose
// nothing to the cancellation of p log p against p log q, and a common error of all log q (that of the row's sum) drops
// out.  In 64 bits: k + 1 values a row.  Where q is far larger than p nothing cancels, and p e^-d is q: there p may be a
// subnormal number next to which e^-d overflows (log p below -709).
__device__ __forceinline__ double class_loss(double p, double log_p, double log_q) {
    if (!(p > 0.0)) return p == 0.0 ? exp(log_q) : p;
    const double d = log_p - log_q;
    if (d < -30.0) return p * (d - 1.0) + exp(log_q);
    return p * (d + expm1(-d));
}

// The base of a sum in 64 bits, where products of two floats are exact, and the logarithm of e^(x / T) relative to it.
__device__ __forceinline__ double base_of(float m, float c) {
    const float b = __fmul_rn(m, c);
    return is_near(b) ? (double)b : (double)m * (double)c;
}
__device__ __forceinline__ double log_rel(float x, double base, float c) { return ((double)x * (double)c - base) * 0.69314718055994530942; }

// Loss of a row whose sums are there.  One warp.
__device__ __forceinline__ float loss_of_row(const DistillParams& p, const Teacher* te) {
    const int lane = (int)threadIdx.x & 31;
    const double total = te->total;
    const double keep = p.tail ? 1.0 : (total > 0.0 ? 1.0 / total : 0.0);
    const double mass = p.tail ? total : (total == 0.0 ? 0.0 : total * keep);
    const double r = p.tail && te->s_rest > 0.0f ? fmax(0.0, 1.0 - mass) : 0.0;
    const double log_s = log((double)te->s), log_keep = p.tail || mass == 0.0 ? 0.0 : log(keep);
    const double base = base_of(te->m, p.c);
    double loss = 0.0;
    for (int i = lane; i < p.k; i += 32) {
        if (te->index[i] < 0) continue;
        const double log_q = log_rel(te->x[i], base, p.c) - log_s;
        loss += class_loss(te->p[i] * keep, ((double)te->logp[i] - (double)te->log_base) + log_keep, log_q);
        if (!te->first[i]) loss -= exp(log_q);  // its q counts once
    }
    loss = warp_sum(loss);
    const double log_rho = (base_of(te->m_rest, p.c) - base) * 0.69314718055994530942 + log((double)te->s_rest) - log_s;
    loss += class_loss(r, log(r), log_rho) + (mass + r - 1.0);
    if (mass == 0.0 && r == 0.0) loss = 0.0;  // the teacher says nothing
    return te->none ? quiet_nan() : (float)loss;
}

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// The gradient of a token that the teacher does not name, f 2^(c (x - m)).  FOLDED: the magnitude of f is part of the exponent, which
// saves a product and a sum, and the sign is left.  The sum log2|f| - c m is rounded, so this is for bf16 and sums below 2^10: the result
// is off by 2^-15 of itself then, a hundredth of half a step (and by the error of the logarithm, 2^-18).
template <typename T, bool FOLDED>
struct RestGrad {
    float c, from, f;  // FOLDED: log2|f| - c m, and 1 or -1

    __device__ __forceinline__ RestGrad(float f_, float m, float c_) : c(c_), from(-m), f(f_) {
        if (FOLDED) {
            const float b = __fmul_rn(m, c);
            from = (log2f(fabsf(f)) - fmaf(m, c, -b)) - b;
            f = f < 0.0f ? -1.0f : 1.0f;
        }
    }
    // (-inf: all results are zero)
    __device__ __forceinline__ bool fits() const { return fabsf(from) <= 1024.0f || from == neg_inf(); }
    __device__ __forceinline__ f32x2 exponents(f32x2 x) const {
        const f32x2 c2 = pack2(c, c), from2 = pack2(from, from);
        return FOLDED ? fma2(x, c2, from2) : mul2(add2(x, from2), c2);
    }
    __device__ __forceinline__ T operator()(float x) const {
        float a, b;
        unpack2(exponents(pack2(x, x)), a, b);
        return from_float<T>(ex2(a) * f);
    }
    // of a vector
    __device__ __forceinline__ uint4 operator()(const uint4& x) const {
        constexpr int E = Elem<T>::E;
        const f32x2 f2 = pack2(f, f);
        const uint32_t sign = f < 0.0f ? 0x80008000u : 0u;
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            float a, b;
            unpack2(exponents(pack2(Elem<T>::at(x, i), Elem<T>::at(x, i + 1))), a, b);
            a = ex2(a);
            b = ex2(b);
            if (!FOLDED) unpack2(mul2(pack2(a, b), f2), a, b);
            if constexpr (sizeof(T) == 4) {
                y[i] = __float_as_uint(a);
                y[i + 1] = __float_as_uint(b);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
                memcpy(&y[i / 2], &h, 4);
                if (FOLDED) y[i / 2] ^= sign;
            }
        }
        return make_uint4(y[0], y[1], y[2], y[3]);
    }
};

// The vector that begins `d` elements into a and goes on in b, 0 < d < E.
template <typename T>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int d) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const int half = d * (int)sizeof(T) / 2;  // in half words
    if (half & 4) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (half & 2) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (half & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Written once and not read here: it leaves L2 before the logits that are read again.
__device__ __forceinline__ void st_stream(uint4* p, const uint4& v) {
    asm volatile("st.global.cs.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Elements [first, last) of a row.
template <typename T>
__device__ __forceinline__ void zero_row(T* out, int first, int last, int tid, int threads) {
    constexpr int E = Elem<T>::E;
    const int before = min(last - first, (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(out + first) & 15u)) & 15u) / sizeof(T)));
    const int from = first + before, count = (last - from) / E, after = from + count * E;
    for (int v = tid; v < count; v += threads) st_stream(reinterpret_cast<uint4*>(out + from) + v, make_uint4(0u, 0u, 0u, 0u));
    if (tid < before) out[first + tid] = from_float<T>(0.0f);
    if (tid < last - after) out[after + tid] = from_float<T>(0.0f);
}

constexpr int kDistillThreads = 256;  // that go through a row; one more warp helps them

// Loss, and with GRAD the gradient.  A CTA (or a cluster of them) goes from row to row for the loss, as far as the grid leaves it
// several, and has one row for the gradient (the grid has a cluster for each).  Eight warps go through the logits: once for the sums,
// and for the gradient once more, backwards, which finds the end of the row in L1 and most of the rest in L2 (2048 rows of 50257, bf16: 109 us forwards and past L1,
// 97 so).  A ninth has the teacher's list, whose loads depend on one another, and the loss, which is a chain of logarithms in 64 bits:
// a row ahead of the others and a row behind where there are several, so neither holds up the loads, of which two batches a thread are
// always on their way.  Barriers: `ready` when a row's tokens are marked, `listed` when the rest of its list is there, `done` when its
// sums are and its list is no longer read; each for odd and for even rows.
// The gradient of 2048 rows of 50257, bf16: 93 us; with the row kept in shared memory 139 (a CTA a row, two CTAs an SM), 119 (one CTA an SM that writes a row's gradient while it takes the next one's sums, through
// registers) and 127 (the same by bulk copies).  One CTA an SM has too few warps for the fixed part of a row, and
// what the SM's L2 traffic saves comes back as waits.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(kDistillThreads + 32, 3)
distill_kernel(const T* logits, T* grad, const DistillParams p) {
    constexpr int NT = kDistillThreads, E = Elem<T>::E;
    constexpr uint32_t kReady = 2, kListed = 4, kDone = 6;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Stats part[NT / 32];
    constexpr int kSlots = GRAD ? 1 : 2;  // rows that are in hand at a time
    __shared__ Stats mine[kSlots];
    __shared__ Teacher teachers[kSlots];
    const int tid = (int)threadIdx.x, rank = (int)blockIdx.x & (p.ctas - 1);
    const int step = (int)gridDim.x >> p.lg;
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem);
    for (int i = tid; i < kSlots * p.marks_bytes / 4; i += NT + 32) marks[i] = 0;
    __syncthreads();
    pdl_wait();
    auto share = [&](int row) { return Share<T>(logits + (long long)row * p.ld, p.vocab, rank, p.lg); };
    int row = (int)blockIdx.x >> p.lg;

    if (tid >= NT) {
        int it = 0;
        for (;; row += step, ++it) {
            const bool there = GRAD ? it == 0 : row < p.n;
            const int slot = it & (kSlots - 1);
            if (there) {
                prepare_row<T>(p, share(row), row, &teachers[slot], marks + slot * (p.marks_bytes / 4), it >= 2, [&] {
                    __syncwarp();
                    asm volatile("bar.arrive %0, %1;" ::"r"(kReady + slot), "n"(NT + 32) : "memory");
                });
                asm volatile("bar.arrive %0, %1;" ::"r"(kListed + slot), "n"(NT + 32) : "memory");
            }
            if (it > 0) {
                const int last = (it - 1) & (kSlots - 1);
                ptx::named_bar_sync(kDone + last, NT + 32);
                if (rank == 0 && p.loss != nullptr) {
                    const float loss = loss_of_row(p, &teachers[last]);
                    if (tid == NT) p.loss[row - step] = loss;
                }
                __syncwarp();
            }
            if (!there) break;
            if (p.ctas > 1) ptx::cluster_sync();  // (that of join_row)
        }
    } else {
        uint4 va[kBatch], vb[kBatch];
        Stream<T, NT, GRAD>(share(row)).start(va, vb);
        // (one turn for the gradient; said here, that makes for an order of instructions that costs fp32 6 %, 176 us and not 166)
        for (int it = 0; row < p.n; row += step, ++it) {
            const int slot = it & (kSlots - 1);
            const Share<T> sh = share(row);
            const Stream<T, NT, GRAD> stream(sh);
            const float single = sh.single >= 0 ? Elem<T>::get(sh.row + sh.single) : 0.0f;
            Teacher* te = &teachers[slot];
            const uint8_t* mark = reinterpret_cast<const uint8_t*>(marks) + slot * p.marks_bytes;
            ptx::named_bar_sync(kReady + slot, NT + 32);
            Running<T, false> run;
            stream.run(va, vb, [&](auto whole, int b, uint4(&v)[kBatch], int have) {
                const int at = b * (kBatch * NT) + tid + 1;
                uint32_t bits[kBatch], any = 0;
#pragma unroll
                for (int u = 0; u < kBatch; ++u) any |= bits[u] = decltype(whole)::value || u < have ? mark[at + u * NT] : 0;
                if (any) {
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
                        if (bits[u]) Elem<T>::mask(v[u], bits[u]);
                }
                run.template batch<decltype(whole)::value>(v, have, p.c);
            });
            if (sh.single >= 0) {
                const int at = mark_place(sh, sh.single);
                if (!((mark[at / E] >> (at % E)) & 1)) run.one(single, p.c);
            }
            // what comes next is on its way while the sums are joined: the row again, or the next one
            if (GRAD) stream.start_back(va, vb);
            else if (row + step < p.n) Stream<T, NT>(share(row + step)).start(va, vb);
            const Stats rest = join_row<NT>(run, part, &mine[slot], p.ctas, p.c);
            ptx::named_bar_sync(kListed + slot, NT + 32);
            const float own_m = te->own_m, m = fmaxf(rest.m, own_m), base = m == neg_inf() ? 0.0f : m;
            const float down = ex2(fmaxf(rel_base(rest.m, base, p.c), kFloor));
            const float s = te->own_s * ex2(fmaxf(rel_base(own_m, base, p.c), kFloor)) + rest.s * down;
            // The rest keeps its own maximum: rho may be too small for a float where its logarithm, and the shares of its
            // tokens in it, are not.
            const float m_rest = rest.m == neg_inf() ? 0.0f : rest.m;
            const bool none = rest.bad || te->bad || !(s > 0.0f);
            if (tid == 0) {
                te->m = base;
                te->s = s;
                te->m_rest = m_rest;
                te->s_rest = rest.s;
                te->none = none;
            }
            if (GRAD) {
                // a row that counts nothing has no gradient, whatever its logits hold; one without a distribution has NaN
                const float w = te->w;
                const bool zero = w == 0.0f;
                const float r = rest.s > 0.0f ? te->r : 0.0f, f = w * p.inv_t, mass = te->mass + r;
                // Sums relative to c times their maxima, without the rounding of their bases: a small result would be 0 with it.
                const float to_base = ex2(base_error(base, p.c)) / s, r_share = r > 0.0f ? r / rest.s * ex2(base_error(m_rest, p.c)) : 0.0f;
                const float f_rest = none ? quiet_nan() : f * (mass * (ex2((rest.m - base) * p.c) * to_base) - r_share);
                const float f_own = none ? quiet_nan() : f * mass * to_base;
                T* out = grad + (long long)row * p.ldd;
                auto others = [&](const auto& g) {
                    if (((reinterpret_cast<uintptr_t>(out + sh.head) ^ reinterpret_cast<uintptr_t>(sh.row + sh.head)) & 15u) == 0) {
                        uint4* out_vec = reinterpret_cast<uint4*>(out + sh.head) + sh.v0 + tid;
                        stream.run_back(va, vb, [&](auto whole, int b, uint4(&v)[kBatch], int have) {
#pragma unroll
                            for (int u = 0; u < kBatch; ++u)
                                if (decltype(whole)::value || u < have) st_stream(out_vec + b * (kBatch * NT) + u * NT, g(v[u]));
                        });
                        if (sh.single >= 0) out[sh.single] = g(single);
                    } else {
                        // The result's rows start elsewhere than the logits': its whole vectors, each from two of the logits',
                        // where both are this CTA's; single elements for the rest.
                        const int from = sh.head + sh.v0 * E;  // of the elements in whole vectors of logits
                        const int before = (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(out + from) & 15u)) & 15u) / sizeof(T));
                        const int count = max(0, sh.v1 - sh.v0 - 1);
                        uint4* out_vec = reinterpret_cast<uint4*>(out + from + before);
                        for (int v = (count - 1) / (kBatch * NT) * (kBatch * NT) + tid; v >= 0; v -= kBatch * NT) {
                            const uint4* at = sh.vec(sh.v0 + v);  // (a neighbour's vector is in L1 by then, or on its way)
#pragma unroll
                            for (int u = 0; u < kBatch; ++u)
                                if (v + u * NT < count) {
                                    va[u] = ld(at + u * NT);
                                    vb[u] = ld(at + u * NT + 1);
                                }
#pragma unroll
                            for (int u = 0; u < kBatch; ++u)
                                if (v + u * NT < count) st_stream(out_vec + v + u * NT, g(shifted<T>(va[u], vb[u], before)));
                        }
                        const int lo = count > 0 ? from + before : sh.last, hi = from + before + count * E;
                        for (int j = sh.first + tid; j < min(lo, sh.last); j += NT) out[j] = g(Elem<T>::get(sh.row + j));
                        for (int j = hi + tid; count > 0 && j < sh.last; j += NT) out[j] = g(Elem<T>::get(sh.row + j));
                    }
                };
                // (the teacher's tokens, whose exponent may overflow here, are written after the others)
                if (zero) {
                    zero_row(out, sh.first, sh.last, tid, NT);
                } else if constexpr (sizeof(T) == 4) {
                    others(RestGrad<T, false>(f_rest, m_rest, p.c));
                } else {
                    const RestGrad<T, true> g(f_rest, m_rest, p.c);
                    if (g.fits()) others(g);
                    else others(RestGrad<T, false>(f_rest, m_rest, p.c));
                }
                row_sync<NT>();
                if (tid < p.k && te->first[tid] && te->index[tid] >= sh.first && te->index[tid] < sh.last) {
                    const float q = ex2((te->x[tid] - base) * p.c) * f_own;
                    out[te->index[tid]] = from_float<T>(zero ? 0.0f : q - te->mass_of[tid] * f);
                }
            }
            asm volatile("bar.arrive %0, %1;" ::"r"(kDone + slot), "n"(NT + 32) : "memory");
        }
    }
    __syncwarp();
    if (p.ctas > 1) ptx::cluster_sync();  // nobody's memory goes away while it is read
}

// ---------------------------------------------------------------- host side

bcq_status check_rows(int n, int vocab, const void* logits, size_t ld, int dtype, float temperature) {
    if (n < 0 || vocab < 1 || ld < (size_t)vocab) return BCQ_ERR_SHAPE;
    if (vocab > kVocabMax || n > kRowsMax) return BCQ_ERR_UNSUPPORTED;
    if (dtype != BCQ_F32 && dtype != BCQ_BF16) return BCQ_ERR_UNSUPPORTED;
    if (!(temperature >= 1e-3f && temperature <= 1e3f)) return BCQ_ERR_SHAPE;
    if (n > 0 && logits == nullptr) return BCQ_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(logits) & (dtype == BCQ_BF16 ? 1u : 3u)) != 0) return BCQ_ERR_ALIGN;
    return BCQ_OK;
}

float exponent_scale(float temperature) { return (float)(1.4426950408889634074 / (double)temperature); }

// CTAs of a row: as many as leave every SM no more than `per_sm` CTAs, and every CTA a batch or so.
int ctas_for(int n, int vocab, int elem_bytes, int threads, int per_sm) {
    const long long nvec = (long long)vocab * elem_bytes / 16;
    int ctas = 1;
    while (ctas < 8 && (long long)n * ctas * 2 <= (long long)sm_count() * per_sm && nvec / (ctas * 2) >= threads) ctas *= 2;
    return ctas;
}

int log2_of(int ctas) { return ctas == 8 ? 3 : ctas / 2; }

int max_vectors(int vocab, int elem_bytes, int ctas) { return ceil_div(vocab * elem_bytes / 16, ctas); }

template <typename T, int LIST>
bcq_status launch_logprobs_as(int n, const void* logits, const LogprobParams& p, cudaStream_t s) {
    const int nv = max_vectors(p.vocab, (int)sizeof(T), p.ctas);
    const size_t smem = LIST ? sizeof(TopShared) + (size_t)ceil_div(nv, kBatch * kLpThreads) * kLpThreads * 4 : 0;
    if (LIST) {
        const bcq_status st = ensure_dynamic_smem(token_logprobs_kernel<T, LIST>, smem);
        if (st != BCQ_OK) return st;
    }
    BCQ_CUDA_TRY(launch_pdl(token_logprobs_kernel<T, LIST>, dim3((unsigned)(n * p.ctas)), LIST ? kLpThreads : kLpThreadsPlain, smem, s,
                            (unsigned)p.ctas, (const T*)logits, p));
    return BCQ_OK;
}

template <typename T>
bcq_status launch_logprobs(int n, const void* logits, const LogprobParams& p, cudaStream_t s) {
    if (p.top == 0) return launch_logprobs_as<T, 0>(n, logits, p, s);
    return p.top > kLongList ? launch_logprobs_as<T, 2>(n, logits, p, s) : launch_logprobs_as<T, 1>(n, logits, p, s);
}

template <typename T, bool GRAD>
bcq_status launch_distill(int n, const void* logits, void* grad, DistillParams p, cudaStream_t s) {
    p.ctas = ctas_for(n, p.vocab, (int)sizeof(T), kDistillThreads, 3);
    p.lg = log2_of(p.ctas);
    p.marks_bytes = (int)align_up((size_t)max_vectors(p.vocab, (int)sizeof(T), p.ctas) + 2, 16);
    const size_t smem = (GRAD ? 1 : 2) * (size_t)p.marks_bytes;
    const bcq_status st = ensure_dynamic_smem(distill_kernel<T, GRAD>, smem);
    if (st != BCQ_OK) return st;
    // The loss goes from row to row (2048 rows of 50272, fp32: 69 us, a CTA for each 74); the gradient, whose rows take longer than a CTA's
    // start, has a CTA for each (2048 of 50257, bf16: 93 us, from row to row 97).
    const int clusters = GRAD ? n : std::min(n, std::max(1, sm_count() * 3 / p.ctas));
    BCQ_CUDA_TRY(launch_pdl(distill_kernel<T, GRAD>, dim3((unsigned)(clusters * p.ctas)), kDistillThreads + 32, smem, s, (unsigned)p.ctas,
                            (const T*)logits, (T*)grad, p));
    return BCQ_OK;
}

bcq_status check_teacher(int n, int k, const int* index, const float* logp) {
    if (k < 1) return BCQ_ERR_SHAPE;
    if (k > kTopMax) return BCQ_ERR_UNSUPPORTED;
    if (n > 0 && (!index || !logp)) return BCQ_ERR_NULL;
    return BCQ_OK;
}

}  // namespace

extern "C" bcq_status bcq_token_logprobs(int n, int vocab, const void* logits, size_t ld, int dtype, const long long* targets,
                                         int top_k, float temperature, float* logprob, float* entropy, float* top_logprob,
                                         int* top_index, void* stream) {
    const bcq_status st = check_rows(n, vocab, logits, ld, dtype, temperature);
    if (st != BCQ_OK) return st;
    if (top_k < 0) return BCQ_ERR_SHAPE;
    if (top_k > kTopMax) return BCQ_ERR_UNSUPPORTED;
    if (n == 0) return BCQ_OK;
    if ((targets == nullptr) != (logprob == nullptr)) return BCQ_ERR_NULL;
    if (top_k > 0 && (!top_logprob || !top_index)) return BCQ_ERR_NULL;
    LogprobParams p;
    p.vocab = vocab; p.top = top_k;
    p.ld = (long long)ld;
    p.targets = targets;
    p.c = exponent_scale(temperature); p.inv_t = 1.0f / temperature;
    p.logprob = logprob; p.entropy = entropy; p.top_logprob = top_logprob; p.top_index = top_index;
    p.ctas = top_k > 0 ? ctas_for(n, vocab, dtype == BCQ_BF16 ? 2 : 4, kLpThreads, 3) : ctas_for(n, vocab, dtype == BCQ_BF16 ? 2 : 4, kLpThreadsPlain, 6);
    p.lg = log2_of(p.ctas);
    cudaStream_t s = (cudaStream_t)stream;
    return dtype == BCQ_BF16 ? launch_logprobs<__nv_bfloat16>(n, logits, p, s) : launch_logprobs<float>(n, logits, p, s);
}

extern "C" bcq_status bcq_distill_loss(int n, int vocab, int k, const void* logits, size_t ld, int dtype, const int* top_index,
                                       const float* top_logprob, float temperature, int tail, float* loss, void* stream) {
    bcq_status st = check_rows(n, vocab, logits, ld, dtype, temperature);
    if (st != BCQ_OK) return st;
    if ((st = check_teacher(n, k, top_index, top_logprob)) != BCQ_OK) return st;
    if (n == 0) return BCQ_OK;
    if (!loss) return BCQ_ERR_NULL;
    DistillParams p;
    p.n = n; p.vocab = vocab; p.k = k; p.tail = tail != 0; p.ld = (long long)ld; p.ldd = 0;
    p.index = top_index; p.logp = top_logprob; p.dloss = nullptr;
    p.c = exponent_scale(temperature); p.inv_t = 1.0f / temperature;
    p.loss = loss;
    cudaStream_t s = (cudaStream_t)stream;
    return dtype == BCQ_BF16 ? launch_distill<__nv_bfloat16, false>(n, logits, nullptr, p, s)
                             : launch_distill<float, false>(n, logits, nullptr, p, s);
}

extern "C" bcq_status bcq_distill_grad(int n, int vocab, int k, const void* logits, size_t ld, int dtype, const int* top_index,
                                       const float* top_logprob, float temperature, int tail, const float* dloss, float* loss,
                                       void* dlogits, size_t lddl, void* stream) {
    bcq_status st = check_rows(n, vocab, logits, ld, dtype, temperature);
    if (st != BCQ_OK) return st;
    if ((st = check_teacher(n, k, top_index, top_logprob)) != BCQ_OK) return st;
    if (lddl < (size_t)vocab) return BCQ_ERR_SHAPE;
    if (n == 0) return BCQ_OK;
    if (!dloss || !dlogits) return BCQ_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(dlogits) & (dtype == BCQ_BF16 ? 1u : 3u)) != 0) return BCQ_ERR_ALIGN;
    if (dlogits == logits && lddl != ld) return BCQ_ERR_SHAPE;
    DistillParams p;
    p.n = n; p.vocab = vocab; p.k = k; p.tail = tail != 0; p.ld = (long long)ld; p.ldd = (long long)lddl;
    p.index = top_index; p.logp = top_logprob; p.dloss = dloss;
    p.c = exponent_scale(temperature); p.inv_t = 1.0f / temperature;
    p.loss = loss;
    cudaStream_t s = (cudaStream_t)stream;
    return dtype == BCQ_BF16 ? launch_distill<__nv_bfloat16, true>(n, logits, dlogits, p, s) : launch_distill<float, true>(n, logits, dlogits, p, s);
}
