// Matrix product in 8-bit integers with a scale for each token and each channel.
//
//   y[m][n] = epilogue(s_a[m] s_w[n] sum_k qa[m][k] qw[n][k] + b[n]),
//   s_a[m] = max_k |x[m][k]| / 127,   qa[m][k] = round(127 x[m][k] / max_k |x[m][k]|)
//
// The tensor core of this part has no fast 8-bit integer kind.  Whole numbers
// up to 128 are exact in fp16, their products and, below 2^24, their sums in
// fp32, so the product runs at the fp16 rate, with the integer's result as long as
// the sums stay below 2^24 in magnitude: whatever the numbers to a depth of 1024 (1040 for
// numbers to 127), for most rows much further (random ones grow with the root of the depth).  Past
// it a sum is fp32's, each step of 16 off by 2^-23 of it at most.  The
// weights stay 8 bits wide in memory, which is what a step of few tokens
// waits for.  The tokens are quantised by a kernel of their own (as fp16 whole
// numbers, ready for TMA); the weights are widened on their way into tensor
// memory, where they are the MMA's A operand: 128 channels are its rows, up to
// 192 tokens its columns.
#include <cuda_fp16.h>

#include <algorithm>

#include "xc_branch.cuh"
#include "xc_kernels.cuh"
#include "xc_ptx.cuh"

namespace xc {

// ------------------------------------------------------------- quantisation
// Eight elements of a row.
template <typename T> struct Vec8;
template <> struct Vec8<bf16> {
    uint4 u;
    __device__ __forceinline__ void load(const bf16 *p) { u = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(bf16 *p) const { *reinterpret_cast<uint4 *>(p) = u; }
    // largest magnitude of the eight and m, as bits (NaN above infinity above the rest)
    __device__ __forceinline__ unsigned top(unsigned m) const {
        unsigned x = __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
        x = max(x << 16, x & 0xffff0000u);
        return max(m, x);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const float4 *>(p)[0];
        b = reinterpret_cast<const float4 *>(p)[1];
    }
    __device__ __forceinline__ void store(float *p) const {
        reinterpret_cast<float4 *>(p)[0] = a;
        reinterpret_cast<float4 *>(p)[1] = b;
    }
    __device__ __forceinline__ unsigned top(unsigned m) const {
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};

constexpr float ROUND_MAGIC = 12582912.0f;   // 1.5 * 2^23: adding it rounds to whole numbers, held in the low bits

// A row's divisor: the largest magnitude's bits, and what is made of them.
struct QuantRow {
    float a, r, f;             // divisor (times f), 127 / a; f: a power of two for both sides of the quotient
    bool finite, plain;        // plain: f = 1

    __device__ __forceinline__ QuantRow(unsigned top) {
        finite = top < 0x7f800000u;
        const float m = __uint_as_float(top);
        // far from 1 both sides are scaled, so that nothing over- or underflows
        f = m > 0x1p100f ? 0x1p-100f : (m < 0x1p-60f ? 0x1p80f : 1.0f);
        plain = f == 1.0f;
        a = m * f;
        r = finite && m > 0.0f ? __fdiv_rn(127.0f, a) : 0.0f;
    }
};
__device__ __forceinline__ float quant_scale(unsigned top) {
    return top < 0x7f800000u ? __fdiv_rn(__uint_as_float(top), 127.0f) : __uint_as_float(0x7fffffffu);
}
// 127 x / a of eight numbers, rounded to the nearest whole number, halves to even, decided as
// the exact quotient would be.  r = 127 / a is off by 2^-24 and the product by
// as much, 2e-5 in all: eight among which a quotient t is that near to a half are decided by the
// sign of 127 x - (k + 1/2) a, k = floor(t), each product as a sum of two floats: near the half the
// difference of the leading ones is exact, and that of the others is off by 2^-48, where sides that
// differ do so by 2^-32 or more (31 and 32 bits).  One test for eight: with one each, 12960 rows of 5120 took 52 us instead of 40.
template <typename T> __device__ __forceinline__ void quant8(const Vec8<T> &z, const QuantRow &row, float (&q)[8]) {
    float x[8], far = row.plain ? 0.0f : 1.0f;
    z.get(x);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float2 t = __fmul2_rn(make_float2(x[i], x[i + 1]), make_float2(row.r, row.r));
        const float2 w = __fadd2_rn(__fadd2_rn(t, make_float2(ROUND_MAGIC, ROUND_MAGIC)), make_float2(-ROUND_MAGIC, -ROUND_MAGIC));
        const float2 d = __fadd2_rn(t, make_float2(-w.x, -w.y));
        far = fmaxf(far, fmaxf(fabsf(d.x), fabsf(d.y)));
        q[i] = w.x;
        q[i + 1] = w.y;
    }
    if (__builtin_expect(far > 0.4999f, 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = fabsf(x[i] * row.f), k = floorf(v * row.r), c = k + 0.5f;
            const float p = 127.0f * v, h = c * row.a;
            const float d = (p - h) + (fmaf(127.0f, v, -p) - fmaf(c, row.a, -h));
            q[i] = copysignf(d > 0.0f ? k + 1.0f : d < 0.0f ? k : rintf(c), x[i]);
        }
        if (row.a == 0.0f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = 0.0f;
        }
    }
    if (!row.finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = 0.0f;
    }
}

// Eight whole numbers as fp16, as bytes.
__device__ __forceinline__ uint4 half8(const float (&e)[8]) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(e[2 * i], e[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint2 pack8(const float (&e)[8]) {
    unsigned w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        unsigned b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(e[4 * h + i] + ROUND_MAGIC);
        w[h] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
    return make_uint2(w[0], w[1]);
}

// TPR threads a row, rows in turn; a thread keeps KEEP vectors of eight elements of its row in
// registers, the next row's on their way meanwhile, and reads what a longer row has beyond
// them again.  HBM bound (12960 x 5120 bf16 to fp16: 45 us, 4.7 TB/s; 8961 x 1536 fp32 to 8 bits: 17).
// A row without a finite largest magnitude gets scale NaN and zeros.
template <typename T, typename Q, int TPR, int KEEP>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, TPR == 512 ? 1 : TPR == 256 ? 3 : 5)
    quantize_rows_kernel(const T *__restrict__ x, Q *__restrict__ q, float *__restrict__ scale, const int M, const int K) {
    pdl_wait();
    pdl_release();
    constexpr int CTA = TPR < 128 ? 128 : TPR, RPC = CTA / TPR;
    __shared__ unsigned sh[2][CTA / 32];
    const int t = threadIdx.x % TPR, nv = K / 8;
    int row = blockIdx.x * RPC + threadIdx.x / TPR;
    Vec8<T> next[KEEP];
    auto load = [&](int r) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (r < M && t + i * TPR < nv) next[i].load(x + (size_t)r * K + 8 * (t + i * TPR));
    };
    load(row);
    for (int turn = 0; TPR > 32 ? row - (int)(threadIdx.x / TPR) < M : row < M; row += gridDim.x * RPC, turn ^= 1) {
        Vec8<T> keep[KEEP];
#pragma unroll
        for (int i = 0; i < KEEP; ++i) keep[i] = next[i];
        load(row + gridDim.x * RPC);
        const T *src = x + (size_t)row * K;
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (t + i * TPR < nv) top = keep[i].top(top);
        for (int v = t + KEEP * TPR; v < nv; v += TPR) {
            Vec8<T> z;
            z.load(src + 8 * v);
            top = z.top(top);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if constexpr (TPR > 32) {                      // (two turns' maxima: one barrier a row)
            if ((threadIdx.x & 31) == 0) sh[turn][threadIdx.x >> 5] = top;
            __syncthreads();
            top = 0;
#pragma unroll
            for (int w = 0; w < CTA / 32; ++w) top = max(top, sh[turn][w]);
        }
        if (t == 0) scale[row] = quant_scale(top);
        const QuantRow qr(top);
        Q *dst = q + (size_t)row * K;
        auto put = [&](const Vec8<T> &z, int v) {
            float e[8];
            quant8<T>(z, qr, e);
            if constexpr (sizeof(Q) == 1) {
                *reinterpret_cast<uint2 *>(dst + 8 * v) = pack8(e);
            } else {
                *reinterpret_cast<uint4 *>(dst + 8 * v) = half8(e);
            }
        };
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (t + i * TPR < nv) put(keep[i], t + i * TPR);
        for (int v = t + KEEP * TPR; v < nv; v += TPR) {
            Vec8<T> z;
            z.load(src + 8 * v);
            put(z, v);
        }
    }
}

// Few rows: a CTA a row, which waits in shared memory for its largest magnitude.  Latency bound, and the code
// is short: a loop over a row in registers is unrolled, and its instructions have to be fetched too.
constexpr int QFEW_BYTES = 48 * 1024 - 256;     // with the warps' maxima, what a CTA has without asking
template <typename T, typename Q, int THREADS>
__global__ void __launch_bounds__(THREADS) quantize_few_kernel(const T *__restrict__ x, Q *__restrict__ q, float *__restrict__ scale, const int K) {
    extern __shared__ __align__(16) uint8_t quant_row[];
    __shared__ unsigned sh[THREADS / 32];
    pdl_wait();
    pdl_release();
    const int t = threadIdx.x, nv = K / 8, row = blockIdx.x;
    const T *src = x + (size_t)row * K;
    T *stage = reinterpret_cast<T *>(quant_row);
    unsigned top = 0;
    for (int v0 = t; v0 < nv; v0 += 4 * THREADS) {
        Vec8<T> z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v0 + i * THREADS < nv) z[i].load(src + 8 * (v0 + i * THREADS));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v0 + i * THREADS < nv) {
                z[i].store(stage + 8 * (v0 + i * THREADS));
                top = z[i].top(top);
            }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if ((t & 31) == 0) sh[t >> 5] = top;
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, sh[t & (THREADS / 32 - 1)]);
    if (t == 0) scale[row] = quant_scale(top);
    const QuantRow qr(top);
    Q *dst = q + (size_t)row * K;
#pragma unroll 1
    for (int v = t; v < nv; v += THREADS) {
        Vec8<T> z;
        float e[8];
        z.load(stage + 8 * v);
        quant8<T>(z, qr, e);
        if constexpr (sizeof(Q) == 1) {
            *reinterpret_cast<uint2 *>(dst + 8 * v) = pack8(e);
        } else {
            *reinterpret_cast<uint4 *>(dst + 8 * v) = half8(e);
        }
    }
}

template <typename T, typename Q>
static cudaError_t quantize_launch(const T *x, Q *q, float *scale, int M, int K, cudaStream_t st) {
    const int nv = K / 8, sms = device_sms();
    constexpr int KEEP = sizeof(T) == 2 ? 5 : 3;
    auto launch = [&](auto kernel, int tpr, int per_sm) {
        const int cta = tpr < 128 ? 128 : tpr, ctas = (M + cta / tpr - 1) / (cta / tpr);
        return launch_pdl(kernel, dim3(std::min(ctas, per_sm * sms)), dim3(cta), 0, st, x, q, scale, M, K);
    };
    auto few = [&](auto kernel, int threads) {
        return launch_pdl(kernel, dim3(M), dim3(threads), (size_t)K * sizeof(T), st, x, q, scale, K);
    };
    // Few rows at one time, with the more threads the fewer and the longer they are (8 x 5120 bf16: 6.2 us with
    // 512 threads, 6.5 with 256; 331 x 13824: 20.9 and 22.7; 560 x 1536: 7.8 and 6.7; in registers 6.5, 23.2 and 7.7).
    if (nv > 32 && M <= 4 * sms && (size_t)K * sizeof(T) <= QFEW_BYTES)
        return nv > 1024 || (nv > 256 && M <= 2 * sms) ? few(quantize_few_kernel<T, Q, 512>, 512) : few(quantize_few_kernel<T, Q, 256>, 256);
    // Many: the fewest threads that hold a row in registers, so that an SM has many rows' loads under way.
    if (nv <= 32 * KEEP) return launch(quantize_rows_kernel<T, Q, 32, KEEP>, 32, 5);
    if (nv <= 128 * KEEP) return launch(quantize_rows_kernel<T, Q, 128, KEEP>, 128, 5);
    if (nv <= 256 * KEEP) return launch(quantize_rows_kernel<T, Q, 256, KEEP>, 256, 3);
    return launch(quantize_rows_kernel<T, Q, 512, KEEP>, 512, 1);
}
cudaError_t quantize_rows(int dtype, int M, int K, const void *x, signed char *q, float *scale, cudaStream_t st) {
    return dtype == XC_BF16 ? quantize_launch(reinterpret_cast<const bf16 *>(x), q, scale, M, K, st)
                            : quantize_launch(reinterpret_cast<const float *>(x), q, scale, M, K, st);
}

// Two whole numbers in [-128, 127] out of four bytes, as fp16: the byte plus 128
// in the low bits of 1024 is 1152 more than the number.
__device__ __forceinline__ void widen4(unsigned w, unsigned &lo, unsigned &hi) {
    const __half2 off = __half2half2(__ushort_as_half(0x6480));
    const unsigned u = w ^ 0x80808080u;
    unsigned a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
    lo = *reinterpret_cast<const unsigned *>(&x);
    hi = *reinterpret_cast<const unsigned *>(&y);
}

// Tokens that the caller quantised: 8-bit whole numbers to fp16, scales to where the product reads them.
__global__ void __launch_bounds__(256) widen_kernel(const uint4 *q, uint4 *out, const long n, const float *scale, float *scale_out,
                                                     const int M) {
    pdl_wait();
    pdl_release();
    const long stride = (long)gridDim.x * 256, i0 = (long)blockIdx.x * 256 + threadIdx.x;
    for (long i = i0; i < n; i += stride) {
        const uint4 v = q[i];
        uint4 a, b;
        widen4(v.x, a.x, a.y);
        widen4(v.y, a.z, a.w);
        widen4(v.z, b.x, b.y);
        widen4(v.w, b.z, b.w);
        out[2 * i] = a;
        out[2 * i + 1] = b;
    }
    for (long i = i0; i < M; i += stride) scale_out[i] = scale[i];
}

// ------------------------------------------------------------------ product
constexpr int I8_BM = 128, I8_BK = 128;        // channels and depth of a weight tile
constexpr int I8_W_BYTES = I8_BM * I8_BK, I8_MAX_W = 8, I8_MAX_B = 16, I8_MAX_A = 8;
constexpr int I8_THREADS = 640, I8_SMEM = 220 * 1024;
constexpr int I8_NT = 192;                     // most tokens of a tile: two sets of sums and four slots of widened weights

struct I8Sched {
    int M, N, NT;              // tokens, channels, tokens of a tile (a multiple of 16)
    int m_tiles, n_pairs, KT;  // tiles of tokens, pairs of tiles of channels, tiles along the depth
    int n_full, P;             // tile pairs that CTA pairs run whole, in rounds (the rest is cut); CTA pairs
    int wst, bst;              // slots in shared memory: weights of depth 128, tokens of depth 64
    int as, acs;               // slots of depth 64 in tensor memory; columns of a set of sums
    int epi, vec;              // vec: 16-byte outputs
    const float *a_scale, *w_scale, *bias, *gate;
    const void *resid;
    void *out;
    float *part;               // [4 P][NT][128] sums of cut tiles

    __host__ __device__ __forceinline__ unsigned line() const { return (unsigned)(m_tiles * n_pairs - n_full) * KT; }
};

// Tile pairs in super-rows of 8 pairs of channel blocks, channels fastest: the tiles that
// run at one time share their weights and tokens in L2.
__host__ __device__ __forceinline__ void i8_tile(const I8Sched &s, int tile, int &mb, int &pb) {
    const int per = 8 * s.m_tiles, grp = tile / per, first = 8 * grp, loc = tile - grp * per;
    const int gn = s.n_pairs - first < 8 ? s.n_pairs - first : 8;
    pb = first + loc % gn;
    mb = loc / gn;
}
// The cut tiles' depth as one line over the CTA pairs.
struct I8Line {
    unsigned q, r;
    __host__ __device__ __forceinline__ I8Line(unsigned T, unsigned P) : q(T / P), r(T - q * P) {}
    __host__ __device__ __forceinline__ unsigned begin(unsigned c) const { return q * c + (c < r ? c : r); }
    __host__ __device__ __forceinline__ unsigned owner(unsigned x) const {
        const unsigned longer = r * (q + 1);
        return x < longer ? x / (q + 1) : r + (x - longer) / q;
    }
};
// The pieces of a CTA pair, as each role walks them: whole tile pairs c, c + P, ..., then
// its share of the line, which touches two tile pairs at most.
struct I8Walk {
    int mb, nb;                // tile of tokens, of channels (this CTA's of the pair)
    int k0, k1, slot;          // slot: of the sums of a cut piece, -1: a whole tile
    int next_full;
    unsigned x, end;
    int first;
    __device__ __forceinline__ I8Walk(const I8Sched &s, int c) : mb(0), nb(0), k0(0), k1(0), slot(-1), next_full(c), first(1) {
        const I8Line l(s.line(), s.P);
        x = l.begin(c);
        end = l.begin(c + 1);
    }
    __device__ __forceinline__ bool next(const I8Sched &s) {
        int tile;
        if (next_full < s.n_full) {
            tile = next_full;
            next_full += s.P;
            k0 = 0;
            k1 = s.KT;
        } else {
            if (x >= end) return false;
            const int t = x / s.KT;
            tile = s.n_full + t;
            k0 = x - t * s.KT;
            k1 = min(s.KT, k0 + (int)(end - x));
            x += k1 - k0;
            slot = k1 - k0 == s.KT ? -1 : 2 * (int)blockIdx.x + (first ? 0 : 1);
            first = 0;
        }
        int pb;
        i8_tile(s, tile, mb, pb);
        nb = 2 * pb + ((int)blockIdx.x & 1);
        return true;
    }
};

template <typename T> __device__ __forceinline__ float i8_gelu(float y) {
    // y (1 + tanh u) / 2 = y / (1 + exp(-2 u)): no cancellation where tanh is near -1
    const float u2 = -1.5957691216057308f * (y + 0.044715f * y * y * y);
    if constexpr (sizeof(T) == 2) return __fdividef(y, 1.0f + __expf(u2));
    else return y / (1.0f + expf(u2));
}
// One output of channel n (its scale, bias, gate in registers).
template <typename T>
__device__ __forceinline__ float i8_epilogue(int epi, float acc, float sa, float sw, float b, float g, float resid) {
    const float y = fmaf(acc * sa, sw, b);
    if (epi == EPI_GELU) return i8_gelu<T>(y);
    if (epi == EPI_RESID_GATE) return fmaf(g, y, resid);
    return y;
}

// The products of one slot of depth 64 (A in tensor memory) and what their end tells: one
// lane is elected for all of it (an election for each instruction took the issuing warp as long
// as the products take).
__device__ __forceinline__ void i8_issue_slot(uint32_t acc, uint32_t a, uint64_t b, uint32_t idesc, uint32_t first, uint64_t *a_empty,
                                              uint64_t *b_empty) {
    asm volatile(
        "{\n\t.reg .pred e, p, t;\n\t.reg .b32 r, a1, a2, a3;\n\t.reg .b64 b1, b2, b3;\n\t"
        "elect.sync r|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.eq.b32 t, %4, %4;\n\t"
        "add.u32 a1, %1, 8;\n\tadd.u32 a2, %1, 16;\n\tadd.u32 a3, %1, 24;\n\t"
        "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, t;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, t;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, t;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t}"
        ::"r"(acc), "r"(a), "l"(b), "r"(idesc), "r"(first), "r"(smem_u32(a_empty)), "r"(smem_u32(b_empty))
        : "memory");
}

// Exchanges between lanes that turn a lane's 16 tokens of one channel into 8 consecutive
// channels of two tokens: on return x[8 r + c] is channel 8 (lane / 8) + c of token 8 r + lane % 8.
__device__ __forceinline__ void i8_turn(float (&x)[16], int lane) {
    float y[16];
#pragma unroll
    for (int t = 0; t < 8; ++t) {                      // y[2 t + c]: channel pair of token 2 t + lane % 2
        const float got = __shfl_xor_sync(0xffffffffu, (lane & 1) ? x[2 * t] : x[2 * t + 1], 1);
        y[2 * t] = (lane & 1) ? got : x[2 * t];
        y[2 * t + 1] = (lane & 1) ? x[2 * t + 1] : got;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)                        // x[4 q + c]: 4 channels of token 4 q + lane % 4
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float got = __shfl_xor_sync(0xffffffffu, (lane & 2) ? y[4 * q + c] : y[4 * q + 2 + c], 2);
            x[4 * q + c] = (lane & 2) ? got : y[4 * q + c];
            x[4 * q + 2 + c] = (lane & 2) ? y[4 * q + 2 + c] : got;
        }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float got = __shfl_xor_sync(0xffffffffu, (lane & 4) ? x[8 * r + c] : x[8 * r + 4 + c], 4);
            const float lo = (lane & 4) ? got : x[8 * r + c], hi = (lane & 4) ? x[8 * r + 4 + c] : got;
            y[8 * r + c] = lo;
            y[8 * r + 4 + c] = hi;
        }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = y[i];
}

// Two CTAs run neighbouring tiles of channels with the same tokens at the same time, so that
// one of them finds the tokens in L2; each loads its own, and neither touches the other's shared
// memory.  (One copy into both, by multicast, took 3 % off a chunk.  But the tokens are in the caller's workspace,
// which nothing here shows to be this GPU's memory, and replicas on several GPUs run this kernel too.)
// Warps: 0 loads weights, 1 issues the products, 2 loads tokens, 4-11 widen the weights (thread = channel =
// TMEM lane, a half of each tile's depth to either four warps), 12-19 write the outputs (two
// per TMEM quadrant, half of the tokens each).
// 12960 tokens x 13824 x 5120: 1066 us, 1.72 PFLOP/s; 331 tokens x 5120 x 13824: 28 us from
// the first product to the last.  A depth of 128 takes 1045 and 900 cycles where the products of 192 and 176 tokens
// take 768 and 704, with 3 % of the time spent waiting for operands (clock counters): probably shared memory's bandwidth, of which
// the products read 64 bytes a clock, the copies write 85 and the widening reads 22, 171 of 128.
template <typename T>
__global__ void __launch_bounds__(I8_THREADS, 1)
    linear_i8_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                     const __grid_constant__ I8Sched s, int *err) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * I8_MAX_W + 2 * I8_MAX_B + 2 * I8_MAX_A + 5];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(16) float sh_scale[8][I8_NT / 2 + 16];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int b_bytes = s.NT * 128;
    uint8_t *sW = smem, *sB = smem + s.wst * I8_W_BYTES;
    uint64_t *w_full = bars, *w_empty = w_full + I8_MAX_W, *b_full = w_empty + I8_MAX_W, *b_empty = b_full + I8_MAX_B;
    uint64_t *a_full = b_empty + I8_MAX_B, *a_empty = a_full + I8_MAX_A;
    uint64_t *acc_full = a_empty + I8_MAX_A, *acc_empty = acc_full + 2, *drained = acc_empty + 2;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < s.wst; ++i) {
            mbar_init(&w_full[i], 1);
            mbar_init(&w_empty[i], 256);
        }
        for (int i = 0; i < s.bst; ++i) {
            mbar_init(&b_full[i], 1);
            mbar_init(&b_empty[i], 1);
        }
        for (int i = 0; i < s.as; ++i) {
            mbar_init(&a_full[i], 128);
            mbar_init(&a_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 256);
        }
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(&tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = 0;                           // all 512 columns are this CTA's (a constant stays in uniform registers)
    const int a_col = 2 * s.acs;
    I8Walk w(s, blockIdx.x >> 1);

    if (warp == 0) {
        // The kernel before this one in the stream (the quantisation) began after
        // everything before it had ended, so the weights need no wait.
        if (lane == 0) {
            int i = 0, it = 0;
            uint32_t ph = 1;
            bool ok = true;
            while (ok && w.next(s)) {
                for (int kt = w.k0; kt < w.k1; ++kt, ++it) {
                    if (!(ok = mbar_wait(&w_empty[i], ph, err, ERR_WAIT_PRODUCER))) break;
                    mbar_expect_tx(&w_full[i], I8_W_BYTES);
                    tma_load_2d(sW + i * I8_W_BYTES, &tmW, &w_full[i], kt * I8_BK, w.nb * I8_BM);
                    if (++i == s.wst) {
                        i = 0;
                        ph ^= 1;
                    }
                }
            }
            for (int j = max(it - s.wst, 0); j < it; ++j)         // every copy has landed before the CTA exits
                mbar_wait(&w_full[j % s.wst], (j / s.wst) & 1, err, ERR_WAIT_PRODUCER);
        }
    } else if (warp == 2) {
        if (lane == 0) {
            pdl_wait();
            int i = 0, it = 0;
            uint32_t ph = 1;
            bool ok = true;
            while (ok && w.next(s)) {
                for (int kt = 2 * w.k0; kt < 2 * w.k1; ++kt, ++it) {
                    if (!(ok = mbar_wait(&b_empty[i], ph, err, ERR_WAIT_PRODUCER))) break;
                    mbar_expect_tx(&b_full[i], b_bytes);
                    tma_load_2d(sB + i * b_bytes, &tmA, &b_full[i], 64 * kt, w.mb * s.NT);
                    if (++i == s.bst) {
                        i = 0;
                        ph ^= 1;
                    }
                }
            }
            for (int j = max(it - s.bst, 0); j < it; ++j)
                mbar_wait(&b_full[j % s.bst], (j / s.bst) & 1, err, ERR_WAIT_PRODUCER);
        }
    } else if (warp == 1) {
        // D f32, A and B f16, N = NT, M = 128
        const uint32_t idesc = (1u << 4) | ((uint32_t)(s.NT >> 3) << 17) | ((uint32_t)(I8_BM >> 4) << 24);
        const uint64_t d0 = sdesc_sw128(smem_u32(sB), 16, 1024);
        auto wait = [&](uint64_t *b, uint32_t parity) {
            return __all_sync(0xffffffffu, mbar_wait(b, parity & 1, err, ERR_WAIT_MMA)) != 0;
        };
        int local = 0, i = 0, a = 0;
        uint32_t ph = 0, a_ph = 0;
        bool ok = true;
        while (ok && w.next(s)) {
            const int buf = local & 1, use = local >> 1;
            ++local;
            if (!(ok = wait(&acc_empty[buf], use ^ 1))) break;
            tc_fence_after();
            const uint32_t acc = tmem + buf * s.acs;
            bool there = false;                        // the next slot has been seen to be ready
#pragma unroll 1
            for (int n = 2 * (w.k1 - w.k0), first = 0; n > 0; --n, first = 1) {
                if (!__all_sync(0xffffffffu, there) && !(ok = wait(&b_full[i], ph) && wait(&a_full[a], a_ph))) break;
                tc_fence_after();
                const uint64_t db = d0 + (uint64_t)((i * b_bytes) >> 4);
                const uint32_t ta = tmem + a_col + 32 * a;
                uint64_t *a_done = &a_empty[a], *b_done = &b_empty[i];
                if (++a == s.as) {
                    a = 0;
                    a_ph ^= 1;
                }
                if (++i == s.bst) {
                    i = 0;
                    ph ^= 1;
                }
                there = mbar_test2(&b_full[i], ph, &a_full[a], a_ph);
                i8_issue_slot(acc, ta, db, idesc, first, a_done, b_done);
            }
            // (the outputs wait for this one, which comes after the slots' commits: the CTA outlives them all)
            if (ok) tc_commit_warp(&acc_full[buf]);
        }
        if (!ok) {                                     // a wait ran out: no product is under way when the CTA ends
            tc_commit_warp(drained);
            wait(drained, 0);
        }
    } else if (warp >= 4 && warp < 12) {
        const int g = (warp - 4) >> 2, q = warp & 3, r = 32 * q + lane;
        const uint32_t t0 = tmem + ((uint32_t)(32 * q) << 16) + a_col;
        // slots of the two rings, and the parities of their turns: this group has every other slot
        int i = 0, a = g;
        uint32_t ph = 0, a_ph = 1;
        bool ok = true;
        while (ok && w.next(s)) {
            for (int kt = w.k0; kt < w.k1; ++kt) {
                if (a >= s.as) {
                    a -= s.as;
                    a_ph ^= 1;
                }
                ok = mbar_wait(&w_full[i], ph, err, ERR_WAIT_TMA);
                ok = ok && mbar_wait(&a_empty[a], a_ph, err, ERR_WAIT_MMA);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                tc_fence_after();
                const uint8_t *src = sW + i * I8_W_BYTES + r * 128;
                uint32_t x[32];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(src + (((4 * g + c) ^ (r & 7)) << 4));
                    widen4(v.x, x[8 * c], x[8 * c + 1]);
                    widen4(v.y, x[8 * c + 2], x[8 * c + 3]);
                    widen4(v.z, x[8 * c + 4], x[8 * c + 5]);
                    widen4(v.w, x[8 * c + 6], x[8 * c + 7]);
                }
                tmem_st32_sync(t0 + 32 * a, x);
                // only now have the loads returned for certain: an arrival may overtake them, and the copy
                // that follows it does not wait for loads of the other proxy
                mbar_arrive(&w_empty[i]);
                tc_fence_before();
                mbar_arrive(&a_full[a]);
                a += 2;
                if (++i == s.wst) {
                    i = 0;
                    ph ^= 1;
                }
            }
        }
    } else if (warp >= 12) {
        pdl_wait();                                    // the tokens' scales
        const int q = warp & 3, half = (warp - 12) >> 2;
        const uint32_t tq = tmem + ((uint32_t)(32 * q) << 16);
        const T *resid = reinterpret_cast<const T *>(s.resid);
        T *out = reinterpret_cast<T *>(s.out);
        float *scale = sh_scale[warp - 12];
        const int nc = s.NT / 16, ch0 = half ? (nc + 1) / 2 : 0, ch1 = half ? nc : (nc + 1) / 2;   // this warp's tokens, by 16
        int local = 0;
        bool ok = true;
        while (ok && w.next(s)) {
            const int buf = local & 1, use = local >> 1;
            ++local;
            const int m0 = w.mb * s.NT, n_base = w.nb * I8_BM + 32 * q, n = n_base + lane, nl = min(n, s.N - 1);
            const int cols = min(s.NT, s.M - m0), last = min(ch1, (cols + 15) / 16);
            const float sw = s.w_scale[nl], b = s.bias[nl], gt = s.epi == EPI_RESID_GATE ? s.gate[nl] : 0.0f;
            __syncwarp();
            for (int x = lane; x < 16 * (last - ch0); x += 32) scale[x] = s.a_scale[min(m0 + 16 * ch0 + x, s.M - 1)];
            __syncwarp();
            ok = mbar_wait(&acc_full[buf], use & 1, err, ERR_WAIT_EPI);
            if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
            tc_fence_after();
            for (int c = ch0; c < last; ++c) {
                const int mc = m0 + 16 * c, left = cols - 16 * c;
                float v[16];
                tmem_ld16_sync(tq + buf * s.acs + 16 * c, v);
                if (c + 1 == last) {
                    tc_fence_before();
                    mbar_arrive(&acc_empty[buf]);
                }
                if (w.slot >= 0) {
                    float *dst = s.part + ((size_t)w.slot * s.NT + 16 * c) * I8_BM + 32 * q + lane;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < left) dst[i * I8_BM] = v[i];
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const float4 sa = *reinterpret_cast<const float4 *>(scale + 16 * (c - ch0) + i);
                    v[i] = fmaf(v[i] * sa.x, sw, b);
                    v[i + 1] = fmaf(v[i + 1] * sa.y, sw, b);
                    v[i + 2] = fmaf(v[i + 2] * sa.z, sw, b);
                    v[i + 3] = fmaf(v[i + 3] * sa.w, sw, b);
                }
                if (s.epi == EPI_GELU) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = i8_gelu<T>(v[i]);
                } else if (s.epi == EPI_RESID_GATE) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] *= gt;
                }
                if (sizeof(T) == 2 && s.vec) {         // whole 16 bytes: N is a multiple of 8
                    i8_turn(v, lane);
                    const int nv = n_base + (lane & ~7);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int i = 8 * r + (lane & 7);
                        if (i >= left || nv >= s.N) continue;
                        const size_t at = (size_t)(mc + i) * s.N + nv;
                        float y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = v[8 * r + j];
                        if (s.epi == EPI_RESID_GATE) {
                            float x[8];
                            loadW<T, 8>(resid + at, x);
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] += x[j];
                        }
                        storeW<T, 8>(out + at, y);
                    }
                } else if (n < s.N) {
                    float x[16];
                    if (s.epi == EPI_RESID_GATE) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = i < left ? to_f(resid[(size_t)(mc + i) * s.N + n]) : 0.0f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] += x[i];
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < left) out[(size_t)(mc + i) * s.N + n] = from_f<T>(v[i]);
                }
            }
            if (ch0 >= last) mbar_arrive(&acc_empty[buf]);
        }
    }
    pdl_release();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Adds the pieces of a cut tile in CTA order: a thread has four channels of two tokens, a
// CTA 16 tokens.  331 tokens x 5120: 6 us, all in L2; bound by latency (six CTAs an SM instead of four spill: no gain).
constexpr int I8M_THREADS = 256, I8M_TOKENS = 16;
template <typename T>
__global__ void __launch_bounds__(I8M_THREADS) linear_i8_merge_kernel(const __grid_constant__ I8Sched s) {
    pdl_wait();
    pdl_release();
    const I8Line l(s.line(), s.P);
    const int rank = blockIdx.x & 1;
    const unsigned x0 = (blockIdx.x >> 1) * (unsigned)s.KT;
    const int c0 = l.owner(x0), c1 = l.owner(x0 + s.KT - 1);
    if (c0 == c1) return;                              // run whole
    int mb, pb;
    i8_tile(s, s.n_full + (blockIdx.x >> 1), mb, pb);
    const int ch = 4 * (threadIdx.x & 31), t0 = blockIdx.y * I8M_TOKENS + (threadIdx.x >> 5), n0 = (2 * pb + rank) * I8_BM + ch;
    const int cols = min(s.NT, s.M - mb * s.NT);
    if (t0 >= cols || n0 >= s.N) return;
    const bool two = t0 + 8 < cols;
    float4 sum[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 4
    for (int c = c0; c <= c1; ++c) {
        const float *src = s.part + ((size_t)(2 * (2 * c + rank) + (l.begin(c) >= x0 ? 0 : 1)) * s.NT + t0) * I8_BM + ch;
        const float4 a = *reinterpret_cast<const float4 *>(src);
        const float4 b = two ? *reinterpret_cast<const float4 *>(src + 8 * I8_BM) : make_float4(0.f, 0.f, 0.f, 0.f);
        sum[0] = make_float4(sum[0].x + a.x, sum[0].y + a.y, sum[0].z + a.z, sum[0].w + a.w);
        sum[1] = make_float4(sum[1].x + b.x, sum[1].y + b.y, sum[1].z + b.z, sum[1].w + b.w);
    }
    const T *resid = reinterpret_cast<const T *>(s.resid);
    T *out = reinterpret_cast<T *>(s.out);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (t == 1 && !two) break;
        const int m = mb * s.NT + t0 + 8 * t;
        const float sa = s.a_scale[m], v[4] = {sum[t].x, sum[t].y, sum[t].z, sum[t].w};
        const size_t at = (size_t)m * s.N + n0;
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = min(n0 + j, s.N - 1);
            const float r = s.epi == EPI_RESID_GATE && n0 + j < s.N ? to_f(resid[at + j]) : 0.0f;
            y[j] = i8_epilogue<T>(s.epi, v[j], sa, s.w_scale[n], s.bias[n], s.epi == EPI_RESID_GATE ? s.gate[n] : 0.0f, r);
        }
        if (sizeof(T) == 2 && s.vec) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(y[0], y[1]), b = __floats2bfloat162_rn(y[2], y[3]);
            *reinterpret_cast<uint2 *>(out + at) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n0 + j < s.N) out[at + j] = from_f<T>(y[j]);
        }
    }
}

// -------------------------------------------------------------- few tokens
// A step of a few tokens waits for the weights' bytes, so everything else goes
// into the one kernel: each CTA (one an SM) quantises all tokens into its shared
// memory as fp16, in the order of the MMA's fragments, and streams its share of the
// channels, N / G each.  The share is a line of (16 channels, depth 128) units that its 16 warps split evenly; a lane loads 16 consecutive
// weights of two channels straight into registers, I8S_AHEAD units ahead, and widens them there.
// (An MMA may take its depth in any order, so the 16 are its numbers 4 j .. 4 j + 3 of product j,
// and no lane exchanges anything.  The tensor core's 8-bit integer products need no widening, but took
// 18.8 us where these take 11 with 4 tokens, 15360 channels and depth 5120.)  The warps' sums
// meet in shared memory, in warp order.  4 x 15360 x 5120: 18.3 us, of which some 3 until the
// tokens are quantised and 2 the sums and outputs; the stream between them is near HBM's rate, and near that of
// the half-rate integer pipe, which 3 of the 5 instructions that widen 4 weights share.  (Asking the weights into L2
// at the kernel's start: 18.9 us.)
constexpr int I8S_THREADS = 512, I8S_WARPS = I8S_THREADS / 32, I8S_AHEAD = 4, I8S_GROUPS = 16;
constexpr int I8S_MAX_M = 32, I8S_TOKEN_BYTES = 144 * 1024;

__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_stream(const void *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

struct I8Small {
    int M, N, K, KB, G;        // KB: units of depth 128
    int epi;
    const void *A;
    const float *a_scale;      // or NULL: quantised here
    const signed char *W;
    const float *w_scale, *bias, *gate;
    const void *resid;
    void *out;
};

// Quantises (or widens) the tokens into dst: vector v of 8 numbers of token m at
// [v / 8][v % 2][m][v / 2 % 4].  A token has 16 / M warps (a power of two, at least one).
template <typename T>
__device__ __forceinline__ void i8_stage_tokens(const I8Small &s, uint4 *dst, float *sh_scale, unsigned *sh_top) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nv = s.K / 8, nvp = s.KB * 16;
    auto place = [&](int m, int v) -> uint4 & { return dst[((size_t)((v >> 3) * 2 + (v & 1)) * s.M + m) * 4 + ((v >> 1) & 3)]; };
    if (s.a_scale != nullptr) {
        const uint2 *A = reinterpret_cast<const uint2 *>(s.A);
        for (int x = tid; x < s.M * nvp; x += I8S_THREADS) {
            const int m = x / nvp, v = x - m * nvp;
            uint4 u = make_uint4(0, 0, 0, 0);
            if (v < nv) {
                const uint2 w = A[(size_t)m * nv + v];
                widen4(w.x, u.x, u.y);
                widen4(w.y, u.z, u.w);
            }
            place(m, v) = u;
        }
        if (tid < s.M) sh_scale[tid] = s.a_scale[tid];
        return;
    }
    constexpr int KEEP = sizeof(T) == 2 ? 8 : 4;       // vectors of a lane's first token that stay in registers
    const T *A = reinterpret_cast<const T *>(s.A);
    int wpr = 1;
    while (2 * wpr * s.M <= I8S_WARPS) wpr *= 2;
    const int per = I8S_WARPS / wpr, m0 = warp / wpr, v0 = (warp % wpr) * 32 + lane, dv = 32 * wpr;
    Vec8<T> x[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (m0 < s.M && v0 + i * dv < nv) x[i].load(A + (size_t)m0 * s.K + 8 * (v0 + i * dv));
    for (int m = m0; m < s.M; m += per) {
        const T *row = A + (size_t)m * s.K;
        unsigned top = 0;
        int v = v0;
        if (m == m0) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if (v0 + i * dv < nv) top = x[i].top(top);
            v = v0 + KEEP * dv;
        }
        for (; v < nv; v += dv) {
            Vec8<T> z;
            z.load(row + 8 * v);
            top = z.top(top);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) atomicMax(&sh_top[m], top);
    }
    __syncthreads();
    for (int m = m0; m < s.M; m += per) {
        const T *row = A + (size_t)m * s.K;
        const QuantRow qr(sh_top[m]);
        if (v0 == 0) sh_scale[m] = quant_scale(sh_top[m]);
        float e[8];
        int v = v0;
        if (m == m0) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if (v0 + i * dv < nv) {
                    quant8<T>(x[i], qr, e);
                    place(m, v0 + i * dv) = half8(e);
                }
            v = v0 + KEEP * dv;
        }
        for (; v < nv; v += dv) {
            Vec8<T> z;
            z.load(row + 8 * v);
            quant8<T>(z, qr, e);
            place(m, v) = half8(e);
        }
        for (v = nv + v0; v < nvp; v += dv) place(m, v) = make_uint4(0, 0, 0, 0);      // depth past K
    }
}

template <typename T, int NT8>
__global__ void __launch_bounds__(I8S_THREADS, 1) linear_i8_small_kernel(const __grid_constant__ I8Small s) {
    extern __shared__ __align__(16) uint4 sm_small[];
    __shared__ float sh_scale[I8S_MAX_M];
    __shared__ unsigned sh_top[I8S_MAX_M];
    constexpr int MP = 8 * NT8;
    uint4 *tok = sm_small;                             // [2 KB][2][M][4]
    float *part = reinterpret_cast<float *>(tok + (size_t)s.KB * 16 * s.M);       // [slot][16][MP]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    const int row0 = (int)((long long)s.N * blockIdx.x / s.G), row1 = (int)((long long)s.N * (blockIdx.x + 1) / s.G);
    if (tid < I8S_MAX_M) sh_top[tid] = 0;
    __syncthreads();
    pdl_wait();
    pdl_release();
    i8_stage_tokens<T>(s, tok, sh_scale, sh_top);
    const bool tail = s.K % 128 != 0;
    for (int p0 = row0; p0 < row1; p0 += 16 * I8S_GROUPS) {
        const int rows = min(row1 - p0, 16 * I8S_GROUPS), groups = (rows + 15) / 16;
        const int U = groups * s.KB, q = U / I8S_WARPS, rem = U - q * I8S_WARPS;
        const int u0 = warp * q + min(warp, rem), u1 = u0 + q + (warp < rem ? 1 : 0);
        uint4 w[I8S_AHEAD][4];
        // The next unit to load: this lane's 16 weights of rows gid and gid + 8 in either half of the depth.  Rows
        // and depth that do not exist are read as others that do: no output takes those rows, and the
        // tokens are zero there.
        int g = u0 / s.KB, k = u0 - g * s.KB, lu = u0, lk = k, lg = g;
        const signed char *pa, *pb;
        auto rows_of = [&]() {
            const int r = 16 * lg + gid, off = 128 * lk + 16 * tig;
            pa = s.W + (size_t)(p0 + min(r, rows - 1)) * s.K + off;
            pb = s.W + (size_t)(p0 + min(r + 8, rows - 1)) * s.K + off;
        };
        rows_of();
        auto fetch = [&](uint4 (&x)[4]) {
            if (lu >= u1) return;
            int o0 = 0, o1 = 64;
            if (tail && lk + 1 == s.KB) {
                const int most = s.K - 16 - (128 * lk + 16 * tig);
                o0 = min(o0, most);
                o1 = min(o1, most);
            }
            x[0] = load_stream(pa + o0);
            x[1] = load_stream(pb + o0);
            x[2] = load_stream(pa + o1);
            x[3] = load_stream(pb + o1);
            ++lu;
            pa += 128;
            pb += 128;
            if (++lk == s.KB) {
                lk = 0;
                ++lg;
                rows_of();
            }
        };
#pragma unroll
        for (int i = 0; i < I8S_AHEAD; ++i) fetch(w[i]);
        __syncthreads();                               // tokens staged; the last pass's sums read
        const uint4 *t = tok + (size_t)k * 16 * s.M + 4 * gid + tig;
        // four products a half: sums of their own where registers allow, as each waits for the one it adds to
        constexpr int SETS = NT8 == 1 ? 4 : NT8 == 2 ? 2 : 1;
        float acc[SETS][NT8][4] = {};
        // warp w's sums of group g: slot g + w (both only grow)
        auto flush = [&]() {
            float *dst = part + (size_t)(g + warp) * 16 * MP;
#pragma unroll
            for (int n = 0; n < NT8; ++n) {
#pragma unroll
                for (int i = 1; i < SETS; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[0][n][j] += acc[i][n][j];
                        acc[i][n][j] = 0.0f;
                    }
                *reinterpret_cast<float2 *>(dst + gid * MP + 8 * n + 2 * tig) = make_float2(acc[0][n][0], acc[0][n][1]);
                *reinterpret_cast<float2 *>(dst + (gid + 8) * MP + 8 * n + 2 * tig) = make_float2(acc[0][n][2], acc[0][n][3]);
                acc[0][n][0] = acc[0][n][1] = acc[0][n][2] = acc[0][n][3] = 0.0f;
            }
        };
        for (int u = u0; u < u1; u += I8S_AHEAD) {
#pragma unroll
            for (int i = 0; i < I8S_AHEAD; ++i) {
                if (u + i >= u1) break;
#pragma unroll
                for (int hk = 0; hk < 2; ++hk) {
                    const unsigned *x0 = reinterpret_cast<const unsigned *>(&w[i][2 * hk]), *x1 = reinterpret_cast<const unsigned *>(&w[i][2 * hk + 1]);
                    unsigned a[4][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        widen4(x0[j], a[j][0], a[j][2]);
                        widen4(x1[j], a[j][1], a[j][3]);
                    }
                    if (hk == 1) fetch(w[i]);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int n = 0; n < NT8; ++n) {
                            uint4 b = make_uint4(0, 0, 0, 0);
                            if (8 * n + gid < s.M) b = t[32 * n + 4 * h * s.M];
                            mma_f16(acc[(2 * h) % SETS][n], a[2 * h][0], a[2 * h][1], a[2 * h][2], a[2 * h][3], b.x, b.y);
                            mma_f16(acc[(2 * h + 1) % SETS][n], a[2 * h + 1][0], a[2 * h + 1][1], a[2 * h + 1][2], a[2 * h + 1][3], b.z, b.w);
                        }
                    t += 8 * s.M;
                }
                if (++k == s.KB) {
                    flush();
                    k = 0;
                    ++g;
                    t -= (size_t)s.KB * 16 * s.M;
                }
            }
        }
        if (u1 > u0 && k > 0) flush();
        __syncthreads();
        // every output of the pass: its group's sums
        const T *resid = reinterpret_cast<const T *>(s.resid);
        T *out = reinterpret_cast<T *>(s.out);
        for (int x = tid; x < rows * s.M; x += I8S_THREADS) {
            const int m = x / rows, r = x - m * rows, grp = r >> 4, n = p0 + r;
            const int a0 = grp * s.KB, a1 = a0 + s.KB - 1, longer = rem * (q + 1);
            const int w0 = a0 < longer ? a0 / (q + 1) : rem + (a0 - longer) / q, w1 = a1 < longer ? a1 / (q + 1) : rem + (a1 - longer) / q;
            float v = 0.0f;
            for (int y = w0; y <= w1; ++y) v += part[((size_t)(grp + y) * 16 + (r & 15)) * MP + m];
            const size_t at = (size_t)m * s.N + n;
            const float res = s.epi == EPI_RESID_GATE ? to_f(resid[at]) : 0.0f, gt = s.epi == EPI_RESID_GATE ? s.gate[n] : 0.0f;
            out[at] = from_f<T>(i8_epilogue<T>(s.epi, v, sh_scale[m], s.w_scale[n], s.bias[n], gt, res));
        }
    }
}

// ------------------------------------------------------------------- host
// Tokens that fit every CTA's shared memory go with the weights' stream.  Against the three kernels, us, weights from DRAM
// (K 5120, N 15360) or L2 (1536, 4608): 4 tokens 19.2 and 26.4, 5.9 and 8.8; 8 tokens 21.3 and 26.8, 6.4 and 9.3; 16 tokens
// of 1536 8.5 and 10.3.  The rule is the memory's, and takes the slower side where a warp's sums are
// many beside its products or the tokens fill the memory: 12 tokens of 5120 32.5 and 27.2, 24 and 32 of 1536
// 16.7 and 10.6, 17.4 and 11.0, 5 of 13824 (N 5120) 29.1 and 24.9.
static bool i8_small(int M, int K) { return M <= I8S_MAX_M && (long)M * ((K + 127) / 128 * 128) * 2 <= I8S_TOKEN_BYTES; }

template <typename T, int NT8>
static cudaError_t i8_small_launch(const I8Small &s, cudaStream_t st) {
    static DeviceSet asked{0};
    const int part = (I8S_GROUPS + I8S_WARPS) * 16 * 8 * NT8 * 4;
    const cudaError_t e = allow_smem(linear_i8_small_kernel<T, NT8>, I8S_TOKEN_BYTES + part, asked);
    if (e != cudaSuccess) return e;
    return launch_pdl(linear_i8_small_kernel<T, NT8>, dim3(s.G), dim3(I8S_THREADS), s.M * s.KB * 256 + part, st, s);
}
template <typename T>
static cudaError_t i8_small_run(const LinearI8Args &a, cudaStream_t st) {
    I8Small s{};
    s.M = a.M;
    s.N = a.N;
    s.K = a.K;
    s.KB = (a.K + 127) / 128;
    s.G = std::min(device_sms(), (a.N + 7) / 8);
    s.epi = a.epi;
    s.A = a.A;
    s.a_scale = a.a_scale;
    s.W = a.W;
    s.w_scale = a.w_scale;
    s.bias = a.bias;
    s.gate = a.gate;
    s.resid = a.resid;
    s.out = a.out;
    if (a.M <= 8) return i8_small_launch<T, 1>(s, st);
    if (a.M <= 16) return i8_small_launch<T, 2>(s, st);
    return i8_small_launch<T, 4>(s, st);
}

struct I8Plan {
    I8Sched s;
    size_t off_scale, off_part, bytes;
    int smem, cut;             // cut: whether a tile may be cut
};
static I8Plan i8_plan(int M, int N, int K) {
    I8Plan p;
    I8Sched &s = p.s;
    s = I8Sched{};
    s.M = M;
    s.N = N;
    const int mt = (M + I8_NT - 1) / I8_NT;
    s.NT = ((M + mt - 1) / mt + 15) / 16 * 16;         // the tiles of tokens as even as they come
    s.m_tiles = (M + s.NT - 1) / s.NT;
    s.n_pairs = (N + 2 * I8_BM - 1) / (2 * I8_BM);
    s.KT = (K + I8_BK - 1) / I8_BK;
    const int tiles = s.m_tiles * s.n_pairs;
    s.P = (int)std::min<long long>(std::max(device_sms() / 2, 1), (long long)tiles * s.KT);
    s.n_full = tiles / s.P * s.P;
    p.cut = s.n_full < tiles;
    s.acs = (s.NT + 31) / 32 * 32;
    s.as = std::min(I8_MAX_A, (512 - 2 * s.acs) / 32);
    // as deep as fits, the weights' ring half a tile deeper than the tokens'
    const int b_bytes = 128 * s.NT;
    s.wst = std::min(I8_MAX_W, (I8_SMEM + I8_W_BYTES / 2) / (I8_W_BYTES + 2 * b_bytes) + 1);
    s.bst = std::min(I8_MAX_B, (I8_SMEM - s.wst * I8_W_BYTES) / b_bytes);
    p.smem = s.wst * I8_W_BYTES + s.bst * b_bytes + 1024;
    p.off_scale = ((size_t)M * K * 2 + 255) / 256 * 256;
    p.off_part = p.off_scale + ((size_t)s.m_tiles * s.NT + 16) * sizeof(float);
    p.off_part = (p.off_part + 255) / 256 * 256;
    p.bytes = p.off_part + (p.cut ? (size_t)4 * s.P * s.NT * I8_BM * sizeof(float) : 0);
    return p;
}
size_t linear_i8_workspace_bytes(int M, int N, int K) { return i8_small(M, K) ? 0 : i8_plan(M, N, K).bytes; }

template <typename T>
static cudaError_t i8_launch(const I8Plan &p, const CUtensorMap &tw, const CUtensorMap &ta, int *err, cudaStream_t st) {
    static DeviceSet asked{0};
    cudaError_t e = allow_smem(linear_i8_kernel<T>, I8_SMEM + 1024, asked);
    if (e != cudaSuccess) return e;
    e = launch_pdl(linear_i8_kernel<T>, dim3(2 * p.s.P), dim3(I8_THREADS), p.smem, st, tw, ta, p.s, err);
    if (e != cudaSuccess || !p.cut) return e;
    return launch_pdl(linear_i8_merge_kernel<T>, dim3(2 * (p.s.m_tiles * p.s.n_pairs - p.s.n_full), (p.s.NT + I8M_TOKENS - 1) / I8M_TOKENS), dim3(I8M_THREADS), 0, st, p.s);
}

cudaError_t linear_i8(const LinearI8Args &a, void *ws, int *err, cudaStream_t st) {
    if (i8_small(a.M, a.K)) return a.dtype == XC_BF16 ? i8_small_run<bf16>(a, st) : i8_small_run<float>(a, st);
    I8Plan p = i8_plan(a.M, a.N, a.K);
    I8Sched &s = p.s;
    char *w = reinterpret_cast<char *>(ws);
    __half *tokens = reinterpret_cast<__half *>(w);
    float *scale = reinterpret_cast<float *>(w + p.off_scale);
    s.epi = a.epi;
    s.a_scale = scale;
    s.w_scale = a.w_scale;
    s.bias = a.bias;
    s.gate = a.gate;
    s.resid = a.resid;
    s.out = a.out;
    s.part = reinterpret_cast<float *>(w + p.off_part);
    s.vec = a.N % 8 == 0 && ((reinterpret_cast<uintptr_t>(a.out) | reinterpret_cast<uintptr_t>(a.resid)) & 15) == 0;
    CUtensorMap tw, ta;
    if (!make_tmap_2d(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.W, a.N, a.K, I8_BM, 128) ||
        !make_tmap_2d(&ta, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, tokens, a.M, a.K, s.NT, 64))
        return cudaErrorInvalidValue;
    cudaError_t e;
    if (a.a_scale != nullptr) {
        const long n = (long)a.M * a.K / 16;
        const long ctas = std::min<long>((n + 255) / 256, (long)device_sms() * 8);
        e = launch_pdl(widen_kernel, dim3((unsigned)ctas), dim3(256), 0, st, reinterpret_cast<const uint4 *>(a.A),
                       reinterpret_cast<uint4 *>(tokens), n, a.a_scale, scale, a.M);
    } else {
        e = a.dtype == XC_BF16 ? quantize_launch(reinterpret_cast<const bf16 *>(a.A), tokens, scale, a.M, a.K, st)
                               : quantize_launch(reinterpret_cast<const float *>(a.A), tokens, scale, a.M, a.K, st);
    }
    if (e != cudaSuccess) return e;
    return a.dtype == XC_BF16 ? i8_launch<bf16>(p, tw, ta, err, st) : i8_launch<float>(p, tw, ta, err, st);
}

}  // namespace xc
