// 8-bit products: rows quantised to int8 with a scale each, int8 x int8 -> int32 products with
// scales per token and per output channel, and the gated feed-forward block made of them.
//
//   s_t = max_k |x_tk| / 127 (fp32),  q_tk = the whole number nearest to x_tk / s_t
//   y_tn = (sum_k q_tk w_nk) s_t c_n
//
// The int32 sums are exact (k <= 131071: 2^14 k < 2^31), so a product differs from its definition
// by the three fp32 roundings of its scaling and the last one to the output's type.
#include "dense.h"

namespace elb {

namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// The whole number nearest to x / s (ties to even), from one that is off by at most one: the
// remainder x - q s is exact near a half (x and s have 24 bits, and it is a multiple of the smaller
// one's last) and decides.
__device__ __forceinline__ float settle(float q, float x, float s) {
    const float r = fmaf(-q, s, x), a = 2.0f * fabsf(r);
    if (a > s || (a == s && fmodf(q, 2.0f) != 0.0f)) q += copysignf(1.0f, r);
    return fminf(fmaxf(q, -127.0f), 127.0f);
}

// A row's scale s and its reciprocal; a small s (whose reciprocal may be infinite) times 2^64, as
// its values then are.
struct RowScale {
    float s, su, inv, up;
    __device__ __forceinline__ explicit RowScale(float amax) {
        s = amax / 127.0f;
        up = s < 1e-30f ? 0x1p64f : 1.0f;
        su = s * up;
        inv = s > 0.0f ? 1.0f / su : 0.0f;
    }
};

// Eight values to whole numbers, four to a word.  x / s is taken as x inv, off by 2^-24 of itself,
// at most 2^-17, and rounded by adding 3 2^22, which leaves the whole number in the low bits; where
// it lies within 2^-14 of a half (one value in 8000 of fp32 rows; of bf16 rows, whose quotients are ratios
// of 8 bits and meet halves exactly, one in 500 to 6000), or s is small, the remainder settles it.
template <class X>  // eight values: an array of floats, or as loaded
__device__ __forceinline__ u32x2_t quantize8(const X& x, const RowScale& r) {
    constexpr float kMagic = 12582912.0f;
    uint32_t u[8];
    float far = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = fmaf(x[e], r.inv, kMagic);
        u[e] = __float_as_uint(t);
        far = fmaxf(far, fabsf(fmaf(x[e], r.inv, -(t - kMagic))));
    }
    if (far > 0.5f - 0x1p-14f || r.up != 1.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = x[e] * r.up, q = __builtin_rintf(v * r.inv);
            u[e] = r.s > 0.0f ? (uint32_t)(int)settle(q, v, r.su) : 0u;
        }
    }
    u32x2_t w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(u[4 * h + 1], u[4 * h], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(u[4 * h + 3], u[4 * h + 2], 0x0c0c0400u);
        w[h] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
    return w;
}

// maxima in which NaN is the largest (fmaxf drops it): a row that holds one has a scale of NaN, and
// so have its products
__device__ __forceinline__ float max_nan(float a, float b) {
    return __builtin_elementwise_maximum(a, b);
}
template <class X>
__device__ __forceinline__ float max8(const X& x, float m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(x[e]));
    return m;
}
// the largest over a wave of values of at least zero (lanes without a source get zero)
__device__ __forceinline__ float wave_max(float m) {
#define ELB_MAX_STEP(ctrl, rows)                                                             \
    m = max_nan(m, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(m), ctrl,  \
                                                               rows, 0xf, false)))
    ELB_MAX_STEP(0x111, 0xf);  // row_shr:1, 2, 4, 8: lane 15 of each row of 16 has the row's
    ELB_MAX_STEP(0x112, 0xf);
    ELB_MAX_STEP(0x114, 0xf);
    ELB_MAX_STEP(0x118, 0xf);
    ELB_MAX_STEP(0x142, 0xa);  // row_bcast:15 to rows 1 and 3, row_bcast:31 to rows 2 and 3
    ELB_MAX_STEP(0x143, 0xc);
#undef ELB_MAX_STEP
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), 63));
}

typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(1)));

// N threads a row (a wave, or a block of 256), 256 / N rows a block.  A thread keeps the first
// four groups of eight values in registers between the maximum and the rounding; longer rows are
// read again, from L2.
template <class T, int N>
__global__ __launch_bounds__(256) void quantize_rows(const T* __restrict__ x, int64_t d,
                                                     int64_t rows, int8_t* __restrict__ q,
                                                     float* __restrict__ scale, Counters clear) {
    constexpr int KEEP = 4;
    clear_counters(clear.p, clear.n);
    const int tid = threadIdx.x % N;
    const int64_t row = (int64_t)dense_block_number() * (256 / N) + threadIdx.x / N;
    if (row >= rows) return;  // a whole wave, or a whole block
    const T* const xr = x + row * d;
    Eight<T> keep[KEEP];
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t c = (i * N + tid) * 8;
        if (c < d) keep[i].load(xr + c);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if ((i * N + tid) * 8 < d) mx = max8(keep[i], mx);
    for (int64_t c = (KEEP * N + tid) * 8; c < d; c += N * 8) {
        float v[8];
        load8(xr + c, v);
        mx = max8(v, mx);
    }
    mx = wave_max(mx);
    if constexpr (N == 256) {
        __shared__ float part[4];
        if ((tid & 63) == 0) part[tid >> 6] = mx;
        __syncthreads();
        mx = max_nan(max_nan(part[0], part[1]), max_nan(part[2], part[3]));
    }
    const RowScale r(mx);
    if (tid == 0) scale[row] = r.s;
    int8_t* const qr = q + row * d;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t c = (i * N + tid) * 8;
        if (c < d) *reinterpret_cast<u32x2_any_t*>(qr + c) = quantize8(keep[i], r);
    }
    for (int64_t c = (KEEP * N + tid) * 8; c < d; c += N * 8) {
        float v[8];
        load8(xr + c, v);
        *reinterpret_cast<u32x2_any_t*>(qr + c) = quantize8(v, r);
    }
}

// ------------------------------------------------------------------------------------------
// The split form with the quantisation in it, for few rows: every block quantises its TM rows of x
// into LDS (as the product's k-tiles) and then multiplies them with its weight rows, whose first
// k-tiles are copied meanwhile.  The blocks repeat each other's quantisation, 16 or 32 rows of at
// most KMAX values.  For up to some ten rows that takes them less than the launch that it saves, for
// more rows about as long, and longer from some hundred on (us on the GPU, here / in its own launch,
// 2048 values to 2048 channels, fp32: one row 5.0 / 7.0, 8 rows 5.8 / 7.8, 16 rows 7.5 / 7.9, 40 rows
// 8.5 / 8.5, 128 rows 12.2 / 9.2; one token through the bf16 block of d = 2048, m = 1024 10.6 / 14.2).
// bf16 rows take longer where many quotients are settled (quantize8): gaussian ones 40 rows 10 to 14 /
// 9.2, with one channel in 64 eight times as large 6.7 to 7.3 / 8.2.
// ------------------------------------------------------------------------------------------
template <class T, int TM, int TN, int NW, bool PAIR, int S, int KMAX>
struct QuantForm {
    static constexpr int FM = TM / 16, FN = TN / 16;
    static constexpr int BU = TN * 128, AU = TM * 128;
    static constexpr int RING = NW * S * BU, XQ = TM * KMAX;
    static constexpr int LDS = RING + XQ + TM * 4;
    typedef SplitJoin<I8, TM, TN, NW, PAIR> Join;
    static_assert(NW * Join::PART <= RING + XQ && KMAX % 512 == 0 && LDS <= 160 * 1024, "");
    typedef Copier<KC, TN, 1, 1, PAIR, true> CB;

    template <class Epi>
    static __device__ __forceinline__ void run(const TileIn& in, char* sm, Epi epi) {
        const int lane = threadIdx.x & 63;
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        char* const xq = sm + RING;
        float* const scales = reinterpret_cast<float*>(sm + RING + XQ);
        const int K = (int)in.K, kend = (K + 127) / 128 * 128;
        // a wave's rows, loaded before the weights' copies are issued (loads return in order); lanes
        // past K have zeros, rows past the last one are left out: they give no result
        constexpr int G = KMAX / 512, RW = TM / NW;  // groups of eight values a lane, rows
        Eight<T> x[RW][G];
#pragma unroll
        for (int j = 0; j < RW; ++j)
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const int r = w + j * NW, c = (i * 64 + lane) * 8;
                x[j][i] = Eight<T>{};
                if (r < in.rows && c < K)
                    x[j][i].load(reinterpret_cast<const T*>(in.a + r * in.lda) + c);
            }
        CB cb;
        cb.init(in.b, in.b2, in.ldb, in.cols, in.K, lane, 0);
        Reader<I8, 16, KC, TM> ra;
        Reader<I8, 16, KC, TN> rb;
        ra.init(0, lane);
        rb.init(0, lane);
        char* const ring = sm + w * S * BU;
        const uint32_t lds = __builtin_amdgcn_readfirstlane(
            (uint32_t)(uintptr_t)(lds_void_t*)sm + (uint32_t)(w * S * BU));
        const int nt = in.t1, t0 = nt * w / NW, t1 = nt * (w + 1) / NW;
#pragma unroll
        for (int p = 0; p < S; ++p) cb.issue(t0 + p, t1, lds + p * BU, ring + p * BU, lane, 0);

        float mx[RW];
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            mx[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < G; ++i) mx[j] = max8(x[j][i], mx[j]);
        }
#pragma unroll
        for (int j = 0; j < RW; ++j) mx[j] = wave_max(mx[j]);
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            const int r = w + j * NW;
            if (r >= in.rows) break;
            const RowScale s(mx[j]);
            if (lane == 0) scales[r] = s.s;
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const int c = (i * 64 + lane) * 8;
                if (c < kend)
                    *reinterpret_cast<u32x2_t*>(xq + c / 128 * AU + r * 128 +
                                                kc_swz(r, c % 128 / 16) * 16 + c % 16) =
                        quantize8(x[j][i], s);
            }
        }
        __syncthreads();

        typename Mma<I8, 16>::acc acc[FM][FN];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = i32x4_t{};
        int u = 0;
        for (int t = t0; t < t1; ++t) {
            ELB_WAIT_VMCNT((S - 1) * CB::N);
            asm volatile("" ::: "memory");
            const char* const pa = xq + t * AU;
            const char* const pb = ring + u * BU;
            i32x4_t fa[2][FM], fb[2][FN];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[ks][j] = rb.load(pb, j, ks);
#pragma unroll
                for (int i = 0; i < FM; ++i) fa[ks][i] = ra.load(pa, i, ks);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the unit is free again
            cb.issue(t + S, t1, lds + u * BU, ring + u * BU, lane, 0);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = Mma<I8, 16>::mma(fb[ks][j], fa[ks][i], acc[i][j]);
            u = u + 1 == S ? 0 : u + 1;
        }
        epi.s = scales;
        Join::run(acc, in, sm, lane, w, epi);
    }
};

template <class T, int TM, int TN, int NW, bool PAIR, int S, int KMAX, class Epi>
__global__ __launch_bounds__(NW * 64) void dense_quant(DenseIn d, int mt, int nt, Epi epi) {
    typedef QuantForm<T, TM, TN, NW, PAIR, S, KMAX> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    int m, n;
    if (!dense_tile(dense_block_number(), mt, nt, m, n)) return;
    dense_block<Form, I8, TM, TN, KC, KC, PAIR>(d, m, n, sm, epi);
}

// v = v s c from left to right, eight values of a row.  FAR, for waves with a row whose |s| is 2^96
// or more: that s over 2^64 on the way, since v s alone (v up to 2^31) would pass the largest fp32 where
// c brings it back.  Powers of two: no rounding differs.  A scalar branch chooses (us, 16384 x 4096 x
// 512, mostly epilogue: never FAR 73.0, chosen 74.8, always 75.0; 2048 and 8192 deep 0 to 1 %).
__device__ __forceinline__ bool any_far(float s) {
    return __builtin_expect(__builtin_amdgcn_ballot_w64(fabsf(s) >= 0x1p96f) != 0, 0);
}
template <bool FAR>
__device__ __forceinline__ void scale8(float (&v)[8], float s, const Eight<float>& c) {
#pragma clang fp contract(off)  // the same roundings in every kernel
    const bool far = FAR && fabsf(s) >= 0x1p96f;
    const float down = far ? s * 0x1p-64f : s, up = far ? 0x1p64f : 1.0f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        v[q] = v[q] * down * c[q];
        if (FAR) v[q] *= up;
    }
}

template <class T>
struct ScaledOut {  // y = [res +] v s_row c_col
    static constexpr bool kMayHalve = true;
    T* y;
    const T* res;
    const float *s, *c;
    int64_t ld;
    __device__ __forceinline__ ScaledOut at(int64_t r0, int c0) const {
        const int64_t o = r0 * ld + c0;
        return {y + o, res ? res + o : nullptr, s ? s + r0 : nullptr, c + c0, ld};
    }
    struct Extra {
        Eight<float> c;
        float s;
        Eight<T> r;
    };
    __device__ __forceinline__ void fetch(int row, int col, Extra& e) const {
        e.c.load(c + col);
        e.s = s[row];
        if (res) e.r.load(res + row * ld + col);
    }
    __device__ __forceinline__ void put(int row, int col, float (&v)[8], const Extra& e) const {
#pragma clang fp contract(off)  // the same roundings in every kernel
        if (any_far(e.s)) scale8<true>(v, e.s, e.c);
        else scale8<false>(v, e.s, e.c);
        if (res) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += e.r[q];
        }
        store8(y + row * ld + col, v);
    }
};

// h = silu(g) u in fp32: rounded to bf16 first (2^-9 of a value, up to a quarter of a step), one h
// in eight of those at 64 steps or more would move to the next whole number when it is quantised
// (8192 columns, gaussian g and u: 13.7 %; of all h 1.1 %)
struct ScaledGateOut {
    static constexpr bool kMayHalve = false;
    float* h;
    const float *s, *c;  // c: m scales of the gate rows, then m of the up rows
    int64_t m;
    __device__ __forceinline__ ScaledGateOut at(int64_t r0, int c0) const {
        return {h + r0 * m + c0, s ? s + r0 : nullptr, c + c0, m};
    }
    struct Extra {
        Eight<float> g, u;
        float s;
    };
    __device__ __forceinline__ void fetch(int row, int col, Extra& e) const {
        e.g.load(c + col);
        e.u.load(c + m + col);
        e.s = s[row];
    }
    __device__ __forceinline__ void put(int row, int col, float (&g)[8], float (&u)[8],
                                        const Extra& e) const {
#pragma clang fp contract(off)
        if (any_far(e.s)) {
            scale8<true>(g, e.s, e.g);
            scale8<true>(u, e.s, e.u);
        } else {
            scale8<false>(g, e.s, e.g);
            scale8<false>(u, e.s, e.u);
        }
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = g[q] * sigma_f32(g[q]) * u[q];
        store8(h + row * m + col, v);
    }
};

template <class T>
hipError_t quantize(const void* x, int64_t rows, int d, int8_t* q, float* scale, Counters clear,
                    hipStream_t s) {
    ProfileScope prof("quantize_rows", s);
    // a wave per row where its lanes can keep it and the rows fill the chip (us, wave / block a row:
    // 65536 x 512 24.5 / 60.9, 16384 x 2048 23.0 / 24.8, 8192 x 1024 9.6 / 11.8, 4096 x 2048 12.4 /
    // 10.2, 300 x 2048 8.7 / 4.1)
    if (d <= 2048 && rows >= 8192)
        ELB_LAUNCH((quantize_rows<T, 64>), grid_of((rows + 3) / 4), dim3(256), 0, s, (const T*)x,
                   (int64_t)d, rows, q, scale, clear);
    else
        ELB_LAUNCH((quantize_rows<T, 256>), grid_of(rows), dim3(256), 0, s, (const T*)x,
                   (int64_t)d, rows, q, scale, clear);
    return hipGetLastError();
}

template <bool PAIR, class Epi>
void product(const int8_t* a, const int8_t* w, int64_t rows, int cols, int64_t K, const Epi& epi,
             hipStream_t s, void* part = nullptr) {
    const DenseIn d{(const char*)a, (const char*)w, K, K, rows, cols, K, (char*)part, nullptr, 0};
    run_product<I8, KC, PAIR>(d, aligned16(a, w), epi, s);
}

template <class T, int TM, int TN, int NW, bool PAIR, int S, int KMAX, class Epi>
void run_quant(const DenseIn& d, const Epi& epi, hipStream_t s) {
    const int mt = tiles(d.rows, TM), nt = tiles(d.cols, PAIR ? TN / 2 : TN);
    ELB_LAUNCH((dense_quant<T, TM, TN, NW, PAIR, S, KMAX, Epi>), grid_of(up8((int64_t)mt * nt)),
               dim3(NW * 64), 0, s, d, mt, nt, epi);
}

// Whether the product of float rows takes a form that quantises them itself.
bool quant_fused(const int8_t* w, int64_t rows, int64_t cols, int64_t K) {
    return aligned16(w, w) &&
           form_quantises(pick_form(rows, cols, (K + 127) / 128, false, true), K);
}

// x [rows, K] of type T times w; only where quant_fused() says so
template <class T, bool PAIR, class Epi>
void product_of(const void* x, const int8_t* w, int64_t rows, int cols, int64_t K,
                const Epi& epi, hipStream_t s) {
    const DenseIn d{(const char*)x, (const char*)w, K * (int64_t)sizeof(T), K, rows, cols, K,
                    nullptr, nullptr, 0};
    switch (pick_form(rows, PAIR ? 2 * (int64_t)cols : cols, (K + 127) / 128, false, true)) {
        case kSplit16x16: return run_quant<T, 16, 16, 8, PAIR, 4, kFusedK>(d, epi, s);
        case kSplit16x32: return run_quant<T, 16, 32, 8, PAIR, 3, kFusedK>(d, epi, s);
        case kSplit16x64: return run_quant<T, 16, 64, 4, PAIR, 3, kFusedK>(d, epi, s);
        default: return run_quant<T, 32, 32, 8, PAIR, 2, kFusedK>(d, epi, s);
    }
}

template <class T, class O>
void linear_of(const void* x, const int8_t* w, const float* c, const void* res, int64_t rows, int n,
               int k, void* y, hipStream_t s) {
    product_of<T, false>(x, w, rows, n, k, ScaledOut<O>{(O*)y, (const O*)res, nullptr, c, n}, s);
}

template <class T>
hipError_t linear(const void* x, const int8_t* w, const float* c, const void* res, int64_t rows,
                  int n, int k, int out, void* y, int8_t* q, float* scale, void* part,
                  hipStream_t s) {
    constexpr int in = sizeof(T) == 2 ? ELB_BF16 : ELB_F32;
    if (quant_fused(w, rows, n, k)) {
        ProfileScope prof("linear_i8", s);
        if (out == ELB_BF16) linear_of<T, bf16_t>(x, w, c, res, rows, n, k, y, s);
        else linear_of<T, float>(x, w, c, res, rows, n, k, y, s);
        return hipGetLastError();
    }
    if (hipError_t e = launch_quantize_rows(x, rows, k, in, q, scale, s, part, n)) return e;
    return launch_gemm_i8(q, scale, w, c, res, rows, n, k, out, y, s, part);
}

template <class T>
hipError_t gate_up(const void* x, const int8_t* w, const float* c, int64_t rows, int d, int m,
                   float* h, int8_t* q, float* scale, hipStream_t s) {
    constexpr int in = sizeof(T) == 2 ? ELB_BF16 : ELB_F32;
    const bool fused = quant_fused(w, rows, 2 * (int64_t)m, d);
    if (!fused)
        if (hipError_t e = launch_quantize_rows(x, rows, d, in, q, scale, s)) return e;
    ProfileScope prof("gate_up_i8", s);
    if (fused) product_of<T, true>(x, w, rows, m, d, ScaledGateOut{h, nullptr, c, m}, s);
    else product<true>(q, w, rows, m, d, ScaledGateOut{h, scale, c, m}, s);
    return hipGetLastError();
}

}  // namespace

size_t i8_halves_bytes(int64_t T, int n, int k, bool most) {
    return (most ? halves_reserve : halves_bytes)(T, n, ((int64_t)k + 127) / 128, false);
}

hipError_t launch_quantize_rows(const void* x, int64_t rows, int d, int dtype, int8_t* q,
                                float* scale, hipStream_t s, void* part, int n) {
    const Counters c = halves_counters((char*)part, rows, n, (d + 127) / 128, false);
    return dtype == ELB_BF16 ? quantize<bf16_t>(x, rows, d, q, scale, c, s)
                             : quantize<float>(x, rows, d, q, scale, c, s);
}

hipError_t launch_gemm_i8(const int8_t* a, const float* a_scale, const int8_t* w,
                          const float* w_scale, const void* res, int64_t T, int n, int k,
                          int dtype, void* y, hipStream_t s, void* part) {
    ProfileScope prof("product_i8", s);
    if (dtype == ELB_BF16)
        product<false>(a, w, T, n, k, ScaledOut<bf16_t>{(bf16_t*)y, (const bf16_t*)res, a_scale,
                                                        w_scale, n}, s, part);
    else
        product<false>(a, w, T, n, k, ScaledOut<float>{(float*)y, (const float*)res, a_scale,
                                                       w_scale, n}, s, part);
    return hipGetLastError();
}

hipError_t launch_linear_i8(const void* x, int in, const int8_t* w, const float* w_scale,
                            const void* res, int64_t T, int n, int k, int out, void* y, int8_t* q,
                            float* scale, void* part, hipStream_t s) {
    return in == ELB_BF16
               ? linear<bf16_t>(x, w, w_scale, res, T, n, k, out, y, q, scale, part, s)
               : linear<float>(x, w, w_scale, res, T, n, k, out, y, q, scale, part, s);
}

hipError_t launch_gate_up_i8(const void* x, int dtype, const int8_t* w, const float* w_scale,
                             int64_t T, int d, int m, float* h, int8_t* q, float* scale,
                             hipStream_t s) {
    return dtype == ELB_BF16 ? gate_up<bf16_t>(x, w, w_scale, T, d, m, h, q, scale, s)
                             : gate_up<float>(x, w, w_scale, T, d, m, h, q, scale, s);
}

}  // namespace elb
