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

// The whole number nearest to x / s (ties to even): the rounded product with 1 / s is off by one
// at most, where x / s is within 2^-15 of a half; the remainder x - q s is exact there (x and s
// have 24 bits, and it is a multiple of the smaller one's last) and decides.
__device__ __forceinline__ float nearest(float x, float s, float inv) {
    float q = __builtin_rintf(x * inv);
    const float r = fmaf(-q, s, x), a = 2.0f * fabsf(r);
    if (a > s || (a == s && fmodf(q, 2.0f) != 0.0f)) q += copysignf(1.0f, r);
    return fminf(fmaxf(q, -127.0f), 127.0f);
}

typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(1)));

constexpr int kQuantThreads = 256;
constexpr int kQuantKeep = 4;  // groups of 8 elements that a thread keeps in registers

// a block per row
template <class T>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows(const T* __restrict__ x, int64_t d,
                                                               int64_t rows, int8_t* __restrict__ q,
                                                               float* __restrict__ scale,
                                                               Counters clear) {
    clear_counters(clear.p, clear.n);
    const int64_t row = dense_block_number();
    if (row >= rows) return;
    const T* const xr = x + row * d;
    const int tid = threadIdx.x;
    float keep[kQuantKeep][8];
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i) {
        const int64_t c = ((int64_t)i * kQuantThreads + tid) * 8;
        if (c < d) {
            load8(xr + c, keep[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(keep[i][e]));
        }
    }
    for (int64_t c = ((int64_t)kQuantKeep * kQuantThreads + tid) * 8; c < d;
         c += kQuantThreads * 8) {
        float v[8];
        load8(xr + c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(v[e]));
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    __shared__ float part[kQuantThreads / 64];
    if ((tid & 63) == 0) part[tid >> 6] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQuantThreads / 64; ++i) mx = fmaxf(mx, part[i]);
    const float s = mx / 127.0f;
    if (tid == 0) scale[row] = s;
    // a subnormal scale has no finite reciprocal: both sides of the quotient times 2^64
    const float up = s < 1e-30f ? 0x1p64f : 1.0f;
    const float su = s * up, inv = s > 0.0f ? 1.0f / su : 0.0f;
    auto put = [&](int64_t c, const float (&v)[8]) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int n = s > 0.0f ? (int)nearest(v[e] * up, su, inv) : 0;
            w[e >> 2] |= (uint32_t)(n & 255) << (8 * (e & 3));
        }
        *reinterpret_cast<u32x2_any_t*>(q + row * d + c) = u32x2_any_t{w[0], w[1]};
    };
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i) {
        const int64_t c = ((int64_t)i * kQuantThreads + tid) * 8;
        if (c < d) put(c, keep[i]);
    }
    for (int64_t c = ((int64_t)kQuantKeep * kQuantThreads + tid) * 8; c < d;
         c += kQuantThreads * 8) {
        float v[8];
        load8(xr + c, v);
        put(c, v);
    }
}

template <class T>
struct ScaledOut {  // y = [res +] v s_row c_col
    T* y;
    const T* res;
    const float *s, *c;
    int64_t ld;
    __device__ __forceinline__ ScaledOut at(int64_t r0, int c0) const {
        const int64_t o = r0 * ld + c0;
        return {y + o, res ? res + o : nullptr, s + r0, c + c0, ld};
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
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = v[q] * e.s * e.c[q];
        if (res) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += e.r[q];
        }
        store8(y + row * ld + col, v);
    }
};

// h = silu(g) u in fp32: rounded to bf16 first, one h in eight would move to the next whole number
// when it is quantised (2^-9 of a value is up to a quarter of a step)
struct ScaledGateOut {
    float* h;
    const float *s, *c;  // c: m scales of the gate rows, then m of the up rows
    int64_t m;
    __device__ __forceinline__ ScaledGateOut at(int64_t r0, int c0) const {
        return {h + r0 * m + c0, s + r0, c + c0, m};
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
    __device__ __forceinline__ void put(int row, int col, const float (&g)[8],
                                        const float (&u)[8], const Extra& e) const {
#pragma clang fp contract(off)
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float gg = g[q] * e.s * e.g[q];
            v[q] = gg / (1.0f + expf(-gg)) * (u[q] * e.s * e.u[q]);
        }
        store8(h + row * m + col, v);
    }
};

template <class T>
hipError_t quantize(const void* x, int64_t rows, int d, int8_t* q, float* scale, Counters clear,
                    hipStream_t s) {
    ProfileScope prof("quantize_rows", s);
    ELB_LAUNCH(quantize_rows<T>, grid_of(rows), dim3(kQuantThreads), 0, s, (const T*)x,
               (int64_t)d, rows, q, scale, clear);
    return hipGetLastError();
}

template <bool PAIR, class Epi>
void product(const int8_t* a, const int8_t* w, int64_t rows, int cols, int64_t K, const Epi& epi,
             hipStream_t s, void* part = nullptr) {
    const DenseIn d{(const char*)a, (const char*)w, K, K, rows, cols, K, (char*)part, nullptr, 0};
    run_product<I8, KC, PAIR>(d, aligned16(a, w), epi, s);
}

}  // namespace

size_t i8_halves_bytes(int64_t T, int n, int k) { return halves_bytes(T, n, (k + 127) / 128, false); }

hipError_t launch_quantize_rows(const void* x, int64_t rows, int d, int dtype, int8_t* q,
                                float* scale, hipStream_t s, void* part, int n) {
    const Counters c = halves_counters((char*)part, rows, n, (d + 127) / 128, false);
    return dtype == ELB_BF16 ? quantize<bf16_t>(x, rows, d, q, scale, c, s)
                             : quantize<float>(x, rows, d, q, scale, c, s);
}

hipError_t launch_gemm_i8(const int8_t* a, const float* a_scale, const int8_t* w,
                          const float* w_scale, const void* res, int64_t T, int n, int k,
                          int dtype, void* y, hipStream_t s, void* part) {
    ProfileScope prof("gemm_i8", s);
    if (dtype == ELB_BF16)
        product<false>(a, w, T, n, k, ScaledOut<bf16_t>{(bf16_t*)y, (const bf16_t*)res, a_scale,
                                                        w_scale, n}, s, part);
    else
        product<false>(a, w, T, n, k, ScaledOut<float>{(float*)y, (const float*)res, a_scale,
                                                       w_scale, n}, s, part);
    return hipGetLastError();
}

hipError_t launch_gate_up_i8(const int8_t* a, const float* a_scale, const int8_t* w,
                             const float* w_scale, int64_t T, int d, int m, float* h,
                             hipStream_t s) {
    ProfileScope prof("gate_up_i8", s);
    product<true>(a, w, T, m, d, ScaledGateOut{h, a_scale, w_scale, m}, s);
    return hipGetLastError();
}

}  // namespace elb
