// Products with 4-bit weights (f4.h), and the dense gated feed-forward block made of them.
//
//   y = [res +] x W^T,  W_ni = e2m1(q_ni) 2^(b_n,i/32 - 127)
//
// Every product of a bf16 x is exact in fp32; an fp32 x is cut into three bf16 parts of its 24 bits,
// which add up to it, and multiplied as three.  Sums are fp32 in a fixed order.
#include "f4.h"

namespace elb {

namespace {

// ---- quantisation: a thread per group of 32 ----
// b: the least power of two by which the group's largest magnitude is at most 6, from 2 to 252 (so that
// every value is a normal number; a group of zeros has 2, larger values saturate); 255 for a group with
// an infinity or a NaN.  Values round to nearest, ties to the even code.
template <class T>
__global__ __launch_bounds__(256) void quantize_f4(const T* __restrict__ x, int64_t groups,
                                                   uint8_t* __restrict__ q,
                                                   uint8_t* __restrict__ scale) {
    const int64_t g = (int64_t)dense_block_number() * 256 + threadIdx.x;
    if (g >= groups) return;
    Eight<T> v[4];
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i].load(x + g * 32 + 8 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t a = __float_as_uint(v[i][e]) & 0x7fffffffu;  // magnitudes in order, NaN last
            mx = a > mx ? a : mx;
        }
    // mx = m 2^e, 1 <= m < 2: at most 6 2^(e - 2) where m <= 1.5, else 6 2^(e - 1)
    int b = (int)(mx >> 23) - 2 + ((mx & 0x7fffffu) > 0x400000u ? 1 : 0);
    b = b < 2 ? 2 : b > 252 ? 252 : b;
    const float inv = __uint_as_float((uint32_t)(254 - b) << 23);  // 2^(127 - b)
    if (mx >= 0x7f800000u) b = 255;
    u32x4_t out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = v[i][e], a = fabsf(t) * inv;
            uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) +
                         (a >= 3.5f) + (a > 5.0f);
            c |= __float_as_uint(t) >> 31 << 3;
            w |= c << (4 * e);
        }
        out[i] = w;
    }
    *reinterpret_cast<u32x4_byte_t*>(q + g * 16) = out;
    scale[g] = (uint8_t)b;
}

// ---- conversion to dtype for the dense forms: a thread per 8 values ----
template <class T>
__global__ __launch_bounds__(256) void expand_f4(const uint8_t* __restrict__ q,
                                                 const uint8_t* __restrict__ scale, int64_t eights,
                                                 T* __restrict__ w, Counters clear) {
    clear_counters(clear.p, clear.n);
    const int64_t i = (int64_t)dense_block_number() * 256 + threadIdx.x;
    if (i >= eights) return;
    typedef uint32_t u32_byte_t __attribute__((aligned(1)));
    const uint32_t v = *reinterpret_cast<const u32_byte_t*>(q + i * 4);
    const bf16x8_t f = f4_to_bf16(v, f4_scale(scale[i >> 2]));
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<bf16x8_t*>(w + i * 8) = f;
    } else {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (float)f[e];
        store8(w + i * 8, o);
    }
}

// ---- tokens' operand: eight values as P bf16 parts whose sum they are ----
template <class X>
struct Tok;
template <>
struct Tok<bf16_t> {
    static constexpr int P = 1;
    u32x4_t v;
    __device__ __forceinline__ void load(const bf16_t* p) {
        v = *reinterpret_cast<const u32x4_any_t*>(p);
    }
    __device__ __forceinline__ void zero() { v = u32x4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void parts(bf16x8_t (&o)[1]) const {
        o[0] = __builtin_bit_cast(bf16x8_t, v);
    }
};
template <>
struct Tok<float> {
    static constexpr int P = 3;
    f32x4_t a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4_any_t*>(p);
        b = *reinterpret_cast<const f32x4_any_t*>(p + 4);
    }
    __device__ __forceinline__ void zero() { a = b = f32x4_t{0, 0, 0, 0}; }
    // the leading 8 bits, the next 8 and the rest: differences of a float and its leading bits are
    // exact.  (An infinity leaves NaN in the second part, and so in the sums.)
    __device__ __forceinline__ void parts(bf16x8_t (&o)[3]) const {
        u32x4_t w[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[2], hi[2], mid[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x[e] = i < 2 ? a[2 * i + e] : b[2 * i - 4 + e];
                hi[e] = __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
                x[e] -= hi[e];
                mid[e] = __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
                x[e] -= mid[e];
            }
            w[0][i] = __builtin_amdgcn_perm(__float_as_uint(hi[1]), __float_as_uint(hi[0]),
                                            0x07060302u);
            w[1][i] = __builtin_amdgcn_perm(__float_as_uint(mid[1]), __float_as_uint(mid[0]),
                                            0x07060302u);
            w[2][i] = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]),
                                            0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) o[p] = __builtin_bit_cast(bf16x8_t, w[p]);
    }
};

template <class X>
struct StreamIn {
    const X* x;
    const uint8_t *w, *scale;
    const X* res;  // PLAIN
    X* out;
    int64_t T;
    int cols, k;  // output columns; PAIR: weight rows [0, cols) gates, [cols, 2 cols) ups
};

// ------------------------------------------------------------------------------------------
// A few tokens: 16 MT of them against NF fragments of 16 weight rows a block (PAIR: half of them gate
// rows and the other half the matching up rows), the contraction in eight waves, whose partial tiles
// are added in LDS in order.  Bound by the weights' stream, or by the latency of its start.
// ------------------------------------------------------------------------------------------
template <class X, int NF, int MT, int R, bool PAIR>
__global__ __launch_bounds__(512) void stream_f4(StreamIn<X> in) {
    constexpr int NW = 8, OF = PAIR ? NF / 2 : NF;  // output fragments
    __shared__ f32x4_t part[NW][MT][NF][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = (int)blockIdx.x * 16 * OF;
    const int64_t t0 = (int64_t)blockIdx.y * 16 * MT;
    const int steps = (in.k + WF4::KS - 1) / WF4::KS;
    const int s0 = steps * wave / NW, s1 = steps * (wave + 1) / NW;
    const WF4 W{in.w, in.scale, in.k};
    // columns are multiples of 16: a fragment is a tensor's or wholly past it, where the last is read
    int64_t wrow[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        int c = c0 + 16 * (f % OF);
        c = c < in.cols ? c : in.cols - 16;
        wrow[f] = (PAIR && f >= OF ? (int64_t)in.cols : 0) + c + l16;
    }
    const X* xp[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t r = t0 + 16 * t + l16;
        xp[t] = in.x + (r < in.T ? r : in.T - 1) * in.k;
    }
    struct Slot {
        WF4::Frag w[NF];
        Tok<X> x[MT][4];
    };
    f32x4_t acc[MT][NF];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[t][f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    ring<R, Slot>(
        s1 - s0,
        [&](int j, Slot& s) {
            // quarters past the contraction: the row's last weights, and zeros for the tokens
            int k = (s0 + j) * WF4::KS + 32 * hq;
            const bool in_k = k < in.k;
            k = in_k ? k : in.k - 32;
#pragma unroll
            for (int f = 0; f < NF; ++f) W.load(s.w[f], wrow[f], k);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s.x[t][i].load(xp[t] + k + 8 * i);
        },
        [&](int j, Slot& s) {
            if ((s0 + j + 1) * WF4::KS > in.k && (s0 + j) * WF4::KS + 32 * hq >= in.k) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s.x[t][i].zero();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bf16x8_t a[NF];
#pragma unroll
                for (int f = 0; f < NF; ++f) a[f] = WF4::get(s.w[f], i);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    bf16x8_t b[Tok<X>::P];
                    s.x[t][i].parts(b);
#pragma unroll
                    for (int p = Tok<X>::P - 1; p >= 0; --p)
#pragma unroll
                        for (int f = 0; f < NF; ++f)
                            acc[t][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[f], b[p],
                                                                                acc[t][f], 0, 0, 0);
                }
            }
        });
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) part[wave][t][f][lane] = acc[t][f];
    __syncthreads();
    // a lane of a tile's fragment has columns 16 f + 4 (lane / 16) .. + 3 of token 16 t + lane % 16
    for (int i = threadIdx.x; i < MT * OF * 64; i += NW * 64) {
        const int l = i & 63, f = i / 64 % OF, t = i / (64 * OF);
        auto sum = [&](int ff) {
            f32x4_t v = part[0][t][ff][l];
#pragma unroll
            for (int w = 1; w < NW; ++w) v += part[w][t][ff][l];
            return v;
        };
        f32x4_t v = sum(f);
        const int64_t r = t0 + 16 * t + (l & 15);
        const int c = c0 + 16 * f + 4 * (l >> 4);
        if (r >= in.T || c >= in.cols) continue;
        const int64_t o = r * in.cols + c;
        if constexpr (PAIR) {
            const f32x4_t u = sum(f + OF);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = v[q] * (sizeof(X) == 2 ? sigma_bf16(v[q]) : sigma_f32(v[q])) * u[q];
        }
        if constexpr (sizeof(X) == 2) {
            typedef uint32_t u32x2_el_t __attribute__((ext_vector_type(2), aligned(2)));
            if (!PAIR && in.res) {
                const u32x2_el_t e = *reinterpret_cast<const u32x2_el_t*>(in.res + o);
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] += bf16_to_f32((bf16_t)(e[q / 2] >> (q % 2 * 16)));
            }
            *reinterpret_cast<u32x2_el_t*>(in.out + o) = u32x2_el_t{pack2(v[0], v[1]),
                                                                    pack2(v[2], v[3])};
        } else {
            if (!PAIR && in.res) v += *reinterpret_cast<const f32x4_any_t*>(in.res + o);
            *reinterpret_cast<f32x4_any_t*>(in.out + o) = v;
        }
    }
}

template <class X, int NF, int MT, int R, bool PAIR>
void run_stream(const StreamIn<X>& in, hipStream_t s) {
    constexpr int OC = 16 * (PAIR ? NF / 2 : NF);
    const dim3 grid((unsigned)((in.cols + OC - 1) / OC), (unsigned)((in.T + 16 * MT - 1) / (16 * MT)));
    ELB_LAUNCH((stream_f4<X, NF, MT, R, PAIR>), grid, dim3(512), 0, s, in);
}

template <class X, bool PAIR>
void stream(const StreamIn<X>& in, hipStream_t s) {
    constexpr bool F = sizeof(X) == 4;
    if (in.T <= 16) {
        if (!PAIR && in.cols <= 16 * 512) return run_stream<X, PAIR ? 2 : 1, 1, F ? 3 : 4, PAIR>(in, s);
        if (in.cols <= 16 * (PAIR ? 512 : 1024)) return run_stream<X, 2, 1, F ? 3 : 4, PAIR>(in, s);
        return run_stream<X, 4, 1, F ? 3 : 4, PAIR>(in, s);
    }
    if (in.T <= 32) return run_stream<X, 2, 2, F ? 2 : 3, PAIR>(in, s);
    return run_stream<X, 2, F ? 2 : 4, F ? 2 : 2, PAIR>(in, s);
}

template <class T>
hipError_t expand(const uint8_t* q, const uint8_t* scale, int64_t values, void* w, Counters clear,
                  hipStream_t s) {
    ProfileScope prof("expand_f4", s);
    ELB_LAUNCH(expand_f4<T>, grid_of((values / 8 + 255) / 256), dim3(256), 0, s, q, scale, values / 8,
               (T*)w, clear);
    return hipGetLastError();
}

template <class T>
hipError_t linear(const void* x, const uint8_t* W, const uint8_t* W_scale, const void* res,
                  int64_t T_, int n, int k, int dtype, void* y, void* w, void* part,
                  hipStream_t s) {
    if (f4_streams(T_, dtype)) {
        ProfileScope prof("linear_f4", s);
        stream<T, false>({(const T*)x, W, W_scale, (const T*)res, (T*)y, T_, n, k}, s);
        return hipGetLastError();
    }
    const int64_t kt = ((int64_t)k * sizeof(T) + 127) / 128;
    if (hipError_t e = expand<T>(W, W_scale, (int64_t)n * k, w,
                                 halves_counters((char*)part, T_, n, kt, sizeof(T) == 4), s))
        return e;
    return launch_linear(x, w, res, T_, n, k, dtype, part, y, s);
}

template <class T>
hipError_t block(const void* x, const uint8_t* Wgu, const uint8_t* gu_scale, const uint8_t* Wd,
                 const uint8_t* d_scale, const void* res, int64_t T_, int d, int m, int dtype,
                 void* h, void* wgu, void* wd, void* part, void* y, hipStream_t s) {
    if (f4_streams(T_, dtype)) {
        {
            ProfileScope prof("gate_up_f4", s);
            stream<T, true>({(const T*)x, Wgu, gu_scale, nullptr, (T*)h, T_, m, d}, s);
            if (hipError_t e = hipGetLastError()) return e;
        }
        return linear<T>(h, Wd, d_scale, res, T_, d, m, dtype, y, nullptr, nullptr, s);
    }
    if (hipError_t e = expand<T>(Wgu, gu_scale, (int64_t)2 * m * d, wgu, {}, s)) return e;
    if (hipError_t e = expand<T>(Wd, d_scale, (int64_t)m * d, wd, {}, s)) return e;
    return launch_ffn_forward(x, wgu, wd, res, T_, d, m, dtype, h, part, nullptr, y, s);
}

}  // namespace

bool f4_streams(int64_t T, int) { return T <= 64; }

hipError_t launch_quantize_f4(const void* x, int64_t rows, int d, int dtype, uint8_t* q,
                              uint8_t* scale, hipStream_t s) {
    ProfileScope prof("quantize_f4", s);
    const int64_t groups = rows * (d / 32);
    if (dtype == ELB_BF16)
        ELB_LAUNCH(quantize_f4<bf16_t>, grid_of((groups + 255) / 256), dim3(256), 0, s,
                   (const bf16_t*)x, groups, q, scale);
    else
        ELB_LAUNCH(quantize_f4<float>, grid_of((groups + 255) / 256), dim3(256), 0, s,
                   (const float*)x, groups, q, scale);
    return hipGetLastError();
}

hipError_t launch_linear_f4(const void* x, const uint8_t* W, const uint8_t* W_scale,
                            const void* res, int64_t T, int n, int k, int dtype, void* y, void* w,
                            void* part, hipStream_t s) {
    return (dtype == ELB_BF16 ? linear<bf16_t> : linear<float>)(x, W, W_scale, res, T, n, k, dtype, y,
                                                                w, part, s);
}

hipError_t launch_ffn_f4(const void* x, const uint8_t* Wgu, const uint8_t* gu_scale,
                         const uint8_t* Wd, const uint8_t* d_scale, const void* res, int64_t T,
                         int d, int m, int dtype, void* h, void* wgu, void* wd, void* part, void* y,
                         hipStream_t s) {
    return (dtype == ELB_BF16 ? block<bf16_t> : block<float>)(x, Wgu, gu_scale, Wd, d_scale, res, T, d,
                                                              m, dtype, h, wgu, wd, part, y, s);
}

}  // namespace elb
