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

// ---- conversion to dtype for the dense forms: a thread per 8 values (2048 x 8192 to bf16 8.2 us, 5.2
// TB/s; the product of 4096 tokens after it 113) ----
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
    // values 128 h + 32 i + 8 c .. + 7 of row r of a unit of 256, in LDS as four k-tiles of TM rows
    template <int TM>
    __device__ __forceinline__ void read(const char* p, int r, int h, int i, int c) {
        v = *reinterpret_cast<const u32x4_t*>(p + (2 * h + i / 2) * TM * 128 + r * 128 +
                                              kc_swz(r, i % 2 * 4 + c) * 16);
    }
    __device__ __forceinline__ void parts(bf16x8_t (&o)[1]) const {
        o[0] = __builtin_bit_cast(bf16x8_t, v);
    }
};
template <>
struct Tok<float> {
    static constexpr int P = 3;
    f32x4_t a, b;
    template <int TM>
    __device__ __forceinline__ void read(const char* p, int r, int h, int i, int c) {
        const char* const q = p + (4 * h + i) * TM * 128 + r * 128;
        a = *reinterpret_cast<const f32x4_t*>(q + kc_swz(r, 2 * c) * 16);
        b = *reinterpret_cast<const f32x4_t*>(q + kc_swz(r, 2 * c + 1) * 16);
    }
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
    // shares > 1: a tile's contraction in that many blocks; their partial sums [tiles, shares, TM, 16 NF],
    // and how many of a tile's are written (zero before the launch)
    int shares;
    float* part;
    uint32_t* count;
    Counters clear;  // the next launch's counters
};

// ------------------------------------------------------------------------------------------
// A few tokens: TM of them against NF fragments of 16 weight rows a block (PAIR: half of them gate rows
// and the other half the matching up rows).  Each of NW waves has a share of the contraction and walks
// it alone: a unit's weights and tokens are copied into the wave's LDS, read into registers, and the
// next unit's copies run while this one is multiplied; no barrier until the waves' partial tiles are
// added, in order.  Bound by the weights' stream, or by the latency of its start.  Where tiles are few,
// blocks share the contraction of one (blockIdx.z): the last of them to write its partial sums adds all,
// in the order of the shares; none waits for another.  One token, 8192 to 2048: 6.2 us (1.4 TB/s, two units
// a wave); 48 tokens, 2048 to 16384 gate and up rows 10.1, 8192 to 2048 in four shares 8.9.
// ------------------------------------------------------------------------------------------
template <class X, int TM, int NF, int NW, bool PAIR, bool DMA>
__global__ __launch_bounds__(64 * NW) void stream_f4(StreamIn<X> in) {
    constexpr int OF = PAIR ? NF / 2 : NF;  // output fragments
    constexpr int MT = (TM + 15) / 16, SUB = 256 * sizeof(X) / 128;
    typedef Stream<WF4, NF, PAIR, DMA> B;
    typedef Copier<KC, TM, sizeof(X), 1, false, DMA> A;
    constexpr int AB = SUB * TM * 128, SLOT = (AB + B::BYTES + 255) / 256 * 256;
    static_assert(MT * NF * 1024 <= SLOT && NW * SLOT <= 160 * 1024, "");
    __shared__ __attribute__((aligned(1024))) char sm[NW * SLOT];
    const int lane = threadIdx.x & 63, l16 = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = (int)blockIdx.x * 16 * OF;
    const int64_t t0 = (int64_t)blockIdx.y * TM;
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
        for (int i = threadIdx.x; i < in.clear.n; i += 64 * NW) in.clear.p[i] = 0;
    const int units = (in.k + 255) / 256, ways = NW * in.shares, way = NW * blockIdx.z + wave;
    const int u0 = units * way / ways, u1 = units * (way + 1) / ways;
    char* const slot = sm + wave * SLOT;
    const uint32_t lds = lds_address(slot);
    A a;
    a.init(in.x + t0 * in.k, nullptr, (int64_t)in.k * sizeof(X),
           in.T - t0 < TM ? (int)(in.T - t0) : TM, in.k, lane, 0);
    B b;
    b.init(in.w, in.scale, c0, in.cols - c0, in.cols, PAIR ? 2 * (int64_t)in.cols : in.cols, in.k,
           lane);
    typename B::Pending pending = {};
    auto issue = [&](int u) {
        const bool whole = DMA && (u + 1) * 256 <= in.k;
#pragma unroll
        for (int q = 0; q < SUB; ++q) {
            const int t = SUB * u + q;
            if (whole) issue_whole(a, (uint32_t)t * 128u, lds + q * TM * 128);
            else a.issue(t, SUB * u1, lds + q * TM * 128, slot + q * TM * 128, lane, 0);
        }
        b.issue(u, u1, lds + AB, slot + AB, lane, pending);
    };
    f32x4_t acc[MT][NF];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[t][f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (u0 < u1) issue(u0);
    for (int u = u0; u < u1; ++u) {
        ELB_WAIT_VMCNT(0);
        b.settle(pending, slot + AB, lane);
        asm volatile("" ::: "memory");  // the copies write LDS behind the compiler's back
        WF4::Half w[NF][2];
        Tok<X> x[MT][2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
                WF4::read(w[f][h], slot + AB, 16 * NF, f, h, l16, hq);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[t][h][i].template read<TM>(slot, TM < 16 ? l16 % TM : 16 * t + l16, h, i, hq);
        }
        // every read of the unit has returned before the next one's copies overwrite it
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (u + 1 < u1) issue(u + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (u * 256 + 128 * h + 32 * i >= in.k) break;
                bf16x8_t wf[NF];
#pragma unroll
                for (int f = 0; f < NF; ++f) wf[f] = w[f][h].get(i);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    bf16x8_t xf[Tok<X>::P];
                    x[t][h][i].parts(xf);
#pragma unroll
                    for (int p = Tok<X>::P - 1; p >= 0; --p)
#pragma unroll
                        for (int f = 0; f < NF; ++f)
                            acc[t][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[f], xf[p],
                                                                                acc[t][f], 0, 0, 0);
                }
            }
    }
    // partial tiles, each in its wave's own LDS
    auto part = [&](int w, int t, int f, int l) {
        return reinterpret_cast<f32x4_t*>(sm + w * SLOT) + (t * NF + f) * 64 + l;
    };
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) *part(wave, t, f, lane) = acc[t][f];
    __syncthreads();
    // fragment f of token tile t in the block's sum, four values a lane
    auto sum = [&](int t, int f, int l) {
        f32x4_t v = *part(0, t, f, l);
#pragma unroll
        for (int w = 1; w < NW; ++w) v += *part(w, t, f, l);
        return v;
    };
    // a lane of a tile's fragment has columns 16 f + 4 (lane / 16) .. + 3 of token 16 t + lane % 16
    auto put = [&](int t, int f, int l, f32x4_t v, f32x4_t u) {
        const int64_t r = t0 + 16 * t + (l & 15);
        const int c = c0 + 16 * f + 4 * (l >> 4);
        if (r >= in.T || 16 * t + (l & 15) >= TM || c >= in.cols) return;
        const int64_t o = r * in.cols + c;
        if constexpr (PAIR) {
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
    };
    constexpr int PIECES = MT * OF * 64;  // of four values
    if (PAIR || in.shares == 1) {
        for (int i = threadIdx.x; i < PIECES; i += NW * 64) {
            const int l = i & 63, f = i / 64 % OF, t = i / (64 * OF);
            put(t, f, l, sum(t, f, l), PAIR ? sum(t, (f + OF) % NF, l) : f32x4_t{});
        }
        return;
    }
    if constexpr (!PAIR) {
        // The partial sums go past the L2, which blocks elsewhere on the chip do not share: agent-scope
        // stores, done when the counter goes up, and agent-scope loads.  (A release fence would
        // write the whole L2 back, for each block: the few-token layer's, 31 us.)
        const int64_t tile = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
        float* const mine = in.part + tile * in.shares * (PIECES * 4);
        __shared__ int last;
        for (int i = threadIdx.x; i < PIECES; i += NW * 64) {
            const f32x4_t v = sum(i / (64 * OF), i / 64 % OF, i & 63);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                __hip_atomic_store(mine + ((int64_t)blockIdx.z * 4 + q) * PIECES + i, v[q],
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        ELB_WAIT_VMCNT(0);
        __syncthreads();
        if (threadIdx.x == 0)
            last = __hip_atomic_fetch_add(in.count + tile, 1u, __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)in.shares - 1;
        __syncthreads();
        if (!last) return;
        for (int i = threadIdx.x; i < PIECES; i += NW * 64) {
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int z = 0; z < in.shares; ++z)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    v[q] += __hip_atomic_load(mine + ((int64_t)z * 4 + q) * PIECES + i,
                                              __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            put(i / (64 * OF), i / 64 % OF, i & 63, v, f32x4_t{});
        }
    }
}

template <class X, int TM, int NF, int NW, bool PAIR>
void run_stream(const StreamIn<X>& in, hipStream_t s) {
    constexpr int OC = 16 * (PAIR ? NF / 2 : NF);
    const dim3 grid((unsigned)((in.cols + OC - 1) / OC), (unsigned)((in.T + TM - 1) / TM),
                    (unsigned)in.shares);
    if (aligned16(in.x, in.w))
        ELB_LAUNCH((stream_f4<X, TM, NF, NW, PAIR, true>), grid, dim3(64 * NW), 0, s, in);
    else
        ELB_LAUNCH((stream_f4<X, TM, NF, NW, PAIR, false>), grid, dim3(64 * NW), 0, s, in);
}

// the counters of a shared product's scratch, or none
Counters f4_counters(const F4Plan& p, void* part) {
    if (!p.part) return {nullptr, 0};
    return {reinterpret_cast<uint32_t*>((char*)part + p.sums()), p.tiles};
}

template <class X, bool PAIR>
hipError_t stream(StreamIn<X> in, const StreamForm& f, hipStream_t s) {
    in.shares = f.shares;
    const bool known = with_form<sizeof(X) == 4, PAIR>(f, [&](auto t) {
        typedef decltype(t) Form;
        run_stream<X, Form::TM, Form::NF, Form::NW, PAIR>(in, s);
    });
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

__global__ __launch_bounds__(256) void clear_f4(Counters c) { clear_counters(c.p, c.n); }

template <class T>
hipError_t expand(const uint8_t* q, const uint8_t* scale, int64_t values, void* w, Counters clear,
                  hipStream_t s) {
    ProfileScope prof("expand_f4", s);
    ELB_LAUNCH(expand_f4<T>, grid_of((values / 8 + 255) / 256), dim3(256), 0, s, q, scale, values / 8,
               (T*)w, clear);
    return hipGetLastError();
}

// y = [res +] x W^T, streamed; cleared: an earlier launch of the call has set the counters to zero
template <class T>
hipError_t streamed(const F4Plan& p, const void* x, const uint8_t* W, const uint8_t* W_scale,
                    const void* res, int64_t T_, int n, int k, void* y, void* part, bool cleared,
                    hipStream_t s) {
    const Counters c = f4_counters(p, part);
    if (c.n && !cleared) {
        ProfileScope prof("clear_f4", s);
        ELB_LAUNCH(clear_f4, dim3(1), dim3(256), 0, s, c);
    }
    ProfileScope prof("linear_f4", s);
    return stream<T, false>({(const T*)x, W, W_scale, (const T*)res, (T*)y, T_, n, k, 1, (float*)part,
                             c.p, {nullptr, 0}}, p.form, s);
}

template <class T>
hipError_t linear(const F4Plan& p, const void* x, const uint8_t* W, const uint8_t* W_scale,
                  const void* res, int64_t T_, int n, int k, int dtype, void* y, void* w, void* part,
                  hipStream_t s) {
    if (p.streams) return streamed<T>(p, x, W, W_scale, res, T_, n, k, y, part, false, s);
    const int64_t kt = ((int64_t)k * sizeof(T) + 127) / 128;
    if (hipError_t e = expand<T>(W, W_scale, (int64_t)n * k, w,
                                 halves_counters((char*)part, T_, n, kt, sizeof(T) == 4), s))
        return e;
    return launch_linear(x, w, res, T_, n, k, dtype, part, y, s);
}

template <class T>
hipError_t block(const F4Plan& p, const void* x, const uint8_t* Wgu, const uint8_t* gu_scale,
                 const uint8_t* Wd, const uint8_t* d_scale, const void* res, int64_t T_, int d, int m,
                 int dtype, void* h, void* wgu, void* wd, void* part, void* y, hipStream_t s) {
    if (p.streams) {
        {
            ProfileScope prof("gate_up_f4", s);
            if (hipError_t e = stream<T, true>({(const T*)x, Wgu, gu_scale, nullptr, (T*)h, T_, m, d, 1,
                                                nullptr, nullptr, f4_counters(p, part)}, p.up, s))
                return e;
        }
        return streamed<T>(p, h, Wd, d_scale, res, T_, d, m, y, part, true, s);
    }
    if (hipError_t e = expand<T>(Wgu, gu_scale, (int64_t)2 * m * d, wgu, {}, s)) return e;
    if (hipError_t e = expand<T>(Wd, d_scale, (int64_t)m * d, wd, {}, s)) return e;
    return launch_ffn_forward(x, wgu, wd, res, T_, d, m, dtype, h, part, nullptr, y, s);
}

}  // namespace

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

hipError_t launch_linear_f4(const F4Plan& p, const void* x, const uint8_t* W, const uint8_t* W_scale,
                            const void* res, int64_t T, int n, int k, int dtype, void* y, void* w,
                            void* part, hipStream_t s) {
    return (dtype == ELB_BF16 ? linear<bf16_t> : linear<float>)(p, x, W, W_scale, res, T, n, k, dtype,
                                                                y, w, part, s);
}

hipError_t launch_ffn_f4(const F4Plan& p, const void* x, const uint8_t* Wgu, const uint8_t* gu_scale,
                         const uint8_t* Wd, const uint8_t* d_scale, const void* res, int64_t T,
                         int d, int m, int dtype, void* h, void* wgu, void* wd, void* part, void* y,
                         hipStream_t s) {
    return (dtype == ELB_BF16 ? block<bf16_t> : block<float>)(p, x, Wgu, gu_scale, Wd, d_scale, res, T,
                                                              d, m, dtype, h, wgu, wd, part, y, s);
}

}  // namespace elb
