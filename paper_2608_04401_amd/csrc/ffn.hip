// The dense gated feed-forward block, forward and backward (bf16 and fp32).
//
//   forward   g = x Wg^T, u = x Wu^T, h = silu(g) * u      one kernel: both projections share the
//                                                          token tile, SwiGLU on the accumulators
//             y = [residual +] h Wd^T
//   backward  dh = dy Wd, s = sigma(g): dg = dh u s (1 + g (1 - s)), du = dh g s, h = g s u
//             dx = dg Wg + du Wu = [dg du] [Wg; Wu]        one product of contraction 2 m
//             dWg = dg^T x, dWu = du^T x, dWd = dy^T h     [dg du]^T x, and beside it dy^T h
//
// Roundings to bf16: h before the down product, dg, du and h before the gradients' products (they
// are matrix operands), and every output.  g and u reach the backward in fp32: rounded to
// bf16, their errors would add to those of dg and du through sigma' in every gradient.
#include "dense.h"

namespace elb {

namespace {

__device__ __forceinline__ float sigma(float g, bf16_t) { return sigma_bf16(g); }
__device__ __forceinline__ float sigma(float g, float) { return sigma_f32(g); }

// ---- what becomes of the products' results ----
template <class T>
struct GateOut {  // h = silu(g) u; keep [T, 2m] fp32: g and u for the backward
    static constexpr bool kMayHalve = false;
    T* h;
    float* keep;
    int64_t m;
    __device__ __forceinline__ GateOut at(int64_t r0, int c0) const {
        return {h + r0 * m + c0, keep ? keep + r0 * 2 * m + c0 : nullptr, m};
    }
    typedef Nothing Extra;
    __device__ __forceinline__ void fetch(int, int, Extra&) const {}
    __device__ __forceinline__ void put(int row, int col, const float (&g)[8],
                                        const float (&u)[8], const Extra&) const {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            v[q] = g[q] * sigma(g[q], T()) * u[q];
        store8(h + row * m + col, v);
        if (keep) {
            store8(keep + row * 2 * m + col, g);
            store8(keep + row * 2 * m + m + col, u);
        }
    }
};

template <class T>
struct GateGradOut {  // from dh, g and u: dg and du [T, 2m], h [T, m]
    static constexpr bool kMayHalve = false;
    const float* keep;
    T* dgu;
    T* h;
    int64_t m;
    __device__ __forceinline__ GateGradOut at(int64_t r0, int c0) const {
        const int64_t o = r0 * 2 * m + c0;
        return {keep + o, dgu + o, h + r0 * m + c0, m};
    }
    struct Extra {
        Eight<float> g, u;
    };
    __device__ __forceinline__ void fetch(int row, int col, Extra& e) const {
        e.g.load(keep + row * 2 * m + col);
        e.u.load(keep + row * 2 * m + m + col);
    }
    __device__ __forceinline__ void put(int row, int col, const float (&dh)[8],
                                        const Extra& e) const {
        const int64_t o = row * 2 * m + col;
        const Eight<float>&g = e.g, &u = e.u;
        float dg[8], du[8], hh[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float s = sigma(g[q], T());
            const float gs = g[q] * s;
            // the larger of dh and u times sigma' first: no step leaves fp32's range where dg does not
            // (dh u may pass the largest number before a closed gate, the smaller times sigma' the
            // smallest)
            const bool up = fabsf(u[q]) > fabsf(dh[q]);
            dg[q] = (s + gs * (1.0f - s)) * (up ? u[q] : dh[q]) * (up ? dh[q] : u[q]);
            du[q] = dh[q] * gs;
            hh[q] = gs * u[q];
        }
        store8(dgu + o, dg);
        store8(dgu + o + m, du);
        store8(h + row * m + col, hh);
    }
};

template <class E, class T>
struct Block {
    template <int LB, bool PAIR, class Epi>
    static void product(const void* a, int64_t lda, const void* b, int64_t ldb, int64_t rows,
                        int cols, int64_t K, const Epi& epi, hipStream_t s, void* part = nullptr,
                        Counters clear = {}) {
        const DenseIn d{(const char*)a, (const char*)b, lda * E::SZ, ldb * E::SZ, rows, cols, K,
                        (char*)part, clear.p, clear.n};
        run_product<E, LB, PAIR>(d, aligned16(a, b), epi, s);
    }

    static int64_t ktiles(int64_t K) { return (K * E::SZ + 127) / 128; }

    static hipError_t forward(const void* x, const void* Wgu, const void* Wd, const void* res,
                              int64_t T_, int d, int m, void* h, void* part, float* keep,
                              void* y, hipStream_t s) {
        {
            ProfileScope prof("ffn_gate_up", s);
            product<KC, true>(x, d, Wgu, d, T_, m, d, GateOut<T>{(T*)h, keep, m}, s, nullptr,
                              halves_counters((char*)part, T_, d, ktiles(m), E::SZ == 4));
            if (hipError_t e = hipGetLastError()) return e;
        }
        ProfileScope prof("ffn_down", s);
        product<KC, false>(h, m, Wd, m, T_, d, m, PlainOut<T>{(T*)y, (const T*)res, d}, s,
                           part);
        return hipGetLastError();
    }

    static hipError_t linear(const void* x, const void* W, const void* res, int64_t T_, int n, int k,
                             void* part, void* y, hipStream_t s) {
        ProfileScope prof("linear", s);
        product<KC, false>(x, k, W, k, T_, n, k, PlainOut<T>{(T*)y, (const T*)res, n}, s, part);
        return hipGetLastError();
    }

    static hipError_t backward(const void* dy, const void* x, const void* Wgu, const void* Wd,
                               const float* keep, int64_t T_, int d, int m, void* dgu, void* h,
                               void* part, void* dx, void* dWgu, void* dWd, hipStream_t s) {
        {
            ProfileScope prof("ffn_dh", s);
            product<KR, false>(dy, d, Wd, m, T_, m, d,
                               GateGradOut<T>{keep, (T*)dgu, (T*)h, m}, s, nullptr,
                               halves_counters((char*)part, T_, d, ktiles(2 * (int64_t)m),
                                               E::SZ == 4));
            if (hipError_t e = hipGetLastError()) return e;
        }
        if (dx) {
            ProfileScope prof("ffn_dx", s);
            product<KR, false>(dgu, 2 * (int64_t)m, Wgu, d, T_, d, 2 * (int64_t)m,
                               PlainOut<T>{(T*)dx, nullptr, d}, s, part);
            if (hipError_t e = hipGetLastError()) return e;
        }
        if (dWgu || dWd) {
            ProfileScope prof("ffn_dw", s);
            const DenseIn a{(const char*)dgu, (const char*)x, 2 * (int64_t)m * E::SZ,
                            (int64_t)d * E::SZ, dWgu ? 2 * (int64_t)m : 0, d, T_,
                            nullptr, nullptr, 0};
            const DenseIn b{(const char*)dy, (const char*)h, (int64_t)d * E::SZ,
                            (int64_t)m * E::SZ, dWd ? d : 0, m, T_, nullptr, nullptr, 0};
            run_product2<E>(a, b, aligned16(dy, x), PlainOut<T>{(T*)dWgu, nullptr, d},
                            PlainOut<T>{(T*)dWd, nullptr, m}, s);
        }
        return hipGetLastError();
    }
};

}  // namespace

size_t ffn_halves_bytes(int64_t T, int d, int64_t K, int dtype, bool most) {
    const int64_t kt = (K * (dtype == ELB_BF16 ? 2 : 4) + 127) / 128;
    return (most ? halves_reserve : halves_bytes)(T, d, kt, dtype != ELB_BF16);
}

hipError_t launch_ffn_forward(const void* x, const void* Wgu, const void* Wd, const void* res,
                              int64_t T, int d, int m, int dtype, void* h, void* part,
                              float* gate_up, void* y, hipStream_t s) {
    return dtype == ELB_BF16
               ? Block<Bf16, bf16_t>::forward(x, Wgu, Wd, res, T, d, m, h, part, gate_up, y, s)
               : Block<F32, float>::forward(x, Wgu, Wd, res, T, d, m, h, part, gate_up, y, s);
}

hipError_t launch_linear(const void* x, const void* W, const void* res, int64_t T, int n, int k,
                         int dtype, void* part, void* y, hipStream_t s) {
    return dtype == ELB_BF16 ? Block<Bf16, bf16_t>::linear(x, W, res, T, n, k, part, y, s)
                             : Block<F32, float>::linear(x, W, res, T, n, k, part, y, s);
}

hipError_t launch_ffn_backward(const void* dy, const void* x, const void* Wgu, const void* Wd,
                               const float* gate_up, int64_t T, int d, int m, int dtype, void* dgu,
                               void* h, void* part, void* dx, void* dWgu, void* dWd,
                               hipStream_t s) {
    return dtype == ELB_BF16 ? Block<Bf16, bf16_t>::backward(dy, x, Wgu, Wd, gate_up, T, d, m, dgu,
                                                             h, part, dx, dWgu, dWd, s)
                             : Block<F32, float>::backward(dy, x, Wgu, Wd, gate_up, T, d, m, dgu,
                                                           h, part, dx, dWgu, dWd, s);
}

}  // namespace elb
