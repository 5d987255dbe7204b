// The whole layer for at most 16 tokens in two launches.
//
//   launch 1  router, routing, h_tj = w_tj silu(W_gate x_t) * (W_up x_t) for each selected expert
//   launch 2  y_t = [residual_t +] sum_j W_down[e_j] h_tj
//
// All tokens are one MFMA tile of 16 rows.  In launch 1 every block routes all of them for itself (the
// same bits as the other router paths: the same chains, sums and per-token code), instead of waiting
// for a launch that does, and then takes its share of the used experts' gate and up rows.  In launch 2
// the experts lie one behind the other in one long contraction: a token's h is zero for experts that it
// has not selected, its routing weight is in h already, so the products' sum is the combine.
#include "f4.h"
#include "route_lane.h"

namespace elb {

namespace {

constexpr int kUpWaves = 8, kDownWaves = 16;

// The experts that some token has selected, and the slot t K + j that token t has of each (-1: none)
struct Slots {
    int16_t slot[64][16];
    int list[64];
    int used;
};

// k, ids: the routing of T tokens (at most 16 x 16 slots); by the whole block, which it synchronises
__device__ __forceinline__ void find_slots(Slots& s, const int* k, const int* ids, int T, int K,
                                           int N) {
    for (int i = threadIdx.x; i < 64 * 8; i += blockDim.x)
        reinterpret_cast<uint32_t*>(s.slot)[i] = 0xffffffffu;
    __syncthreads();
    if ((int)threadIdx.x < T * K) {
        const int t = threadIdx.x / K, j = threadIdx.x - t * K;
        const int e = ids[threadIdx.x];
        if (j < k[t] && e >= 0 && e < N) s.slot[e][t] = (int16_t)threadIdx.x;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint32_t* const row = reinterpret_cast<const uint32_t*>(s.slot[threadIdx.x]);
        uint32_t all = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < 8; ++i) all &= row[i];
        const uint64_t used = __ballot(all != 0xffffffffu);
        if (all != 0xffffffffu)
            s.list[__popcll(used & ((1ull << threadIdx.x) - 1))] = threadIdx.x;
        if (threadIdx.x == 0) s.used = __popcll(used);
    }
    __syncthreads();
}

template <class W>
__device__ __forceinline__ W expert(const void* w, const uint8_t* scale, int64_t at, int64_t ld);
template <>
__device__ __forceinline__ WBf16 expert<WBf16>(const void* w, const uint8_t*, int64_t at, int64_t ld) {
    return {(const bf16_t*)w + at, ld};
}
template <>
__device__ __forceinline__ WF4 expert<WF4>(const void* w, const uint8_t* scale, int64_t at,
                                           int64_t ld) {
    return {(const uint8_t*)w + at / 2, scale + at / 32, ld};
}

struct FewIn {
    const bf16_t *x, *router;
    const void *gate_up, *down;
    const uint8_t *gu_scale, *d_scale;
    const bf16_t* residual;
    int T, d, N, m, K, mode, renorm;
    float eps;
    bf16_t* h;
    bf16_t* y;
    int *k, *ids;
    float* w;
};

// NG: groups of 16 experts
template <class W, int NG, int KMAX, int R>
__global__ __launch_bounds__(64 * kUpWaves) void few_up(FewIn in, XTable xt) {
    __shared__ float logits[RW][16 * 65];
    __shared__ f32x4_t part[kUpWaves][4][64];
    __shared__ Slots slots;
    __shared__ int sk[16], sids[16 * kLaneMaxK];
    __shared__ float sw[16 * kLaneMaxK];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int T = in.T, d = in.d, N = in.N, m = in.m, K = in.K;
    const bf16_t* const xr = in.x + (int64_t)(l16 < T ? l16 : T - 1) * d;

    // ---- router: wave w has slice w % 4 of the contraction and every other group of experts ----
    {
        constexpr int G = (NG + 1) / 2;
        struct Slot {
            u32x4_t a, b[G];
        };
        int first, count;
        router_slice(d, wave & 3, first, count);
        const bf16_t* wr[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int n = 16 * (2 * g + (wave >> 2)) + l16;
            wr[g] = in.router + (int64_t)(n < N ? n : N - 1) * d;
        }
        f32x4_t acc[G];
#pragma unroll
        for (int g = 0; g < G; ++g) acc[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        ring<8, Slot>(
            count,
            [&](int j, Slot& s) {
                const int c = (first + j) * 32 + hq * 8;
                s.a = *reinterpret_cast<const u32x4_any_t*>(xr + c);
#pragma unroll
                for (int g = 0; g < G; ++g)
                    s.b[g] = *reinterpret_cast<const u32x4_any_t*>(wr[g] + c);
            },
            [&](int, Slot& s) {
#pragma unroll
                for (int g = 0; g < G; ++g)
                    acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8_t, s.a), __builtin_bit_cast(bf16x8_t, s.b[g]),
                        acc[g], 0, 0, 0);
            });
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                logits[wave & 3][(4 * hq + r) * 65 + 16 * (2 * g + (wave >> 2)) + l16] = acc[g][r];
    }
    __syncthreads();
    if (tid < 256) {  // whole waves: 16 lanes a token
        const int t = tid >> 4, sl = tid & 15;
        float l4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = 4 * sl + i;
            l4[i] = -INFINITY;
            if (n < N) {
                float v = logits[0][t * 65 + n];
#pragma unroll
                for (int q = 1; q < RW; ++q) v += logits[q][t * 65 + n];
                l4[i] = v;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) logits[0][t * 65 + 4 * sl + i] = l4[i];
    }
    __syncthreads();
    if (tid < 256)
        route_token_x16<KMAX>(logits[0] + (tid >> 4) * 65, N, K, in.eps, in.mode, in.renorm, xt,
                              tid >> 4, (tid >> 4) < T, sk, sids, sw);
    __syncthreads();
    if (blockIdx.x == 0) {
        if (tid < T * K) {
            in.ids[tid] = sids[tid];
            in.w[tid] = sw[tid];
        }
        if (tid < T) in.k[tid] = sk[tid];
    }
    find_slots(slots, sk, sids, T, K, N);

    // ---- tasks: 32 columns of h of an expert, its 32 gate rows and the matching up rows ----
    const int per_e = m / 32, tasks = slots.used * per_e;
    const int steps = (d + W::KS - 1) / W::KS;
    const int s0 = steps * wave / kUpWaves, s1 = steps * (wave + 1) / kUpWaves;
    for (int task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int u = task / per_e, c = task - u * per_e;
        const int e = __builtin_amdgcn_readfirstlane(slots.list[u]);
        const W w = expert<W>(in.gate_up, in.gu_scale, (int64_t)e * 2 * m * d, d);
        struct Slot {
            typename W::Frag w[4];
            u32x4_t x[W::J];
        };
        f32x4_t acc[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        ring<R, Slot>(
            s1 - s0,
            [&](int j, Slot& s) {
                int k = (s0 + j) * W::KS + W::KS / 4 * hq;
                k = k < d ? k : d - W::KS / 4;
#pragma unroll
                for (int f = 0; f < 4; ++f)
                    w.load(s.w[f], (f < 2 ? 0 : m) + 32 * c + 16 * (f & 1) + l16, k);
#pragma unroll
                for (int i = 0; i < W::J; ++i)
                    s.x[i] = *reinterpret_cast<const u32x4_any_t*>(xr + k + 8 * i);
            },
            [&](int j, Slot& s) {
                const bool past = (s0 + j) * W::KS + W::KS / 4 * hq >= d;
#pragma unroll
                for (int i = 0; i < W::J; ++i) {
                    if (past) s.x[i] = u32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            W::get(s.w[f], i), __builtin_bit_cast(bf16x8_t, s.x[i]), acc[f], 0, 0,
                            0);
                }
            });
        if (task != (int)blockIdx.x) __syncthreads();  // the last task's partial tiles have been read
#pragma unroll
        for (int f = 0; f < 4; ++f) part[wave][f][lane] = acc[f];
        __syncthreads();
        // thread: token tid / 32, column tid % 32; a lane holds rows 4 (lane / 16) .. + 3 of its
        // fragment for token lane % 16
        const int t = tid >> 5, col = tid & 31, f = col >> 4;
        const int l = ((col & 15) >> 2) * 16 + t, i = col & 3;
        const int slot = slots.slot[e][t];
        if (slot >= 0) {
            float g = part[0][f][l][i], up = part[0][f + 2][l][i];
#pragma unroll
            for (int q = 1; q < kUpWaves; ++q) {
                g += part[q][f][l][i];
                up += part[q][f + 2][l][i];
            }
            in.h[(int64_t)slot * m + 32 * c + col] = f32_to_bf16(g * sigma_bf16(g) * up * sw[slot]);
        }
    }
}

// 16 columns of y a block; the used experts' contractions one behind the other, cut evenly into
// sixteen waves
template <class W, int R>
__global__ __launch_bounds__(64 * kDownWaves) void few_down(FewIn in) {
    __shared__ f32x4_t part[kDownWaves][64];
    __shared__ Slots slots;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int d = in.d, m = in.m;
    find_slots(slots, in.k, in.ids, in.T, in.K, in.N);
    const int per = (m + W::KS - 1) / W::KS, steps = slots.used * per;
    const int s0 = steps * wave / kDownWaves, s1 = steps * (wave + 1) / kDownWaves;
    const int64_t row = (int64_t)blockIdx.x * 16 + l16;
    struct Slot {
        typename W::Frag w;
        u32x4_t x[W::J];
        bool live;
    };
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    int u = s0 / per, s = s0 - u * per;  // of the next step to load
    ring<R, Slot>(
        s1 - s0,
        [&](int, Slot& sl) {
            const int e = __builtin_amdgcn_readfirstlane(slots.list[u]);
            const int slot = slots.slot[e][l16];
            int k = s * W::KS + W::KS / 4 * hq;
            sl.live = slot >= 0 && k < m;
            k = k < m ? k : m - W::KS / 4;
            expert<W>(in.down, in.d_scale, (int64_t)e * d * m, m).load(sl.w, row, k);
            const bf16_t* const hr = in.h + (int64_t)(slot >= 0 ? slot : 0) * m + k;
#pragma unroll
            for (int i = 0; i < W::J; ++i)
                sl.x[i] = *reinterpret_cast<const u32x4_any_t*>(hr + 8 * i);
            if (++s == per) s = 0, ++u;
        },
        [&](int, Slot& sl) {
#pragma unroll
            for (int i = 0; i < W::J; ++i) {
                if (!sl.live) sl.x[i] = u32x4_t{0, 0, 0, 0};
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    W::get(sl.w, i), __builtin_bit_cast(bf16x8_t, sl.x[i]), acc, 0, 0, 0);
            }
        });
    part[wave][lane] = acc;
    __syncthreads();
    if (tid >= 256) return;
    const int t = tid >> 4, col = tid & 15;
    if (t >= in.T) return;
    const int l = (col >> 2) * 16 + t, i = col & 3;
    float v = part[0][l][i];
#pragma unroll
    for (int q = 1; q < kDownWaves; ++q) v += part[q][l][i];
    const int64_t o = (int64_t)t * d + (int64_t)blockIdx.x * 16 + col;
    if (in.residual) v += bf16_to_f32(in.residual[o]);
    in.y[o] = f32_to_bf16(v);
}

template <class W, int NG, int RU>
void run_up(const FewIn& in, unsigned blocks, hipStream_t s) {
    const XTable xt = make_xtable(in.N);
    if (in.K <= 8)
        ELB_LAUNCH((few_up<W, NG, 8, RU>), dim3(blocks), dim3(64 * kUpWaves), 0, s, in, xt);
    else
        ELB_LAUNCH((few_up<W, NG, kLaneMaxK, RU>), dim3(blocks), dim3(64 * kUpWaves), 0, s, in, xt);
}

template <class W, int RU, int RD>
hipError_t few(const FewIn& in, int cus, hipStream_t s) {
    {
        ProfileScope prof("few_up", s);
        const int most = (in.T * in.K < in.N ? in.T * in.K : in.N) * (in.m / 32);
        const unsigned blocks = most < cus ? most : cus;
        if (in.N > 48) run_up<W, 4, RU>(in, blocks, s);
        else if (in.N > 32) run_up<W, 3, RU>(in, blocks, s);
        else if (in.N > 16) run_up<W, 2, RU>(in, blocks, s);
        else run_up<W, 1, RU>(in, blocks, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    ProfileScope prof("few_down", s);
    ELB_LAUNCH((few_down<W, RD>), dim3(in.d / 16), dim3(64 * kDownWaves), 0, s, in);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_moe_few(const void* x, const void* Wr, const void* Wgu, const uint8_t* gu_scale,
                          const void* Wd, const uint8_t* d_scale, const void* res, int64_t T, int d,
                          int N, int m, const elb_route_params& p, void* h, void* y, int* k,
                          int* ids, float* w, int cus, hipStream_t s) {
    const FewIn in{(const bf16_t*)x, (const bf16_t*)Wr, Wgu, Wd, gu_scale, d_scale,
                   (const bf16_t*)res, (int)T, d, N, m, p.K, p.mode, p.renormalize, p.eps,
                   (bf16_t*)h, (bf16_t*)y, k, ids, w};
    return gu_scale ? few<WF4, 4, 4>(in, cus, s) : few<WBf16, 8, 8>(in, cus, s);
}

}  // namespace elb
