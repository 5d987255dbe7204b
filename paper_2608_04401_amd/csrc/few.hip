// The whole layer for at most 16 tokens in two launches.
//
//   launch 1  router, routing, h_tj = w_tj silu(W_gate x_t) * (W_up x_t) for each selected expert
//   launch 2  y_t = [residual_t +] sum_j W_down[e_j] h_tj
//
// All tokens are one MFMA tile of 16 rows.  In launch 1 every block routes all of them for itself (the
// same bits as the other router paths: the same chains, sums and per-token code), instead of waiting
// for a launch that does, and then takes its share of the used experts' gate and up rows.  In launch 2
// the experts lie one behind the other in one long contraction, of which a token's sums take what belongs
// to experts that it has selected; its routing weight is in h already, so the products' sum is the combine.
#include "f4.h"
#include "route_lane.h"

namespace elb {

namespace {

constexpr int kUpWaves = 8, kDownWaves = 16;
constexpr int kDownFrags = 2;  // of 16 columns, a block of launch 2

// The experts that some token has selected (list[0 .. used)), and of each its tokens: a bit for each,
// the slot t K + j of each (where its bit is set), and their slots in order.
struct Slots {
    uint32_t tokens[64];
    int16_t slot[64][16], row[64][16];
    int list[64];
    int used;
};

// k, ids: the routing of T tokens (at most 16 x 16 slots); by the whole block, which it synchronises
__device__ __forceinline__ void find_slots(Slots& s, const int* k, const int* ids, int T, int K,
                                           int N) {
    const int q = threadIdx.x;
    int e = -1;
    const int t = q / K;
    if (q < T * K) {
        e = ids[q];
        if (q - t * K >= k[t] || e >= N) e = -1;
    }
    if (q < 64) s.tokens[q] = 0;
    __syncthreads();
    if (e >= 0) atomicOr(&s.tokens[e], 1u << t);
    __syncthreads();
    if (e >= 0) {
        s.slot[e][t] = (int16_t)q;
        s.row[e][__popc(s.tokens[e] & ((1u << t) - 1))] = (int16_t)q;
    }
    if (q < 64) {
        const uint64_t used = __ballot(s.tokens[q] != 0);
        if (s.tokens[q] != 0) s.list[__popcll(used & ((1ull << q) - 1))] = q;
        if (q == 0) s.used = __popcll(used);
    }
    __syncthreads();
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
    float* part;  // shares > 1: partial sums of launch 2 [column tiles, shares, 16, columns], and
    int* count;   // how many of a column tile's are written (zeroed by launch 1)
    int shares;
};

// A wave's tokens of 16 bytes a lane: row l16, values 8 hq .. of a run of 32
__device__ __forceinline__ bf16x8_t as_frag(u32x4_t v) { return __builtin_bit_cast(bf16x8_t, v); }

// ------------------------------------------------------------------------------------------
// Launch 1.  XR: rows of x, 8 or 16; DMA: x, W_router and the weights on 16-byte boundaries.
// 64 experts of 2048 x 1024, top 8: one token 18.2 us (4 bits 13.4), of which the routing 6.6; 13 tokens in 4
// bits 34.7, the weights at 4.6 TB/s after it.
// ------------------------------------------------------------------------------------------
template <class W, int XR, bool DMA>
__global__ __launch_bounds__(64 * kUpWaves) void few_up(FewIn in, XTable xt) {
    typedef Stream<W, 4, true, DMA, true> B;
    // a wave's LDS: a unit of weights, then its partial tiles; before that RN units of the router, as
    // many as fit
    constexpr int PART = (B::BYTES + 255) / 256 * 256;
    constexpr int RUNIT = 32 * 128 + XR * 128, RN = XR == 8 ? 3 : 2;  // 32 rows of W_router, XR of x
    constexpr int SLOT = PART + 4096 > RN * RUNIT ? PART + 4096 : RN * RUNIT;
    __shared__ __attribute__((aligned(1024))) char sm[kUpWaves * SLOT];
    __shared__ float logits[RW][16 * 65];
    __shared__ Slots slots;
    __shared__ float sorted[XR][64];
    __shared__ int order[XR][64], rank[XR][64];
    __shared__ int sk[16], sids[16 * kLaneMaxK];
    __shared__ float sw[16 * kLaneMaxK];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int T = in.T, d = in.d, N = in.N, m = in.m, K = in.K;
    char* const slot = sm + wave * SLOT;
    const uint32_t lds = lds_address(slot);

    if (blockIdx.x == 0 && in.shares > 1)
        for (int i = tid; i < d / (16 * kDownFrags); i += 64 * kUpWaves) in.count[i] = 0;
    for (int i = wave; i < XR; i += kUpWaves) rank[i][lane] = 0;

    // the tokens' operands of this wave's share of the contraction, where it is at most 256 long
    const int units = (d + W::KU - 1) / W::KU;
    const int u0 = units * wave / kUpWaves, u1 = units * (wave + 1) / kUpWaves;
    const bool held = (units + kUpWaves - 1) / kUpWaves * W::KU <= 256;
    const bf16_t* const xr = in.x + (int64_t)(l16 < T ? l16 : T - 1) * d + 8 * hq;
    u32x4_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = u0 * W::KU + 32 * i;
        x[i] = *reinterpret_cast<const u32x4_any_t*>(xr + (k < d ? k : d - 32));
    }

    // ---- router: wave w has slice w % 4 of the contraction and experts 32 (w / 4) .. + 31 ----
    {
        int first, count;
        router_slice(d, wave & 3, first, count);
        const int e0 = 32 * (wave >> 2);
        const int n = (count + 1) / 2;  // units of two steps of 32
        // Byte offsets of the lane's copies: rows 8 i + lane / 8 of W_router and of x (past the last
        // one that again, whose logits no token or expert takes), chunk kc_swz(row, lane % 8).  (Copier's
        // bounds for each unit take longer than its copies: one token's router 5.0 us with them, 3.8 with
        // these.)
        uint32_t off[4 + XR / 8], swz[2];
#pragma unroll
        for (int i = 0; i < 4 + XR / 8; ++i) {
            int r = 8 * (i < 4 ? i : i - 4) + (lane >> 3);
            if (i < 2) swz[i] = kc_swz(r, lane & 7) * 16;
            if (i < 4) r = e0 + r < N ? e0 + r : N - 1;
            else r = r < T ? r : T - 1;
            off[i] = ((uint32_t)r * (uint32_t)d + (uint32_t)first * 32u) * 2u;
        }
        auto issue = [&](int u, int at) {
            u = u < n ? u : n - 1;  // past the last one: that again, so that the waits' counts hold
            const bool whole = 2 * u + 1 < count;
#pragma unroll
            for (int i = 0; i < 4 + XR / 8; ++i) {
                // of a unit of one step the lower half alone is read
                const uint32_t o = off[i] + (uint32_t)u * 128u + (whole ? swz[i & 1] : swz[i & 1] & 63u);
                const char* const src = (const char*)(i < 4 ? in.router : in.x);
                if constexpr (DMA)
                    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2"
                                 :: "s"(lds + at * RUNIT + i * 1024), "v"(o), "s"(src)
                                 : "memory", "m0");
                else
                    copy16_any(slot + at * RUNIT + i * 1024 + lane * 16, src + o);
            }
        };
        f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        constexpr int RI = 4 + XR / 8;  // copy instructions of a unit
#pragma unroll
        for (int u = 0; u < RN; ++u)
            if (n > 0) issue(u, u);
        int at = 0;
        for (int u = 0; u < n; ++u) {
            ELB_WAIT_VMCNT((RN - 1) * RI);  // all but the units after this one
            asm volatile("" ::: "memory");
            const char* const p = slot + at * RUNIT;
            const int xr = l16 % XR;
            u32x4_t a[2], b[2][2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                a[s] = *reinterpret_cast<const u32x4_t*>(p + 4096 + xr * 128 +
                                                         kc_swz(xr, 4 * s + hq) * 16);
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    b[s][g] = *reinterpret_cast<const u32x4_t*>(p + (16 * g + l16) * 128 +
                                                                kc_swz(l16, 4 * s + hq) * 16);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the unit is free again
            issue(u + RN, at);
            at = at + 1 == RN ? 0 : at + 1;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (2 * u + s >= count) break;
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(a[s]), as_frag(b[s][g]),
                                                                     acc[g], 0, 0, 0);
            }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                logits[wave & 3][(4 * hq + r) * 65 + e0 + 16 * g + l16] = acc[g][r];
    }
    ELB_WAIT_VMCNT(0);  // the last copies, before their LDS is used again; and x
    __syncthreads();
    // A lane per expert has its logit, and its rank by counting the (key, id) pairs before it, in the
    // order of route_token_x16's network: a token or two a wave, or several waves a token (from here to
    // the selection, one token 3.4 us, 4.5 by the network; from 9 tokens on the two take as long).
    {
        const int parts = XR > 8 || T > 4 ? 1 : T > 2 ? 2 : T > 1 ? 4 : 8;  // waves a token
        const int part = wave % parts;
        float key[XR / 8];
#pragma unroll
        for (int h = 0; h < XR / 8; ++h) {
            const int t = 8 * h + wave / parts;
            key[h] = 0.0f;
            if (t >= T) continue;
            float l = -INFINITY;
            if (lane < N) {
                l = logits[0][t * 65 + lane];
#pragma unroll
                for (int q = 1; q < RW; ++q) l += logits[q][t * 65 + lane];
            }
            key[h] = N == 64 ? order_key(l) : order_key_any(l);
            const int image = ord_flip32(__float_as_int(key[h]));
            const int64_t mine = ((int64_t)image << 32) | (uint32_t)(63 - lane);
            int before = 0;
            const int n = 64 / parts;
            for (int j0 = n * part; j0 < n * (part + 1); j0 += 8)
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int j = j0 + q;
                    const int64_t other =
                        ((int64_t)__builtin_amdgcn_readlane(image, j) << 32) | (uint32_t)(63 - j);
                    before += other > mine;
                }
            atomicAdd(&rank[t][lane], before);
        }
        __syncthreads();
        if (part == 0) {
#pragma unroll
            for (int h = 0; h < XR / 8; ++h) {
                const int t = 8 * h + wave / parts;
                if (t >= T) continue;
                const int r = rank[t][lane];
                sorted[t][r] = key[h];
                order[t][r] = lane;
            }
        }
        __syncthreads();
        if (tid < 16 * XR) {  // whole waves: 16 lanes a token
            const int t = tid >> 4, sl = tid & 15;
            float k4[4];
            int id[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                k4[i] = sorted[t][4 * sl + i];
                id[i] = order[t][4 * sl + i];
            }
            route_sorted_x16(k4, id, N, K, in.eps, in.mode, in.renorm, xt, t, t < T, sk, sids, sw);
        }
    }
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
    const int64_t w_bytes = W::row_bytes((int64_t)2 * m * d);  // of an expert
    int task = blockIdx.x;
    B b;
    typename B::Pending pending = {};
    auto begin = [&](int t) {
        const int u = t / per_e;
        const int e = __builtin_amdgcn_readfirstlane(slots.list[u]);
        b.init((const char*)in.gate_up + e * w_bytes,
               W::SCALES ? in.gu_scale + (int64_t)e * 2 * m * (d / 32) : nullptr,
               32 * (t - u * per_e), 32, m, 2 * (int64_t)m, d, lane);
        if (u0 < u1) b.issue(u0, u1, lds, slot, lane, pending);
        return e;
    };
    int e = task < tasks ? begin(task) : 0;
    while (task < tasks) {
        f32x4_t acc[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const int next = task + gridDim.x;
        int next_e = 0;
        for (int u = u0; u < u1; ++u) {
            if (!held) {
#pragma unroll
                for (int i = 0; i < W::KU / 32; ++i) {
                    const int k = u * W::KU + 32 * i;
                    x[i] = *reinterpret_cast<const u32x4_any_t*>(xr + (k < d ? k : d - 32));
                }
            }
            ELB_WAIT_VMCNT(0);
            b.settle(pending, slot, lane);
            asm volatile("" ::: "memory");
            typename W::Half w[4][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int f = 0; f < 4; ++f) W::read(w[f][h], slot, 64, f, h, l16, hq);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the unit is free again
            if (u + 1 < u1) b.issue(u + 1, u1, lds, slot, lane, pending);
            else if (next < tasks) next_e = begin(next);
            __builtin_amdgcn_sched_barrier(0);
            auto multiply = [&](int at) {  // at: the unit's first operand in x
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < W::J; ++i) {
                        if (u * W::KU + h * (W::KU / 2) + 32 * i >= d) break;
#pragma unroll
                        for (int f = 0; f < 4; ++f)
                            acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                w[f][h].get(i), as_frag(x[at + h * W::J + i]), acc[f], 0, 0, 0);
                    }
            };
            if constexpr (W::KU == 256) {
                multiply(0);
            } else {
                switch (held ? u - u0 : 0) {  // registers have no index
                    case 0: multiply(0); break;
                    case 1: multiply(2); break;
                    case 2: multiply(4); break;
                    default: multiply(6); break;
                }
            }
        }
        if (u0 == u1 && next < tasks) next_e = begin(next);
        f32x4_t* const part = reinterpret_cast<f32x4_t*>(slot + PART);
#pragma unroll
        for (int f = 0; f < 4; ++f) part[f * 64 + lane] = acc[f];
        __syncthreads();
        // thread: token tid / 32, column tid % 32; a lane holds rows 4 (lane / 16) .. + 3 of its
        // fragment for token lane % 16
        const int t = tid >> 5, col = tid & 31, f = col >> 4;
        const int l = ((col & 15) >> 2) * 16 + t, i = col & 3;
        if (slots.tokens[e] >> t & 1) {
            const int at = slots.slot[e][t];
            float g = 0.f, up = 0.f;
#pragma unroll
            for (int q = 0; q < kUpWaves; ++q) {
                const float* const p = reinterpret_cast<const float*>(sm + q * SLOT + PART);
                g += p[(f * 64 + l) * 4 + i];
                up += p[((f + 2) * 64 + l) * 4 + i];
            }
            in.h[(int64_t)at * m + 32 * (task - task / per_e * per_e) + col] =
                f32_to_bf16(g * sigma_bf16(g) * up * sw[at]);
        }
        __syncthreads();  // the partial tiles have been read
        task = next;
        e = next_e;
    }
}

// ------------------------------------------------------------------------------------------
// Launch 2.  A block has 32 columns of y and one of `shares` shares of the contraction, the used
// experts' units one behind the other (per expert as often as its tokens fill tiles of eight); its
// waves take every sixteenth unit.  The last block of a column tile to write its partial sums adds all
// of them, in the order of the shares; none waits for another.  64 experts of 2048 x 1024, top 8: one
// token 9.8 us (4 bits 7.3), 13 tokens in 4 bits 16.1 (64 columns and eight waves: 10.2, 8.0, 17.1).
// ------------------------------------------------------------------------------------------
template <class W, bool DMA>
__global__ __launch_bounds__(64 * kDownWaves) void few_down(FewIn in) {
    constexpr int NF = kDownFrags, COLS = 16 * NF;
    typedef Stream<W, NF, false, DMA, true> B;
    constexpr int SUB = W::KU / 64, AB = SUB * 8 * 128;  // eight rows of h
    constexpr int SLOT = (AB + B::BYTES + 255) / 256 * 256;
    static_assert(SLOT >= NF * 1024, "");
    __shared__ __attribute__((aligned(1024))) char sm[kDownWaves * SLOT];
    __shared__ Slots slots;
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int d = in.d, m = in.m, T = in.T;
    const int tile = blockIdx.x, share = blockIdx.y;
    find_slots(slots, in.k, in.ids, T, in.K, in.N);
    char* const slot = sm + wave * SLOT;
    const uint32_t lds = lds_address(slot);
    const int per = (m + W::KU - 1) / W::KU, units = slots.used * per;
    const int v0 = units * share / in.shares + wave, v1 = units * (share + 1) / in.shares;
    const int64_t w_bytes = W::row_bytes((int64_t)d * m);
    B b0;
    b0.init(in.down, in.d_scale, COLS * tile, COLS, 0, d, m, lane);
    // rows of h: chunk lane % 8 of row lane / 8, in each of the unit's k-tiles of 64
    const uint64_t hb = (uint64_t)in.h;
    const u32x4_t hr = {uniform((uint32_t)hb), uniform((uint32_t)(hb >> 32)) & 0xffffu,
                        uniform((uint32_t)(T * in.K) * (uint32_t)m * 2u), 0x00027000u};
    const int chunk = kc_swz(lane >> 3, lane & 7) * 16;
    typename B::Pending pending = {};
    auto issue = [&](int v, int pass) {
        const int u = v / per, unit = v - u * per;
        const int e = __builtin_amdgcn_readfirstlane(slots.list[u]);
        b0.moved(e * w_bytes, W::SCALES ? (int64_t)e * d * (m / 32) : 0)
            .issue(unit, per, lds + AB, slot + AB, lane, pending);
        const int rank = 8 * pass + (lane >> 3);
        const int at = rank < __popc(slots.tokens[e]) ? slots.row[e][rank] : -1;
#pragma unroll
        for (int q = 0; q < SUB; ++q) {
            const int k = unit * W::KU + 64 * q;  // m is a multiple of 64
            const uint32_t off = at < 0 || k >= m ? kOutOfBounds
                                                  : (uint32_t)at * (uint32_t)m * 2u +
                                                        (uint32_t)k * 2u + chunk;
            asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                         :: "s"(lds + q * 1024), "v"(off), "s"(hr) : "memory", "m0");
        }
        return e;
    };
    f32x4_t acc[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int pass = 0, e = v0 < v1 ? issue(v0, 0) : 0;
    for (int v = v0; v < v1;) {
        ELB_WAIT_VMCNT(0);
        b0.settle(pending, slot + AB, lane);
        asm volatile("" ::: "memory");
        const uint32_t tokens = slots.tokens[e];
        const int rank = __popc(tokens & ((1u << l16) - 1)) - 8 * pass;
        const bool live = (tokens >> l16 & 1) && rank >= 0 && rank < 8;
        const int r = live ? rank : 0;
        typename W::Half w[NF][2];
        u32x4_t x[2][W::J];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int f = 0; f < NF; ++f) W::read(w[f][h], slot + AB, COLS, f, h, l16, hq);
#pragma unroll
            for (int i = 0; i < W::J; ++i) {
                const int run = h * W::J + i;  // of 32 values
                x[h][i] = *reinterpret_cast<const u32x4_t*>(
                    slot + run / 2 * 1024 + r * 128 + kc_swz(r, run % 2 * 4 + hq) * 16);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the unit is free again
        const int k0 = v % per * W::KU;
        // an expert of more than eight tokens takes another pass
        if (8 * (pass + 1) < __popc(tokens)) {
            ++pass;
        } else {
            pass = 0;
            v += kDownWaves;
        }
        if (v < v1) e = issue(v, pass);
        __builtin_amdgcn_sched_barrier(0);
        // A lane's sums are those of token l16: where that has not selected the expert they stay what they
        // were.  (Zeros for its h would not do: 0 times a weight that is infinite or NaN is NaN.)
        f32x4_t sum[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) sum[f] = acc[f];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < W::J; ++i) {
                if (k0 + (h * W::J + i) * 32 >= m) break;
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    sum[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f][h].get(i),
                                                                     as_frag(x[h][i]), sum[f], 0, 0,
                                                                     0);
            }
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[f][q] = live ? sum[f][q] : acc[f][q];
    }
    f32x4_t* const part = reinterpret_cast<f32x4_t*>(slot);
#pragma unroll
    for (int f = 0; f < NF; ++f) part[f * 64 + lane] = acc[f];
    __syncthreads();
    // value i: token i / COLS, column i % COLS
    auto sum = [&](int i) {
        const int t = i / COLS, col = i % COLS;
        const int at = ((col >> 4) * 64 + ((col & 15) >> 2) * 16 + t) * 4 + (col & 3);
        float v = reinterpret_cast<const float*>(sm)[at];
#pragma unroll
        for (int q = 1; q < kDownWaves; ++q)
            v += reinterpret_cast<const float*>(sm + q * SLOT)[at];
        return v;
    };
    float* const mine = in.part + (int64_t)tile * in.shares * (16 * COLS);
    auto put = [&](int i, float v) {
        const int64_t o = (int64_t)(i / COLS) * d + COLS * tile + i % COLS;
        if (in.residual) v += bf16_to_f32(in.residual[o]);
        in.y[o] = f32_to_bf16(v);
    };
    if (in.shares == 1) {
        for (int i = tid; i < T * COLS; i += 64 * kDownWaves) put(i, sum(i));
        return;
    }
    // The partial sums go past the L2, which blocks elsewhere on the chip do not share: agent-scope
    // stores, done when the counter goes up, and agent-scope loads: 2.5 us of a token's 7.  (A release
    // fence would write the whole L2 back, for each block: 31 us more.)
    for (int i = tid; i < T * COLS; i += 64 * kDownWaves)
        __hip_atomic_store(mine + share * (16 * COLS) + i, sum(i), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    ELB_WAIT_VMCNT(0);
    __syncthreads();
    if (tid == 0)
        last = __hip_atomic_fetch_add(in.count + tile, 1, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT) == in.shares - 1;
    __syncthreads();
    if (!last) return;
    for (int i = tid; i < T * COLS; i += 64 * kDownWaves) {
        float p[16], v = 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q)
            p[q] = q < in.shares ? __hip_atomic_load(mine + q * (16 * COLS) + i, __ATOMIC_RELAXED,
                                                     __HIP_MEMORY_SCOPE_AGENT)
                                 : 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q) v += p[q];
        put(i, v);
    }
}

// shares of launch 2's contraction: so many that its blocks fill the compute units
int few_tiles(int d) { return d / (16 * kDownFrags); }
int few_shares(int d) {
    const int n = 256 / few_tiles(d);
    return n < 1 ? 1 : n > 16 ? 16 : n;
}

template <class W, bool DMA>
hipError_t few(const FewIn& in, int cus, hipStream_t s) {
    {
        ProfileScope prof("few_up", s);
        const int most = (in.T * in.K < in.N ? in.T * in.K : in.N) * (in.m / 32);
        const unsigned blocks = most < cus ? most : cus;
        const XTable xt = make_xtable(in.N);
        if (in.T <= 8)
            ELB_LAUNCH((few_up<W, 8, DMA>), dim3(blocks), dim3(64 * kUpWaves), 0, s, in, xt);
        else
            ELB_LAUNCH((few_up<W, 16, DMA>), dim3(blocks), dim3(64 * kUpWaves), 0, s, in, xt);
        if (hipError_t e = hipGetLastError()) return e;
    }
    ProfileScope prof("few_down", s);
    ELB_LAUNCH((few_down<W, DMA>), dim3(few_tiles(in.d), in.shares), dim3(64 * kDownWaves), 0, s,
               in);
    return hipGetLastError();
}

}  // namespace

// no share joins another where there is one alone
size_t few_part_bytes(int d) {
    const int n = few_shares(d);
    return n > 1 ? (size_t)n * 16 * d * 4 : 0;
}
size_t few_count_bytes(int d) { return few_shares(d) > 1 ? (size_t)few_tiles(d) * 4 : 0; }

hipError_t launch_moe_few(const void* x, const void* Wr, const void* Wgu, const uint8_t* gu_scale,
                          const void* Wd, const uint8_t* d_scale, const void* res, int64_t T, int d,
                          int N, int m, const elb_route_params& p, void* h, float* part, int* count,
                          void* y, int* k, int* ids, float* w, int cus, hipStream_t s) {
    const FewIn in{(const bf16_t*)x, (const bf16_t*)Wr, Wgu, Wd, gu_scale, d_scale,
                   (const bf16_t*)res, (int)T, d, N, m, p.K, p.mode, p.renormalize, p.eps,
                   (bf16_t*)h, (bf16_t*)y, k, ids, w, part, count, few_shares(d)};
    const bool dma = aligned16(x, Wr) && aligned16(Wgu, Wd);
    if (!gu_scale) return dma ? few<WBf16, true>(in, cus, s) : few<WBf16, false>(in, cus, s);
    return dma ? few<WF4, true>(in, cus, s) : few<WF4, false>(in, cus, s);
}

}  // namespace elb
