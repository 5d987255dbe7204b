// Norms before and after a block, with its gate and residual scale, forward and backward.
//
//   forward   r_b = 1 / sqrt(mean(b^2) + eps),  p = w_post b r_b          (no w_post: p = b)
//             s = alpha res + beta gate p,  r_s = 1 / sqrt(mean(s^2) + eps),  n = w_pre s r_s
//   backward  S = ds + r_s (w_pre dn - s^ mean(s^ w_pre dn)),  s^ = s r_s,  dres = alpha S
//             dp = beta S gate,  db = r_b (w_post dp - b^ mean(b^ w_post dp)),  b^ = b r_b
//             dgate = beta S p, dw_post = dp b^, dw_pre = dn s^, summed over what they are broadcast to
//
// Every tensor is read once and written once: a row stays in registers between the two
// reductions that it needs (its second waits for the first: s is made of b's norm).  n is taken from
// s before its rounding; the backward reads s as stored, whose rounding moves s^ by half a step of it.
#include "dense.h"

namespace elb {

namespace {

// the sum over a wave, in lane order of a fixed tree; every lane gets it
__device__ __forceinline__ float wave_sum(float v) {
#define ELB_SUM_STEP(ctrl, rows)                                                              \
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), ctrl, rows, 0xf, false))
    ELB_SUM_STEP(0x111, 0xf);  // row_shr:1, 2, 4, 8: lane 15 of each row of 16 has the row's sum
    ELB_SUM_STEP(0x112, 0xf);
    ELB_SUM_STEP(0x114, 0xf);
    ELB_SUM_STEP(0x118, 0xf);
    ELB_SUM_STEP(0x142, 0xa);  // row_bcast:15 to rows 1 and 3, row_bcast:31 to rows 2 and 3
    ELB_SUM_STEP(0x143, 0xc);
#undef ELB_SUM_STEP
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// The sum over the N threads of a row (whole waves; N > 64: through sh, one word per wave of the
// block, whose waves all call this).  A caller alternates between two sh, so that a word is read by
// all before it is written again.
template <int N>
__device__ __forceinline__ float row_sum(float v, float* sh) {
    v = wave_sum(v);
    if constexpr (N == 64) return v;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) sh[wave] = v;
    __syncthreads();
    constexpr int W = N / 64;
    const float* const mine = sh + wave / W * W;
    float t = mine[0];
#pragma unroll
    for (int i = 1; i < W; ++i) t += mine[i];
    return t;
}

// Two of them behind one barrier
template <int N>
__device__ __forceinline__ void row_sum2(float& v, float& u, float* sh, float* sh2) {
    v = wave_sum(v);
    u = wave_sum(u);
    if constexpr (N > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            sh[wave] = v;
            sh2[wave] = u;
        }
        __syncthreads();
        constexpr int W = N / 64;
        const int at = wave / W * W;
        v = sh[at];
        u = sh2[at];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            v += sh[at + i];
            u += sh2[at + i];
        }
    }
}

// 1 / sqrt(mean of v^2 + eps) of a row.  Where that leaves fp32's range it is taken again of v 2^-72 and
// eps 2^-144: the largest squares are below 2^112 then, and 16384 of them below 2^126.  Near the lower end
// (eps and the row both tiny), where squares lose digits, of v 2^72 and eps 2^144: less than 2^42 and at
// least 2^-5.  (The branch is the same for all that work on the row.)
template <int N, int KEEP>
__device__ __forceinline__ float row_rstd(const float (&v)[KEEP][8], int d, float eps, float* sh) {
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) a = fmaf(v[i][q], v[i][q], a);
    a = row_sum<N>(a, sh);
    const float ms = a / (float)d + eps;
    if (__builtin_expect(ms < INFINITY && ms >= 0x1p-102f, 1)) return 1.0f / sqrtf(ms);
    const float scale = ms < 1.0f ? 0x1p72f : 0x1p-72f;
    a = 0.0f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float t = v[i][q] * scale;
            a = fmaf(t, t, a);
        }
    if (N > 64) __syncthreads();
    a = row_sum<N>(a, sh);
    return scale / sqrtf(a / (float)d + eps * scale * scale);
}

// Eight values as loaded, in as many registers as they have words (dense.h's Eight lets the compiler
// split bf16 pairs, twice the registers: the backward of 4096 rows of 2048 then spilled, 60 us)
template <class T>
struct Packed;
template <>
struct Packed<bf16_t> {
    u32x4_t v;
    __device__ __forceinline__ void load(const bf16_t* p) {
        v = *reinterpret_cast<const u32x4_any_t*>(p);
    }
    __device__ __forceinline__ float operator[](int i) const {
        return __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
    }
};
template <>
struct Packed<float> {
    f32x4_t a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4_any_t*>(p);
        b = *reinterpret_cast<const f32x4_any_t*>(p + 4);
    }
    __device__ __forceinline__ float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
};
__device__ __forceinline__ float one_value(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float one_value(const float* p) { return *p; }

template <class T>
struct NormIn {
    const T *residual, *block, *gate, *w_post, *w_pre;
    int64_t rows;
    int d, gate_kind;
    float alpha, beta;
};

// the gate of row `row` at the eight columns from c on
template <class T>
__device__ __forceinline__ void load_gate(const NormIn<T>& in, int64_t row, int c, Packed<T>& g) {
    if (in.gate_kind == ELB_GATE_CHANNEL) g.load(in.gate + c);
    else if (in.gate_kind == ELB_GATE_FULL) g.load(in.gate + row * in.d + c);
}

// Blocks of up to 1024 threads in rows of 2^20: a launch dimension stays below 2^32 threads.
constexpr int kNormRow = 1 << 20;

// N threads a row (a wave, or the whole block), eight columns of each of KEEP groups a thread.  Bound by
// memory: 16384 rows of 2048, bf16, with a gate per element 59.5 us, 5.6 TB/s; one row 2.6 us.
template <class T, int N, int KEEP>
__global__ __launch_bounds__(N == 64 ? 256 : N) void norm_forward(NormIn<T> in, float eps,
                                                                  T* sum, T* normed, float* r_post,
                                                                  float* r_pre) {
    __shared__ float sh[2][16];
    constexpr int RPB = N == 64 ? 4 : 1;
    const int tid = threadIdx.x % N, d = in.d;
    const int64_t row = ((int64_t)blockIdx.y * kNormRow + blockIdx.x) * RPB + threadIdx.x / N;
    if (row >= in.rows) return;  // a whole wave, or a whole block
    Packed<T> x[KEEP], b[KEEP], g[KEEP], wp[KEEP], wn[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int c = (i * N + tid) * 8;
        if (c >= d) continue;
        if (in.block) b[i].load(in.block + row * d + c);
        if (in.residual) x[i].load(in.residual + row * d + c);
        load_gate(in, row, c, g[i]);
        if (in.w_post) wp[i].load(in.w_post + c);
        if (normed) wn[i].load(in.w_pre + c);
    }
    float v[KEEP][8];
    float scale = in.beta;
    if (in.gate_kind == ELB_GATE_TOKEN) scale *= one_value(in.gate + row);
    if (in.block) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[i][q] = (i * N + tid) * 8 < d ? b[i][q] : 0.0f;
        float r = 1.0f;
        if (in.w_post) {
            r = row_rstd<N>(v, d, eps, sh[0]);
            if (r_post && tid == 0) r_post[row] = r;
        }
        const bool gated = in.gate_kind == ELB_GATE_CHANNEL || in.gate_kind == ELB_GATE_FULL;
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float p = v[i][q] * r;
                if (in.w_post) p *= wp[i][q];
                if (gated) p *= g[i][q];
                v[i][q] = (i * N + tid) * 8 < d ? p * scale : 0.0f;
            }
    } else {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[i][q] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int c = (i * N + tid) * 8;
        if (c >= d) continue;
        if (in.residual) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[i][q] = fmaf(in.alpha, x[i][q], v[i][q]);
        }
        if (sum) store8(sum + row * d + c, v[i]);
    }
    if (!normed) return;  // kernel-uniform
    const float r = row_rstd<N>(v, d, eps, sh[1]);
    if (r_pre && tid == 0) r_pre[row] = r;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int c = (i * N + tid) * 8;
        if (c >= d) continue;
        float o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = v[i][q] * r * wn[i][q];
        store8(normed + row * d + c, o);
    }
}

template <class T>
struct NormGradIn {
    const T *ds, *dn, *sum;
    const float *r_post, *r_pre;
    T *dres, *dblock, *dgate;
    float* part;  // sums over a block's rows [blocks, 3, d]: of w_pre, w_post, the gate per channel
    int cols;     // bit j: sum j is wanted
};

// What a row brings, as loaded
template <class T, int KEEP>
struct RowIn {
    Packed<T> ds[KEEP], dn[KEEP], s[KEEP], b[KEEP], g[KEEP];
    float rs, rb, gt;  // r_pre, r_post (1 without w_post), a gate per token
};

// RPB rows of N threads at a time, the block's rows RPB gridDim apart.  The sums over the rows stay in
// registers until the end, then the RPB of the block are added in LDS, in order.  (The next rows loaded
// ahead of the present ones' work take registers that the block's other rows need: 39 us for 25.)
// 4096 rows of 2048, bf16, gate per channel: 23.7 us, 4.2 TB/s, and the sums over the blocks 4.0.
template <class T, int N, int KEEP, int RPB>
__global__ __launch_bounds__(N* RPB) void norm_backward(NormIn<T> in, NormGradIn<T> gr) {
    constexpr int W = N * RPB / 64;
    __shared__ float sh[3][2][W];  // per sum and parity of the round
    // a row's threads and eight words more, which put the eight columns of a thread in other banks
    constexpr int CN = N + 8;
    __shared__ float cols[3][RPB > 1 ? RPB * 8 * CN : 1];
    const int tid = threadIdx.x % N, sub = threadIdx.x / N, d = in.d;
    const float inv_d = 1.0f / (float)d;
    float acc[3][KEEP][8];
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[j][i][q] = 0.0f;
    const bool branch = gr.dblock || gr.dgate || (gr.cols & 6);
    const bool gated = in.gate_kind == ELB_GATE_CHANNEL || in.gate_kind == ELB_GATE_FULL;
    typedef RowIn<T, KEEP> R;
    auto load = [&](int64_t row, R& r) {
        const bool live = row < in.rows;
        r.rs = r.rb = r.gt = 1.0f;
        if (live && gr.dn) r.rs = gr.r_pre[row];
        if (live && branch && in.w_post) r.rb = gr.r_post[row];
        if (live && branch && in.gate_kind == ELB_GATE_TOKEN) r.gt = one_value(in.gate + row);
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int c = (i * N + tid) * 8;
            r.ds[i] = r.dn[i] = r.s[i] = r.b[i] = r.g[i] = Packed<T>{};
            if (c >= d || !live) continue;
            const int64_t o = row * d + c;
            if (gr.ds) r.ds[i].load(gr.ds + o);
            if (gr.dn) {
                r.dn[i].load(gr.dn + o);
                r.s[i].load(gr.sum + o);
            }
            if (branch) {
                r.b[i].load(in.block + o);
                if (in.gate_kind == ELB_GATE_FULL) r.g[i].load(in.gate + o);
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * RPB;
    int ph = 0;
    R r;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < in.rows; r0 += step) {
        const int64_t row = r0 + sub;
        const bool live = row < in.rows;
        load(row, r);
        // the norms' weights and a gate per channel are the same for every row, but are read again, from
        // L1, rather than held in registers
        asm volatile("" ::: "memory");
        float S[KEEP][8];
        float a = 0.0f;
        if (gr.dn) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                Packed<T> wn = {};
                if ((i * N + tid) * 8 < d) wn.load(in.w_pre + (i * N + tid) * 8);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float t = wn[q] * r.dn[i][q], hat = r.s[i][q] * r.rs;
                    S[i][q] = t;
                    a = fmaf(t, hat, a);
                    acc[0][i][q] = fmaf(r.dn[i][q], hat, acc[0][i][q]);
                }
            }
            a = row_sum<N>(a, sh[0][ph]) * inv_d;
        }
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int c = (i * N + tid) * 8;
            float o[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float t = r.ds[i][q];
                if (gr.dn) t += r.rs * fmaf(-r.s[i][q] * r.rs, a, S[i][q]);
                S[i][q] = t;
                o[q] = in.alpha * t;
            }
            if (gr.dres && live && c < d) store8(gr.dres + row * d + c, o);
        }
        if (branch) {
            float m = 0.0f, tok = 0.0f;
            float u[KEEP][8];
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                const int c = (i * N + tid) * 8;
                Packed<T> wp = {}, gc = {};
                if (c < d && in.w_post) wp.load(in.w_post + c);
                if (c < d && in.gate_kind == ELB_GATE_CHANNEL) gc.load(in.gate + c);
                float o[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float bh = r.b[i][q] * r.rb, qv = in.beta * S[i][q];
                    const float g = !gated ? r.gt : in.gate_kind == ELB_GATE_FULL ? r.g[i][q]
                                                                                  : gc[q];
                    const float dp = qv * g, w = in.w_post ? wp[q] : 1.0f;
                    o[q] = qv * (w * bh);
                    tok += o[q];
                    acc[2][i][q] += o[q];
                    acc[1][i][q] = fmaf(dp, bh, acc[1][i][q]);
                    u[i][q] = w * dp;
                    m = fmaf(u[i][q], bh, m);
                }
                if (gr.dgate && in.gate_kind == ELB_GATE_FULL && live && c < d)
                    store8(gr.dgate + row * d + c, o);
            }
            if (in.w_post || (gr.dgate && in.gate_kind == ELB_GATE_TOKEN)) {
                row_sum2<N>(m, tok, sh[1][ph], sh[2][ph]);
                m *= inv_d;
            }
            if (gr.dgate && in.gate_kind == ELB_GATE_TOKEN && live && tid == 0) {
                if constexpr (sizeof(T) == 2) gr.dgate[row] = f32_to_bf16(tok);
                else gr.dgate[row] = tok;
            }
            if (gr.dblock) {
#pragma unroll
                for (int i = 0; i < KEEP; ++i) {
                    const int c = (i * N + tid) * 8;
                    if (c >= d || !live) continue;
                    float o[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        o[q] = in.w_post ? r.rb * fmaf(-r.b[i][q] * r.rb, m, u[i][q]) : u[i][q];
                    store8(gr.dblock + row * d + c, o);
                }
            }
        }
        ph ^= 1;
    }
    // the block's sums, one row of d floats of `part` for each
    float* const out = gr.part + (int64_t)blockIdx.x * 3 * d;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int c = (i * N + tid) * 8;
        if constexpr (RPB > 1) {
            static_assert(KEEP == 1, "one pass through LDS");
#pragma unroll
            for (int j = 0; j < 3; ++j)
#pragma unroll
                for (int q = 0; q < 8; ++q) cols[j][(sub * 8 + q) * CN + tid] = acc[j][i][q];
            __syncthreads();
            // 3 times 8 N sums by N RPB threads, in the order of the columns
#pragma unroll
            for (int j = 0; j < 3; ++j)
                for (int k = threadIdx.x; k < 8 * N; k += N * RPB) {
                    const int at = k % 8 * CN + k / 8;
                    float t = cols[j][at];
#pragma unroll
                    for (int p = 1; p < RPB; ++p) t += cols[j][p * 8 * CN + at];
                    if (k < d && (gr.cols >> j & 1)) out[(int64_t)j * d + k] = t;
                }
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (c < d && (gr.cols >> j & 1)) store8(out + (int64_t)j * d + c, acc[j][i]);
        }
    }
}

// The sums over all blocks of the backward: 64 columns a block, sixteen threads a column, each of which
// adds a sixteenth of the blocks in order.
template <class T>
__global__ __launch_bounds__(1024) void norm_columns(const float* __restrict__ part, int blocks,
                                                     int d, T* o0, T* o1, T* o2) {
    __shared__ float sh[16][64];
    const int j = blockIdx.y, l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + l;
    T* const out = j == 0 ? o0 : j == 1 ? o1 : o2;
    if (!out) return;  // block-uniform
    float t = 0.0f;
    if (c < d) {
        const float* const p = part + (int64_t)j * d + c;
        const int b1 = blocks * (w + 1) / 16;
#pragma unroll 16
        for (int b = blocks * w / 16; b < b1; ++b) t += p[(int64_t)b * 3 * d];
    }
    sh[w][l] = t;
    __syncthreads();
    if (w == 0 && c < d) {
        t = sh[0][l];
#pragma unroll
        for (int i = 1; i < 16; ++i) t += sh[i][l];
        if constexpr (sizeof(T) == 2) out[c] = f32_to_bf16(t);
        else out[c] = t;
    }
}

template <class T, int N, int KEEP>
void forward(const NormIn<T>& in, float eps, T* sum, T* normed, float* r_post, float* r_pre,
             hipStream_t s) {
    const int64_t blocks = N == 64 ? (in.rows + 3) / 4 : in.rows;
    const dim3 grid((unsigned)(blocks < kNormRow ? blocks : kNormRow),
                    (unsigned)((blocks + kNormRow - 1) / kNormRow));
    ELB_LAUNCH((norm_forward<T, N, KEEP>), grid, dim3(N == 64 ? 256 : N), 0, s, in, eps, sum, normed,
               r_post, r_pre);
}

template <class T>
hipError_t forward_of(const elb_norm& p, void* sum, void* normed, float* r_post, float* r_pre,
                      hipStream_t s) {
    ProfileScope prof("norm_forward", s);
    const NormIn<T> in{(const T*)p.residual, (const T*)p.block, (const T*)p.gate,
                       (const T*)p.w_post, (const T*)p.w_pre, p.T, p.d, p.gate_kind,
                       p.residual_scale, p.block_scale};
    T *const o = (T*)sum, *const n = (T*)normed;
    if (p.d <= 512) forward<T, 64, 1>(in, p.eps, o, n, r_post, r_pre, s);
    else if (p.d <= 1024) forward<T, 128, 1>(in, p.eps, o, n, r_post, r_pre, s);
    else if (p.d <= 2048) forward<T, 256, 1>(in, p.eps, o, n, r_post, r_pre, s);
    else if (p.d <= 4096) forward<T, 256, 2>(in, p.eps, o, n, r_post, r_pre, s);
    else if (p.d <= 8192) forward<T, 1024, 1>(in, p.eps, o, n, r_post, r_pre, s);
    else forward<T, 1024, 2>(in, p.eps, o, n, r_post, r_pre, s);
    return hipGetLastError();
}

// The backward's shape by row length: as many threads a row as leave a thread eight values, and rows to
// fill a block of 512 threads.  (4096 rows of 2048, bf16, one row a block 29.4 us with the sums over the
// blocks, two 28.1, four 29.4; 16384 rows 88, 86, 93; 2048 rows of 4096, 256 threads and sixteen values 43.)
struct BackShape {
    int threads, rows;
};
BackShape back_shape(int d) {
    if (d <= 512) return {64, 8};
    if (d <= 1024) return {128, 4};
    if (d <= 2048) return {256, 2};
    return {d <= 4096 ? 512 : 1024, 1};
}

template <class T, int N, int KEEP, int RPB>
void backward(const NormIn<T>& in, const NormGradIn<T>& g, int blocks, hipStream_t s) {
    ELB_LAUNCH((norm_backward<T, N, KEEP, RPB>), dim3(blocks), dim3(N * RPB), 0, s, in, g);
}

template <class T>
hipError_t backward_of(const elb_norm& p, const void* ds, const void* dn, const void* sum,
                       const float* r_post, const float* r_pre, void* dres, void* dblock,
                       void* dgate, void* dw_post, void* dw_pre, void* part, hipStream_t s) {
    const NormIn<T> in{nullptr, (const T*)p.block, (const T*)p.gate, (const T*)p.w_post,
                       (const T*)p.w_pre, p.T, p.d, p.gate_kind, p.residual_scale,
                       p.block_scale};
    const bool channel = p.gate_kind == ELB_GATE_CHANNEL;
    const int cols = (dw_pre ? 1 : 0) | (dw_post ? 2 : 0) | (dgate && channel ? 4 : 0);
    const NormGradIn<T> g{(const T*)ds, (const T*)dn, (const T*)sum, r_post, r_pre, (T*)dres,
                          (T*)dblock, (T*)dgate, (float*)part, cols};
    const int blocks = norm_backward_blocks(p.T, p.d);
    if (blocks) {
        ProfileScope prof("norm_backward", s);
        if (p.d <= 512) backward<T, 64, 1, 8>(in, g, blocks, s);
        else if (p.d <= 1024) backward<T, 128, 1, 4>(in, g, blocks, s);
        else if (p.d <= 2048) backward<T, 256, 1, 2>(in, g, blocks, s);
        else if (p.d <= 4096) backward<T, 512, 1, 1>(in, g, blocks, s);
        else if (p.d <= 8192) backward<T, 1024, 1, 1>(in, g, blocks, s);
        else backward<T, 1024, 2, 1>(in, g, blocks, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (!cols) return hipSuccess;
    ProfileScope prof("norm_columns", s);
    ELB_LAUNCH(norm_columns<T>, dim3((p.d + 63) / 64, 3), dim3(1024), 0, s, (const float*)part,
               blocks, p.d, (T*)dw_pre, (T*)dw_post, channel ? (T*)dgate : nullptr);
    return hipGetLastError();
}

}  // namespace

// at most 1024 threads a compute unit
int norm_backward_blocks(int64_t T, int d) {
    const BackShape b = back_shape(d);
    const int64_t n = (T + b.rows - 1) / b.rows, most = 256 * 1024 / (b.threads * b.rows);
    return (int)(n < most ? n : most);
}

hipError_t launch_norm_forward(const elb_norm& p, void* sum, void* normed, float* r_post,
                               float* r_pre, hipStream_t s) {
    return p.dtype == ELB_BF16 ? forward_of<bf16_t>(p, sum, normed, r_post, r_pre, s)
                               : forward_of<float>(p, sum, normed, r_post, r_pre, s);
}

hipError_t launch_norm_backward(const elb_norm& p, const void* ds, const void* dn, const void* sum,
                                const float* r_post, const float* r_pre, void* dres, void* dblock,
                                void* dgate, void* dw_post, void* dw_pre, void* part,
                                hipStream_t s) {
    return (p.dtype == ELB_BF16 ? backward_of<bf16_t> : backward_of<float>)(
        p, ds, dn, sum, r_post, r_pre, dres, dblock, dgate, dw_post, dw_pre, part, s);
}

}  // namespace elb
