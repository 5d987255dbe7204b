// Tile products of the dense operators (the gated feed-forward block and the 8-bit products):
// global -> LDS copies with bounds, MFMA operand reads, and the block forms built of them.
//
//   C[r, c] = sum_k A(r, k) B(c, k),  r < rows, c < cols, k < K
//
// An operand is stored either with its contraction contiguous (KC: x W^T has both so) or with
// the contraction as its row index (KR: the gradients' products dy W and dy^T x read their
// operands "down" the rows).  A k-tile is 128 bytes of contraction per operand row: 64 bf16, 128
// int8 or 32 fp32; a unit is one operand's share of a k-tile, TR rows x 128 bytes whatever the
// layout (KR: 128 / SZ contraction rows of TR elements).
#pragma once

#include "common.h"
#include "forms.h"

namespace elb {

namespace {

enum Lay { KC = 0, KR = 1 };

// ---- element types: the MFMA shape and its operand and accumulator registers ----
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef int32_t i32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <class E, int MF>
struct Mma;
struct Bf16 {
    static constexpr int SZ = 2;
    typedef bf16x8_t frag;
    typedef float acc1;
};
struct I8 {
    static constexpr int SZ = 1;
    typedef i32x4_t frag;
    typedef int32_t acc1;
};
struct F32 {
    static constexpr int SZ = 4;
    typedef f32x4_t frag;
    typedef float acc1;
};
// The first MFMA operand is the one whose rows become output COLUMNS: a lane then holds four
// consecutive output columns per group of four accumulators.
template <>
struct Mma<Bf16, 32> {
    typedef f32x16_t acc;
    static __device__ __forceinline__ acc mma(bf16x8_t b, bf16x8_t a, acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
    }
};
template <>
struct Mma<Bf16, 16> {
    typedef f32x4_t acc;
    static __device__ __forceinline__ acc mma(bf16x8_t b, bf16x8_t a, acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
    }
};
template <>
struct Mma<I8, 32> {
    typedef i32x16_t acc;
    static __device__ __forceinline__ acc mma(i32x4_t b, i32x4_t a, acc c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(b, a, c, 0, 0, 0);
    }
};
template <>
struct Mma<I8, 16> {
    typedef i32x4_t acc;
    static __device__ __forceinline__ acc mma(i32x4_t b, i32x4_t a, acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(b, a, c, 0, 0, 0);
    }
};
template <>
struct Mma<F32, 16> {  // four k of one row per operand: a permutation both operands share
    typedef f32x4_t acc;
    static __device__ __forceinline__ acc mma(f32x4_t b, f32x4_t a, acc c) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[q], a[q], c, 0, 0, 0);
        return c;
    }
};

// ---- LDS layouts ----
// KC unit: TR rows of 128 bytes, the eight 16-byte chunks of row r XOR-swizzled so that 16
// consecutive rows' reads of one logical chunk hit distinct banks.
__device__ __forceinline__ int kc_swz(int r, int c) {
    return c ^ (((r >> 1) ^ ((r & 1) << 2)) & 7);
}
// KR unit: 128 / SZ rows of TR elements.  bf16: granules of 16 columns (32 bytes), swizzled so
// that what 32 lanes of a transposing read touch lies in distinct banks, four rows x two granules
// (MFMAs of 32) or two times four rows, eight apart, of one granule (of 16); fp32: granules of 16
// columns (64 bytes), four rows apart in distinct banks.  Returns the XOR on the 16-byte chunk of
// row k.
template <int TR, int SZ>
__device__ __forceinline__ int kr_swz(int k) {
    if (SZ == 4) return TR >= 64 ? ((k >> 2) & 3) << 2 : 0;
    const int far = ((k >> 3) & 1) << 1;
    return TR >= 128 ? (k & 3) << 2 | far : TR == 64 ? ((k >> 1) & 1) << 2 | far
           : TR == 32 ? far : 0;
}

// ---- global -> LDS copies ----
// 16 bytes from global memory at any byte boundary
typedef uint32_t u32x4_byte_t __attribute__((ext_vector_type(4), aligned(1)));

// the same value in every lane, in a scalar register
__device__ __forceinline__ uint32_t uniform(uint32_t v) {
    return __builtin_amdgcn_readfirstlane(v);
}

constexpr uint32_t kOutOfBounds = 0x7fffff00u;  // past every buffer: spans stay below 2^31 - 512

// One wave's share of a unit's copies: NW waves copy TR rows, 1 KB per instruction
// (buffer_load_dwordx4 ... lds).  The buffer's bound is set per unit, so lanes past the operand's
// last row, column or contraction index write zeros to LDS: tails need no clamping, and nothing
// they read is out of the tensor.  PAIR (KC): rows [0, TR / 2) and [TR / 2, TR) of the unit come
// from two places (gate rows and the matching up rows).  DMA = false: ordinary loads, for tensors
// off a 16-byte boundary.
template <int LAY, int TR, int SZ, int NW, bool PAIR, bool DMA>
struct Copier {
    static constexpr int N = TR / 8 / NW;  // copy instructions per unit
    static constexpr int NB = (PAIR && NW == 1) ? 2 : 1;
    static constexpr int KT = 128 / SZ;    // contraction depth of a k-tile
    static constexpr int P = TR * SZ;      // KR: bytes of a contraction row in LDS
    static_assert(TR % (8 * NW) == 0 && !(PAIR && LAY == KR) && !(PAIR && NW == 1 && N % 2), "");
    const char* base[NB];
    uint32_t off[N];
    int kchunk[2];   // KC: byte offset in the k-tile of copies i and i + 1 (i even)
    int64_t ld;      // bytes between the operand's rows
    int64_t span;    // KC: bytes of the tile's rows; KR: bytes of the tile's columns
    int64_t klen;    // KC: bytes of contraction; KR: contraction rows

    // p0: the tile's first row (KC) or column (KR) at contraction 0; p1: with PAIR its first row
    // of the second half; ext: valid rows or columns from there on (of each half with PAIR)
    __device__ __forceinline__ void init(const void* p0, const void* p1, int64_t ld_, int ext,
                                         int64_t K, int lane, int w) {
        ld = ld_;
        constexpr int HR = PAIR ? TR / 2 : TR;
        if (LAY == KC) {
            span = (int64_t)(ext < HR ? ext : HR) * ld_;
            klen = K * SZ;
        } else {
            span = (int64_t)(ext < TR ? ext : TR) * SZ;
            klen = ext > 0 ? K : 0;  // a tile past the last column reads nothing
        }
        base[0] = (const char*)(PAIR && NB == 1 && w >= NW / 2 ? p1 : p0);
        if (NB == 2) base[NB - 1] = (const char*)p1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (LAY == KC) {
                int r = 8 * (w * N + i) + (lane >> 3);
                if (i < 2) kchunk[i] = kc_swz(r, lane & 7) * 16;
                if (PAIR) r = r >= HR ? r - HR : r;
                off[i] = (uint32_t)r * (uint32_t)ld_ + kchunk[i & 1];
            } else {
                constexpr int LPR = P / 16;  // lanes per contraction row
                const int k = (w * N + i) * (64 / LPR) + lane / LPR;
                off[i] = (uint32_t)k * (uint32_t)ld_ + ((lane % LPR) ^ kr_swz<TR, SZ>(k)) * 16;
            }
        }
        if (LAY == KC && N == 1) kchunk[1] = kchunk[0];
    }
    // a k-tile's buffer bounds
    struct Unit {
        u32x4_t rs[NB];
        int64_t at, rec, left;
    };
    // k-tile t; past tend nothing is read (zeros are written), so that the count of copies in
    // flight is the same
    __device__ __forceinline__ Unit unit(int t, int tend) const {
        Unit u;
        if (LAY == KC) {
            u.at = (int64_t)t * 128;
            u.rec = span - u.at;
            u.left = klen - u.at;
        } else {
            u.at = (int64_t)t * KT * ld;
            u.left = klen - (int64_t)t * KT;
            u.rec = u.left <= 0 ? 0 : ((u.left < KT ? u.left : KT) - 1) * ld + span;
        }
        if (t >= tend || u.rec < 0) u.rec = 0;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint64_t p = (uint64_t)(base[b] + u.at);
            u.rs[b] = u32x4_t{uniform((uint32_t)p), uniform((uint32_t)(p >> 32)) & 0xffffu,
                              uniform((uint32_t)u.rec), 0x00027000u};
        }
        return u;
    }
    // copy instruction i of the unit at LDS byte address lds (ldsp: the same as a pointer)
    __device__ __forceinline__ void one(const Unit& u, int i, uint32_t lds, char* ldsp, int lane,
                                        int w) const {
        const int b = (NB == 2 && i >= N / 2) ? NB - 1 : 0;
        uint32_t vo = off[i];
        if (LAY == KC && u.left < 128) vo = kchunk[i & 1] < u.left ? vo : kOutOfBounds;
        if constexpr (DMA) {
            const uint32_t la = lds + (uint32_t)(w * N + i) * 1024;
            // inline assembly: the compiler cannot tell which unit a copy writes, and would wait
            // for every copy in flight before each LDS read; waits are explicit
            asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                         :: "s"(la), "v"(vo), "s"(u.rs[b]) : "memory", "m0");
        } else {
            u32x4_t v = {0, 0, 0, 0};
            if ((int64_t)vo < u.rec)
                v = *reinterpret_cast<const u32x4_byte_t*>(base[b] + u.at + vo);
            *reinterpret_cast<u32x4_t*>(ldsp + (w * N + i) * 1024 + lane * 16) = v;
        }
    }
    __device__ __forceinline__ void issue(int t, int tend, uint32_t lds, char* ldsp, int lane,
                                          int w) const {
        const Unit u = unit(t, tend);
#pragma unroll
        for (int i = 0; i < N; ++i) one(u, i, lds, ldsp, lane, w);
    }
};

// ---- MFMA operand reads ----
// Fragment i of MF rows at row0 + MF i of the unit, k-step ks (of 64 / MF) of the k-tile.
template <class E, int MF, int LAY, int TR>
struct Reader {
    static constexpr int P = TR * E::SZ;
    static constexpr int KS = MF / 8;   // k-steps of a k-tile
    static constexpr int KD = 512 / MF; // KR, bf16: contraction rows of a k-step
    int at, ofs[LAY == KC ? KS : 1];
    int row;
    __device__ __forceinline__ void init(int row0, int lane) {
        const int l = lane & (MF - 1), g = lane / MF;
        row = row0;
        if (LAY == KC) {
            at = (row0 + l) * 128;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                ofs[ks] = kc_swz(l, ks * (64 / MF) + g) * 16;
        } else if (E::SZ == 2) {
            // transposing reads: the 16 lanes of a group bring four contraction rows of 16
            // columns, and lane j of the group receives column j
            const int p = lane & 15;
            const int kh = MF == 32 ? (lane >> 5) : (lane >> 4);
            at = (8 * kh + (p >> 2)) * P + (p & 3) * 8;
            ofs[0] = (kr_swz<TR, 2>(8 * kh + (p >> 2)) * 16) ^ (MF == 32 ? ((lane >> 4) & 1) * 32 : 0);
        } else {
            at = 4 * g * P + l * 4;
            ofs[0] = kr_swz<TR, 4>(4 * g) * 16;
        }
    }
    __device__ __forceinline__ typename E::frag load(const char* unit, int i, int ks) const {
        typename E::frag v;
        if constexpr (LAY == KC) {
            v = *reinterpret_cast<const typename E::frag*>(unit + at + i * MF * 128 + ofs[ks]);
        } else if constexpr (E::SZ == 2) {
            const int c = ((row + MF * i) * 2) ^ ofs[0];
            const char* const q = unit + at + c + ks * KD * P;
            typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
            const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
            const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q + 4 * P));
            v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const char* const q = unit + at + (((row + MF * i) * 4) ^ ofs[0]) + ks * 16 * P;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = *reinterpret_cast<const float*>(q + c * P);
        }
        return v;
    }
};

// ---- results: eight consecutive columns of a row at a time ----
__device__ __forceinline__ void read8(const char* p, float (&v)[8], float) {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p);
    const f32x4_t b = *reinterpret_cast<const f32x4_t*>(p + 16);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = a[q], v[q + 4] = b[q];
}
__device__ __forceinline__ void read8(const char* p, float (&v)[8], int32_t) {
    const i32x4_t a = *reinterpret_cast<const i32x4_t*>(p);
    const i32x4_t b = *reinterpret_cast<const i32x4_t*>(p + 16);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = (float)a[q], v[q + 4] = (float)b[q];
}

typedef __bf16 bf16x2_pk_t __attribute__((ext_vector_type(2)));
typedef float f32x2_pk_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const f32x2_pk_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_pk_t));
}
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
// eight values from / to a tensor at any element boundary, rounded once to its type
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
    const u32x4_any_t a = *reinterpret_cast<const u32x4_any_t*>(p);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v[2 * q] = __uint_as_float(a[q] << 16);
        v[2 * q + 1] = __uint_as_float(a[q] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const f32x4_any_t a = *reinterpret_cast<const f32x4_any_t*>(p);
    const f32x4_any_t b = *reinterpret_cast<const f32x4_any_t*>(p + 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = a[q], v[q + 4] = b[q];
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
    const u32x4_any_t a = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]),
                           pack2(v[6], v[7])};
    *reinterpret_cast<u32x4_any_t*>(p) = a;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<f32x4_any_t*>(p) = f32x4_any_t{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any_t*>(p + 4) = f32x4_any_t{v[4], v[5], v[6], v[7]};
}

// One tile's operands: A has the rows, B the columns of the result; b2: the second half's first
// row with PAIR.  rows, cols: valid ones from the tile's first on (PAIR: output columns, half of
// the tile's B rows); k-tiles [t0, t1).
struct TileIn {
    const char *a, *b, *b2;
    int64_t lda, ldb;
    int rows, cols;
    int64_t K;
    int t0, t1;
    char* part;       // TurnForm with HALVES: the tile's two partial results,
    uint32_t* count;  // the number of them that are written,
    int half;         // and the one that is this block's
};

// ------------------------------------------------------------------------------------------
// Block form 1: a TM x TN tile by four waves (WM x WN), operands in a ring of S k-tiles.  At the
// barrier that opens k-tile t every wave has read tile t - 1, whose units then receive tile
// t + S - 1.
// ------------------------------------------------------------------------------------------
template <class E, int MF, int TM, int TN, int WM, int LA, int LB, bool PAIR, bool DMA, int S>
struct TileForm {
    static constexpr int WN = 4 / WM;
    static constexpr int WTM = TM / WM, WTN = TN / WN;  // a wave's rows and columns
    static constexpr int FM = WTM / MF, FN = WTN / MF;
    static constexpr int HJ = PAIR ? FN / 2 : FN;       // PAIR: the gate rows' fragments
    static constexpr int AU = TM * 128, BU = TN * 128;  // bytes of a unit
    static constexpr int RING = S * (AU + BU);
    static constexpr int PITCH = WTN * 4 + 16;          // bytes per staged row
    static constexpr int STAGE = MF * PITCH;            // a wave's staging area
    static constexpr int LDS = RING > 4 * STAGE ? RING : 4 * STAGE;
    static_assert(WTM % MF == 0 && WTN % MF == 0 && (!PAIR || FN % 2 == 0), "");
    typedef typename Mma<E, MF>::acc acc_t;
    typedef Copier<LA, TM, E::SZ, 4, false, DMA> CA;
    typedef Copier<LB, TN, E::SZ, 4, PAIR, DMA> CB;

    template <class Epi>
    static __device__ __forceinline__ void run(const TileIn& in, char* sm, const Epi& epi) {
        const int lane = threadIdx.x & 63;
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = w / WN, wn = w % WN;
        CA ca;
        CB cb;
        ca.init(in.a, nullptr, in.lda, in.rows, in.K, lane, w);
        cb.init(in.b, in.b2, in.ldb, in.cols, in.K, lane, w);
        Reader<E, MF, LA, TM> ra;
        Reader<E, MF, LB, TN> rb;
        ra.init(wm * WTM, lane);
        rb.init(PAIR ? wn * (WTN / 2) : wn * WTN, lane);
        const uint32_t lds = __builtin_amdgcn_readfirstlane(
            (uint32_t)(uintptr_t)(lds_void_t*)sm);
        acc_t acc[FM][FN];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = acc_t{};
        auto issue = [&](int t, int u) {
            ca.issue(t, in.t1, lds + u * (AU + BU), sm + u * (AU + BU), lane, w);
            cb.issue(t, in.t1, lds + u * (AU + BU) + AU, sm + u * (AU + BU) + AU, lane, w);
        };
#pragma unroll
        for (int p = 0; p < S - 1; ++p) issue(in.t0 + p, p);
        int u = 0;
        for (int t = in.t0; t < in.t1; ++t) {
            ELB_WAIT_VMCNT((S - 2) * (CA::N + CB::N));
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            issue(t + S - 1, u == 0 ? S - 1 : u - 1);
            const char* const pa = sm + u * (AU + BU);
            const char* const pb = pa + AU;
#pragma unroll
            for (int ks = 0; ks < MF / 8; ++ks) {
                typename E::frag fa[FM], fb[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    fb[j] = rb.load(pb + (j >= HJ ? BU / 2 : 0), j % HJ, ks);
#pragma unroll
                for (int i = 0; i < FM; ++i) fa[i] = ra.load(pa, i, ks);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = Mma<E, MF>::mma(fb[j], fa[i], acc[i][j]);
            }
            u = u + 1 == S ? 0 : u + 1;
        }
        // results through LDS, each wave in its own area: MF rows at a time
        ELB_WAIT_VMCNT(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        results<Epi>(acc, in, sm + w * STAGE, lane, wm, wn, epi);
    }

    template <class Epi>
    static __device__ __forceinline__ void results(const acc_t (&acc)[FM][FN], const TileIn& in,
                                                   char* stg, int lane, int wm, int wn,
                                                   const Epi& epi) {
        typedef typename E::acc1 a1;
        typedef a1 a4 __attribute__((ext_vector_type(4)));
        constexpr int OC = PAIR ? WTN / 2 : WTN;  // output columns of the wave
        constexpr int CPR = OC / 8, RPI = 64 / CPR;
        const int l = lane & (MF - 1), g = lane / MF;
        const int cc = lane % CPR, r0 = lane / CPR;
        const int col = wn * OC + cc * 8;
        constexpr int NP = (MF + RPI - 1) / RPI;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            typename Epi::Extra extra[NP];
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int r = r0 + p * RPI, row = wm * WTM + i * MF + r;
                if ((RPI <= MF || r < MF) && row < in.rows && col < in.cols)
                    epi.fetch(row, col, extra[p]);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < MF * MF / 256; ++q) {
                    const a4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                                  acc[i][j][4 * q + 3]};
                    const int c = j * MF + (MF == 32 ? 8 * q + 4 * g : 4 * g);
                    *reinterpret_cast<a4*>(stg + l * PITCH + c * 4) = v;
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int r = r0 + p * RPI, row = wm * WTM + i * MF + r;
                if ((RPI > MF && r >= MF) || row >= in.rows || col >= in.cols) continue;
                float v[8];
                read8(stg + r * PITCH + cc * 32, v, a1{});
                if constexpr (PAIR) {
                    float v2[8];
                    read8(stg + r * PITCH + (OC + cc * 8) * 4, v2, a1{});
                    epi.put(row, col, v, v2, extra[p]);
                } else {
                    epi.put(row, col, v, extra[p]);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// The end of a split form: the waves' partial TM x TN tiles, summed in LDS in the order of the
// contraction.
template <class E, int TM, int TN, int NW, bool PAIR>
struct SplitJoin {
    static constexpr int FM = TM / 16, FN = TN / 16;
    static constexpr int PITCH = TN * 4 + 16;
    static constexpr int PART = TM * PITCH;  // a wave's partial tile
    typedef typename Mma<E, 16>::acc acc_t;

    template <class Epi>
    static __device__ __forceinline__ void run(const acc_t (&acc)[FM][FN], const TileIn& in,
                                               char* sm, int lane, int w, const Epi& epi) {
        typedef typename E::acc1 a1;
        typedef a1 a4 __attribute__((ext_vector_type(4)));
        ELB_WAIT_VMCNT(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const int l16 = lane & 15, hq = lane >> 4;
        char* const part = sm + w * PART;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
                *reinterpret_cast<a4*>(part + (16 * i + l16) * PITCH + (16 * j + 4 * hq) * 4) =
                    acc[i][j];
        __syncthreads();
        constexpr int OC = PAIR ? TN / 2 : TN;
        constexpr int CPR = OC / 8, ITEMS = TM * CPR;
        for (int it = threadIdx.x; it < ITEMS; it += NW * 64) {
            const int row = it / CPR, cc = it % CPR;
            if (row >= in.rows || cc * 8 >= in.cols) continue;
            typename Epi::Extra extra;
            epi.fetch(row, cc * 8, extra);
            float v[8], v2[8];
            sum8<a1>(sm + row * PITCH + cc * 32, v);
            if constexpr (PAIR) {
                sum8<a1>(sm + row * PITCH + (OC + cc * 8) * 4, v2);
                epi.put(row, cc * 8, v, v2, extra);
            } else {
                epi.put(row, cc * 8, v, extra);
            }
        }
    }
    template <class a1>
    static __device__ __forceinline__ void sum8(const char* p, float (&v)[8]) {
        typedef a1 a4 __attribute__((ext_vector_type(4)));
        a4 a = *reinterpret_cast<const a4*>(p), b = *reinterpret_cast<const a4*>(p + 16);
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            a += *reinterpret_cast<const a4*>(p + w * PART);
            b += *reinterpret_cast<const a4*>(p + w * PART + 16);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (float)a[q], v[q + 4] = (float)b[q];
    }
};

// ------------------------------------------------------------------------------------------
// Block form 2, for few rows: NW waves take a share of the contraction each, every one of them
// the whole TM x TN tile, with a ring of S k-tiles of its own and no barrier in the loop; their
// partial tiles are then summed in LDS in the order of the contraction.
// ------------------------------------------------------------------------------------------
template <class E, int TM, int TN, int NW, int LA, int LB, bool PAIR, int S>
struct SplitForm {
    static constexpr int MF = 16;
    static constexpr int FM = TM / 16, FN = TN / 16;
    static constexpr int AU = TM * 128, BU = TN * 128;
    static constexpr int WRING = S * (AU + BU);  // a wave's ring
    static constexpr int PART = SplitJoin<E, TM, TN, NW, PAIR>::PART;
    static constexpr int LDS = NW * (WRING > PART ? WRING : PART);
    typedef typename Mma<E, 16>::acc acc_t;
    typedef Copier<LA, TM, E::SZ, 1, false, true> CA;
    typedef Copier<LB, TN, E::SZ, 1, PAIR, true> CB;

    template <class Epi>
    static __device__ __forceinline__ void run(const TileIn& in, char* sm, const Epi& epi) {
        const int lane = threadIdx.x & 63;
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        CA ca;
        CB cb;
        ca.init(in.a, nullptr, in.lda, in.rows, in.K, lane, 0);
        cb.init(in.b, in.b2, in.ldb, in.cols, in.K, lane, 0);
        Reader<E, 16, LA, TM> ra;
        Reader<E, 16, LB, TN> rb;
        ra.init(0, lane);
        rb.init(0, lane);
        char* const ring = sm + w * WRING;
        const uint32_t lds = __builtin_amdgcn_readfirstlane(
            (uint32_t)(uintptr_t)(lds_void_t*)sm + (uint32_t)w * WRING);
        acc_t acc[FM][FN];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = acc_t{};
        const int nt = in.t1 - in.t0;
        const int t0 = in.t0 + nt * w / NW, t1 = in.t0 + nt * (w + 1) / NW;
        auto issue = [&](int t, int u) {
            ca.issue(t, t1, lds + u * (AU + BU), ring + u * (AU + BU), lane, 0);
            cb.issue(t, t1, lds + u * (AU + BU) + AU, ring + u * (AU + BU) + AU, lane, 0);
        };
#pragma unroll
        for (int p = 0; p < S; ++p) issue(t0 + p, p);
        int u = 0;
        for (int t = t0; t < t1; ++t) {
            ELB_WAIT_VMCNT((S - 1) * (CA::N + CB::N));
            asm volatile("" ::: "memory");
            const char* const pa = ring + u * (AU + BU);
            const char* const pb = pa + AU;
            typename E::frag fa[2][FM], fb[2][FN];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[ks][j] = rb.load(pb, j, ks);
#pragma unroll
                for (int i = 0; i < FM; ++i) fa[ks][i] = ra.load(pa, i, ks);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the units are free again
            issue(t + S, u);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = Mma<E, 16>::mma(fb[ks][j], fa[ks][i], acc[i][j]);
            u = u + 1 == S ? 0 : u + 1;
        }
        SplitJoin<E, TM, TN, NW, PAIR>::run(acc, in, sm, lane, w, epi);
    }
};

// ------------------------------------------------------------------------------------------
// Block form 3, for many rows: a TM x TN tile by eight waves, two on each SIMD, that take turns:
// while the waves 0 .. 3 feed themselves (LDS reads, copies), the waves 4 .. 7 keep the matrix
// units busy, and the other way round.  The tile is four quadrants (row half x column half) of
// QM x QN; a wave owns the same QM / WM x QN / WN piece of each.  A k-tile is then four phases, each
// a quadrant:
//     phase   LDS reads           copies issued       matrix products
//       0     A0 (tile t)         A1 (tile t + 1)     A0 BF
//       1     BG                  A0 (tile t + 2)     A0 BG
//       2     A1                  BF (tile t + 2)     A1 BG
//       3     BG (tile t + 1)     BG (tile t + 2)     A1 BF
// AHEAD, where A's contraction is contiguous: F is 0 in even k-tiles and 1 in odd ones, G = 1 - F, so
// that the half of B that a k-tile starts with is read in phase 3 before, where its registers
// have just become free.  Otherwise F is always 0, and phase 0 reads BF too, phase 3 nothing (us,
// otherwise / AHEAD: gate and up of 4096 tokens, m = 8192 250 / 244, their down product 127 / 121;
// both weight gradients, which read A and B down the rows with twice the instructions, 332 / 357).
// Each half of a phase (reads and copies; products) ends with a barrier of all waves; the second
// group starts one half later.  A unit is overwritten (by the copies of two k-tiles later, two
// buffers) at the earliest two halves after its last read by the first group, one after that by
// the second, whose reads are waited for before its barrier.  Every unit is copied five to seven
// phases before its first read; the waits leave what is not needed yet in flight.  Copies are
// issued, and arrive, in the order ... A0, BF, BG (tile t + 1; phases 1, 2, 3 of tile t - 1), A1
// (phase 0 of tile t), A0, BF, BG (t + 2) ...  Phase 1 waits for A1 of tile t (five units are later);
// AHEAD, phase 0 for BG of tile t (five), phase 2 for the first half of B of tile t + 1, and with
// it its A0 (four); otherwise phase 3 for A0, BF and BG of tile t + 1 (four).
// HALVES: two blocks share a tile, each with half of the contraction (two halves of 128 tiles fill the
// chip where one block each would leave half of it idle; of 320 tiles, 640 blocks fill two and a half
// rounds of half the length where whole tiles take two).  The block that finds its partner's
// partial result written adds it to its own and finishes the tile; one that does not writes its
// own.  Neither waits: where both come at once both write, and the second one to count goes on.  A sum
// of two does not depend on its order.
//
// The 16 x 16 MFMAs run it faster than the 32 x 32 ones of the same rate (us, 32 / 16: 4096 x 16384 x
// 2048 with SwiGLU 227 / 211, 8192 x 4096 x 8192 442 / 403, int8 of twice the depth 456 / 410).
// ------------------------------------------------------------------------------------------
template <int V>
struct Half {
    static constexpr int value = V;
};
template <class E, int TM, int TN, int WM, int LA, int LB, bool PAIR, bool HALVES = false>
struct TurnForm {
    static constexpr int MF = 16, KS = 2;  // MFMA rows and columns, k-steps of a k-tile
    static constexpr bool AHEAD = LA == KC;
    static constexpr int WN = 8 / WM;
    static constexpr int QM = TM / 2, QN = TN / 2;
    static constexpr int PM = QM / WM, PN = QN / WN;  // a wave's piece of a quadrant
    static constexpr int FM = PM / MF, FN = PN / MF;
    static constexpr int AU = QM * 128, BU = QN * 128, BUF = 2 * (AU + BU);
    static constexpr int PITCH = 2 * PN * 4 + 16, STAGE = 32 * PITCH;
    static constexpr int LDS = 2 * BUF > 8 * STAGE ? 2 * BUF : 8 * STAGE;
    static_assert(FM * MF * WM == QM && FN * MF * WN == QN, "");
    typedef typename Mma<E, MF>::acc acc_t;
    typedef Copier<LA, QM, E::SZ, 8, false, true> CA;
    typedef Copier<LB, QN, E::SZ, 8, false, true> CB;

    template <class Epi>
    static __device__ __forceinline__ void run(const TileIn& in, char* sm, const Epi& epi) {
        const int lane = threadIdx.x & 63;
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = w / WN, wn = w % WN;
        const bool second = w >= 4;
        CA ca[2];
        CB cb[2];
        ca[0].init(in.a, nullptr, in.lda, in.rows, in.K, lane, w);
        ca[1].init(in.a + QM * (LA == KC ? in.lda : E::SZ), nullptr, in.lda,
                   in.rows > QM ? in.rows - QM : 0, in.K, lane, w);
        cb[0].init(in.b, nullptr, in.ldb, in.cols, in.K, lane, w);
        cb[1].init(PAIR ? in.b2 : in.b + QN * (LB == KC ? in.ldb : E::SZ), nullptr, in.ldb,
                   PAIR ? in.cols : in.cols > QN ? in.cols - QN : 0, in.K, lane, w);
        Reader<E, MF, LA, QM> ra;
        Reader<E, MF, LB, QN> rb;
        ra.init(wm * PM, lane);
        rb.init(wn * PN, lane);
        const uint32_t lds = __builtin_amdgcn_readfirstlane(
            (uint32_t)(uintptr_t)(lds_void_t*)sm);
        acc_t acc[2][2][FM][FN];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[a][b][i][j] = acc_t{};
        auto copy_a = [&](int h, int t) {
            const int at = ((t - in.t0) & 1) * BUF + h * AU;
            ca[h].issue(t, in.t1, lds + at, sm + at, lane, w);
        };
        auto copy_b = [&](int h, int t) {
            const int at = ((t - in.t0) & 1) * BUF + 2 * AU + h * BU;
            cb[h].issue(t, in.t1, lds + at, sm + at, lane, w);
        };
        typename E::frag fa[FM][KS], fb[2][FN][KS];
        auto read_a = [&](const char* unit) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < FM; ++i) fa[i][k] = ra.load(unit, i, k);
        };
        auto read_b = [&](const char* unit, int h) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[h][j][k] = rb.load(unit, j, k);
        };
        auto half = [&]() {  // the end of a half phase
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto products = [&](int a, int b) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[a][b][i][j] =
                            Mma<E, MF>::mma(fb[b][j][k], fa[i][k], acc[a][b][i][j]);
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };

        const int t0 = in.t0;
        auto buffer = [&](int t) { return sm + ((t - t0) & 1) * BUF; };
        auto tile = [&](int t, auto first) {
            constexpr int F = decltype(first)::value, G = 1 - F;
            const char* const buf = buffer(t);
            if (!AHEAD) read_b(buf + 2 * AU, F);
            read_a(buf);
            copy_a(1, t + 1);
            if (AHEAD) ELB_WAIT_VMCNT(3 * CA::N + 2 * CB::N);
            half();
            products(0, F);
            read_b(buf + 2 * AU + G * BU, G);
            copy_a(0, t + 2);
            ELB_WAIT_VMCNT(3 * CA::N + 2 * CB::N);
            half();
            products(0, G);
            read_a(buf + AU);
            copy_b(F, t + 2);
            if (AHEAD) ELB_WAIT_VMCNT(2 * CA::N + 2 * CB::N);
            half();
            products(1, G);
            if (AHEAD) read_b(buffer(t + 1) + 2 * AU + G * BU, G);
            copy_b(G, t + 2);
            if (!AHEAD) ELB_WAIT_VMCNT(2 * CA::N + 2 * CB::N);
            half();
            products(1, F);
        };
        copy_a(0, t0);
        copy_b(0, t0);
        copy_b(1, t0);
        copy_a(1, t0);
        copy_a(0, t0 + 1);
        copy_b(AHEAD, t0 + 1);
        copy_b(!AHEAD, t0 + 1);
        ELB_WAIT_VMCNT(2 * CA::N + 2 * CB::N);
        half();
        if (AHEAD) read_b(buffer(t0) + 2 * AU, 0);
        if (second) asm volatile("s_barrier" ::: "memory");
        for (int t = t0; t < in.t1; t += 2) {
            tile(t, Half<0>());
            if (t + 1 < in.t1) tile(t + 1, Half<AHEAD ? 1 : 0>());
        }
        if (!second) asm volatile("s_barrier" ::: "memory");
        ELB_WAIT_VMCNT(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

        typedef typename E::acc1 a1;
        typedef a1 a4 __attribute__((ext_vector_type(4)));
        if constexpr (HALVES) {
            static_assert(8 * STAGE + 4 <= LDS, "the flag beside the staging areas");
            constexpr int NV = 4 * FM * FN;  // 16-byte pieces of a lane's results
            uint32_t* const flag = reinterpret_cast<uint32_t*>(sm + LDS - 4);
            auto piece = [&](int half, int i) {
                return reinterpret_cast<a4*>(in.part + half * (TM * TN * 4)) +
                       ((w * NV + i) * 64 + lane);
            };
            if (threadIdx.x == 0)
                *flag = __hip_atomic_load(in.count, __ATOMIC_ACQUIRE, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (*flag == 0) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const acc_t& c = acc[i / (2 * FM * FN)][i / (FM * FN) % 2][i / FN % FM][i % FN];
                    *piece(in.half, i) = c;
                    if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
                }
                // every wave's stores have reached L2 before the barrier; then one wave's release
                // (which writes L2 back) covers them all (by all eight waves: 35 us more)
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0)
                    *flag = __hip_atomic_fetch_add(in.count, 1u, __ATOMIC_ACQ_REL,
                                                   __HIP_MEMORY_SCOPE_AGENT);
                __syncthreads();
                if (*flag == 0) return;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                acc[i / (2 * FM * FN)][i / (FM * FN) % 2][i / FN % FM][i % FN] +=
                    *piece(1 - in.half, i);
                // eight loads at a time: all of them at once have no registers
                if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
            }
        }

        // results through LDS, each wave in its own area: 32 rows of a row half at a time
        char* const stg = sm + w * STAGE;
        constexpr int HC = PN / 8;                    // 8-column chunks of a column half
        constexpr int CPR = PAIR ? HC : 2 * HC, RPI = 64 / CPR;
        const int l = lane & (MF - 1), g = lane / MF;
        const int cc = lane % CPR, r0 = lane / CPR;
        const int col = (cc / HC) * QN + wn * PN + (cc % HC) * 8;
        constexpr int NP = 32 / RPI;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < PM / 32; ++i) {
                typename Epi::Extra extra[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int row = a * QM + wm * PM + i * 32 + r0 + p * RPI;
                    if (row < in.rows && col < in.cols) epi.fetch(row, col, extra[p]);
                }
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < FN; ++j)
                            *reinterpret_cast<a4*>(stg + (h * 16 + l) * PITCH +
                                                   (b * PN + j * 16 + 4 * g) * 4) =
                                acc[a][b][2 * i + h][j];
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int r = r0 + p * RPI, row = a * QM + wm * PM + i * 32 + r;
                    if (row >= in.rows || col >= in.cols) continue;
                    float v[8];
                    read8(stg + r * PITCH + cc * 32, v, a1{});
                    if constexpr (PAIR) {
                        float v2[8];
                        read8(stg + r * PITCH + (PN + cc * 8) * 4, v2, a1{});
                        epi.put(row, col, v, v2, extra[p]);
                    } else {
                        epi.put(row, col, v, extra[p]);
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
    }
};

// ------------------------------------------------------------------------------------------
// Block form 4, for tiles that are few (one round over the chip): a 128 x 128 tile by two groups of
// four waves (2 x 2 of 64 x 64) that take the k-tiles in turn, one group the even, the other the
// odd ones, so that a compute unit has two waves per SIMD without a second tile.  A group
// reads a whole k-tile into registers while the other one multiplies, and the other way round
// (barriers of all waves between the halves, the second group one half behind).  A group's
// k-tile i + 2 is copied over k-tile i as soon as its waves have read that.  The two partial tiles
// are added in LDS, each group finishing one half of every wave's rows.
// ------------------------------------------------------------------------------------------
template <class E, int LA, int LB, bool PAIR>
struct PairForm {
    static constexpr int TM = 128, TN = 128;
    static constexpr int AU = TM * 128, BU = TN * 128, BUF = AU + BU;
    static constexpr int PITCH = 64 * 4 + 16, STAGE = 32 * PITCH;
    static constexpr int LDS = 16 * STAGE > 4 * BUF ? 16 * STAGE : 4 * BUF;
    typedef typename Mma<E, 32>::acc acc_t;
    typedef Copier<LA, TM, E::SZ, 4, false, true> CA;
    typedef Copier<LB, TN, E::SZ, 4, PAIR, true> CB;

    template <class Epi>
    static __device__ __forceinline__ void run(const TileIn& in, char* sm, const Epi& epi) {
        typedef typename E::acc1 a1;
        typedef a1 a4 __attribute__((ext_vector_type(4)));
        const int lane = threadIdx.x & 63;
        const int w8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int grp = w8 >> 2, w = w8 & 3;
        const int wm = w >> 1, wn = w & 1;
        CA ca;
        CB cb;
        ca.init(in.a, nullptr, in.lda, in.rows, in.K, lane, w);
        cb.init(in.b, in.b2, in.ldb, in.cols, in.K, lane, w);
        Reader<E, 32, LA, TM> ra;
        Reader<E, 32, LB, TN> rb;
        ra.init(wm * 64, lane);
        rb.init(PAIR ? wn * 32 : wn * 64, lane);
        char* const ring = sm + grp * 2 * BUF;
        const uint32_t lds = __builtin_amdgcn_readfirstlane(
            (uint32_t)(uintptr_t)(lds_void_t*)sm + (uint32_t)(grp * 2 * BUF));
        acc_t acc[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = acc_t{};
        auto copy = [&](int i) {  // the group's i-th k-tile
            const int t = in.t0 + 2 * i + grp, at = (i & 1) * BUF;
            ca.issue(t, in.t1, lds + at, ring + at, lane, w);
            cb.issue(t, in.t1, lds + at + AU, ring + at + AU, lane, w);
        };
        const int n = (in.t1 - in.t0 + 1) / 2;  // of both groups; past the last one zeros
        copy(0);
        copy(1);
        ELB_WAIT_VMCNT(CA::N + CB::N);
        asm volatile("s_barrier" ::: "memory");
        if (grp) asm volatile("s_barrier" ::: "memory");
        for (int i = 0; i < n; ++i) {
            const char* const pa = ring + (i & 1) * BUF;
            const char* const pb = pa + AU;
            typename E::frag fa[2][4], fb[2][4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    fb[j][k] = PAIR ? rb.load(pb + j * (BU / 2), 0, k) : rb.load(pb, j, k);
                    fa[j][k] = ra.load(pa, j, k);
                }
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            const int t2 = in.t0 + 2 * (i + 2) + grp, at2 = (i & 1) * BUF;
            const auto ua = ca.unit(t2, in.t1);
            const auto ub = cb.unit(t2, in.t1);
            // a copy after every other product: one that cannot issue at once then holds up one
            // product, not all of them
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int a = 0; a < 2; ++a) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        acc[a][b] = Mma<E, 32>::mma(fb[b][k], fa[a][k], acc[a][b]);
                    __builtin_amdgcn_sched_barrier(0);
                    if (k < 2) ca.one(ua, 2 * k + a, lds + at2, ring + at2, lane, w);
                    else cb.one(ub, 2 * k + a - 4, lds + at2 + AU, ring + at2 + AU, lane, w);
                    __builtin_amdgcn_sched_barrier(0);
                }
            __builtin_amdgcn_s_setprio(0);
            ELB_WAIT_VMCNT(CA::N + CB::N);
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!grp) asm volatile("s_barrier" ::: "memory");
        ELB_WAIT_VMCNT(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

        // area a of wave w: its rows 32 a .. 32 a + 31, of group 0 and of group 1
        const int l = lane & 31, g = lane >> 5;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            char* const stg = sm + ((w * 2 + a) * 2 + grp) * STAGE + l * PITCH;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const acc_t& c = acc[a][b];
                    *reinterpret_cast<a4*>(stg + (b * 32 + 8 * q + 4 * g) * 4) =
                        a4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
                }
        }
        __syncthreads();
        constexpr int OC = PAIR ? 32 : 64, CPR = OC / 8, RPI = 64 / CPR;
        const int cc = lane % CPR, r0 = lane / CPR;
        const int col = wn * OC + cc * 8;
        const char* const stg = sm + (w * 2 + grp) * 2 * STAGE;
        typename Epi::Extra extra[32 / RPI];
#pragma unroll
        for (int p = 0; p < 32 / RPI; ++p) {
            const int row = wm * 64 + grp * 32 + r0 + p * RPI;
            if (row < in.rows && col < in.cols) epi.fetch(row, col, extra[p]);
        }
#pragma unroll
        for (int p = 0; p < 32 / RPI; ++p) {
            const int r = r0 + p * RPI, row = wm * 64 + grp * 32 + r;
            if (row >= in.rows || col >= in.cols) continue;
            float v[8];
            sum8<a1>(stg + r * PITCH + cc * 32, v);
            if constexpr (PAIR) {
                float v2[8];
                sum8<a1>(stg + r * PITCH + (32 + cc * 8) * 4, v2);
                epi.put(row, col, v, v2, extra[p]);
            } else {
                epi.put(row, col, v, extra[p]);
            }
        }
    }
    template <class a1>
    static __device__ __forceinline__ void sum8(const char* p, float (&v)[8]) {
        typedef a1 a4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const a4 s = *reinterpret_cast<const a4*>(p + 16 * h) +
                         *reinterpret_cast<const a4*>(p + STAGE + 16 * h);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[4 * h + q] = (float)s[q];
        }
    }
};

// ---- tiles over the chip ----
// Blocks go round-robin over the 8 XCDs, each with its own L2: XCD x takes a contiguous range of
// the tiles, which are numbered in groups of GM rows of tiles, down the rows first, so that the
// blocks resident on an XCD share a patch of rows and columns.
// The block's number; blocks of up to 512 threads in rows of 2^22, so that a launch dimension stays
// below 2^32 threads.
constexpr int kDenseRow = 1 << 22;
__device__ __forceinline__ uint32_t dense_block_number() {
    return blockIdx.y * (uint32_t)kDenseRow + blockIdx.x;
}
__device__ __forceinline__ bool dense_tile(uint32_t b, uint32_t mt, uint32_t nt, int& m, int& n) {
    constexpr uint32_t GM = 4;
    const uint32_t total = mt * nt;
    const uint32_t per = (total + 7) >> 3, s = b >> 3, L = (b & 7) * per + s;
    if (s >= per || L >= total) return false;
    const uint32_t span = GM * nt, g = L / span, r = L - g * span;
    const uint32_t gm = mt - g * GM < GM ? mt - g * GM : GM;
    n = (int)(r / gm);
    m = (int)(g * GM + r - n * gm);
    return true;
}

// A dense product: A [rows, K] (KC) or [K, rows] (KR), B [cols, K] or [K, cols]; PAIR: B is
// [2 cols, K], output column c of rows c and cols + c.
struct DenseIn {
    const char *a, *b;
    int64_t lda, ldb;  // bytes between rows in memory
    int64_t rows;
    int cols;
    int64_t K;
    char* part;       // scratch for kHalves (halves_bytes), or null
    uint32_t* clear;  // counters of a later product in this call, set to zero here
    int nclear;
};

__device__ __forceinline__ void clear_counters(uint32_t* c, int n) {
    if (c && dense_block_number() == 0)
        for (int i = threadIdx.x; i < n; i += blockDim.x) c[i] = 0;
}

template <class Form, class E, int TM, int TN, int LA, int LB, bool PAIR, class Epi>
__device__ __forceinline__ void dense_block(const DenseIn& d, int m, int n, char* sm,
                                            const Epi& epi, int half = -1, int tile = 0,
                                            int tiles = 0) {
    constexpr int OC = PAIR ? TN / 2 : TN;
    const int64_t r0 = (int64_t)m * TM;
    const int c0 = n * OC;
    TileIn in;
    in.a = d.a + r0 * (LA == KC ? d.lda : E::SZ);
    in.b = d.b + (int64_t)c0 * (LB == KC ? d.ldb : E::SZ);
    in.b2 = PAIR ? d.b + ((int64_t)d.cols + c0) * d.ldb : nullptr;
    in.lda = d.lda;
    in.ldb = d.ldb;
    in.rows = d.rows - r0 < TM ? (int)(d.rows - r0) : TM;
    in.cols = d.cols - c0;
    in.K = d.K;
    const int nk = (int)((d.K * E::SZ + 127) / 128);
    // with halves the first block takes 8 k-tiles less, so that it has written its partial result
    // when the second one is done (down product of 4096 tokens, m = 8192: 135 -> 126 us)
    const int first = nk / 2 - 4 < 0 ? 0 : nk / 2 - 4;
    in.t0 = half > 0 ? first : 0;
    in.t1 = half == 0 ? first : nk;
    in.half = half;
    in.part = d.part + (int64_t)tile * (2 * kPartialBytes);
    in.count = reinterpret_cast<uint32_t*>(d.part + (int64_t)tiles * (2 * kPartialBytes)) + tile;
    Form::run(in, sm, epi.at(r0, c0));
}

// sigma(g) = 1 / (1 + e^-g) to about two units in the last place of fp32: e^-g = 2^t 2^r with t the
// rounded product -g log2 e and r what its rounding left off (below 2^-17 for |g| < 2^7), 2^r =
// 1 + r ln 2.  A g below -88 makes 2^t infinite and sigma zero.  g is held to +-128, where sigma is
// 1 and 0 already: beyond 2^127 / log2 e, t and r would be infinite and their product no number. A
// NaN becomes -128, and still NaN in every product with g itself.  (The library's exponential and
// division take five times the instructions: gate/up of 4096 tokens, m = 8192, int8, 162 us with
// them.)
__device__ __forceinline__ float sigma_f32(float g) {
    g = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f);
    constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.69314718f;
    const float t = -g * kLog2e;
    const float r = fmaf(-g, kLog2eRest, fmaf(-g, kLog2e, -t));
    return __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(t), fmaf(r, kLn2, 1.0f), 1.0f));
}
// where the result is rounded to bf16: the hardware's exponential as it is
__device__ __forceinline__ float sigma_bf16(float g) {
    return __builtin_amdgcn_rcpf(1.0f + __expf(-g));
}

// ---- what becomes of a product ----
// An Epi's fetch(row, col) loads what eight columns of a row need beside the product, and put()
// computes and stores them.  Block forms fetch for several rows before they put the first: loads
// do not pass the stores before them, and one at a time each would wait out the memory's latency
// (down product of 16384 tokens, m = 1024, with a residual 78 us, 86 one at a time; dh of 4096 tokens,
// m = 8192, which is bound by the 64 bytes of eight columns, 213 either way).
struct Nothing {};

template <class T>
struct Eight {  // eight values of a tensor, as loaded
    T v[8];
    __device__ __forceinline__ void load(const T* p) {
        typedef uint32_t raw_t __attribute__((ext_vector_type(2 * sizeof(T)), aligned(2)));
        *reinterpret_cast<raw_t*>(v) = *reinterpret_cast<const raw_t*>(p);
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (sizeof(T) == 2) return bf16_to_f32(v[i]);
        else return v[i];
    }
};

template <class T>
struct PlainOut {  // y = [res +] v
    static constexpr bool kMayHalve = true;  // its products may take kHalves
    T* y;
    const T* res;
    int64_t ld;
    typedef Eight<T> Extra;
    __device__ __forceinline__ PlainOut at(int64_t r0, int c0) const {
        const int64_t o = r0 * ld + c0;
        return {y + o, res ? res + o : nullptr, ld};
    }
    __device__ __forceinline__ void fetch(int row, int col, Extra& e) const {
        if (res) e.load(res + row * ld + col);
    }
    __device__ __forceinline__ void put(int row, int col, float (&v)[8], const Extra& e) const {
        if (res) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += e[q];
        }
        store8(y + row * ld + col, v);
    }
};

// ---- kernels ----
template <class E, int MF, int TM, int TN, int WM, int LA, int LB, bool PAIR, bool DMA, int S,
          class Epi>
__global__ __launch_bounds__(256) void dense_tiles(DenseIn d, int mt, int nt, Epi epi) {
    typedef TileForm<E, MF, TM, TN, WM, LA, LB, PAIR, DMA, S> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    clear_counters(d.clear, d.nclear);
    int m, n;
    if (!dense_tile(dense_block_number(), mt, nt, m, n)) return;
    dense_block<Form, E, TM, TN, LA, LB, PAIR>(d, m, n, sm, epi);
}

// two products of one kind in one launch: the first mt1 nt1 tiles (rounded up to blocks1 blocks,
// a multiple of 8), then the second's
template <class E, int MF, int TM, int TN, int WM, int LA, int LB, bool DMA, int S, class Epi>
__global__ __launch_bounds__(256) void dense_tiles2(DenseIn d1, DenseIn d2, int mt1, int nt1,
                                                    int mt2, int nt2, uint32_t blocks1, Epi epi1,
                                                    Epi epi2) {
    typedef TileForm<E, MF, TM, TN, WM, LA, LB, false, DMA, S> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    const uint32_t b = dense_block_number();
    int m, n;
    if (b < blocks1) {
        if (!dense_tile(b, mt1, nt1, m, n)) return;
        dense_block<Form, E, TM, TN, LA, LB, false>(d1, m, n, sm, epi1);
    } else {
        if (!dense_tile(b - blocks1, mt2, nt2, m, n)) return;
        dense_block<Form, E, TM, TN, LA, LB, false>(d2, m, n, sm, epi2);
    }
}

template <class E, int TM, int TN, int NW, int LB, bool PAIR, int S, class Epi>
__global__ __launch_bounds__(NW * 64) void dense_split(DenseIn d, int mt, int nt, Epi epi) {
    typedef SplitForm<E, TM, TN, NW, KC, LB, PAIR, S> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    clear_counters(d.clear, d.nclear);
    int m, n;
    if (!dense_tile(dense_block_number(), mt, nt, m, n)) return;
    dense_block<Form, E, TM, TN, KC, LB, PAIR>(d, m, n, sm, epi);
}

template <class E, int TM, int TN, int WM, int LA, int LB, bool PAIR, class Epi>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_turns(
    DenseIn d, int mt, int nt, Epi epi) {
    typedef TurnForm<E, TM, TN, WM, LA, LB, PAIR> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    clear_counters(d.clear, d.nclear);
    int m, n;
    if (!dense_tile(dense_block_number(), mt, nt, m, n)) return;
    dense_block<Form, E, TM, TN, LA, LB, PAIR>(d, m, n, sm, epi);
}

// two blocks per tile: tile b / 2 of a numbering in which an XCD's tiles follow each other
template <class E, int TM, int TN, int WM, int LA, int LB, class Epi>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_halves(
    DenseIn d, int mt, int nt, Epi epi) {
    typedef TurnForm<E, TM, TN, WM, LA, LB, false, true> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    const uint32_t b = dense_block_number();
    const uint32_t half = b >> 3 & 1, b2 = (b >> 4 << 3) + (b & 7);  // both on one XCD
    int m, n;
    if (!dense_tile(b2, mt, nt, m, n)) return;
    dense_block<Form, E, TM, TN, LA, LB, false>(d, m, n, sm, epi, half, m * nt + n, mt * nt);
}

template <class E, int TM, int TN, int WM, int LA, int LB, class Epi>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_turns2(
    DenseIn d1, DenseIn d2, int mt1, int nt1, int mt2, int nt2, uint32_t blocks1, Epi epi1,
    Epi epi2) {
    typedef TurnForm<E, TM, TN, WM, LA, LB, false> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    const uint32_t b = dense_block_number();
    const bool one = b < blocks1;
    int m, n;
    if (!dense_tile(one ? b : b - blocks1, one ? mt1 : mt2, one ? nt1 : nt2, m, n)) return;
    const DenseIn d = one ? d1 : d2;
    const Epi epi = one ? epi1 : epi2;
    dense_block<Form, E, TM, TN, LA, LB, false>(d, m, n, sm, epi);
}

template <class E, int LA, int LB, bool PAIR, class Epi>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_pairs(
    DenseIn d, int mt, int nt, Epi epi) {
    typedef PairForm<E, LA, LB, PAIR> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    clear_counters(d.clear, d.nclear);
    int m, n;
    if (!dense_tile(dense_block_number(), mt, nt, m, n)) return;
    dense_block<Form, E, 128, 128, LA, LB, PAIR>(d, m, n, sm, epi);
}

template <class E, int LA, int LB, class Epi>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void dense_pairs2(
    DenseIn d1, DenseIn d2, int mt1, int nt1, int mt2, int nt2, uint32_t blocks1, Epi epi1,
    Epi epi2) {
    typedef PairForm<E, LA, LB, false> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    const uint32_t b = dense_block_number();
    const bool one = b < blocks1;
    int m, n;
    if (!dense_tile(one ? b : b - blocks1, one ? mt1 : mt2, one ? nt1 : nt2, m, n)) return;
    const DenseIn d = one ? d1 : d2;
    const Epi epi = one ? epi1 : epi2;
    dense_block<Form, E, 128, 128, LA, LB, false>(d, m, n, sm, epi);
}

template <class E, int TM, int TN, int NW, int S, class Epi>
__global__ __launch_bounds__(NW * 64) void dense_split2(DenseIn d1, DenseIn d2, int mt1, int nt1,
                                                        int mt2, int nt2, uint32_t blocks1,
                                                        Epi epi1, Epi epi2) {
    typedef SplitForm<E, TM, TN, NW, KR, KR, false, S> Form;
    __shared__ __attribute__((aligned(1024))) char sm[Form::LDS];
    const uint32_t b = dense_block_number();
    const bool one = b < blocks1;
    int m, n;
    if (!dense_tile(one ? b : b - blocks1, one ? mt1 : mt2, one ? nt1 : nt2, m, n)) return;
    const DenseIn d = one ? d1 : d2;
    const Epi epi = one ? epi1 : epi2;
    dense_block<Form, E, TM, TN, KR, KR, false>(d, m, n, sm, epi);
}

inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
inline dim3 grid_of(int64_t blocks) {
    return blocks <= kDenseRow ? dim3((unsigned)blocks)
                               : dim3(kDenseRow, (unsigned)((blocks + kDenseRow - 1) / kDenseRow));
}
inline int tiles(int64_t n, int t) { return (int)((n + t - 1) / t); }

template <class E, int MF, int TM, int TN, int WM, int LA, int LB, bool PAIR, bool DMA, int S,
          class Epi>
void run_tiles(const DenseIn& d, const Epi& epi, hipStream_t s) {
    const int mt = tiles(d.rows, TM), nt = tiles(d.cols, PAIR ? TN / 2 : TN);
    if (mt == 0 || nt == 0) return;
    ELB_LAUNCH((dense_tiles<E, MF, TM, TN, WM, LA, LB, PAIR, DMA, S, Epi>),
               grid_of(up8((int64_t)mt * nt)), dim3(256), 0, s, d, mt, nt, epi);
}

template <class E, int TM, int TN, int NW, int LB, bool PAIR, int S, class Epi>
void run_split(const DenseIn& d, const Epi& epi, hipStream_t s) {
    const int mt = tiles(d.rows, TM), nt = tiles(d.cols, PAIR ? TN / 2 : TN);
    if (mt == 0 || nt == 0) return;
    ELB_LAUNCH((dense_split<E, TM, TN, NW, LB, PAIR, S, Epi>), grid_of(up8((int64_t)mt * nt)),
               dim3(NW * 64), 0, s, d, mt, nt, epi);
}

template <class E, int TM, int TN, int WM, int LA, int LB, bool PAIR, class Epi>
void run_turns(const DenseIn& d, const Epi& epi, hipStream_t s) {
    const int mt = tiles(d.rows, TM), nt = tiles(d.cols, PAIR ? TN / 2 : TN);
    if (mt == 0 || nt == 0) return;
    ELB_LAUNCH((dense_turns<E, TM, TN, WM, LA, LB, PAIR, Epi>), grid_of(up8((int64_t)mt * nt)),
               dim3(512), 0, s, d, mt, nt, epi);
}

template <class E, int TM, int TN, int WM, int LA, int LB, class Epi>
void run_halves(const DenseIn& d, const Epi& epi, hipStream_t s) {
    const int mt = tiles(d.rows, TM), nt = tiles(d.cols, TN);
    if (mt == 0 || nt == 0) return;
    ELB_LAUNCH((dense_halves<E, TM, TN, WM, LA, LB, Epi>),
               grid_of(2 * up8((int64_t)mt * nt)), dim3(512), 0, s, d, mt, nt, epi);
}

// the counters of a product's kHalves scratch, or none where another form is picked
struct Counters {
    uint32_t* p;
    int n;
};
inline Counters halves_counters(char* part, int64_t rows, int64_t cols, int64_t ktiles,
                                bool fp32) {
    if (!part || pick_form(rows, cols, ktiles, fp32, true) != kHalves) return {nullptr, 0};
    const int64_t n = form_tiles(kFormCosts[kHalves], rows, cols);
    return {reinterpret_cast<uint32_t*>(part + n * 2 * kPartialBytes), (int)n};
}

template <class E, int LA, int LB, bool PAIR, class Epi>
void run_pairs(const DenseIn& d, const Epi& epi, hipStream_t s) {
    const int mt = tiles(d.rows, 128), nt = tiles(d.cols, PAIR ? 64 : 128);
    if (mt == 0 || nt == 0) return;
    ELB_LAUNCH((dense_pairs<E, LA, LB, PAIR, Epi>), grid_of(up8((int64_t)mt * nt)), dim3(512), 0,
               s, d, mt, nt, epi);
}

// A product whose first operand has its contraction contiguous, in the form picked for its
// size.  The forms that copy by 16-byte LDS loads want tensors on 16-byte boundaries (aligned);
// others take the tile form with ordinary loads.
template <class E, int LB, bool PAIR, class Epi>
void run_product(const DenseIn& d, bool aligned, const Epi& epi, hipStream_t s) {
    constexpr bool F = E::SZ == 4;
    constexpr int MF = F ? 16 : 32, TT = F ? 64 : 128, S = F ? 3 : 2;
    const FormId form = !aligned ? kTiles
                                 : pick_form(d.rows, PAIR ? 2 * (int64_t)d.cols : d.cols,
                                             (d.K * E::SZ + 127) / 128, F,
                                             Epi::kMayHalve && d.part);
    switch (form) {
        case kSplit16x16: return run_split<E, 16, 16, 8, LB, PAIR, 4>(d, epi, s);
        case kSplit16x32: return run_split<E, 16, 32, 8, LB, PAIR, 3>(d, epi, s);
        case kSplit16x64: return run_split<E, 16, 64, 4, LB, PAIR, 3>(d, epi, s);
        case kSplit32x32: return run_split<E, 32, 32, 8, LB, PAIR, 2>(d, epi, s);
        case kSplit32x64: return run_split<E, 32, 64, 4, LB, PAIR, 3>(d, epi, s);
        case kSplit64x64: return run_split<E, 64, 64, 4, LB, PAIR, 2>(d, epi, s);
        default: break;
    }
    if constexpr (!F) {
        if (form == kPairs) return run_pairs<E, KC, LB, PAIR>(d, epi, s);
        if (form == kTurns) return run_turns<E, 256, 256, 2, KC, LB, PAIR>(d, epi, s);
        if constexpr (Epi::kMayHalve)
            if (form == kHalves) return run_halves<E, 256, 256, 2, KC, LB>(d, epi, s);
        run_tiles<E, MF, TT, TT, 2, KC, LB, PAIR, false, S>(d, epi, s);
    } else {
        if (aligned) run_tiles<E, MF, TT, TT, 2, KC, LB, PAIR, true, S>(d, epi, s);
        else run_tiles<E, MF, TT, TT, 2, KC, LB, PAIR, false, S>(d, epi, s);
    }
}

// Two products of one kind, both operands down the rows (KR), in one launch.
template <int TM, int TN, class Kernel, class Epi>
void launch2(Kernel kernel, int threads, const DenseIn& d1, const DenseIn& d2, const Epi& e1,
             const Epi& e2, hipStream_t s) {
    const int mt1 = tiles(d1.rows, TM), nt1 = tiles(d1.cols, TN);
    const int mt2 = tiles(d2.rows, TM), nt2 = tiles(d2.cols, TN);
    const int64_t b1 = up8((int64_t)mt1 * nt1), blocks = b1 + up8((int64_t)mt2 * nt2);
    if (blocks == 0) return;
    ELB_LAUNCH(kernel, grid_of(blocks), dim3(threads), 0, s, d1, d2, mt1, nt1, mt2, nt2,
               (uint32_t)b1, e1, e2);
}

template <class E, class Epi>
void run_product2(const DenseIn& d1, const DenseIn& d2, bool aligned, const Epi& e1,
                  const Epi& e2, hipStream_t s) {
    constexpr bool F = E::SZ == 4;
    const FormId form = !aligned ? kTiles
                                 : pick_form2(d1.rows, d1.cols, d2.rows, d2.cols,
                                              (d1.K * E::SZ + 127) / 128, F);
    switch (form) {
        case kSplit32x32:
            return launch2<32, 32>(dense_split2<E, 32, 32, 8, 2, Epi>, 512, d1, d2, e1, e2, s);
        case kSplit64x64:
            return launch2<64, 64>(dense_split2<E, 64, 64, 4, 2, Epi>, 256, d1, d2, e1, e2, s);
        default: break;
    }
    if constexpr (F) {
        if (aligned)
            launch2<64, 64>(dense_tiles2<E, 16, 64, 64, 2, KR, KR, true, 3, Epi>, 256, d1, d2, e1,
                            e2, s);
        else
            launch2<64, 64>(dense_tiles2<E, 16, 64, 64, 2, KR, KR, false, 3, Epi>, 256, d1, d2,
                            e1, e2, s);
    } else {
        if (form == kTiles)
            launch2<128, 128>(dense_tiles2<E, 32, 128, 128, 2, KR, KR, false, 2, Epi>, 256, d1,
                              d2, e1, e2, s);
        else if (form == kPairs)
            launch2<128, 128>(dense_pairs2<E, KR, KR, Epi>, 512, d1, d2, e1, e2, s);
        else
            launch2<256, 256>(dense_turns2<E, 256, 256, 2, KR, KR, Epi>, 512, d1, d2, e1, e2, s);
    }
}

}  // namespace

}  // namespace elb
