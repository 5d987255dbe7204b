// 4-bit weights with group scales, and the pieces that stream weights past a few tokens.
//
// A weight is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives: sign, two bits of exponent, one of
// mantissa), two to a byte, the earlier along the contraction in the low half; 32 of them share a
// scale 2^(b - 127), b a byte.  v_cvt_scalef32_pk_bf16_fp4 makes two of them, scaled, bf16 (exactly),
// so a product costs half an instruction a weight before its MFMA.
//
// Weights are streamed in units of 128 bytes of 16 NF rows (64 bf16 or 256 4-bit values of the
// contraction), copied in whole lines into a wave's own LDS and read from there as MFMA operands.
// (Operands loaded straight into registers, 16 rows of 64 bytes an instruction, reached a third of that
// rate: 8 waves of a block read a router of 64 rows of 4 KB in 9 us.)  In LDS a row's eight 16-byte
// chunks are swizzled (kc_swz).  Lane l of a fragment has row l % 16 and quarter c = l / 16 of each
// half of the unit: 8 bf16, one v_mfma_f32_16x16x32_bf16; or 32 4-bit values, which are turned between
// the quarters (a 4 x 4 transposition of words in four swaps) into the operands of four, the i-th
// of them group i of the half, so that the tokens' operand is contiguous in the same way.
#pragma once

#include "dense.h"

namespace elb {

namespace {

typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32_byte_t __attribute__((aligned(1)));

// eight 4-bit weights times a power of two
__device__ __forceinline__ bf16x8_t f4_to_bf16(uint32_t w, float scale) {
    const bf16x2v_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    const bf16x2v_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2v_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    const bf16x2v_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    const u32x4_t v = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
    return __builtin_bit_cast(bf16x8_t, v);
}
__device__ __forceinline__ float f4_scale(uint32_t b) { return __uint_as_float(b << 23); }

// words a and b, each of four quarters of a wave: (a0 a1 b0 b1), (a2 a3 b2 b3)
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
// (a0 b0 a2 b2), (a1 b1 a3 b3)
__device__ __forceinline__ void swap_quarters(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// this wave's lane's 32-bit LDS address of a pointer into LDS, in a scalar register
__device__ __forceinline__ uint32_t lds_address(const char* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)p);
}

// ---- weight types: KU, the contraction of a unit; J, MFMAs of a half of it ----
struct WBf16 {
    static constexpr int KU = 64, J = 1, SCALES = 0;
    struct Half {  // a fragment's operands of half a unit
        u32x4_t v;
        __device__ __forceinline__ bf16x8_t get(int) const { return __builtin_bit_cast(bf16x8_t, v); }
    };
    static __device__ __forceinline__ int64_t row_bytes(int64_t k) { return 2 * k; }
    // half h of the unit in LDS at p, row l16 of fragment f
    static __device__ __forceinline__ void read(Half& o, const char* p, int, int f, int h, int l16,
                                                int c) {
        o.v = *reinterpret_cast<const u32x4_t*>(p + (16 * f + l16) * 128 +
                                                kc_swz(l16, 4 * h + c) * 16);
    }
};
struct WF4 {
    static constexpr int KU = 256, J = 4, SCALES = 8;  // scale bytes of a row
    struct Half {
        uint32_t v[4], s;
        // (the scales of both halves lie in a row's eight bytes: s holds those of this one)
        __device__ __forceinline__ bf16x8_t get(int i) const {
            return f4_to_bf16(v[i], f4_scale(s >> (8 * i) & 255u));
        }
    };
    static __device__ __forceinline__ int64_t row_bytes(int64_t k) { return k / 2; }
    // rows: of the unit, whose scales lie behind them
    static __device__ __forceinline__ void read(Half& o, const char* p, int rows, int f, int h,
                                                int l16, int c) {
        const int r = 16 * f + l16;
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p + r * 128 +
                                                            kc_swz(l16, 4 * h + c) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) o.v[i] = v[i];
        o.s = *reinterpret_cast<const uint32_t*>(p + rows * 128 + r * 8 + 4 * h);
        swap_halves(o.v[0], o.v[2]);
        swap_halves(o.v[1], o.v[3]);
        swap_quarters(o.v[0], o.v[1]);
        swap_quarters(o.v[2], o.v[3]);
    }
};

// A KC copier's k-tile that lies wholly within the contraction, `at` bytes from its start, to LDS at lds:
// one buffer for the tile's rows, whose bound leaves out those past the last, and `at` as the scalar
// offset.  (Copier::issue sets bounds for every k-tile, some twenty instructions for each: 8192 to 2048
// of 512 tokens 37.6 us with it, 34.5 with this; 64 tokens 11.1, 11.2.)
// NT: with the non-temporal hint.
template <bool NT = false, class C>
__device__ __forceinline__ void issue_whole(const C& c, uint32_t at, uint32_t lds) {
    u32x4_t rs[C::NB];
#pragma unroll
    for (int b = 0; b < C::NB; ++b) {
        const uint64_t p = (uint64_t)c.base[b];
        rs[b] = u32x4_t{uniform((uint32_t)p), uniform((uint32_t)(p >> 32)) & 0xffffu,
                        uniform((uint32_t)(c.span > 0 ? c.span : 0)), 0x00027000u};
    }
#pragma unroll
    for (int i = 0; i < C::N; ++i) {
        const u32x4_t& r = rs[C::NB == 2 && i >= C::N / 2 ? C::NB - 1 : 0];
        if constexpr (NT)
            asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                         :: "s"(uniform(lds + i * 1024)), "v"(c.off[i]), "s"(r), "s"(uniform(at))
                         : "memory", "m0");
        else
            asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                         :: "s"(uniform(lds + i * 1024)), "v"(c.off[i]), "s"(r), "s"(uniform(at))
                         : "memory", "m0");
    }
}

// One wave's copies of a unit of weights: 16 NF rows (PAIR: the second half of them `apart` rows of
// the tensor further on) of 128 bytes, and the rows' eight scale bytes behind them.  DMA: weights on
// 16-byte boundaries; otherwise ordinary loads, as for scales whose rows are off 4-byte ones.  NT:
// weights that a call reads once, with the non-temporal hint (few-token layer, bf16, 8 to 16 tokens: 97 %
// to 104 % of the time that elb_moe_forward takes, by card, 108 % to 112 % without).
template <class W, int NF, bool PAIR, bool DMA, bool NT = false>
struct Stream {
    static constexpr int ROWS = 16 * NF;
    static constexpr int BYTES = ROWS * 128 + (W::SCALES ? (ROWS + 31) / 32 * 256 : 0);
    typedef Copier<KC, ROWS, 1, 1, PAIR, DMA> C;
    C copy;
    const uint8_t* scale[(ROWS + 31) / 32];  // of the lane's rows
    int groups;                              // of a row
    const uint8_t* end;                      // of the scales
    bool words;                              // scale rows start on 4-byte boundaries

    // row0: the tile's first row; rows: valid ones from there on (of each half with PAIR); all: rows of
    // the matrix
    __device__ __forceinline__ void init(const void* w, const uint8_t* s, int64_t row0, int rows,
                                         int64_t apart, int64_t all, int64_t k, int lane) {
        const int64_t ld = W::row_bytes(k);
        copy.init((const char*)w + row0 * ld, (const char*)w + (row0 + apart) * ld, ld, rows, ld,
                  lane, 0);
        if (!W::SCALES) return;
        groups = (int)(k / 32);
        end = s + all * groups;
        words = DMA && (groups & 3) == 0 && ((uintptr_t)s & 3) == 0;
        constexpr int HR = PAIR ? ROWS / 2 : ROWS;
#pragma unroll
        for (int i = 0; i < (ROWS + 31) / 32; ++i) {
            int r = 32 * i + (lane >> 1);  // two words a row
            r = r < ROWS ? r : ROWS - 1;
            int64_t row = row0;
            if (PAIR && r >= HR) {
                row += apart;
                r -= HR;
            }
            scale[i] = s + (row + (r < rows ? r : rows - 1)) * groups;
        }
    }
    // scale words on their way to LDS by ordinary loads
    struct Pending {
        uint32_t v[(ROWS + 31) / 32];
    };
    // unit u to LDS at lds (ldsp: the same as a pointer); values past the row's end are zeros
    __device__ __forceinline__ void issue(int u, int uend, uint32_t lds, char* ldsp, int lane,
                                          Pending& pending) const {
        if (DMA && u < uend && (int64_t)(u + 1) * 128 <= copy.klen)
            issue_whole<NT>(copy, (uint32_t)u * 128u, lds);
        else
            copy.issue(u, uend, lds, ldsp, lane, 0);
        if constexpr (W::SCALES != 0) {
            const int g = 8 * u + 4 * (lane & 1);
#pragma unroll
            for (int i = 0; i < (ROWS + 31) / 32; ++i) {
                // groups past the row's last: other bytes of the tensor, which no product takes
                if (words) {
                    const uint8_t* const p = scale[i] + (g < groups ? g : groups - 4);
                    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off"
                                 :: "s"(uniform(lds + ROWS * 128 + i * 256)), "v"(p)
                                 : "memory", "m0");
                } else {
                    // a word at any byte; the tensor's last one moved down to lie in it
                    const uint8_t* const p = scale[i] + (g < groups ? g : 0);
                    const int64_t over = p + 4 - end;
                    const int past = over > 0 ? (int)over : 0;
                    pending.v[i] = *reinterpret_cast<const u32_byte_t*>(p - past) >> (8 * past);
                }
            }
        }
    }
    // after the wait for a unit, before it is read
    __device__ __forceinline__ void settle(const Pending& pending, char* ldsp, int lane) const {
        if constexpr (W::SCALES != 0) {
            if (words) return;
#pragma unroll
            for (int i = 0; i < (ROWS + 31) / 32; ++i)
                *reinterpret_cast<uint32_t*>(ldsp + ROWS * 128 + i * 256 + lane * 4) = pending.v[i];
        }
    }
    // the same rows of another matrix, w_bytes and s_bytes further on
    __device__ __forceinline__ Stream moved(int64_t w_bytes, int64_t s_bytes) const {
        Stream o = *this;
#pragma unroll
        for (int b = 0; b < C::NB; ++b) o.copy.base[b] += w_bytes;
        if (W::SCALES) {
#pragma unroll
            for (int i = 0; i < (ROWS + 31) / 32; ++i) o.scale[i] += s_bytes;
            o.end += s_bytes;
        }
        return o;
    }
};
}  // namespace

}  // namespace elb
