// 4-bit weights with group scales, and the ring that streams weights past a few tokens.
//
// A weight is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives: sign, two bits of exponent, one of
// mantissa), two to a byte, the earlier along the contraction in the low half; 32 of them share a
// scale 2^(b - 127), b a byte.  v_cvt_scalef32_pk_bf16_fp4 makes two of them, scaled, bf16 (exactly),
// so a product costs half an instruction a weight before its MFMA.
//
// Operands lie in registers as they come from memory: a lane loads 16 bytes of weight row (lane & 15),
// its quarter (lane >> 4) of a step of 64 bytes.  That is 8 bf16 or 32 4-bit values, so a step of the
// contraction is one v_mfma_f32_16x16x32_bf16 or four; in the i-th of the four, quarter c multiplies
// values 32 c + 8 i .. + 7 of the step, and the tokens' operand is loaded to match.
#pragma once

#include "dense.h"

namespace elb {

namespace {

typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));

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

// ---- weights of a step: 16 bytes a lane of each fragment of 16 rows ----
struct WBf16 {
    static constexpr int KS = 32, J = 1;  // contraction of a step, MFMAs that it takes
    struct Frag {
        u32x4_t v;
    };
    const bf16_t* w;
    int64_t ld;  // elements
    __device__ __forceinline__ void load(Frag& f, int64_t row, int k) const {
        f.v = *reinterpret_cast<const u32x4_any_t*>(w + row * ld + k);
    }
    static __device__ __forceinline__ bf16x8_t get(const Frag& f, int) {
        return __builtin_bit_cast(bf16x8_t, f.v);
    }
};
struct WF4 {
    static constexpr int KS = 128, J = 4;
    struct Frag {
        u32x4_t v;
        uint32_t s;
    };
    const uint8_t *w, *scale;
    int64_t ld;  // values
    __device__ __forceinline__ void load(Frag& f, int64_t row, int k) const {
        const int64_t o = row * ld + k;
        f.v = *reinterpret_cast<const u32x4_byte_t*>(w + (o >> 1));
        f.s = scale[o >> 5];
    }
    static __device__ __forceinline__ bf16x8_t get(const Frag& f, int i) {
        return f4_to_bf16(f.v[i], f4_scale(f.s));
    }
};

// Steps 0 .. n - 1 through R register slots: R - 1 steps are in flight while one is multiplied.
// load(step, slot) for steps in order (none past the last), mma(step, slot).
template <int R, class Slot, class Load, class Mma>
__device__ __forceinline__ void ring(int n, Load&& load, Mma&& mma) {
    Slot s[R];
#pragma unroll
    for (int p = 0; p < R - 1; ++p)
        if (p < n) load(p, s[p]);
    for (int j = 0; j < n; j += R) {
#pragma unroll
        for (int p = 0; p < R; ++p) {
            if (j + p >= n) break;
            if (j + p + R - 1 < n) load(j + p + R - 1, s[(p + R - 1) % R]);
            // this step's loads before its products, which wait for an earlier step's only
            __builtin_amdgcn_sched_barrier(0);
            mma(j + p, s[p]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

}  // namespace

}  // namespace elb
