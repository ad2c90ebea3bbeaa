// The 4-bit cache format (voxzip_q4_cache): how a row is held, and the warp-level code that makes a packed row.
//
// A row of D channels is D / 32 groups of 32 consecutive channels, each with a bf16 scale s and a 4-bit code
// per channel, stored as c + 8 with c in [-8, 7]; the channel stands for c s, times 2^e for K with the unit's
// exponent e of that channel. 32 channels per 16-bit scale is 4.5 bits per channel.
//   s = bf16(x_m / -8), x_m the element of largest magnitude: it is held at code -8, so that all sixteen codes
//   serve (with s = max / 7 one of them would be idle). Codes are rint(x (1 / s)): one division per group.
// The order of the codes in a row is the one the decode kernel's tensor-core operands want, without moving a
// bit between lanes:
//   K: 4-byte word q J + j (J = D / 32) holds channels 32 j + 8 q + e, e = 0..7, channel e at nibble
//      e / 2 + 4 (e % 2): lane q of a quad loads its J words as one vector, one word per group; the nibbles i
//      and i + 4 of a word lie 16 bits apart, a pair of bf16 operands after one AND.
//   V: 2-byte word g J + j holds channels 32 j + 4 g + i, channel i at nibble i: lane group g loads its J
//      half-words as one vector, and halves of two tokens make a pair of operands.
#pragma once

#include "common.cuh"
#include "evict_policy.cuh"
#include "ptx.cuh"

namespace voxzip {

constexpr int kQ4Group = 32;
constexpr int kQ4MaxExp = 16;

// The views' element types; strides follow from D and C.
struct Q4View {
    uint8_t *k_codes, *v_codes;            // [units][C][D / 2]
    __nv_bfloat16 *k_scale, *v_scale;      // [units][C][D / 32]
    int8_t *k_exp;                         // [units][D]
};

inline Q4View q4_view(const voxzip_q4_cache &c) {
    return Q4View{static_cast<uint8_t *>(c.k_codes), static_cast<uint8_t *>(c.v_codes),
                  static_cast<__nv_bfloat16 *>(c.k_scale), static_cast<__nv_bfloat16 *>(c.v_scale), c.k_exp};
}

__device__ __forceinline__ float exp2_int(int e) {  // 2^e for e in [-126, 127], exact
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Order of "larger magnitude, the positive one on a tie": bits of |x|, then the sign.
__device__ __forceinline__ uint32_t magnitude_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return (b << 1) | ((b >> 31) ^ 1u);
}

// Scale of a group from the key of its element of largest magnitude.
__device__ __forceinline__ float q4_scale(uint32_t key) {
    const uint32_t mag = key >> 1;
    if (mag >= 0x7f800000u) return __uint_as_float(0x7fffffffu);  // not finite: the group reads back as NaN
    const float eighth = __uint_as_float(mag) * 0.125f;
    const float s = __bfloat162float(__float2bfloat16_rn((key & 1u) ? -eighth : eighth));
    return fabsf(s) < 1.17549435e-38f ? 0.f : s;  // below the smallest normal number: a group of zeros
}

// Code + 8 of x under the scale's reciprocal (0 stands for "no codes": scale 0 or NaN).
__device__ __forceinline__ uint32_t q4_code(float x, float inv) {
    return (uint32_t)(min(max(__float2int_rn(__fmul_rn(x, inv)), -8), 7) + 8);
}
__device__ __forceinline__ float q4_inverse(float s) { return s != 0.f && s == s ? __frcp_rn(s) : 0.f; }

// A row packed by a warp: lane l of the first D / 4 lanes holds channels 4 l .. 4 l + 3 (for K already times 2^-e);
// the other lanes hold zeros. All 32 lanes make it; store() may then be called with any row of either memory.
template <int D, bool kIsK>
struct Q4Row {
    static constexpr int J = D / kQ4Group;
    uint32_t bits;  // K: a word, the same in lanes 2 i and 2 i + 1; V: a half-word
    __nv_bfloat16 scale;

    __device__ __forceinline__ explicit Q4Row(const float4 &x) {
        uint32_t key = max(max(magnitude_key(x.x), magnitude_key(x.y)), max(magnitude_key(x.z), magnitude_key(x.w)));
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
        const float s = q4_scale(key), inv = q4_inverse(s);
        scale = __float2bfloat16_rn(s);
        const uint32_t n0 = q4_code(x.x, inv), n1 = q4_code(x.y, inv), n2 = q4_code(x.z, inv), n3 = q4_code(x.w, inv);
        if constexpr (kIsK) {
            bits = (n0 | n1 << 16 | n2 << 4 | n3 << 20) << ((threadIdx.x & 1) * 8);
            bits |= __shfl_xor_sync(0xffffffffu, bits, 1);
        } else {
            bits = n0 | n1 << 4 | n2 << 8 | n3 << 12;
        }
    }
    // codes, scales: the row's own D / 2 bytes and J scales.
    __device__ __forceinline__ void store(uint8_t *codes, __nv_bfloat16 *scales) const {
        const int lane = threadIdx.x & 31, j = lane >> 3;
        if (lane >= D / 4) return;
        if constexpr (kIsK) {
            if (!(lane & 1)) reinterpret_cast<uint32_t *>(codes)[((lane >> 1) & 3) * J + j] = bits;
        } else {
            reinterpret_cast<uint16_t *>(codes)[(lane & 7) * J + j] = (uint16_t)bits;
        }
        if ((lane & 7) == 0) scales[j] = scale;
    }
};

// Host-side launchers.
cudaError_t launch_q4_pack(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                           const void *k_cache, const void *v_cache, const int32_t *len, int32_t *status,
                           cudaStream_t stream);
cudaError_t launch_q4_unpack(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const int32_t *len, int32_t first, int32_t rows, void *k_out, void *v_out, int32_t *status,
                             cudaStream_t stream);
cudaError_t launch_decode_q4(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const void *q, const void *k_new, const void *v_new, const int32_t *new_pos, float *score,
                             int32_t *pos, int32_t *len, float gamma, float sm_scale, int32_t max_len, void *out,
                             int32_t *status, cudaStream_t stream);
cudaError_t launch_decode_q4_rows(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin,
                                  int32_t layer_count, const void *q, const void *k_new, const void *v_new,
                                  const int32_t *new_pos, float *score, int32_t *pos, int32_t *len, float gamma,
                                  float sm_scale, int32_t max_len, void *out, int32_t *status, cudaStream_t stream);
cudaError_t launch_evict_q4(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                            float *score, int32_t *pos, int32_t *len, const int32_t *budget,
                            const voxzip_evict_policy &policy, int32_t *status, cudaStream_t stream);

}  // namespace voxzip
