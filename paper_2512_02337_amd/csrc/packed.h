// The 4-bit cache (specpv_packed_kv): E2M1 values under one power of two for every 32 channels, and its kernels' arguments.
// A row of D channels is D / 2 bytes of codes (channel 2 i in the low nibble of byte i) and D / 32 scale bytes e + 127.
// Every value has two significant bits, so it is exact in bf16, and the conversions of the hardware (four bits to bf16 or
// fp32 and back, with the power of two) are the format's own: all 16 codes under scales 3, 127 and 252, both nibbles, give
// the values, byte 255 gives NaN, and every finite bf16 under its exponent's scales rounds to nearest, ties to even, ends at 6.
#pragma once
#include "internal.h"

namespace specpv {

typedef __attribute__((ext_vector_type(2))) float f32x2;

struct PackedShape {
    Shape s;                     // k, v: codes; sb, sh, st: bytes of codes (a sixteenth of them for the scales)
    const uint8_t *ks, *vs;
    int64_t rows;                // that the memory has: none behind them is read or written, whatever the lengths say
};

constexpr int kPackedGroup = 32;       // channels of a scale
constexpr uint32_t kScaleMin = 3, kScaleMax = 252, kScaleNaN = 255;

// The scale byte of a group by the bits of its largest magnitude: 2^e is the smallest power of two under which that is at
// most 7 (6.x then rounds to 6 by no more than half of the last step), so 7 * 2^e = 1.75 * 2^(e + 2) is the line.  Against the
// exponent alone, which leaves up to 8 to end at 6, and against a line at 6, N(0, 1) in bf16 loses 0.112 of its rms where those lose 0.115.
// The end of the range: values down to 2^-125 stay normal, and the largest finite ones end at 6 * 2^125.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    if (top >= 0x7f800000u) return kScaleNaN;
    const int ex = (int)(top >> 23) - 2;                              // e + 127
    uint32_t byte = ex < (int)kScaleMin ? kScaleMin : (uint32_t)ex;
    byte += top > (((byte + 2u) << 23) | 0x600000u) ? 1u : 0u;
    return byte < kScaleMax ? byte : kScaleMax;
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight codes, channel 0 in the low nibble, from eight values of one group
__device__ __forceinline__ uint32_t encode8(const float *f, float scale)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0], f[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2], f[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4], f[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6], f[7], scale, 3);
    return r;
}
// and back: eight bf16 values (exact)
__device__ __forceinline__ uint4 decode8_bf16(uint32_t code, float scale)
{
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
    return r;
}

// Rows of `src` into the packed cache `p` (see specpv_pack_tokens).  src.ctx_len bounds the source rows; p.s.ctx_len is not read.
struct PackArgs {
    const int32_t *src_begin, *src_rows, *n_rows, *dst_begin;
    int max_rows;
    void *kmax, *kmin;
};
hipError_t launch_pack(const Shape &src, int dtype, const PackedShape &p, const PackArgs &a, hipStream_t st);
hipError_t launch_packed_gather(const PackedShape &p, int dtype, const int32_t *sel_idx, const int32_t *sel_count, int n_sel,
                                void *out_k, void *out_v, int32_t *out_len, hipStream_t st);


// Context part of the attention (packed_attn.hip): part.nsplit splits of row tiles of 16 or 32.
// Whether a chunk's 32 tokens follow each other: the whole cache, or blocks of whole chunks (rows no more than 2^26 bytes apart).
static inline bool packed_runs(const Shape &s, bool lists) { return (!lists || s.B % 32 == 0) && s.st < ((int64_t)1 << 26); }
// Tiles of 16 rows where one is enough (one query token, 16 / 32, us: 16K tokens 12.1 / 13.7, 128K 30.8 / 37.1; 32 rows as two of them: 16K 13.0 /
// 13.1, 128K 39.1 / 39.7).  (fp32 at 128 channels has registers for 16 rows' three operands only)
static inline int packed_row_tile(const Shape &s, int dtype) { return s.M * s.G <= 16 || (dtype == SPECPV_F32 && s.D == 128) ? 16 : 32; }
static inline int packed_row_tiles(const Shape &s, int dtype) { return (s.M * s.G + packed_row_tile(s, dtype) - 1) / packed_row_tile(s, dtype); }
hipError_t launch_packed_attn(const PackedShape &p, int dtype, const int32_t *sel_idx, const int32_t *sel_count, int n_sel, Partials part,
                              int waves, hipStream_t st);   // waves: 8, or (tiles of 32 rows, and fp32) 4

}  // namespace specpv
