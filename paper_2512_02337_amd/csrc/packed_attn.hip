// Context part of the verify attention over the 4-bit cache (specpv_packed_verify_attn): split-KV partials in the form that
// the combine kernel merges with the draft-tree segment.
//
// A cached value is exact in bf16, so the products are those of the bf16 kernels: S^T = K . Q^T and O^T += V^T . P^T by
// v_mfma_f32_32x32x16_bf16, 32 query rows (columns) a wavefront and 32 tokens a chunk, a running maximum and sum per column.
// A wavefront works for itself: the K codes of a chunk are its A operand as they come from memory (a lane holds half of a
// token's row; which channels a step of the product takes does not matter as long as Q's are the same), V goes through a
// piece of LDS of its own as bf16, because its operand has tokens where memory has channels: the transposing LDS reads turn it.
// The next two chunks' codes, 35 bytes a lane each, are under way while one is worked on.
#include "packed.h"
#include "attn_mfma.h"

namespace specpv {

typedef __attribute__((ext_vector_type(4))) short i16x4;

struct PackedAttnArgs {
    PackedShape p;
    Partials part;
    const int32_t *sel_idx, *sel_count;
    int n_sel, row_tiles;
    FastDiv div_B, div_hkv, div_M, div_tiles;
    float scale_log2;
};

constexpr int kPackedWaves = 4;

// One or three bf16 operands whose sum is the value: fp32 has 24 significant bits, bf16 8.
template <typename T> struct Pieces { static constexpr int N = sizeof(T) == 2 ? 1 : 3; };

// Which tokens a chunk has.  RUN: they follow each other in memory (the whole cache, or blocks of whole chunks): a scalar row and a
// count.  Else (blocks of other sizes) a lane looks its token up.
template <bool RUN> struct ChunkTokens;
template <> struct ChunkTokens<true> { int row; };
template <> struct ChunkTokens<false> { int tok; };

template <typename T, int D, bool RUN>
__global__ __launch_bounds__(64 * kPackedWaves, 2) void packed_attn_kernel(PackedAttnArgs a)
{
    constexpr int N = Pieces<T>::N, STEPS = D / 16, GROUPS = D / 32, TILES = D / 32, VLOADS = D / 64;
    constexpr int RING = N == 1 ? 3 : 2;              // chunks in registers: this one and those under way
    constexpr int VROW = D * 2;                       // bytes of a V row in LDS
    __shared__ __align__(16) char lds[kPackedWaves][32 * VROW];
    __shared__ float2 ml_lds[kPackedWaves][64];
    const Shape &s = a.p.s;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int bg = blockIdx.x, b = (int)a.div_hkv.div((uint32_t)bg), g = bg - b * s.Hkv;
    const int split = (int)a.div_tiles.div(blockIdx.y), tile = (int)blockIdx.y - split * a.row_tiles;
    const int R = s.M * s.G, r = tile * 32 + col;
    const bool row_live = r < R;
    const int64_t cap = (int64_t)s.max_blocks * s.B;
    const int L = (int)min((int64_t)max(s.ctx_len[b], 0), cap);
    const int nb = (int)a.div_B.div((uint32_t)L + (uint32_t)s.B - 1u);
    int span = L;
    if (a.sel_idx) span = L ? max(min(a.sel_count[bg], a.n_sel), 0) * s.B : 0;
    const int chunks = (int)(((uint32_t)span + 31u) >> 5);
    const int c0 = (int)((int64_t)chunks * split / a.part.nsplit), c1 = (int)((int64_t)chunks * (split + 1) / a.part.nsplit);

    // ---- query rows: the B operand of step i is channels 32 * (half * GROUPS / 2 + i / 4) + 8 * (i & 3) .. + 7 ----
    bf16x8 q[N][STEPS];
    {
        const int rr = min(r, R - 1), hh = (int)a.div_M.div((uint32_t)rr), j = rr - hh * s.M;
        const T *row = (const T *)s.q + (((int64_t)b * s.M + j) * s.Hq + (int64_t)g * s.G + hh) * D + half * (D / 2);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if constexpr (N == 1) {
                q[0][i] = __builtin_bit_cast(bf16x8, *(const uint4 *)(row + 8 * i));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float f = row[8 * i + e];
#pragma unroll
                    for (int n = 0; n < N; ++n) { q[n][i][e] = (__bf16)f; f -= (float)q[n][i][e]; }
                }
            }
        }
    }

    // ---- where this lane's V loads come from and go to ----
    // D = 128: lanes 4 u .. 4 u + 3 a token's four groups, 16 lanes tokens 0, 4, 8, 12 (+ lane / 16, + 16 x); D = 64: two
    // groups, 16 lanes 8 tokens in a row.  In LDS a row's 64-byte units and their 16-byte pieces are permuted by the token, so that
    // the 16 lanes of a write cover all banks, and so do the four rows of 64 bytes that half a wavefront's transposing read takes.
    auto v_token = [&](int x) { return D == 128 ? 4 * ((lane >> 2) & 3) + (lane >> 4) + 16 * x : lane >> 1; };
    auto v_place = [&](int t, int unit, int piece) {   // byte of a 16-byte piece
        return D == 128 ? t * VROW + ((unit ^ (t & 3)) << 6) + ((piece ^ ((t >> 2) & 3)) << 4)
                        : t * VROW + ((unit ^ ((t >> 1) & 1)) << 6) + ((piece ^ ((t >> 1) & 3)) << 4);
    };
    const int v_group = lane & (GROUPS - 1);
    char *const mine = lds[wave];

    const int64_t base = (int64_t)b * s.sb + (int64_t)g * s.sh;
    const uint8_t *const kc = (const uint8_t *)s.k + base, *const vc = (const uint8_t *)s.v + base;
    const uint8_t *const ksc = a.p.ks + (base >> 4), *const vsc = a.p.vs + (base >> 4);
    const int32_t *const list = a.sel_idx ? a.sel_idx + (int64_t)bg * a.n_sel : nullptr;
    const uint32_t k_lane = (uint32_t)half * (D / 4), v_lane = (uint32_t)v_group * 16, ks_lane = (uint32_t)half * (GROUPS / 2), vs_lane = (uint32_t)v_group;

    typedef ChunkTokens<RUN> Tokens;
    auto tokens_of = [&](int c) {   // of chunk c < c1 (behind it: of the last one once more)
        Tokens x;
        c = min(c, c1 - 1);
        if constexpr (RUN) {
            x.row = 32 * c;
            if (list) {
                const int slot = (int)a.div_B.div((uint32_t)(32 * c)), e = list[slot];
                x.row = e >= 0 && e < nb ? e * s.B + (32 * c - slot * s.B) : -1;
            }
        } else {
            const int p = 32 * c + col;
            x.tok = -1;
            if (p < span) {
                x.tok = p;
                if (list) {
                    const int slot = (int)a.div_B.div((uint32_t)p), e = list[slot];
                    x.tok = e >= 0 && e < nb ? e * s.B + (p - slot * s.B) : -1;
                }
            }
        }
        return x;
    };
    struct Codes {
        uint4 k[GROUPS / 2], v[VLOADS];
        uint32_t ks, vs[VLOADS];
        uint32_t live;       // bit t: token t of the chunk counts
    };
    // Tokens that are not there are read as another of the chunk, which is; a chunk of none as token 0, and is then left out.
    auto fetch = [&](const Tokens &tk, Codes &x) __attribute__((always_inline)) {
        if constexpr (RUN) {
            const int n = tk.row < 0 ? 0 : min(max(L - tk.row, 0), 32);
            x.live = n >= 32 ? 0xffffffffu : (1u << n) - 1u;
            const int row = n > 0 ? tk.row : 0, last = n > 0 ? n - 1 : 0;
            const int64_t at = (int64_t)row * s.st;
            const uint8_t *const k0 = kc + at, *const v0 = vc + at, *const ks0 = ksc + (at >> 4), *const vs0 = vsc + (at >> 4);
            const uint32_t st = (uint32_t)s.st;   // (32 rows lie within 2^31 bytes: launch_packed_attn)
            const uint32_t ko = (uint32_t)min(col, last) * st;
#pragma unroll
            for (int i = 0; i < GROUPS / 2; ++i) x.k[i] = *(const uint4 *)(k0 + (ko + k_lane + 16 * i));
            if constexpr (D == 128) x.ks = *(const uint16_t *)(ks0 + ((ko >> 4) + ks_lane));
            else x.ks = ks0[(ko >> 4) + ks_lane];
#pragma unroll
            for (int i = 0; i < VLOADS; ++i) {
                const uint32_t vo = (uint32_t)min(v_token(i), last) * st;
                x.v[i] = *(const uint4 *)(v0 + (vo + v_lane));
                x.vs[i] = vs0[(vo >> 4) + vs_lane];
            }
        } else {
            const bool there = tk.tok >= 0 && tk.tok < L;
            const unsigned long long who = __ballot(there);
            x.live = (uint32_t)who;
            const int tok = there ? tk.tok : (who ? __builtin_amdgcn_readlane(tk.tok, __builtin_ctzll(who)) : 0);
            const int64_t o = (int64_t)tok * s.st;
#pragma unroll
            for (int i = 0; i < GROUPS / 2; ++i) x.k[i] = *(const uint4 *)(kc + o + k_lane + 16 * i);
            if constexpr (D == 128) x.ks = *(const uint16_t *)(ksc + (o >> 4) + ks_lane);
            else x.ks = ksc[(o >> 4) + ks_lane];
#pragma unroll
            for (int i = 0; i < VLOADS; ++i) {
                const int64_t vo = (int64_t)__shfl(tok, v_token(i)) * s.st;
                x.v[i] = *(const uint4 *)(vc + vo + v_lane);
                x.vs[i] = vsc[(vo >> 4) + vs_lane];
            }
        }
    };

    f32x16 O[TILES];
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[j][i] = 0.f;
    RowState st;

    // the lane's addresses for the transposing reads: token 4 half + (lane & 15) / 4 of eight, its 4 channels of tile j
    uint32_t v_at[2][TILES];
    {
        const int sl = lane & 15, grp = (lane >> 4) & 1;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                const int t = 8 * hf + 4 * half + (sl >> 2), byte = 32 * grp + 8 * (sl & 3);
                v_at[hf][j] = (uint32_t)(v_place(t, j, byte >> 4) + (byte & 15));
            }
    }
    typedef __attribute__((address_space(3))) i16x4 *lds_i16x4;

    auto work = [&](const Codes &x) __attribute__((always_inline)) {
        if (x.live == 0) return;
        // V as bf16 into LDS
#pragma unroll
        for (int i = 0; i < VLOADS; ++i) {
            const int t = v_token(i);
            const float sc = scale_of(x.vs[i]);
            const uint32_t w[4] = {x.v[i].x, x.v[i].y, x.v[i].z, x.v[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) *(uint4 *)(mine + v_place(t, v_group, e)) = decode8_bf16(w[e], sc);
        }
        f32x16 S;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const uint4 c4 = x.k[i >> 2];
            const uint32_t w = (i & 3) == 0 ? c4.x : ((i & 3) == 1 ? c4.y : ((i & 3) == 2 ? c4.z : c4.w));
            const float sc = scale_of((i >> 2) ? x.ks >> 8 : x.ks & 0xffu);
            const bf16x8 kf = __builtin_bit_cast(bf16x8, decode8_bf16(w, sc));
#pragma unroll
            for (int n = 0; n < N; ++n) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[n][i], S, 0, 0, 0);
        }
        mask_scores(x.live, half, S);
        follow_max(tile_max(S), a.scale_log2, st, O);
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = __builtin_amdgcn_exp2f(fmaf(S[i], a.scale_log2, st.neg_ref));
        // (the sum of the weights themselves, not of the rounded ones: the log-sum-exp is an output in 32 bits)
        float sum[4] = {S[0], S[1], S[2], S[3]};
#pragma unroll
        for (int i = 4; i < 16; ++i) sum[i & 3] += S[i];
        st.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 pf[N];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float f = S[8 * ks + e];
#pragma unroll
                for (int n = 0; n < N; ++n) { pf[n][e] = (__bf16)f; f -= (float)pf[n][e]; }
            }
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(mine + v_at[0][j] + ks * 16 * VROW));
                const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(mine + v_at[1][j] + ks * 16 * VROW));
                const auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int n = 0; n < N; ++n) O[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), pf[n], O[j], 0, 0, 0);
            }
        }
    };

    if (c0 + wave < c1) {
        Codes ring[RING];
        int c = c0 + wave;
#pragma unroll
        for (int x = 0; x < RING - 1; ++x) fetch(tokens_of(c + x * kPackedWaves), ring[x]);
        Tokens next = tokens_of(c + (RING - 1) * kPackedWaves);
        for (;;) {
            bool done = false;
#pragma unroll
            for (int x = 0; x < RING; ++x) {   // (in turn, so that no registers move)
                const Tokens now = next;
                next = tokens_of(c + RING * kPackedWaves);
                fetch(now, ring[(x + RING - 1) % RING]);
                work(ring[x]);
                c += kPackedWaves;
                if (c >= c1) { done = true; break; }
            }
            if (done) break;
        }
    }
    float l = sum_xor32(st.l), m = l != 0.f ? -st.neg_ref : -INFINITY;   // (l may be NaN)

    // ---- the wavefronts' results into one: 2 and 3 into 0 and 1, then 1 into 0 ----
    constexpr int kParts = TILES * 16;   // values of a lane
    float *const room = (float *)lds;    // [2][kParts][64]
    static_assert(2 * kParts * 64 * 4 <= (int)sizeof(lds), "room for two wavefronts' results");
#pragma unroll
    for (int n = kPackedWaves / 2; n > 0; n >>= 1) {
        __syncthreads();
        if (wave >= n && wave < 2 * n) {
            ml_lds[wave - n][lane] = make_float2(m, l);
#pragma unroll
            for (int j = 0; j < TILES; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) room[((wave - n) * kParts + j * 16 + i) * 64 + lane] = O[j][i];
        }
        __syncthreads();
        if (wave < n) {
            const float2 o = ml_lds[wave][lane];
            const float m_new = fmaxf(m, o.x), ref = m_new == -INFINITY ? 0.f : m_new;
            const float w0 = __builtin_amdgcn_exp2f(m - ref), w1 = __builtin_amdgcn_exp2f(o.x - ref);
            l = l * w0 + o.y * w1;
            m = m_new;
#pragma unroll
            for (int j = 0; j < TILES; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[j][i] = O[j][i] * w0 + room[(wave * kParts + j * 16 + i) * 64 + lane] * w1;
        }
    }
    if (wave || !row_live) return;
    const int64_t prow = ((int64_t)bg * a.part.nsplit + split) * R + r;
    // (the combine kernel takes a partial by l > 0: a sum that is no number is handed on in the maximum's place)
    if (half == 0) ((float2 *)a.part.ml)[prow] = l == l ? make_float2(m, l) : make_float2(l, 1.f);
    if (a.part.o_half) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
        typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
        _Float16 *out = (_Float16 *)a.part.o + prow * D;
#pragma unroll
        for (int j = 0; j < TILES; ++j)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                f16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float o = O[j][i + e] * inv;
                    v[e] = (_Float16)(o > 65504.f ? 65504.f : (o < -65504.f ? -65504.f : o));   // (NaN stays)
                }
                *(f16x4 *)(out + 32 * j + 8 * (i >> 2) + 4 * half) = v;
            }
    } else {
        float *out = a.part.o + prow * D;
#pragma unroll
        for (int j = 0; j < TILES; ++j)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(float4 *)(out + partial_pos(32 * j + 8 * (i >> 2) + 4 * half, D)) = make_float4(O[j][i], O[j][i + 1], O[j][i + 2], O[j][i + 3]);
    }
}

hipError_t launch_packed_attn(const PackedShape &p, int dtype, const int32_t *sel_idx, const int32_t *sel_count, int n_sel, Partials part, hipStream_t st)
{
    const Shape &s = p.s;
    const int tiles = packed_row_tiles(s);
    const PackedAttnArgs a{p, part, sel_idx, sel_count, n_sel, tiles, make_fastdiv((uint32_t)s.B), make_fastdiv((uint32_t)s.Hkv),
                           make_fastdiv((uint32_t)s.M), make_fastdiv((uint32_t)tiles), kLog2e / sqrtf((float)s.D)};
    const dim3 grid(s.batch * s.Hkv, tiles * part.nsplit);
    const bool run = (!sel_idx || s.B % 32 == 0) && s.st < ((int64_t)1 << 26);
#define SPECPV_ATTN(T, DD)                                                                                             \
    do {                                                                                                               \
        if (run) hipLaunchKernelGGL((packed_attn_kernel<T, DD, true>), grid, dim3(64 * kPackedWaves), 0, st, a);       \
        else hipLaunchKernelGGL((packed_attn_kernel<T, DD, false>), grid, dim3(64 * kPackedWaves), 0, st, a);          \
    } while (0)
    if (dtype == SPECPV_BF16) {
        if (s.D == 128) SPECPV_ATTN(bf16_t, 128); else SPECPV_ATTN(bf16_t, 64);
    } else {
        if (s.D == 128) SPECPV_ATTN(float, 128); else SPECPV_ATTN(float, 64);
    }
#undef SPECPV_ATTN
    return hipGetLastError();
}

}  // namespace specpv
