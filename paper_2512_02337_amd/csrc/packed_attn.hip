// Context part of the verify attention over the 4-bit cache (specpv_packed_verify_attn): split-KV partials in the form that
// the combine kernel merges with the draft-tree segment.
//
// A cached value is exact in bf16, so the products are those of the bf16 kernels: S^T = K . Q^T and O^T += V^T . P^T by
// v_mfma_f32_32x32x16_bf16, 32 query rows (columns) a wavefront and 32 tokens a chunk, a running maximum and sum per column.
// A wavefront works for itself: the K codes of a chunk are its A operand as they come from memory (a lane holds half of a
// token's row; which channels a step of the product takes does not matter as long as Q's are the same), V goes through a
// piece of LDS of its own as bf16, because its operand has tokens where memory has channels: the transposing LDS reads turn it.
// Bound by memory for few rows (one token over 8 heads of 128K, 142 MB: 25.2 us, 5.6 TB/s), by matrix and vector units at the clock that the
// chip's power leaves for many (78 over 64K: 105 us, 800 TFLOP/s at 1.55 GHz).
// The next chunk's codes, 68 bytes a lane at 128 channels, are under way while one is worked on.  (Two of them: 13.8 us for 12.9 over 32K tokens, 30.5 for
// 29.1 over 128K, 50.6 for 49.0 over 32 sequences of 8K: a split's end reads more for nothing, and there are wavefronts enough.)
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


// One or three bf16 operands whose sum is the value: fp32 has 24 significant bits, bf16 8.  Queries have all of theirs, the weights
// what they have in the ordinary calls: all 24 bits for fp32 and for bf16 at 64 channels (one operand / three: 60 query tokens x 4 heads over 32K,
// 8 KV heads, 30.4 / 44.0 us, one over 128K 18.3 / 20.0), bf16's 8 at 128 (one / two: 78 over 64K 109.8 / 142.2, 60 over a list of 4K 16.3 /
// 17.6, one over 128K 29.2 / 30.0; outputs off by 0.0023 / 0.0017 of their size, where their own rounding is 0.0017).
template <typename T, int D> struct Pieces { static constexpr int Q = sizeof(T) == 2 ? 1 : 3, W = sizeof(T) == 2 && D == 128 ? 1 : 3; };

// Which tokens a chunk has.  RUN: they follow each other in memory (the whole cache, or blocks of whole chunks): a scalar row and a
// count.  Else (blocks of other sizes) a lane looks its token up.
template <bool RUN> struct ChunkTokens;
template <> struct ChunkTokens<true> { int row; };
template <> struct ChunkTokens<false> { int tok; };

// Four adjacent channels of a partial's row (see Partials): sums, and the factor that normalises them.
__device__ __forceinline__ void store_partial(const Partials &part, int64_t row, int ch, int D, const float (&o)[4], float inv)
{
    if (part.o_half) {
        typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
        f16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = o[e] * inv;
            v[e] = (_Float16)(y > 65504.f ? 65504.f : (y < -65504.f ? -65504.f : y));   // (NaN stays)
        }
        *(f16x4 *)((_Float16 *)part.o + row * D + ch) = v;
    } else {
        *(float4 *)(part.o + row * D + partial_pos(ch, D)) = make_float4(o[0], o[1], o[2], o[3]);
    }
}

template <bool STREAM, typename V> __device__ __forceinline__ V load_codes(const V *p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    else return *p;
}

// RT query rows a wavefront.  32: v_mfma_f32_32x32x16, two lanes a column; 16: v_mfma_f32_16x16x32, four lanes a column, half of the
// registers and of the softmax, for few rows.  A column's lanes share the channels of the first product and the tokens of the second.
template <int RT, int D> struct RowTile;
template <int D> struct RowTile<32, D> {
    typedef f32x16 Acc;
    static constexpr int REGS = 16, KT = 1, VSTEPS = 2;
    static __device__ __forceinline__ Acc mfma(bf16x8 a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ int token(int, int i, int part) { return 8 * (i >> 2) + 4 * part + (i & 3); }   // of score register i
    static __device__ __forceinline__ float col_max(float x) { return max_xor32(x); }
    static __device__ __forceinline__ float col_sum(float x) { return sum_xor32(x); }
};
template <int D> struct RowTile<16, D> {
    typedef __attribute__((ext_vector_type(4))) float Acc;
    static constexpr int REGS = 4, KT = 2, VSTEPS = 1;
    static __device__ __forceinline__ Acc mfma(bf16x8 a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ int token(int kt, int i, int part) { return 16 * kt + 4 * part + i; }
    static __device__ __forceinline__ float xor16(float x, bool sum)
    {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return sum ? __uint_as_float(r[0]) + __uint_as_float(r[1]) : fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    static __device__ __forceinline__ float col_max(float x) { return max_xor32(xor16(x, false)); }
    static __device__ __forceinline__ float col_sum(float x) { return sum_xor32(xor16(x, true)); }
};

// SHARES: workgroup w has the chunks that are its share of all (sequence, KV head) pairs' (StreamShare), of one pair or of several.
template <typename T, int D, int RT, bool RUN, int WAVES, bool SHARES>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_attn_kernel(PackedAttnArgs a)
{
    typedef RowTile<RT, D> Tile;
    typedef typename Tile::Acc Acc;
    constexpr int N = Pieces<T, D>::Q, NW = Pieces<T, D>::W, GROUPS = D / 32, KT = Tile::KT, REGS = Tile::REGS;
    constexpr int PARTS = 64 / RT, SHARE = D / PARTS, STEPS = SHARE / 8;   // lanes of a column; their channels, and steps of the product
    constexpr int KWORDS = SHARE / 8;                 // 4-byte words of K codes of a lane and tile
    constexpr int OT = D / RT, VLOADS = D / 64;
    constexpr bool STREAM = RT == 16 && N == 1;       // codes past the caches: they are read once (one row tile)
    constexpr int VROW = D * 2;                       // bytes of a V row in LDS
    constexpr int VALUES = OT * REGS;                 // results of a lane
    constexpr int ROOM = 32 * VROW > VALUES * 256 ? 32 * VROW : VALUES * 256;
    __shared__ __align__(16) char lds[WAVES][ROOM];   // V rows of each wavefront; at the end their results
    __shared__ float2 ml_lds[WAVES][64];
    const Shape &s = a.p.s;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & (RT - 1), part = lane / RT;
    const int R = s.M * s.G;
    int x = 0, x1 = 0, seq_chunks = 0, seq_upto = 0;   // SHARES: chunks from here to there, in the row of all pairs' (and see StreamShare)
    if constexpr (SHARES) {
        const StreamShare sh(s, lane, a.part.stream);
        if ((int)blockIdx.x >= sh.wgs) return;
        x = sh.begin((int)blockIdx.x);
        x1 = sh.begin((int)blockIdx.x + 1);
        seq_chunks = sh.chunks;
        seq_upto = sh.upto;
    }
    do {   // (SHARES: pair by pair)
        int bg = blockIdx.x, b, g, tile = blockIdx.y, split = 0, c0, c1;
        int64_t slot;
        if constexpr (SHARES) {
            b = __builtin_ctzll(__ballot(lane < s.batch && seq_upto * s.Hkv > x));
            const int C = __builtin_amdgcn_readlane(seq_chunks, b), from = x - (__builtin_amdgcn_readlane(seq_upto, b) - C) * s.Hkv;
            g = (int)((uint32_t)from / (uint32_t)C);
            c0 = from - g * C;
            c1 = min(C, c0 + x1 - x);
            bg = b * s.Hkv + g;
            slot = (int64_t)blockIdx.x + bg;
        } else {
            b = (int)a.div_hkv.div((uint32_t)bg);
            g = bg - b * s.Hkv;
            split = (int)a.div_tiles.div(blockIdx.y);
            tile -= split * a.row_tiles;
            slot = (int64_t)bg * a.part.nsplit + split;
        }
        const int r = tile * RT + col;
        const bool row_live = r < R;
        const int L = (int)min((int64_t)max(s.ctx_len[b], 0), a.p.rows);   // (SHARES: chunks behind it have nothing)
        const int nb = (int)a.div_B.div((uint32_t)L + (uint32_t)s.B - 1u);
        int span = L;
        if (a.sel_idx) span = L ? max(min(a.sel_count[bg], a.n_sel), 0) * s.B : 0;
        if constexpr (!SHARES) {
            const int chunks = (int)(((uint32_t)span + 31u) >> 5);
            c0 = (int)((int64_t)chunks * split / a.part.nsplit);
            c1 = (int)((int64_t)chunks * (split + 1) / a.part.nsplit);
        }

        // ---- query rows: the B operand of step i is channels part * SHARE + 8 i .. + 7 ----
        bf16x8 q[N][STEPS];
        {
            const int rr = min(r, R - 1), hh = (int)a.div_M.div((uint32_t)rr), j = rr - hh * s.M;
            const T *row = (const T *)s.q + (((int64_t)b * s.M + j) * s.Hq + (int64_t)g * s.G + hh) * D + part * SHARE;
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
        // the 16 lanes of a write cover all banks, and so do the rows that half a wavefront's transposing read takes (RT = 32: four of
        // 64 bytes, RT = 16: eight of 32).
        auto v_token = [&](int x) { return D == 128 ? 4 * ((lane >> 2) & 3) + (lane >> 4) + 16 * x : lane >> 1; };
        auto v_place = [&](int t, int unit, int piece) {   // byte of a 16-byte piece
            const int u = t >> 2 & 3;
            return D == 128 ? t * VROW + ((unit ^ (t & 3)) << 6) + ((piece ^ ((u & 1) << 1 | u >> 1)) << 4)
                            : t * VROW + ((unit ^ ((t >> 1) & 1)) << 6) + ((piece ^ ((t >> 1) & 3)) << 4);
        };
        const int v_group = lane & (GROUPS - 1);
        char *const mine = lds[wave];

        const int64_t base = (int64_t)b * s.sb + (int64_t)g * s.sh;
        const uint8_t *const kc = (const uint8_t *)s.k + base, *const vc = (const uint8_t *)s.v + base;
        const uint8_t *const ksc = a.p.ks + (base >> 4), *const vsc = a.p.vs + (base >> 4);
        const int32_t *const list = a.sel_idx ? a.sel_idx + (int64_t)bg * a.n_sel : nullptr;
        const uint32_t k_lane = (uint32_t)part * (SHARE / 2), v_lane = (uint32_t)v_group * 16, ks_lane = (uint32_t)(part * SHARE) / 32, vs_lane = (uint32_t)v_group;

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
                const int p = 32 * c + (lane & 31);
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
            uint32_t k[KT][KWORDS], ks[KT];
            uint4 v[VLOADS];
            uint32_t vs[VLOADS];
            uint32_t live;       // bit t: token t of the chunk counts
        };
        auto k_words = [&](const uint8_t *p, uint32_t (&w)[KWORDS]) __attribute__((always_inline)) {
            if constexpr (KWORDS == 2) {
                const u32x2 u = load_codes<STREAM>((const u32x2 *)p);
                w[0] = u[0]; w[1] = u[1];
            } else {
#pragma unroll
                for (int i = 0; i < KWORDS; i += 4) {
                    const u32x4 u = load_codes<STREAM>((const u32x4 *)(p + 4 * i));
                    w[i] = u[0]; w[i + 1] = u[1]; w[i + 2] = u[2]; w[i + 3] = u[3];
                }
            }
        };
        auto k_scale = [&](const uint8_t *p) __attribute__((always_inline)) { return SHARE == 64 ? (uint32_t) * (const uint16_t *)p : (uint32_t)*p; };
        // Tokens that are not there are read as another of the chunk, which is; a chunk of none as token 0, and is then left out.
        auto fetch = [&](const Tokens &tk, Codes &x) __attribute__((always_inline)) {
            if constexpr (RUN) {
                const int n = tk.row < 0 ? 0 : min(max(L - tk.row, 0), 32);
                x.live = n >= 32 ? 0xffffffffu : (1u << n) - 1u;
                const int row = n > 0 ? tk.row : 0, last = n > 0 ? n - 1 : 0;
                const int64_t at = (int64_t)row * s.st;
                const uint8_t *const k0 = kc + at, *const v0 = vc + at, *const ks0 = ksc + (at >> 4), *const vs0 = vsc + (at >> 4);
                const uint32_t st = (uint32_t)s.st;   // (32 rows lie within 2^31 bytes: packed_runs)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const uint32_t ko = (uint32_t)min(col + RT * kt, last) * st;
                    k_words(k0 + (ko + k_lane), x.k[kt]);
                    x.ks[kt] = k_scale(ks0 + ((ko >> 4) + ks_lane));
                }
#pragma unroll
                for (int i = 0; i < VLOADS; ++i) {
                    const uint32_t vo = (uint32_t)min(v_token(i), last) * st;
                    x.v[i] = __builtin_bit_cast(uint4, load_codes<STREAM>((const u32x4 *)(v0 + (vo + v_lane))));
                    x.vs[i] = vs0[(vo >> 4) + vs_lane];
                }
            } else {
                const bool there = tk.tok >= 0 && tk.tok < L;
                const unsigned long long who = __ballot(there);
                x.live = (uint32_t)who;
                const int tok = there ? tk.tok : (who ? __builtin_amdgcn_readlane(tk.tok, __builtin_ctzll(who)) : 0);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const int64_t o = (int64_t)(KT == 1 ? tok : __shfl(tok, col + RT * kt)) * s.st;
                    k_words(kc + o + k_lane, x.k[kt]);
                    x.ks[kt] = k_scale(ksc + (o >> 4) + ks_lane);
                }
#pragma unroll
                for (int i = 0; i < VLOADS; ++i) {
                    const int64_t vo = (int64_t)__shfl(tok, v_token(i)) * s.st;
                    x.v[i] = __builtin_bit_cast(uint4, load_codes<STREAM>((const u32x4 *)(vc + vo + v_lane)));
                    x.vs[i] = vsc[(vo >> 4) + vs_lane];
                }
            }
        };

        Acc O[OT];
#pragma unroll
        for (int j = 0; j < OT; ++j)
#pragma unroll
            for (int i = 0; i < REGS; ++i) O[j][i] = 0.f;
        float neg_ref = 3e38f, sum_l = 0.f;   // minus the reference maximum, in log2 units; the lane's sum

        // the lane's addresses for the transposing reads: its token of the four that 16 lanes turn, its 4 channels of tile j
        uint32_t v_at[2][OT];
        {
            const int sl = lane & 15;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int j = 0; j < OT; ++j) {
                    const int t = (RT == 32 ? 8 : 16) * hf + 4 * part + (sl >> 2);
                    const int byte = 2 * RT * j + (RT == 32 ? 32 * ((lane >> 4) & 1) : 0) + 8 * (sl & 3);   // of the row
                    v_at[hf][j] = (uint32_t)(v_place(t, byte >> 6, (byte >> 4) & 3) + (byte & 15));
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
            Acc S[KT];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
                for (int i = 0; i < REGS; ++i) S[kt][i] = 0.f;
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    const float sc = scale_of(SHARE == 64 ? (i >> 2 ? x.ks[kt] >> 8 : x.ks[kt] & 0xffu) : x.ks[kt]);
                    const bf16x8 kf = __builtin_bit_cast(bf16x8, decode8_bf16(x.k[kt][i], sc));
#pragma unroll
                    for (int n = 0; n < N; ++n) S[kt] = Tile::mfma(kf, q[n][i], S[kt]);
                }
            }
            if (x.live != 0xffffffffu) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < REGS; ++i) S[kt][i] = x.live >> Tile::token(kt, i, part) & 1u ? S[kt][i] : -INFINITY;
            }
            // The reference maximum moves where the weights say that it has been left behind: one above 2^12 makes its lane's sum larger
            // than that (so does the first chunk's, by a reference of -3e38, and one that is no number).  No maximum is looked for elsewhere.
            float w[KT * REGS], sum;
            auto weigh = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < KT * REGS; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(S[i / REGS][i % REGS], a.scale_log2, neg_ref));
                // (the sum of the weights themselves, not of the rounded ones: the log-sum-exp is an output in 32 bits)
                float t[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
                for (int i = 4; i < KT * REGS; ++i) t[i & 3] += w[i];
                sum = (t[0] + t[1]) + (t[2] + t[3]);
            };
            weigh();
            if (__any(!(sum <= 4096.f))) {
                float top = S[0][0];
#pragma unroll
                for (int i = 1; i < KT * REGS; ++i) top = fmaxf(top, S[i / REGS][i % REGS]);
                const float z = Tile::col_max(top) * a.scale_log2, ref = -neg_ref, ref_new = z > ref ? z : ref;
                const float alpha = __builtin_amdgcn_exp2f(ref - ref_new);
                neg_ref = -ref_new;
                sum_l *= alpha;
#pragma unroll
                for (int j = 0; j < OT; ++j)
#pragma unroll
                    for (int i = 0; i < REGS; ++i) O[j][i] *= alpha;
                weigh();
            }
            sum_l += sum;
            const Bf16Halves halves;
#pragma unroll
            for (int ks = 0; ks < Tile::VSTEPS; ++ks) {
                uint32_t pk[NW][4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f0 = w[8 * ks + 2 * e], f1 = w[8 * ks + 2 * e + 1];
#pragma unroll
                    for (int n = 0; n < NW; ++n) {
                        pk[n][e] = pack_bf16x2(f0, f1);
                        if (n + 1 < NW) { f0 = halves.sub_lo(f0, pk[n][e]); f1 = halves.sub_hi(f1, pk[n][e]); }
                    }
                }
                bf16x8 pf[NW];
#pragma unroll
                for (int n = 0; n < NW; ++n) pf[n] = __builtin_bit_cast(bf16x8, make_uint4(pk[n][0], pk[n][1], pk[n][2], pk[n][3]));
#pragma unroll
                for (int j = 0; j < OT; ++j) {
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(mine + v_at[0][j] + ks * 16 * VROW));
                    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(mine + v_at[1][j] + ks * 16 * VROW));
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int n = 0; n < NW; ++n) O[j] = Tile::mfma(vf, pf[n], O[j]);
                }
            }
        };

        if (c0 + wave < c1) {
            Codes even, odd;   // (in turn, so that no registers move)
            int c = c0 + wave;
            fetch(tokens_of(c), even);
            Tokens next = tokens_of(c + WAVES);
            for (;;) {
                fetch(next, odd);
                next = tokens_of(c + 2 * WAVES);
                work(even);
                if ((c += WAVES) >= c1) break;
                fetch(next, even);
                next = tokens_of(c + 2 * WAVES);
                work(odd);
                if ((c += WAVES) >= c1) break;
            }
        }
        // ---- the wavefronts' results into one: all of them to LDS, and each wavefront merges and stores every so-manieth four channels ----
        float l = Tile::col_sum(sum_l), m = l != 0.f ? -neg_ref : -INFINITY;   // (l may be NaN)
        ml_lds[wave][lane] = make_float2(m, l);
        float4 *const own = (float4 *)lds[wave];     // [VALUES / 4][64]
#pragma unroll
        for (int i = 0; i < VALUES / 4; ++i) {
            const Acc &o = O[4 * i / REGS];
            own[i * 64 + lane] = make_float4(o[4 * i % REGS], o[4 * i % REGS + 1], o[4 * i % REGS + 2], o[4 * i % REGS + 3]);
        }
        __syncthreads();
        float wt[WAVES];
        m = -INFINITY;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) m = fmaxf(m, ml_lds[x][lane].x);
        const float ref = m == -INFINITY ? 0.f : m;
        l = 0.f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            const float2 o = ml_lds[x][lane];
            wt[x] = __builtin_amdgcn_exp2f(o.x - ref);
            l = fmaf(o.y, wt[x], l);
        }
        if (row_live) {
            const int64_t prow = slot * R + r;
            // (the combine kernel takes a partial by l > 0: a sum that is no number is handed on in the maximum's place)
            if (wave == 0 && part == 0) ((float2 *)a.part.ml)[prow] = l == l ? make_float2(m, l) : make_float2(l, 1.f);
            const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
            for (int i = 0; i < (VALUES / 4 + WAVES - 1) / WAVES; ++i) {
                const int at = i * WAVES + wave;
                if (at >= VALUES / 4) break;
                float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < WAVES; ++x) {
                    const float4 v = ((const float4 *)lds[x])[at * 64 + lane];
                    o[0] = fmaf(v.x, wt[x], o[0]); o[1] = fmaf(v.y, wt[x], o[1]); o[2] = fmaf(v.z, wt[x], o[2]); o[3] = fmaf(v.w, wt[x], o[3]);
                }
                const int ch = RT == 32 ? 32 * (at >> 2) + 8 * (at & 3) + 4 * part : 16 * at + 4 * part;   // four in a row
                store_partial(a.part, prow, ch, D, o, inv);
            }
        }
        if constexpr (SHARES) {
            x += c1 - c0;
            if (x >= x1) break;
            __syncthreads();   // (the results' places are wanted again)
        }
    } while (SHARES);
}

hipError_t launch_packed_attn(const PackedShape &p, int dtype, const int32_t *sel_idx, const int32_t *sel_count, int n_sel, Partials part,
                              int waves, hipStream_t st)
{
    const Shape &s = p.s;
    const bool run = packed_runs(s, sel_idx != nullptr);
    const int rt = packed_row_tile(s, dtype), tiles = packed_row_tiles(s, dtype);
    const PackedAttnArgs a{p, part, sel_idx, sel_count, n_sel, tiles, make_fastdiv((uint32_t)s.B), make_fastdiv((uint32_t)s.Hkv),
                           make_fastdiv((uint32_t)s.M), make_fastdiv((uint32_t)tiles), kLog2e / sqrtf((float)s.D)};
    const dim3 grid(part.stream ? part.stream : s.batch * s.Hkv, tiles * (part.stream ? 1 : part.nsplit));
#define SPECPV_ATTN_W(T, DD, R, RUN, WAVES, SHARES) \
    hipLaunchKernelGGL((packed_attn_kernel<T, DD, R, RUN, WAVES, SHARES>), grid, dim3(64 * WAVES), 0, st, a)
#define SPECPV_ATTN_S(T, DD, R, RUN)                                                                     \
    do {                                                                                                 \
        if constexpr (RUN) {                                                                             \
            if (part.stream) { SPECPV_ATTN_W(T, DD, R, true, 8, true); break; }                          \
        }                                                                                                \
        if constexpr (sizeof(T) == 4 || R == 32) {                                                       \
            if (waves == 4) { SPECPV_ATTN_W(T, DD, R, RUN, 4, false); break; }                           \
        }                                                                                                \
        SPECPV_ATTN_W(T, DD, R, RUN, 8, false);                                                          \
    } while (0)
#define SPECPV_ATTN_R(T, DD, RUN)                                                                        \
    do {                                                                                                 \
        if (rt == 16) SPECPV_ATTN_S(T, DD, 16, RUN);                                                     \
        else if constexpr (sizeof(T) == 2 || DD == 64) SPECPV_ATTN_S(T, DD, 32, RUN);                    \
    } while (0)
#define SPECPV_ATTN(T, DD) do { if (run) SPECPV_ATTN_R(T, DD, true); else SPECPV_ATTN_R(T, DD, false); } while (0)
    if (dtype == SPECPV_BF16) {
        if (s.D == 128) SPECPV_ATTN(bf16_t, 128); else SPECPV_ATTN(bf16_t, 64);
    } else {
        if (s.D == 128) SPECPV_ATTN(float, 128); else SPECPV_ATTN(float, 64);
    }
#undef SPECPV_ATTN
#undef SPECPV_ATTN_R
#undef SPECPV_ATTN_S
#undef SPECPV_ATTN_W
    return hipGetLastError();
}

}  // namespace specpv
