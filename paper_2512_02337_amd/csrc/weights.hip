// Accumulated attention weights: for each cached token the weight that a pass's query rows gave it, summed over the rows,
// added to what earlier passes gave it (specpv_accumulate_weights).
//
// With the pass's log-sum-exp at hand a weight is one exponential, exp(q . k / sqrt(D) - lse), and nothing has to be merged:
// a wavefront keeps its tokens' K rows in registers as the matrix instruction's A operand (rows = tokens), the query rows go
// by as B (columns), 32 at a time out of LDS, and a lane adds up its column's weights for 16 tokens a tile.  The 32 columns
// are folded once, at the end.  K is read once and nothing else of size is read or written: few rows are bound by that (16 rows over
// 8 heads of 128K, bf16, 268 MB: 53.3 us, 5.0 TB/s), many by products, exponentials and LDS reads together (512 rows over 32K: 46 - 50 us, 690 -
// 740 TFLOP/s; without the exponentials a workgroup takes 77 % of its cycles, without the products 86, without the LDS reads 82).
#include "summarize.h"

namespace specpv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

struct WeighKernelArgs {
    Shape s;
    WeighArgs a;
    FastDiv div_B, div_G;
    float scale_log2, scale_off;   // log2 e / sqrt(D), and by what part of itself it is too small
};

template <typename T> struct Mfma32;
template <> struct Mfma32<bf16_t> {   // 16 channels a step: a lane's 16 bytes are its half of them
    static __device__ __forceinline__ f32x16 step(const uint4 &k, const uint4 &q, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
    }
};
template <> struct Mfma32<float> {    // 8 channels a step, in four products of two
    static __device__ __forceinline__ f32x16 step(const uint4 &k, const uint4 &q, f32x16 c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.x), __uint_as_float(q.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.y), __uint_as_float(q.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.z), __uint_as_float(q.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.w), __uint_as_float(q.w), c, 0, 0, 0);
    }
};

// Sums over the 32 lanes of a half wavefront of sixteen values: lane l (of a half) ends up with the sum of value
// 8 * bit 0 + 4 * bit 1 + 2 * bit 2 + bit 3 of l.  Each exchange halves the values that a lane still has to do with.
template <int CTRL> __device__ __forceinline__ float dpp_any(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float fold32(const float (&v)[16], int lane)
{
    float a[8], b[4], c[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = ((lane & 1) ? v[i + 8] : v[i]) + dpp_any<0xB1>((lane & 1) ? v[i] : v[i + 8]);
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = ((lane & 2) ? a[i + 4] : a[i]) + dpp_any<0x4E>((lane & 2) ? a[i] : a[i + 4]);
#pragma unroll
    for (int i = 0; i < 2; ++i) c[i] = ((lane & 4) ? b[i + 2] : b[i]) + __shfl_xor((lane & 4) ? b[i] : b[i + 2], 4);
    float d = ((lane & 8) ? c[1] : c[0]) + __shfl_xor((lane & 8) ? c[0] : c[1], 8);
    return d + __shfl_xor(d, 16);
}

// A workgroup has WAVES wavefronts, SPLIT of them to each 32 tokens, which share the tiles of query rows between them (launch_weigh).  A
// stage's query rows are found and fetched by all of its threads, on their way to registers while the stage before is worked on; what rows
// cost is the less, the more wavefronts they are fetched for.
template <typename T, int D, int WAVES, int SPLIT> struct WeighTile {
    static constexpr int E = Elem<T>::kPerVec, STEPS = D / (2 * E);        // channels of a lane's 16 bytes; products of a tile
    static constexpr int PIECES = D / E;                                   // 16-byte pieces of a row
    static constexpr int MINE = SPLIT > 1 ? SPLIT * PIECES / (2 * WAVES) : (PIECES == 32 ? 4 : 2);   // pieces of a stage that a thread brings
    static constexpr int ROWS = MINE * 64 * WAVES / PIECES;                // query rows of a stage
    static_assert(ROWS % (32 * SPLIT) == 0, "whole tiles");
    // so that the 16 lanes that LDS serves at a time find their pieces in different banks
    static __device__ __forceinline__ int place(int row, int piece)
    {
        return row * PIECES + (PIECES >= 16 ? piece ^ (row & 15) : piece ^ ((row >> 1) & 7));
    }
};

template <typename T, int D, int WAVES, int SPLIT, bool LISTS>
__global__ __launch_bounds__(64 * WAVES) void weigh_kernel(WeighKernelArgs k)
{
    typedef WeighTile<T, D, WAVES, SPLIT> W;
    constexpr int STEPS = W::STEPS, THREADS = 64 * WAVES;
    __shared__ uint4 q_lds[2][W::ROWS * W::PIECES];
    __shared__ float2 lse_lds[2][W::ROWS];   // -lse * log2 e, and what that is off by, as a factor (below); (-inf, 0): a row that gives nothing
    const Shape &s = k.s;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.y, b = blockIdx.z, half = lane >> 5, col = lane & 31;
    const int64_t bg = (int64_t)b * s.Hkv + g;
    const int64_t cap = (int64_t)s.max_blocks * s.B;
    const int L = (int)min((int64_t)max(s.ctx_len[b], 0), cap);
    const int nb = (int)k.div_B.div((uint32_t)L + (uint32_t)s.B - 1u);
    int span = L;   // positions that there are
    if (LISTS) span = max(min(k.a.sel_count[bg], k.a.n_sel), 0) * s.B;
    const int p0 = (int)blockIdx.x * (WAVES / SPLIT * 32);
    if (p0 >= span || L == 0) return;
    // ---- the wavefront's K rows ----
    int tok = -1;
    uint4 kk[STEPS];
    {
        const int p = p0 + wave / SPLIT * 32 + col;
        if (p < span) {
            tok = p;
            if (LISTS) {
                const int slot = (int)k.div_B.div((uint32_t)p), e = k.a.sel_idx[bg * k.a.n_sel + slot];
                tok = e >= 0 && e < nb ? e * s.B + (p - slot * s.B) : -1;
            }
            if (tok >= L) tok = -1;
        }
        const char *row = (const char *)s.k + ((int64_t)b * s.sb + (int64_t)g * s.sh + (int64_t)max(tok, 0) * s.st) * (int64_t)sizeof(T) + 16 * half;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) kk[i] = *(const uint4 *)(row + 32 * i);   // (a token that is not there: the first one, for nothing)
    }
    // ---- query rows r0 .. r0 + ROWS - 1: this thread's pieces, and the sums of the rows whose first pieces they are ----
    const int nodes = k.a.nodes ? min(k.a.n_nodes[b], k.a.max_nodes) : s.M;
    const int R = max(nodes, 0) * s.G;
    // A weight is 2^x, x = z - lse * log2 e, and large where the two nearly cancel: what either is off by from its rounding is then larger than x's own
    // error.  The product with lse comes in two parts, and z = scale_log2 * (1 + scale_off) * q . k is -lse * log2 e's opposite but for x: both
    // offsets are a factor of the row, which the sums take in without another instruction.
    uint4 qp[W::MINE];
    float2 neg[W::MINE];
    auto row_of = [&](float l) {
        const float n = l * -kLog2e, low = fmaf(l, -kLog2e, -n) - l * 1.925963033500011e-8f;   // (log2 e itself less kLog2e)
        if (l == -INFINITY) return make_float2(-INFINITY, 0.f);                                  // (a row that attended nothing gives nothing)
        return make_float2(n, fabsf(n) < 1e6f ? fmaf(0.693147181f, low - k.scale_off * n, 1.f) : 1.f);   // (beyond, nothing cancels)
    };
    auto fetch = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < W::MINE; ++x) {
            const int at = (int)threadIdx.x + x * THREADS, row = r0 + at / W::PIECES, piece = at % W::PIECES;
            qp[x] = make_uint4(0, 0, 0, 0);
            neg[x] = make_float2(-INFINITY, 0.f);
            if (row < R) {
                const int i = (int)k.div_G.div((uint32_t)row), hh = row - i * s.G;
                const int node = k.a.nodes ? k.a.nodes[(int64_t)b * k.a.max_nodes + i] : i;
                if (node >= 0 && node < s.M) {
                    const int64_t qr = ((int64_t)b * s.M + node) * s.Hq + (int64_t)g * s.G + hh;
                    qp[x] = ((const uint4 *)s.q)[qr * W::PIECES + piece];
                    if (piece == 0) neg[x] = row_of(k.a.lse[qr]);
                }
            }
        }
    };
    float sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    fetch(0);
    for (int r0 = 0, buf = 0; r0 < R; r0 += W::ROWS, buf ^= 1) {
#pragma unroll
        for (int x = 0; x < W::MINE; ++x) {
            const int at = (int)threadIdx.x + x * THREADS, row = at / W::PIECES, piece = at % W::PIECES;
            q_lds[buf][W::place(row, piece)] = qp[x];
            if (piece == 0) lse_lds[buf][row] = neg[x];
        }
        if (r0 + W::ROWS < R) fetch(r0 + W::ROWS);
        // (LDS only.  One meeting a stage: whoever writes a buffer again has met those that have read it)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        const int rows = min(W::ROWS, R - r0);
        for (int t0 = wave % SPLIT * 32; t0 < rows; t0 += 32 * SPLIT) {
            f32x16 sc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) sc = Mfma32<T>::step(kk[i], q_lds[buf][W::place(t0 + col, 2 * i + half)], sc);
            const float2 n = lse_lds[buf][t0 + col];
            // Columns that give nothing: products with an infinite key, or of a query row that is no number, are none either.  (Only in tiles
            // that have such columns.  Without / with: 512 rows over 32K, 47.8 / 48.0 us, 16 over 128K, half a tile, 52.8 / 53.5.)
            if (__any(n.y == 0.f)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = n.y == 0.f ? 0.f : sc[i];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = fmaf(__builtin_amdgcn_exp2f(fmaf(sc[i], k.scale_log2, n.x)), n.y, sum[i]);
        }
    }
    // ---- fold the columns; value i of a tile is its token 8 * (i >> 2) + 4 * half + (i & 3) ----
    float w = fold32(sum, lane);
    if constexpr (SPLIT > 1) {   // the shares of the wavefronts that have the same tokens, in their order
        __shared__ float shares[WAVES][64];
        shares[wave][lane] = w;
        __syncthreads();
        if (wave % SPLIT) return;
#pragma unroll
        for (int x = 1; x < SPLIT; ++x) w += shares[wave + x][lane];
    }
    const int i = ((lane & 1) << 3) | ((lane & 2) << 1) | ((lane & 4) >> 1) | ((lane & 8) >> 3);
    const int t = __shfl(tok, 8 * (i >> 2) + 4 * half + (i & 3));
    if ((lane & 16) || t < 0) return;
    float *to = k.a.weights + bg * cap + t;
    // (a block that is listed m times is added to m times, by the same amount each: the order changes nothing)
    if (LISTS) unsafeAtomicAdd(to, w);
    else *to += w;
}

hipError_t launch_weigh(const Shape &s, int dtype, const WeighArgs &a, hipStream_t st)
{
    const double scale = 1.4426950408889634 / sqrt((double)s.D);
    const WeighKernelArgs k{s, a, make_fastdiv((uint32_t)s.B), make_fastdiv((uint32_t)s.G), (float)scale, (float)(scale / (float)scale - 1.)};
    const int64_t positions = (a.sel_idx ? (int64_t)a.n_sel : (int64_t)s.max_blocks) * s.B;
    if (positions <= 0) return hipSuccess;
    const int64_t rows = (int64_t)(a.nodes ? a.max_nodes : s.M) * s.G;
    // Eight wavefronts from 64 rows on where every CU gets tokens for eight, in bf16 from 192 rows on (there the rows themselves, brought by more
    // threads, are what matters).  (us, 8 KV heads, 4 / 8: bf16, 128 channels, 64 rows 2K 5.2 / 5.5, 4K 5.3 / 6.0, 8K 7.9 / 6.7, 128K 68.2 / 64.1;
    // 240 rows 2K 10.6 / 10.0, 8K 16.0 / 12.0, 32K 36.6 / 30.3; 480 rows 2K 23.4 / 18.3; 64 channels, 64 rows 2K 4.1 / 4.3, 8K 4.9 / 4.3,
    // 240 rows 64K 42.5 / 35.7; fp32, 128 channels, 64 rows 2K 11.9 / 15.6, 8K 18.7 / 17.8, 240 rows 2K 35.4 / 44.7, 8K 52.3 / 47.0; 64 channels, 240 rows
    // 8K 28.3 / 25.4.)  Sixteen for bf16 at 128 channels where every CU gets tokens for those (8 / 16: 128 rows, 8K 8.6 / 10.4, 16K 12.5 / 11.9; 240, 16K
    // 17.3 / 15.9, 32K 30.3 / 29.4; 480, 8K 18.9 / 21.5, 32K 48.9 / 45.1; 64 channels, 240, 64K 35.7 / 36.2; fp32, 64 channels, 128, 32K 46.9 / 47.9): one such
    // workgroup to a CU has nobody to compute while it reads its K rows, but reads each fragment of Q for sixteen.
    // Four wavefronts to the same 32 tokens from 96 rows on where a CU gets 64 tokens or less: a wavefront by itself would work on while most of the
    // chip has nothing to do (one to four of eight wavefronts: bf16, 128 channels, 2K, 52 rows 5.1 / 5.5, 112 6.9 / 6.1, 240 10.0 / 7.9, 480 18.4 / 14.4, 4K,
    // 240 11.3 / 17.2; 64 channels, 2K, 240 7.1 / 5.4; fp32, 128 channels, 2K, 52 11.4 / 11.5, 112 19.1 / 14.1, 240 35.8 / 22.7, 4K, 240 36.0 / 41.8).
    const int64_t each = positions * s.batch * s.Hkv / device_cu_count();   // tokens of a CU
    const bool wide = dtype == SPECPV_BF16 && s.D == 128 && rows >= 128 && each >= 512;
    const bool few = rows >= 96 && each <= 64;
    const bool many = (rows >= 64 && each >= 256) || (dtype == SPECPV_BF16 && rows >= 192);
#define SPECPV_WEIGH_L(T, DD, WAVES, SPLIT, LISTS)                                                                              \
    do {                                                                                                                 \
        const dim3 grid((unsigned)((positions + WAVES / SPLIT * 32 - 1) / (WAVES / SPLIT * 32)), s.Hkv, s.batch);                        \
        hipLaunchKernelGGL((weigh_kernel<T, DD, WAVES, SPLIT, LISTS>), grid, dim3(64 * WAVES), 0, st, k);                       \
    } while (0)
#define SPECPV_WEIGH_W(T, DD, WAVES, SPLIT) do { if (a.sel_idx) SPECPV_WEIGH_L(T, DD, WAVES, SPLIT, true); else SPECPV_WEIGH_L(T, DD, WAVES, SPLIT, false); } while (0)
#define SPECPV_WEIGH(T, DD)                                                                                              \
    do {                                                                                                                 \
        if constexpr (sizeof(T) == 2 && DD == 128) {                                                                     \
            if (wide) { SPECPV_WEIGH_W(T, DD, 16, 1); break; }                                                              \
        }                                                                                                                \
        if (few) SPECPV_WEIGH_W(T, DD, 8, 4); else if (many) SPECPV_WEIGH_W(T, DD, 8, 1); else SPECPV_WEIGH_W(T, DD, 4, 1);                                               \
    } while (0)
    if (dtype == SPECPV_BF16) {
        if (s.D == 128) SPECPV_WEIGH(bf16_t, 128); else SPECPV_WEIGH(bf16_t, 64);
    } else {
        if (s.D == 128) SPECPV_WEIGH(float, 128); else SPECPV_WEIGH(float, 64);
    }
#undef SPECPV_WEIGH
#undef SPECPV_WEIGH_W
#undef SPECPV_WEIGH_L
    return hipGetLastError();
}

}  // namespace specpv
