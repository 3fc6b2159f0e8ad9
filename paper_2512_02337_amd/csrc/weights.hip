// Accumulated attention weights: for each cached token the weight that a pass's query rows gave it, summed over the rows,
// added to what earlier passes gave it (specpv_accumulate_weights).
//
// With the pass's log-sum-exp at hand a weight is one exponential, exp(q . k / sqrt(D) - lse), and nothing has to be merged:
// a wavefront keeps its tokens' K rows in registers as the matrix instruction's A operand (rows = tokens), the query rows go
// by as B (columns), 32 at a time out of LDS, and a lane adds up its column's weights for 16 tokens a tile.  The 32 columns
// are folded once, at the end.  K is read once and nothing else of size is read or written.
#include "internal.h"
#include <type_traits>

namespace specpv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

struct WeighKernelArgs {
    Shape s;
    WeighArgs a;
    FastDiv div_B, div_G;
    float scale_log2;
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

constexpr int kWeighWaves = 4;
template <typename T, int D> struct WeighTile {
    static constexpr int E = Elem<T>::kPerVec, STEPS = D / (2 * E);        // channels of a lane's 16 bytes; products of a tile
    static constexpr int TILES = 1;              // tiles of 32 tokens of a wavefront: 64 registers of K
    static constexpr int PIECES = D / E;                                   // 16-byte pieces of a row
    static constexpr int ROWS = 32768 / (PIECES * 16);                     // query rows in LDS at a time
    // so that the 16 lanes that LDS serves at a time find their pieces in different banks
    static __device__ __forceinline__ int place(int row, int piece)
    {
        return row * PIECES + (PIECES >= 16 ? piece ^ (row & 15) : piece ^ ((row >> 1) & 7));
    }
};

template <typename T, int D, bool LISTS>
__global__ __launch_bounds__(64 * kWeighWaves, 2) void weigh_kernel(WeighKernelArgs k)
{
    typedef WeighTile<T, D> W;
    constexpr int E = W::E, STEPS = W::STEPS, TILES = W::TILES;
    __shared__ uint4 q_lds[W::ROWS * W::PIECES];
    __shared__ float lse_lds[W::ROWS];   // -lse * log2 e; -inf: no such row
    const Shape &s = k.s;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.y, b = blockIdx.z, half = lane >> 5, col = lane & 31;
    const int64_t bg = (int64_t)b * s.Hkv + g;
    const int64_t cap = (int64_t)s.max_blocks * s.B;
    const int L = (int)min((int64_t)max(s.ctx_len[b], 0), cap);
    const int nb = (int)k.div_B.div((uint32_t)L + (uint32_t)s.B - 1u);
    int cnt = 0, span = L;   // entries of the list; positions that there are
    if (LISTS) {
        cnt = min(k.a.sel_count[bg], k.a.n_sel);
        span = max(cnt, 0) * s.B;
    }
    const int p0 = (int)blockIdx.x * (kWeighWaves * 32 * TILES);
    if (p0 >= span) return;
    // ---- the wavefront's K rows ----
    int tok[TILES];
    uint4 kk[TILES][STEPS];
    const char *const k0 = (const char *)s.k + ((int64_t)b * s.sb + (int64_t)g * s.sh) * (int64_t)sizeof(T) + 16 * half;
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
        const int p = p0 + (wave * TILES + x) * 32 + col;
        tok[x] = -1;
        if (p < span) {
            tok[x] = p;
            if (LISTS) {
                const int slot = (int)k.div_B.div((uint32_t)p), e = k.a.sel_idx[bg * k.a.n_sel + slot];
                tok[x] = e >= 0 && e < nb ? e * s.B + (p - slot * s.B) : -1;
            }
            if (tok[x] >= L) tok[x] = -1;
        }
        if (tok[x] >= 0) {
            const char *row = k0 + (int64_t)tok[x] * s.st * (int64_t)sizeof(T);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) kk[x][i] = *(const uint4 *)(row + 32 * i);
        } else {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) kk[x][i] = make_uint4(0, 0, 0, 0);
        }
    }
    float sum[TILES][16];
#pragma unroll
    for (int x = 0; x < TILES; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[x][i] = 0.f;
    const int nodes = k.a.nodes ? min(k.a.n_nodes[b], k.a.max_nodes) : s.M;
    const int R = max(nodes, 0) * s.G;
    for (int r0 = 0; r0 < R; r0 += W::ROWS) {
        const int rows = min(W::ROWS, R - r0), padded = (rows + 31) & ~31;
        if (r0) __syncthreads();
        for (int at = threadIdx.x; at < padded * W::PIECES; at += 64 * kWeighWaves) {
            const int row = at / W::PIECES, piece = at % W::PIECES;
            uint4 v = make_uint4(0, 0, 0, 0);
            float neg = -INFINITY;
            if (row < rows) {
                const int i = (int)k.div_G.div((uint32_t)(r0 + row)), hh = r0 + row - i * s.G;
                const int node = k.a.nodes ? k.a.nodes[(int64_t)b * k.a.max_nodes + i] : i;
                if (node >= 0 && node < s.M) {
                    const int64_t qr = ((int64_t)b * s.M + node) * s.Hq + (int64_t)g * s.G + hh;
                    v = ((const uint4 *)s.q)[qr * W::PIECES + piece];
                    if (piece == 0) {
                        const float l = k.a.lse[qr];
                        neg = l == -INFINITY ? -INFINITY : l * -kLog2e;   // (a row that attended nothing gives nothing)
                    }
                }
            }
            q_lds[W::place(row, piece)] = v;
            if (piece == 0) lse_lds[row] = neg;
        }
        __syncthreads();
        for (int t0 = 0; t0 < padded; t0 += 32) {
            f32x16 sc[TILES];
#pragma unroll
            for (int x = 0; x < TILES; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[x][i] = 0.f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const uint4 qf = q_lds[W::place(t0 + col, 2 * i + half)];
#pragma unroll
                for (int x = 0; x < TILES; ++x) sc[x] = Mfma32<T>::step(kk[x][i], qf, sc[x]);
            }
            const float neg = lse_lds[t0 + col];
#pragma unroll
            for (int x = 0; x < TILES; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[x][i] += __builtin_amdgcn_exp2f(fmaf(sc[x][i], k.scale_log2, neg));
        }
    }
    // ---- fold the columns; value i of a tile is its token 8 * (i >> 2) + 4 * half + (i & 3) ----
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
        const float w = fold32(sum[x], lane);
        const int i = ((lane & 1) << 3) | ((lane & 2) << 1) | ((lane & 4) >> 1) | ((lane & 8) >> 3);
        const int t = __shfl(tok[x], 8 * (i >> 2) + 4 * half + (i & 3));
        if ((lane & 16) || t < 0) continue;
        float *to = k.a.weights + bg * cap + t;
        // (a block that is listed m times is added to m times, by the same amount each: the order changes nothing)
        if (LISTS) unsafeAtomicAdd(to, w);
        else *to += w;
    }
}

hipError_t launch_weigh(const Shape &s, int dtype, const WeighArgs &a, hipStream_t st)
{
    const WeighKernelArgs k{s, a, make_fastdiv((uint32_t)s.B), make_fastdiv((uint32_t)s.G), kLog2e / sqrtf((float)s.D)};
    const int64_t positions = (a.sel_idx ? (int64_t)a.n_sel : (int64_t)s.max_blocks) * s.B;
    if (positions <= 0) return hipSuccess;
#define SPECPV_WEIGH_L(T, DD, LISTS)                                                                            \
    do {                                                                                                        \
        const int64_t per = kWeighWaves * 32 * WeighTile<T, DD>::TILES;                                         \
        const dim3 grid((unsigned)((positions + per - 1) / per), s.Hkv, s.batch);                               \
        hipLaunchKernelGGL((weigh_kernel<T, DD, LISTS>), grid, dim3(64 * kWeighWaves), 0, st, k);               \
    } while (0)
#define SPECPV_WEIGH(T, DD) do { if (a.sel_idx) SPECPV_WEIGH_L(T, DD, true); else SPECPV_WEIGH_L(T, DD, false); } while (0)
    if (dtype == SPECPV_BF16) {
        if (s.D == 128) SPECPV_WEIGH(bf16_t, 128); else SPECPV_WEIGH(bf16_t, 64);
    } else {
        if (s.D == 128) SPECPV_WEIGH(float, 128); else SPECPV_WEIGH(float, 64);
    }
#undef SPECPV_WEIGH
#undef SPECPV_WEIGH_L
    return hipGetLastError();
}

}  // namespace specpv
