// Rows into the 4-bit cache (with the block summaries of Section 3.2, eq. 1, beside it) and out of it again.
#include "packed.h"
#include "summarize.h"

namespace specpv {

// A lane takes eight channels of a row in either type: 16 (or 8) lanes a row, the four lanes of a group of 32 channels find
// its largest magnitude by two exchanges, and a row's codes leave as one dense run of 4 bytes a lane.  Bound by memory: 8 heads of 128K
// tokens, bf16, with their summaries 131 us, 5.2 TB/s; a few rows by the chain of count, row, value and store (22 rows for each of 8
// sequences 6.4 us).
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    uint4 u;
    __device__ __forceinline__ void load(const bf16_t *p) { u = load_stream((const uint4 *)p); }
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void value(float *f) const { Elem<bf16_t>::unpack(u, f); }
};
template <> struct Eight<float> {
    uint4 u[2];
    __device__ __forceinline__ void load(const float *p) { u[0] = load_stream((const uint4 *)p); u[1] = load_stream((const uint4 *)p + 1); }
    __device__ __forceinline__ void zero() { u[0] = u[1] = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void value(float *f) const { Elem<float>::unpack(u[0], f); Elem<float>::unpack(u[1], f + 4); }
};

__device__ __forceinline__ uint32_t quad_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false));   // lane ^ 1
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false));   // lane ^ 2
}

struct PackKernelArgs {
    Shape src;
    PackedShape p;
    PackArgs a;
    int unit;         // tokens of a unit: the block size where there are summaries
    int64_t capacity; // tokens that the packed cache has room for
};

// A unit is one block's K rows or V rows: one wavefront's work, or (WIDE, long blocks) a workgroup's.
template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(256) void pack_kernel(PackKernelArgs k)
{
    constexpr int LPR = D / 8, RPP = 64 / LPR, U = sizeof(T) == 2 ? 8 : 4, WAVES = WIDE ? 4 : 1;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.y, b = blockIdx.z;
    const int at = WIDE ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
    const bool values = at & 1;
    const int L = (int)min((int64_t)k.src.ctx_len[b], (int64_t)k.src.max_blocks * k.src.B);
    const int64_t sb = k.a.src_begin ? k.a.src_begin[b] : 0, db = k.a.dst_begin ? k.a.dst_begin[b] : 0;
    int64_t n = k.a.n_rows ? k.a.n_rows[b] : (k.a.src_rows ? (int64_t)k.a.max_rows : (int64_t)L - sb);
    if (n > k.a.max_rows) n = k.a.max_rows;
    const int64_t end64 = min(db + n, k.capacity);
    const int first = db > 0 ? (int)db / k.unit : 0;
    const int64_t u0 = ((int64_t)first + (at >> 1)) * k.unit;
    const int64_t lo64 = max(u0, db), hi64 = min(u0 + k.unit, end64);
    if (lo64 >= hi64) return;   // (the whole workgroup, WIDE)
    const int lo = (int)lo64, hi = (int)hi64;
    const int c = lane % LPR, rsub = lane / LPR;
    const T *src = (const T *)(values ? k.src.v : k.src.k) + (int64_t)b * k.src.sb + (int64_t)g * k.src.sh + c * 8;
    const int64_t dst0 = (int64_t)b * k.p.s.sb + (int64_t)g * k.p.s.sh;
    uint8_t *const code = (uint8_t *)const_cast<void *>(values ? k.p.s.v : k.p.s.k) + dst0 + c * 4;
    uint8_t *const scale = const_cast<uint8_t *>(values ? k.p.vs : k.p.ks) + (dst0 >> 4) + (c >> 2);
    const int32_t *rows = k.a.src_rows ? k.a.src_rows + (int64_t)b * k.a.max_rows : nullptr;
    const bool sums = k.a.kmax && !values;
    float mx[8], mn[8];
    bool any = false;   // a row that is there
#pragma unroll
    for (int e = 0; e < 8; ++e) { mx[e] = -INFINITY; mn[e] = INFINITY; }
    for (int t = lo + (WIDE ? wave * RPP : 0); t < hi; t += WAVES * U * RPP) {
        Eight<T> x[U];
        bool live[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int tok = t + u * WAVES * RPP + rsub;
            live[u] = tok < hi;
            int64_t row = 0;
            if (live[u]) {
                const int64_t i = tok - db;
                row = rows ? (int64_t)rows[i] : sb + i;
                live[u] = row >= 0 && row < L;
            }
            x[u].zero();
            if (live[u]) x[u].load(src + row * k.src.st);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[8];
            x[u].value(f);
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);   // (NaN above infinity above the rest)
            const uint32_t byte = scale_byte(quad_max(top));
            const uint32_t word = encode8(f, scale_of(byte));
            if (live[u]) {
                const int64_t row = (int64_t)(t + u * WAVES * RPP + rsub) * k.p.s.st;
                *(uint32_t *)(code + row) = word;
                if ((c & 3) == 0) scale[row >> 4] = (uint8_t)byte;
                if (sums) {
                    any = true;
#pragma unroll
                    for (int e = 0; e < 8; ++e) { mx[e] = fmaxf(mx[e], f[e]); mn[e] = fminf(mn[e], f[e]); }
                }
            }
        }
    }
    if (!sums) return;
    any = __any(any);
    // the lanes that hold the same channels, then what the block had before
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { mx[e] = fmaxf(mx[e], __shfl_xor(mx[e], o)); mn[e] = fminf(mn[e], __shfl_xor(mn[e], o)); }
    }
    if constexpr (WIDE) {
        __shared__ float fold[4][2][D];
        __shared__ bool seen[4];
        if (lane == 0) seen[wave] = any;
        if (lane < LPR) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { fold[wave][0][c * 8 + e] = mx[e]; fold[wave][1][c * 8 + e] = mn[e]; }
        }
        __syncthreads();
        if (wave) return;
        any = seen[0] | seen[1] | seen[2] | seen[3];
#pragma unroll
        for (int w = 1; w < 4; ++w) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { mx[e] = fmaxf(mx[e], fold[w][0][c * 8 + e]); mn[e] = fminf(mn[e], fold[w][1][c * 8 + e]); }
        }
    }
    if (!any || lane >= LPR) return;
    const int64_t o = (((int64_t)b * k.p.s.Hkv + g) * k.p.s.max_blocks + u0 / k.unit) * D + c * 8;
    T *const to[2] = {(T *)k.a.kmax + o, (T *)k.a.kmin + o};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        float *f = m ? mn : mx;
        if (u0 < db) {   // older tokens in front
            float old[8];
            constexpr int E = Elem<T>::kPerVec;
#pragma unroll
            for (int v = 0; v < 8 / E; ++v) Elem<T>::unpack(((const uint4 *)to[m])[v], old + v * E);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = m ? fminf(f[e], old[e]) : fmaxf(f[e], old[e]);
        }
        constexpr int E = Elem<T>::kPerVec;
#pragma unroll
        for (int v = 0; v < 8 / E; ++v) ((uint4 *)to[m])[v] = Elem<T>::pack(f + v * E);
    }
}

hipError_t launch_pack(const Shape &src, int dtype, const PackedShape &p, const PackArgs &a, hipStream_t st)
{
    PackKernelArgs k{src, p, a, p.s.B, p.rows};
    if (!a.kmax) k.unit = 64;
    const int64_t most = (k.capacity + k.unit - 1) / k.unit, rows = ((int64_t)a.max_rows + k.unit - 2) / k.unit + 1;
    const int64_t units = 2 * (rows < most ? rows : most);
    // A workgroup to a block where that is no more than eight workgroups to a CU, or the blocks are long (us, wavefronts / workgroups, 8 heads, bf16:
    // blocks of 32, 64 rows 11.3 / 10.0, 1K 14.6 / 12.3, 2K 15.9 / 14.8, 4K 19.6 / 20.6, 32K 61.7 / 94.9; of 64, 64 rows 14.4 / 10.5, 1K 18.3 / 12.7, 8K
    // 31.4 / 29.1, 32K 61.6 / 72.7; of 128, 1K 28.0 / 15.0, 32K 61.7 / 63.1, 128K 245 / 237; of 256, 128K 250 / 233; fp32, of 64, 4K 34.5 / 26.2.)  Blocks
    // of 16 are a pass of eight loads or less for a wavefront by itself (1K rows 11.9 / 12.8).
    const bool wide = k.unit > 64 || (k.unit > 16 && units * p.s.Hkv * p.s.batch <= 8 * (int64_t)device_cu_count());
    const dim3 grid((unsigned)(wide ? units : (units + 3) / 4), p.s.Hkv, p.s.batch);
#define SPECPV_PACK(T, DD)                                                                                   \
    do {                                                                                                     \
        if (wide) hipLaunchKernelGGL((pack_kernel<T, DD, true>), grid, dim3(256), 0, st, k);                 \
        else hipLaunchKernelGGL((pack_kernel<T, DD, false>), grid, dim3(256), 0, st, k);                     \
    } while (0)
    if (dtype == SPECPV_BF16) {
        if (p.s.D == 128) SPECPV_PACK(bf16_t, 128); else SPECPV_PACK(bf16_t, 64);
    } else {
        if (p.s.D == 128) SPECPV_PACK(float, 128); else SPECPV_PACK(float, 64);
    }
#undef SPECPV_PACK
    return hipGetLastError();
}

// ---- out of the cache ----------------------------------------------------------------------------------------------------

struct PackedGatherArgs {
    PackedShape p;
    const int32_t *sel_idx, *sel_count;
    int n_sel;
    FastDiv div_B;
    void *out_k, *out_v;
    int32_t *out_len;
};

// Workgroup 0 of a sequence's first head finds the gathered length; the others bring U passes of rows of K and V each.  Bound by memory:
// 8 heads of 128K tokens to bf16, 111 us, 6.1 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_gather_kernel(PackedGatherArgs a)
{
    constexpr int LPR = D / 8, RPP = 256 / LPR, U = 4;
    const Shape &s = a.p.s;
    const int g = blockIdx.y, b = blockIdx.z;
    const int L = (int)min((int64_t)max(s.ctx_len[b], 0), a.p.rows);
    const int nb = (int)a.div_B.div((uint32_t)L + (uint32_t)s.B - 1u);
    if (blockIdx.x == 0) {
        if (g || !a.out_len) return;
        int rows = a.sel_idx ? 0 : L;
        if (a.sel_idx) {
            for (int h = 0; h < s.Hkv; ++h) {
                const int64_t row = (int64_t)b * s.Hkv + h;
                const int cnt = min(a.sel_count[row], a.n_sel);
                for (int i = threadIdx.x; i < cnt; i += 256) {
                    const int e = a.sel_idx[row * a.n_sel + i];
                    if (e >= 0 && e < nb) rows = max(rows, i * s.B + min(s.B, L - e * s.B));
                }
            }
        }
        __shared__ int most[4];
        for (int off = 32; off; off >>= 1) rows = max(rows, __shfl_xor(rows, off));
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = rows;
        __syncthreads();
        if (threadIdx.x == 0) a.out_len[b] = max(max(most[0], most[1]), max(most[2], most[3]));
        return;
    }
    const int64_t bg = (int64_t)b * s.Hkv + g, total = (a.sel_idx ? (int64_t)a.n_sel : (int64_t)s.max_blocks) * s.B;
    const int cnt = a.sel_idx ? a.sel_count[bg] : 0;
    const int c = threadIdx.x % LPR, rsub = threadIdx.x / LPR;
    const int64_t src0 = (int64_t)b * s.sb + (int64_t)g * s.sh;
    const int64_t r0 = (int64_t)(blockIdx.x - 1) * (U * RPP);
    uint32_t code[U][2], byte[U][2];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * RPP + rsub;
        int tok = -1;
        if (r < total) {
            if (a.sel_idx) {
                const int slot = (int)a.div_B.div((uint32_t)r);
                const int e = slot < cnt ? a.sel_idx[bg * a.n_sel + slot] : -1;
                if (e >= 0 && e < nb) tok = e * s.B + (int)(r - (int64_t)slot * s.B);
            } else {
                tok = (int)r;
            }
        }
        live[u] = tok >= 0 && tok < L;
        code[u][0] = code[u][1] = byte[u][0] = byte[u][1] = 0;
        if (live[u]) {
            const int64_t o = src0 + (int64_t)tok * s.st;
            code[u][0] = *(const uint32_t *)((const uint8_t *)s.k + o + c * 4);
            code[u][1] = *(const uint32_t *)((const uint8_t *)s.v + o + c * 4);
            byte[u][0] = a.p.ks[(o >> 4) + (c >> 2)];
            byte[u][1] = a.p.vs[(o >> 4) + (c >> 2)];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * RPP + rsub;
        if (r >= total) continue;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const uint4 v = decode8_bf16(code[u][m], scale_of(byte[u][m]));   // (codes of 0 where nothing is)
            T *out = (T *)(m ? a.out_v : a.out_k) + (bg * total + r) * D + c * 8;
            if constexpr (sizeof(T) == 2) {
                __builtin_nontemporal_store(__builtin_bit_cast(__attribute__((ext_vector_type(4))) uint32_t, v), (__attribute__((ext_vector_type(4))) uint32_t *)out);
            } else {
                float f[8];
                Elem<bf16_t>::unpack(v, f);
                ((uint4 *)out)[0] = Elem<float>::pack(f);
                ((uint4 *)out)[1] = Elem<float>::pack(f + 4);
            }
        }
    }
}

hipError_t launch_packed_gather(const PackedShape &p, int dtype, const int32_t *sel_idx, const int32_t *sel_count, int n_sel,
                                void *out_k, void *out_v, int32_t *out_len, hipStream_t st)
{
    const PackedGatherArgs a{p, sel_idx, sel_count, n_sel, make_fastdiv((uint32_t)p.s.B), out_k, out_v, out_len};
    const int64_t rows = (sel_idx ? (int64_t)n_sel : (int64_t)p.s.max_blocks) * p.s.B, per = 4 * 256 / (p.s.D / 8);
    const dim3 grid((unsigned)(1 + (rows + per - 1) / per), p.s.Hkv, p.s.batch);
#define SPECPV_GATHER(T, DD) hipLaunchKernelGGL((packed_gather_kernel<T, DD>), grid, dim3(256), 0, st, a)
    if (dtype == SPECPV_BF16) {
        if (p.s.D == 128) SPECPV_GATHER(bf16_t, 128); else SPECPV_GATHER(bf16_t, 64);
    } else {
        if (p.s.D == 128) SPECPV_GATHER(float, 128); else SPECPV_GATHER(float, 64);
    }
#undef SPECPV_GATHER
    return hipGetLastError();
}

}  // namespace specpv
