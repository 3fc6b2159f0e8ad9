// Eviction by accumulated attention weight (specpv_evict_tokens): which tokens of each (sequence, KV head) stay, and their
// rows moved, in order, into another cache.
#include "internal.h"
#include "topk.h"

namespace specpv {

// A weight's key: larger is better, -0 and +0 alike, NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : score_bits(w); }

struct EvictKernelArgs {
    Shape s;
    Shape d;              // the cache that the kept tokens go to
    EvictArgs a;
    int64_t cap, dcap;    // tokens that either has room for
};

constexpr int kPickThreads = 1024;

// Inclusive sums over the workgroup, in thread order; `total`: of all.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *wave_tot, uint32_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t in = (uint32_t)wave_inclusive_scan((int)x);
    if (lane == 63) wave_tot[wave] = in;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPickThreads / 64; ++w) {
        const uint32_t v = wave_tot[w];
        before += w < wave ? v : 0u;
        total += v;
    }
    __syncthreads();
    return before + in;
}

// One workgroup to a (sequence, KV head): the key of the k-th best candidate by a radix select (digits of 11, 11 and 10 bits),
// then the kept tokens in order.
__global__ __launch_bounds__(kPickThreads) void pick_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[2048], wave_tot[16], found[3];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const int64_t bg = (int64_t)b * k.s.Hkv + g;
    const int L = (int)min((int64_t)max(k.s.ctx_len[b], 0), k.cap), n_keep = k.a.ns + k.a.k + k.a.nr;
    int32_t *const idx = k.a.keep_idx + bg * n_keep;
    if (g == 0 && tid == 0) const_cast<int32_t *>(k.d.ctx_len)[b] = min(L, n_keep);
    if (L <= n_keep) {
        for (int i = tid; i < n_keep; i += kPickThreads) idx[i] = i < L ? i : -1;
        return;
    }
    const float *const w = k.a.weights + bg * k.cap;
    const int lo = k.a.ns, hi = L - k.a.nr;   // candidates; more than k of them
    uint32_t prefix = 0, need = (uint32_t)k.a.k, ties = 0;   // ties: candidates with the threshold's key that stay
    if (need) {
        int bits = 32;
        while (bits > 0) {
            const int width = bits > 10 ? 11 : 10, shift = bits - width;
            for (int i = tid; i < 2048; i += kPickThreads) hist[i] = 0;
            __syncthreads();
            for (int t0 = lo; t0 < hi; t0 += kPickThreads) {
                const int t = t0 + tid;
                const uint32_t key = t < hi ? weight_key(w[t]) : 0u;
                const bool in = t < hi && (bits == 32 || (key >> bits) == prefix);
                const uint32_t digit = (key >> shift) & ((1u << width) - 1u);
                const unsigned long long who = __ballot(in);
                if (!who) continue;
                // (a wavefront of one digit, as of tokens that nothing has looked at yet, counts itself in at once)
                const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(who));
                if (__ballot(in && digit == one) == who) {
                    if (lane == 0) atomicAdd(&hist[one], (uint32_t)__popcll(who));
                } else if (in) {
                    atomicAdd(&hist[digit], 1u);
                }
            }
            __syncthreads();
            // thread i owns the bins 2047 - 2 i and the one below it: sums from the top
            const uint32_t h1 = hist[2047 - 2 * tid], h0 = hist[2046 - 2 * tid];
            uint32_t total;
            const uint32_t upto = block_scan(h0 + h1, wave_tot, total);
            const uint32_t above1 = upto - h0 - h1, above0 = upto - h0;
            if (above1 < need && above1 + h1 >= need) { found[0] = 2047u - 2u * tid; found[1] = above1; found[2] = h1; }
            if (above0 < need && above0 + h0 >= need) { found[0] = 2046u - 2u * tid; found[1] = above0; found[2] = h0; }
            __syncthreads();
            prefix = prefix << width | found[0];
            need -= found[1];
            bits = shift;
            __syncthreads();
        }
        ties = need;
    } else {
        prefix = 0xffffffffu;   // (no weight has this key)
    }
    // the kept tokens, 4 consecutive ones a thread: better ones and ties before each
    uint32_t done_gt = 0, done_eq = 0;
    for (int t0 = 0; t0 < L; t0 += 4 * kPickThreads) {
        uint32_t mine = 0;
        bool gt[4], eq[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int t = t0 + 4 * tid + x;
            const uint32_t key = t >= lo && t < hi ? weight_key(w[t]) : 0u;
            gt[x] = t < L && (t < lo || t >= hi || (t < hi && key > prefix));
            eq[x] = t >= lo && t < hi && ties && key == prefix;
            mine += (gt[x] ? 1u : 0u) + (eq[x] ? 0x10000u : 0u);
        }
        uint32_t total;
        const uint32_t in = block_scan(mine, wave_tot, total) - mine;
        uint32_t n_gt = done_gt + (in & 0xffffu), n_eq = done_eq + (in >> 16);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (gt[x] || (eq[x] && n_eq < ties)) idx[n_gt + min(n_eq, ties)] = t0 + 4 * tid + x;
            n_gt += gt[x] ? 1u : 0u;
            n_eq += eq[x] ? 1u : 0u;
        }
        done_gt += total & 0xffffu;
        done_eq += total >> 16;
    }
}

// Rows i, i + 1, ... of the new cache from rows keep_idx[i], ...; the weights with them, zeros behind.
template <int ROW>   // bytes of a row
__global__ __launch_bounds__(256) void move_kernel(EvictKernelArgs k, int elem)
{
    constexpr int LPR = ROW / 16, RPP = 256 / LPR, U = 4;
    const int g = blockIdx.y, b = blockIdx.z, n_keep = k.a.ns + k.a.k + k.a.nr;
    const int64_t bg = (int64_t)b * k.s.Hkv + g;
    const int32_t *const idx = k.a.keep_idx + bg * n_keep;
    const int c = threadIdx.x % LPR, rsub = threadIdx.x / LPR;
    const int r0 = (int)blockIdx.x * (U * RPP);
    if (k.a.new_weights) {
        for (int64_t i = r0 + (int)threadIdx.x, x = 0; x < (U * RPP + 255) / 256; ++x, i += 256) {
            if (i >= r0 + U * RPP || i >= k.dcap) break;
            const int t = i < n_keep ? idx[i] : -1;
            k.a.new_weights[bg * k.dcap + i] = t >= 0 ? k.a.weights[bg * k.cap + t] : 0.f;
        }
    }
    const char *const sk = (const char *)k.s.k + ((int64_t)b * k.s.sb + (int64_t)g * k.s.sh) * elem + c * 16;
    const char *const sv = (const char *)k.s.v + ((int64_t)b * k.s.sb + (int64_t)g * k.s.sh) * elem + c * 16;
    char *const dk = (char *)const_cast<void *>(k.d.k) + ((int64_t)b * k.d.sb + (int64_t)g * k.d.sh) * elem + c * 16;
    char *const dv = (char *)const_cast<void *>(k.d.v) + ((int64_t)b * k.d.sb + (int64_t)g * k.d.sh) * elem + c * 16;
    uint4 kk[U], vv[U];
    int t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = r0 + u * RPP + rsub;
        t[u] = r < n_keep ? idx[r] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (t[u] >= 0) {
            kk[u] = *(const uint4 *)(sk + (int64_t)t[u] * k.s.st * elem);
            vv[u] = *(const uint4 *)(sv + (int64_t)t[u] * k.s.st * elem);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = r0 + u * RPP + rsub;
        if (t[u] >= 0) {
            *(uint4 *)(dk + (int64_t)r * k.d.st * elem) = kk[u];
            *(uint4 *)(dv + (int64_t)r * k.d.st * elem) = vv[u];
        }
    }
}

size_t evict_scratch_bytes(int64_t pairs) { return (size_t)pairs * 256; }

hipError_t launch_evict(const Shape &s, const Shape &d, int dtype, const EvictArgs &a, hipStream_t st)
{
    const EvictKernelArgs k{s, d, a, (int64_t)s.max_blocks * s.B, (int64_t)d.max_blocks * d.B};
    hipLaunchKernelGGL(pick_kernel, dim3(s.Hkv, s.batch), dim3(kPickThreads), 0, st, k);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int elem = dtype == SPECPV_BF16 ? 2 : 4, row = s.D * elem, per = 4 * 256 / (row / 16);
    const int64_t rows = a.new_weights ? k.dcap : (int64_t)a.ns + a.k + a.nr;
    const dim3 grid((unsigned)((rows + per - 1) / per), s.Hkv, s.batch);
    if (row == 512) hipLaunchKernelGGL((move_kernel<512>), grid, dim3(256), 0, st, k, elem);
    else if (row == 256) hipLaunchKernelGGL((move_kernel<256>), grid, dim3(256), 0, st, k, elem);
    else hipLaunchKernelGGL((move_kernel<128>), grid, dim3(256), 0, st, k, elem);
    return hipGetLastError();
}

}  // namespace specpv
