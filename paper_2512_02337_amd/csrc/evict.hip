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
    int64_t chunks;       // of kPickMost tokens
};

// ---- which tokens stay -----------------------------------------------------------------------------------------------------
// A radix select on the weights' keys.  Caches of up to kPickMost tokens: one workgroup to a (sequence, KV head) with every key in
// registers, one launch (pick_kernel).  Longer ones by a workgroup to every kPickMost tokens; a launch is what those wait for each
// other by (first_digits, second_digits, collect, resolve): each leaves its histogram of a digit in the workspace, and the next
// launch's workgroups add them up, all of them for themselves (4 KiB a chunk: less than an atomic's way, and nothing to be cleared).
// Two digits of 11 bits leave the few candidates that agree with the threshold in 22 bits, or a great many equal ones
// (tokens that nothing has looked at): those are listed, and every workgroup finds the threshold's key among them for itself.

constexpr int kDigits = 2048;

// Inclusive sums over the workgroup, in thread order; `total`: of all.
template <int WAVES> __device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *wave_tot, uint32_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t in = (uint32_t)wave_inclusive_scan((int)x);
    if (lane == 63) wave_tot[wave] = in;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const uint32_t v = wave_tot[w];
        before += w < wave ? v : 0u;
        total += v;
    }
    __syncthreads();
    return before + in;
}

// hist[digit] + 1 where `in`.  A wavefront of one digit counts itself in at once: equal weights would queue for one address.
__device__ __forceinline__ void count_digit(uint32_t *hist, uint32_t digit, bool in)
{
    const unsigned long long who = __ballot(in);
    if (!who) return;
    const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(who));
    if (__ballot(in && digit == one) == who) {
        if ((threadIdx.x & 63) == __builtin_ctzll(who)) atomicAdd(&hist[one], (uint32_t)__popcll(who));
    } else if (in) {
        atomicAdd(&hist[digit], 1u);
    }
}

// The digit that the need-th largest key has, and how many keys have a larger one.  BINS / THREADS bins a thread, from the top.
template <int BINS, int WAVES> __device__ __forceinline__ void find_digit(const uint32_t *hist, uint32_t need, uint32_t *wave_tot, uint32_t *found)
{
    constexpr int PER = BINS / (64 * WAVES);
    uint32_t h[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { h[i] = hist[BINS - 1 - PER * (int)threadIdx.x - i]; sum += h[i]; }
    uint32_t total;
    uint32_t above = block_scan<WAVES>(sum, wave_tot, total) - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (above < need && above + h[i] >= need) { found[0] = (uint32_t)(BINS - 1 - PER * (int)threadIdx.x - i); found[1] = above; }
        above += h[i];
    }
    __syncthreads();
}

struct Span {   // of one (sequence, KV head)
    int64_t bg;
    int L, lo, hi, n_keep;   // candidates lo .. hi - 1
    const float *w;
    int32_t *idx;
    __device__ __forceinline__ Span(const EvictKernelArgs &k, int b, int g)
    {
        bg = (int64_t)b * k.s.Hkv + g;
        L = (int)min((int64_t)max(k.s.ctx_len[b], 0), k.cap);
        n_keep = k.a.ns + k.a.k + k.a.nr;
        lo = k.a.ns;
        hi = L - k.a.nr;
        w = k.a.weights + bg * k.cap;
        idx = k.a.keep_idx + bg * n_keep;
    }
    __device__ __forceinline__ bool all() const { return L <= n_keep; }
};

// N keys a thread: of tokens t0 + 4 (x WAVES 64 + thread) + 0 .. 3 for x < N / 4; 0 where no candidate is.
template <int N, int WAVES> __device__ __forceinline__ void load_keys(const Span &s, int t0, uint32_t (&key)[N])
{
#pragma unroll
    for (int x = 0; x < N / 4; ++x) {
        const int t = t0 + 4 * (x * WAVES * 64 + (int)threadIdx.x);
        float f[4] = {0.f, 0.f, 0.f, 0.f};
        if (t + 3 < s.L) {   // (rows of weights start at any multiple of four bytes)
            __builtin_memcpy(f, __builtin_assume_aligned(s.w + t, 4), 16);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = t + e < s.L ? s.w[t + e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) key[4 * x + e] = t + e >= s.lo && t + e < s.hi ? weight_key(f[e]) : 0u;
    }
}

// The kept tokens of t0 .. t0 + 64 N WAVES - 1 to their places: those with a key above `limit` and, in order, ties with it while
// there are less than `ties`; gt and eq: how many of either lie in front.
template <int N, int WAVES>
__device__ __forceinline__ void place_kept(const Span &s, int t0, const uint32_t (&key)[N], uint32_t limit, uint32_t ties, uint32_t gt, uint32_t eq, uint32_t *wave_tot)
{
#pragma unroll
    for (int x = 0; x < N / 4; ++x) {
        const int t = t0 + 4 * (x * WAVES * 64 + (int)threadIdx.x);
        uint32_t mine = 0;
        bool is_gt[4], is_eq[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool cand = t + e >= s.lo && t + e < s.hi;
            is_gt[e] = t + e < s.L && (!cand || key[4 * x + e] > limit);
            is_eq[e] = cand && ties && key[4 * x + e] == limit;
            mine += (is_gt[e] ? 1u : 0u) + (is_eq[e] ? 0x10000u : 0u);
        }
        uint32_t total;
        const uint32_t in = block_scan<WAVES>(mine, wave_tot, total) - mine;
        uint32_t n_gt = gt + (in & 0xffffu), n_eq = eq + (in >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (is_gt[e] || (is_eq[e] && n_eq < ties)) s.idx[n_gt + min(n_eq, ties)] = t + e;
            n_gt += is_gt[e] ? 1u : 0u;
            n_eq += is_eq[e] ? 1u : 0u;
        }
        gt += total & 0xffffu;
        eq += total >> 16;
    }
}

constexpr int kPickWaves = 16;
template <int N> __global__ __launch_bounds__(64 * kPickWaves) void pick_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[kDigits], wave_tot[kPickWaves], found[2];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const Span s(k, b, g);
    if (g == 0 && tid == 0) const_cast<int32_t *>(k.d.ctx_len)[b] = min(s.L, s.n_keep);
    if (s.all()) {
        for (int i = tid; i < s.n_keep; i += 64 * kPickWaves) s.idx[i] = i < s.L ? i : -1;
        return;
    }
    uint32_t key[N];
    load_keys<N, kPickWaves>(s, 0, key);
    uint32_t prefix = 0, need = (uint32_t)k.a.k;
    if (need) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int width = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            for (int i = tid; i < kDigits; i += 64 * kPickWaves) hist[i] = 0;
            __syncthreads();
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const int t = 4 * (x / 4 * kPickWaves * 64 + tid) + x % 4;
                if (4 * (x / 4 * kPickWaves * 64) >= s.hi) break;
                count_digit(hist, (key[x] >> shift) & ((1u << width) - 1u), t >= s.lo && t < s.hi && (pass == 0 || (key[x] >> (shift + width)) == prefix));
            }
            __syncthreads();
            find_digit<kDigits, kPickWaves>(hist, need, wave_tot, found);
            prefix = prefix << width | found[0];
            need -= found[1];
            __syncthreads();
        }
    } else {
        prefix = 0xffffffffu;   // (no key)
    }
    place_kept<N, kPickWaves>(s, 0, key, prefix, need, 0, 0, wave_tot);
}

// ---- long caches: scratch of a (sequence, KV head) ----
constexpr int kPickMost = 16384, kKeys = kPickMost / (64 * kPickWaves);
struct PickScratch {             // words
    uint32_t *first, *second;    // [chunks][kDigits / 2] histograms, two 16-bit counts a word
    uint32_t *state;             // first digit, what is needed of it; the 22 bits, what is needed of those
    uint32_t *chunk;             // [chunks][4]: keys above; candidates; their least and largest key
    uint32_t *cand;              // [chunks][kPickMost]
};
static int64_t pick_chunks(int64_t cap) { return (cap + kPickMost - 1) / kPickMost; }
__host__ __device__ constexpr int64_t pick_words(int64_t chunks) { return 64 + chunks * (kDigits + 4 + kPickMost); }
__device__ __forceinline__ PickScratch pick_scratch(const EvictKernelArgs &k, int64_t bg)
{
    PickScratch p;
    p.state = k.a.scratch + bg * pick_words(k.chunks);
    p.first = p.state + 64;
    p.second = p.first + k.chunks * (kDigits / 2);
    p.chunk = p.second + k.chunks * (kDigits / 2);
    p.cand = p.chunk + k.chunks * 4;
    return p;
}
// a chunk's histogram to its place, and those of all chunks added up (thread i has digits 2 i and 2 i + 1)
__device__ __forceinline__ void store_hist(const uint32_t *hist, uint32_t *to, int chunk)
{
    to[chunk * (kDigits / 2) + (int)threadIdx.x] = hist[2 * threadIdx.x] | hist[2 * threadIdx.x + 1] << 16;
}
__device__ __forceinline__ void sum_hist(const uint32_t *from, int first_chunk, int chunks, uint32_t *hist)
{
    static_assert(kDigits == 2 * 64 * kPickWaves, "two digits a thread");
    uint32_t a = 0, b = 0;
#pragma unroll 4
    for (int c = first_chunk; c < chunks; ++c) {
        const uint32_t v = from[(int64_t)c * (kDigits / 2) + threadIdx.x];
        a += v & 0xffffu;
        b += v >> 16;
    }
    hist[2 * threadIdx.x] = a;
    hist[2 * threadIdx.x + 1] = b;
    __syncthreads();
}

// chunks that have candidates: first .. last - 1
struct Chunks { int first, last; };
__device__ __forceinline__ Chunks with_candidates(const Span &s) { return Chunks{s.lo / kPickMost, (s.hi + kPickMost - 1) / kPickMost}; }

__global__ __launch_bounds__(64 * kPickWaves) void first_digits_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[kDigits];
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kPickMost, tid = threadIdx.x;
    const Span s(k, b, g);
    if (s.all() || !k.a.k || t0 >= s.hi || t0 + kPickMost <= s.lo) return;
    uint32_t key[kKeys];
    load_keys<kKeys, kPickWaves>(s, t0, key);
    hist[tid] = hist[tid + 1024] = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kKeys; ++x) {
        const int t = t0 + 4 * (x / 4 * kPickWaves * 64 + tid) + x % 4;
        count_digit(hist, key[x] >> 21, t >= s.lo && t < s.hi);
    }
    __syncthreads();
    store_hist(hist, pick_scratch(k, s.bg).first, blockIdx.x);
}

__global__ __launch_bounds__(64 * kPickWaves) void second_digits_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[kDigits], wave_tot[kPickWaves], found[2];
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kPickMost, tid = threadIdx.x;
    const Span s(k, b, g);
    if (s.all() || !k.a.k || t0 >= s.hi || t0 + kPickMost <= s.lo) return;
    const PickScratch p = pick_scratch(k, s.bg);
    uint32_t key[kKeys];
    load_keys<kKeys, kPickWaves>(s, t0, key);
    const Chunks c = with_candidates(s);
    sum_hist(p.first, c.first, c.last, hist);
    find_digit<kDigits, kPickWaves>(hist, (uint32_t)k.a.k, wave_tot, found);
    const uint32_t digit = found[0];
    if ((int)blockIdx.x == c.first && tid == 0) { p.state[0] = digit; p.state[1] = (uint32_t)k.a.k - found[1]; }
    hist[tid] = hist[tid + 1024] = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kKeys; ++x) {
        const int t = t0 + 4 * (x / 4 * kPickWaves * 64 + tid) + x % 4;
        count_digit(hist, (key[x] >> 10) & 2047u, t >= s.lo && t < s.hi && (key[x] >> 21) == digit);
    }
    __syncthreads();
    store_hist(hist, p.second, blockIdx.x);
}

// What a chunk has above the 22 bits (tokens that stay in any case among them), and the keys that agree with them, in order.
__global__ __launch_bounds__(64 * kPickWaves) void collect_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[kDigits], wave_tot[kPickWaves], found[2], low, high;
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kPickMost;
    const Span s(k, b, g);
    if (s.all() || t0 >= s.L) return;
    const PickScratch p = pick_scratch(k, s.bg);
    uint32_t key[kKeys];
    load_keys<kKeys, kPickWaves>(s, t0, key);
    if (threadIdx.x == 0) { low = 0xffffffffu; high = 0; }
    uint32_t prefix = 0xffffffffu;
    if (k.a.k) {
        const uint32_t need = p.state[1];
        const Chunks c = with_candidates(s);
        sum_hist(p.second, c.first, c.last, hist);
        find_digit<kDigits, kPickWaves>(hist, need, wave_tot, found);
        prefix = p.state[0] << 11 | found[0];
        if (blockIdx.x == 0 && threadIdx.x == 0) { p.state[2] = prefix; p.state[3] = need - found[1]; }
    }
    __syncthreads();
    uint32_t gt = 0, eq = 0;
    uint32_t *const cand = p.cand + (int64_t)blockIdx.x * kPickMost;
#pragma unroll
    for (int x = 0; x < kKeys / 4; ++x) {
        const int t = t0 + 4 * (x * kPickWaves * 64 + (int)threadIdx.x);
        uint32_t mine = 0;
        bool is_eq[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool c = t + e >= s.lo && t + e < s.hi;
            is_eq[e] = c && (key[4 * x + e] >> 10) == prefix;
            const bool is_gt = t + e < s.L && (!c || (k.a.k && (key[4 * x + e] >> 10) > prefix));
            mine += (is_gt ? 1u : 0u) + (is_eq[e] ? 0x10000u : 0u);
        }
        uint32_t total;
        uint32_t at = eq + ((block_scan<kPickWaves>(mine, wave_tot, total) - mine) >> 16);
        if (mine >> 16) {
            uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!is_eq[e]) continue;
                cand[at++] = key[4 * x + e];
                lo = min(lo, key[4 * x + e]);
                hi = max(hi, key[4 * x + e]);
            }
            atomicMin(&low, lo);
            atomicMax(&high, hi);
        }
        gt += total & 0xffffu;
        eq += total >> 16;
    }
    __syncthreads();
    if (threadIdx.x == 0) ((uint4 *)p.chunk)[blockIdx.x] = make_uint4(gt, eq, low, high);
}

// The threshold's key out of the listed ones, by every workgroup for itself, and the chunk's kept tokens in their places.
__global__ __launch_bounds__(64 * kPickWaves) void resolve_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[1024], wave_tot[kPickWaves], found[2], sums[4];
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kPickMost, tid = threadIdx.x;
    const Span s(k, b, g);
    if (g == 0 && blockIdx.x == 0 && tid == 0) const_cast<int32_t *>(k.d.ctx_len)[b] = min(s.L, s.n_keep);
    if (s.all()) {
        for (int i = t0 + tid; i < min(s.n_keep, t0 + kPickMost); i += 64 * kPickWaves) s.idx[i] = i < s.L ? i : -1;
        return;
    }
    const PickScratch p = pick_scratch(k, s.bg);
    if (t0 >= s.L) return;
    uint32_t key[kKeys];
    load_keys<kKeys, kPickWaves>(s, t0, key);
    const int chunks = (s.L + kPickMost - 1) / kPickMost;
    // in front: keys above, candidates; of all: the least and the largest candidate
    if (tid < 4) sums[tid] = tid == 2 ? 0xffffffffu : 0u;
    hist[tid] = 0;
    __syncthreads();
    uint32_t gt = 0, eq = 0, lo = 0xffffffffu, hi = 0;
    for (int c = tid; c < chunks; c += 64 * kPickWaves) {
        const uint4 v = ((const uint4 *)p.chunk)[c];
        if (c < (int)blockIdx.x) { gt += v.x; eq += v.y; }
        lo = min(lo, v.z);
        hi = max(hi, v.w);
    }
    if (tid < chunks) { atomicAdd(&sums[0], gt); atomicAdd(&sums[1], eq); atomicMin(&sums[2], lo); atomicMax(&sums[3], hi); }
    __syncthreads();
    gt = sums[0]; eq = sums[1]; lo = sums[2]; hi = sums[3];
    uint32_t limit = 0xffffffffu, ties = 0;
    if (k.a.k) {
        ties = p.state[3];
        limit = hi;
        if (lo != hi) {   // (else all are equal)
            for (int c = 0; c < chunks; ++c) {
                const uint32_t n = p.chunk[4 * c + 1];
                for (uint32_t i = tid; i < ((n + 63u) & ~63u); i += 64 * kPickWaves) {
                    const uint32_t x = i < n ? p.cand[(int64_t)c * kPickMost + i] : 0u;
                    count_digit(hist, x & 1023u, i < n);
                }
            }
            __syncthreads();
            find_digit<1024, kPickWaves>(hist, ties, wave_tot, found);
            limit = p.state[2] << 10 | found[0];
            ties -= found[1];
            // of the candidates in front
            __syncthreads();
            if (tid < 2) sums[tid] = 0;
            __syncthreads();
            uint32_t more = 0, same = 0;
            for (int c = 0; c < (int)blockIdx.x; ++c) {
                const uint32_t n = p.chunk[4 * c + 1];
                for (uint32_t i = tid; i < n; i += 64 * kPickWaves) {
                    const uint32_t x = p.cand[(int64_t)c * kPickMost + i];
                    more += x > limit ? 1u : 0u;
                    same += x == limit ? 1u : 0u;
                }
            }
            if (more) atomicAdd(&sums[0], more);
            if (same) atomicAdd(&sums[1], same);
            __syncthreads();
            gt += sums[0];
            eq = sums[1];
        }
    }
    place_kept<kKeys, kPickWaves>(s, t0, key, limit, ties, gt, eq, wave_tot);
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
        kk[u] = vv[u] = make_uint4(0, 0, 0, 0);   // (left undefined, they would live in memory)
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

size_t evict_scratch_bytes(int64_t pairs, int64_t cap) { return cap > kPickMost ? (size_t)(pairs * pick_words(pick_chunks(cap))) * sizeof(uint32_t) : 0; }

hipError_t launch_evict(const Shape &s, const Shape &d, int dtype, const EvictArgs &a, hipStream_t st)
{
    const int64_t cap = (int64_t)s.max_blocks * s.B;
    const EvictKernelArgs k{s, d, a, cap, (int64_t)d.max_blocks * d.B, pick_chunks(cap)};
    const dim3 one(s.Hkv, s.batch), grid_c((unsigned)k.chunks, s.Hkv, s.batch), threads(64 * kPickWaves);
    if (cap <= 4096) {
        hipLaunchKernelGGL(pick_kernel<4>, one, threads, 0, st, k);
    } else if (cap <= kPickMost) {
        hipLaunchKernelGGL(pick_kernel<16>, one, threads, 0, st, k);
    } else {
        hipLaunchKernelGGL(first_digits_kernel, grid_c, threads, 0, st, k);
        hipLaunchKernelGGL(second_digits_kernel, grid_c, threads, 0, st, k);
        hipLaunchKernelGGL(collect_kernel, grid_c, threads, 0, st, k);
        hipLaunchKernelGGL(resolve_kernel, grid_c, threads, 0, st, k);
    }
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
