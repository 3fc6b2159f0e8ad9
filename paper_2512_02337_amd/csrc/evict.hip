// Eviction by accumulated attention weight (specpv_evict_tokens): which tokens of each (sequence, KV head) stay, and their
// rows moved, in order, into another cache.
#include "internal.h"
#include "summarize.h"
#include "topk.h"

namespace specpv {

template <bool STREAM> __device__ __forceinline__ void store16(void *p, uint4 v)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    if constexpr (!STREAM) *(uint4 *)p = v;
    else __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4 *)p);
}

// A weight's key: larger is better, -0 and +0 alike, NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : score_bits(w); }

struct EvictKernelArgs {
    Shape s;
    Shape d;              // the cache that the kept tokens go to
    EvictArgs a;
    int64_t cap, dcap;    // tokens that either has room for
    int64_t chunks;       // of kChunk tokens, whole histograms of them
};

// ---- which tokens stay -----------------------------------------------------------------------------------------------------
// A radix select on the weights' keys.  Caches of up to kPickMost tokens: one workgroup to a (sequence, KV head) with every key in
// registers, one launch (pick_kernel).  Longer ones by many; a launch is what those wait for each other by.  first_digits leaves a
// histogram of the leading eleven bits for every 8192 tokens in the workspace; collect's workgroups, 4096 tokens each, add them up, all
// of them for themselves (4 KiB each: less than an atomic's way, and nothing to be cleared), and list the keys that agree with the
// threshold in those bits: sign, exponent and two more, so that a fiftieth of the candidates does, or a great many equal ones (tokens
// that nothing has looked at) do.  resolve's workgroups find the threshold's key among the listed ones, again each for itself, and
// put their kept tokens in their places.  8 heads of 128K, 16K kept: 37 us with a second digit in a launch of its own and workgroups of
// 16384 tokens, 32 without the second digit, 24 so (what is left of each launch is a chain of reads and meetings; the wide
// workgroups issued from a quarter of the CUs).

constexpr int kDigits = 2048;   // of the first digit

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

__device__ __forceinline__ uint32_t wave_total(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane(wave_inclusive_scan((int)x), 63); }

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
    int L, lo, hi, n_keep, cap;   // candidates lo .. hi - 1
    const float *w;
    int32_t *idx;
    __device__ __forceinline__ Span(const EvictKernelArgs &k, int b, int g)
    {
        bg = (int64_t)b * k.s.Hkv + g;
        L = (int)min((int64_t)max(k.s.ctx_len[b], 0), k.cap);
        n_keep = k.a.ns + k.a.k + k.a.nr;
        lo = k.a.ns;
        hi = L - k.a.nr;
        cap = (int)k.cap;
        w = k.a.weights + bg * k.cap;
        idx = k.a.keep_idx + bg * n_keep;
    }
    __device__ __forceinline__ bool all() const { return L <= n_keep; }
};

// N keys a thread: key[4 x + e] is that of token t0 + 4 (64 WAVES x + thread) + e, 0 where no candidate is.
template <int WAVES> __device__ __forceinline__ int token_at(int t0, int i) { return t0 + 4 * (64 * WAVES * (i / 4) + (int)threadIdx.x) + i % 4; }
template <int N, int WAVES> __device__ __forceinline__ void load_keys(const Span &s, int t0, uint32_t (&key)[N])
{
    float f[N];
#pragma unroll
    for (int x = 0; x < N; x += 4) {
        const int t = token_at<WAVES>(t0, x);
        f[x] = f[x + 1] = f[x + 2] = f[x + 3] = 0.f;
        if (t + 3 < s.cap) {   // (whatever the length is, so as not to wait for it; rows of weights start at any multiple of four bytes)
            __builtin_memcpy(f + x, __builtin_assume_aligned(s.w + t, 4), 16);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[x + e] = t + e < s.cap ? s.w[t + e] : 0.f;
        }
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
        const int t = token_at<WAVES>(t0, x);
        key[x] = t >= s.lo && t < s.hi ? weight_key(f[x]) : 0u;
    }
}

// Exclusive sums in token order of X counts a thread (two 16-bit counts a word), and the sum of all: one meeting for all X.
template <int X, int WAVES>
__device__ __forceinline__ uint32_t token_scan(const uint32_t (&mine)[X], uint32_t (*wave_tot)[X], uint32_t (&before)[X])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int x = 0; x < X; ++x) {
        const uint32_t in = (uint32_t)wave_inclusive_scan((int)mine[x]);
        if (lane == 63) wave_tot[wave][x] = in;
        before[x] = in - mine[x];
    }
    __syncthreads();
    uint32_t front = 0;
#pragma unroll
    for (int x = 0; x < X; ++x) {
        uint32_t in_front = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t v = wave_tot[w][x];
            in_front += w < wave ? v : 0u;
            all += v;
        }
        before[x] += front + in_front;
        front += all;
    }
    __syncthreads();
    return front;
}

// The kept tokens of t0 .. t0 + 64 N WAVES - 1 to their places, by way of LDS (`list`: as many entries): those with a key above
// `limit` and, in order, ties with it while there are less than `ties`; gt and eq: how many of either lie in front.
template <int N, int WAVES>
__device__ __forceinline__ void place_kept(const Span &s, int t0, const uint32_t (&key)[N], uint32_t limit, uint32_t ties, uint32_t gt, uint32_t eq,
                                           uint32_t (*wave_tot)[N / 4], int *list)
{
    uint32_t mine[N / 4], before[N / 4], is_gt = 0, is_eq = 0;   // bit x: of token x
#pragma unroll
    for (int x = 0; x < N; ++x) {
        const int t = token_at<WAVES>(t0, x);
        const bool cand = t >= s.lo && t < s.hi;
        is_gt |= t < s.L && (!cand || key[x] > limit) ? 1u << x : 0u;
        is_eq |= cand && ties && key[x] == limit ? 1u << x : 0u;
    }
#pragma unroll
    for (int x = 0; x < N / 4; ++x) mine[x] = (uint32_t)__popc(is_gt >> 4 * x & 15u) | (uint32_t)__popc(is_eq >> 4 * x & 15u) << 16;
    const uint32_t total = token_scan<N / 4, WAVES>(mine, wave_tot, before);
    const uint32_t base = gt + min(eq, ties);
#pragma unroll
    for (int x = 0; x < N / 4; ++x) {
        uint32_t n_gt = gt + (before[x] & 0xffffu), n_eq = eq + (before[x] >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool above = is_gt >> (4 * x + e) & 1u, same = is_eq >> (4 * x + e) & 1u;
            if (above || (same && n_eq < ties)) list[n_gt + min(n_eq, ties) - base] = token_at<WAVES>(t0, 4 * x + e);
            n_gt += above ? 1u : 0u;
            n_eq += same ? 1u : 0u;
        }
    }
    __syncthreads();
    const uint32_t n = gt + (total & 0xffffu) + min(eq + (total >> 16), ties) - base;
    for (uint32_t i = threadIdx.x; i < n; i += 64 * WAVES) s.idx[base + i] = list[i];
}

constexpr int kPickWaves = 16;
template <int N> __global__ __launch_bounds__(64 * kPickWaves) void pick_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[2048], wave_tot[kPickWaves], found[2], tots[kPickWaves][N / 4];
    __shared__ int list[64 * kPickWaves * N];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const Span s(k, b, g);
    uint32_t key[N];
    load_keys<N, kPickWaves>(s, 0, key);
    if (g == 0 && tid == 0) const_cast<int32_t *>(k.d.ctx_len)[b] = min(s.L, s.n_keep);
    if (s.all()) {
        for (int i = tid; i < s.n_keep; i += 64 * kPickWaves) s.idx[i] = i < s.L ? i : -1;
        return;
    }
    uint32_t prefix = 0, need = (uint32_t)k.a.k;
    if (need) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int width = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            for (int i = tid; i < 2048; i += 64 * kPickWaves) hist[i] = 0;
            __syncthreads();
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const int t = token_at<kPickWaves>(0, x);
                count_digit(hist, (key[x] >> shift) & ((1u << width) - 1u), t >= s.lo && t < s.hi && (pass == 0 || (key[x] >> (shift + width)) == prefix));
            }
            __syncthreads();
            find_digit<2048, kPickWaves>(hist, need, wave_tot, found);
            prefix = prefix << width | found[0];
            need -= found[1];
            __syncthreads();
        }
    } else {
        prefix = 0xffffffffu;   // (no key)
    }
    place_kept<N, kPickWaves>(s, 0, key, prefix, need, 0, 0, tots, list);
}

// ---- long caches: scratch of a (sequence, KV head) ----
constexpr int kPickMost = 16384;
constexpr int kHistKeys = 8, kHistTokens = 64 * kPickWaves * kHistKeys;          // of a histogram
constexpr int kWaves = 4, kKeys = 16, kChunk = 64 * kWaves * kKeys;               // of the other launches' workgroups
struct PickScratch {             // words
    uint32_t *state;             // the first digit, what is needed of it
    uint32_t *first;             // [histograms][kDigits / 2], two 16-bit counts a word
    uint32_t *chunk;             // [chunks][4]: keys above; candidates; their least and largest key
    uint32_t *cand;              // [chunks][kChunk]
};
static int64_t pick_chunks(int64_t cap) { return (cap + kHistTokens - 1) / kHistTokens * (kHistTokens / kChunk); }
__host__ __device__ constexpr int64_t pick_words(int64_t chunks) { return 64 + chunks / (kHistTokens / kChunk) * (kDigits / 2) + chunks * (4 + kChunk); }
__device__ __forceinline__ PickScratch pick_scratch(const EvictKernelArgs &k, int64_t bg)
{
    PickScratch p;
    p.state = k.a.scratch + bg * pick_words(k.chunks);
    p.first = p.state + 64;
    p.chunk = p.first + k.chunks / (kHistTokens / kChunk) * (kDigits / 2);
    p.cand = p.chunk + k.chunks * 4;
    return p;
}

__global__ __launch_bounds__(64 * kPickWaves) void first_digits_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[kDigits];
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kHistTokens, tid = threadIdx.x;
    const Span s(k, b, g);
    uint32_t key[kHistKeys];
    load_keys<kHistKeys, kPickWaves>(s, t0, key);
    if (s.all() || !k.a.k || t0 >= s.hi || t0 + kHistTokens <= s.lo) return;
    static_assert(kDigits == 2 * 64 * kPickWaves, "two digits a thread");
    hist[tid] = hist[tid + kDigits / 2] = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kHistKeys; ++x) {
        const int t = token_at<kPickWaves>(t0, x);
        count_digit(hist, key[x] >> 21, t >= s.lo && t < s.hi);
    }
    __syncthreads();
    pick_scratch(k, s.bg).first[(int64_t)blockIdx.x * (kDigits / 2) + tid] = hist[2 * tid] | hist[2 * tid + 1] << 16;
}

// All histograms added up (thread i: the eight digits from 8 i on).
__device__ __forceinline__ void sum_histograms(const Span &s, const uint32_t *from, uint32_t *hist)
{
    static_assert(kDigits == 8 * 64 * kWaves, "eight digits a thread");
    const int last = (s.hi + kHistTokens - 1) / kHistTokens;
    uint32_t n[8] = {};
#pragma unroll 8
    for (int c = s.lo / kHistTokens; c < last; ++c) {
        const uint4 v = *(const uint4 *)(from + (int64_t)c * (kDigits / 2) + 4 * (int)threadIdx.x);
        n[0] += v.x & 0xffffu; n[1] += v.x >> 16; n[2] += v.y & 0xffffu; n[3] += v.y >> 16;
        n[4] += v.z & 0xffffu; n[5] += v.z >> 16; n[6] += v.w & 0xffffu; n[7] += v.w >> 16;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) hist[8 * (int)threadIdx.x + i] = n[i];
    __syncthreads();
}

// What a chunk has above the first digit (tokens that stay in any case among them), and the keys that agree with them, in order.
__global__ __launch_bounds__(64 * kWaves) void collect_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[kDigits], wave_tot[kWaves], found[2], low[kWaves], high[kWaves], tots[kWaves][kKeys / 4];
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kChunk;
    const Span s(k, b, g);
    uint32_t key[kKeys];
    load_keys<kKeys, kWaves>(s, t0, key);
    if (s.all() || t0 >= s.L) return;
    const PickScratch p = pick_scratch(k, s.bg);
    uint32_t prefix = 0xffffffffu;
    if (k.a.k) {
        sum_histograms(s, p.first, hist);
        find_digit<kDigits, kWaves>(hist, (uint32_t)k.a.k, wave_tot, found);
        prefix = found[0];
        if (blockIdx.x == 0 && threadIdx.x == 0) { p.state[0] = prefix; p.state[1] = (uint32_t)k.a.k - found[1]; }
    }
    __syncthreads();
    uint32_t *const cand = p.cand + (int64_t)blockIdx.x * kChunk;
    uint32_t mine[kKeys / 4], before[kKeys / 4], lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int x = 0; x < kKeys / 4; ++x) {
        mine[x] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = token_at<kWaves>(t0, 4 * x + e);
            const bool c = t >= s.lo && t < s.hi;
            const uint32_t digit = key[4 * x + e] >> 21;
            mine[x] += t < s.L && (!c || (k.a.k && digit > prefix)) ? 1u : (c && digit == prefix ? 0x10000u : 0u);
        }
    }
    const uint32_t total = token_scan<kKeys / 4, kWaves>(mine, tots, before);
#pragma unroll
    for (int x = 0; x < kKeys / 4; ++x) {
        uint32_t at = before[x] >> 16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = token_at<kWaves>(t0, 4 * x + e);
            const uint32_t key1 = key[4 * x + e];
            if (!(t >= s.lo && t < s.hi && (key1 >> 21) == prefix)) continue;
            cand[at++] = key1;
            lo = min(lo, key1);
            hi = max(hi, key1);
        }
    }
    lo = wave_min_u32(lo);
    hi = wave_max_u32(hi);
    if ((threadIdx.x & 63) == 0) { low[threadIdx.x >> 6] = lo; high[threadIdx.x >> 6] = hi; }
    __syncthreads();
    if (threadIdx.x == 0) ((uint4 *)p.chunk)[blockIdx.x] = 
        make_uint4(total & 0xffffu, total >> 16, min(min(low[0], low[1]), min(low[2], low[3])), max(max(high[0], high[1]), max(high[2], high[3])));
}

// The threshold's key out of the listed ones, by every workgroup for itself, and the chunk's kept tokens in their places.
// Up to kListed candidates are in registers, whichever chunk they come from; more are read again for each digit.  (Looking for a
// candidate's chunk thread by thread, instead of by chunks into LDS, took 9 us of the launch's 18.)
constexpr int kListEach = 16, kListed = kListEach * 64 * kWaves, kListedChunks = 64 * kWaves;
__global__ __launch_bounds__(64 * kWaves) void resolve_kernel(EvictKernelArgs k)
{
    __shared__ uint32_t hist[2048], wave_tot[kWaves], found[2], upto[kListedChunks], tots[kWaves][kKeys / 4];
    __shared__ int list[kChunk];
    __shared__ uint4 sums[kWaves];
    const int g = blockIdx.y, b = blockIdx.z, t0 = (int)blockIdx.x * kChunk, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Span s(k, b, g);
    uint32_t key[kKeys];
    load_keys<kKeys, kWaves>(s, t0, key);
    if (g == 0 && blockIdx.x == 0 && tid == 0) const_cast<int32_t *>(k.d.ctx_len)[b] = min(s.L, s.n_keep);
    if (s.all()) {   // (the grid has the source's chunks, and more tokens may stay than it has room for)
        for (int64_t c = t0; c < s.n_keep; c += (int64_t)gridDim.x * kChunk)
            for (int i = (int)c + tid; i < min(s.n_keep, (int)c + kChunk); i += 64 * kWaves) s.idx[i] = i < s.L ? i : -1;
        return;
    }
    if (t0 >= s.L) return;
    const PickScratch p = pick_scratch(k, s.bg);
    const int chunks = (s.L + kChunk - 1) / kChunk;
    // in front: keys above, candidates; of all: the least and the largest candidate.  (By wavefront reductions: atomics of a wavefront on
    // one address are a loop over its lanes, 4 us for the four of them.)
    uint32_t gt = 0, eq = 0, lo = 0xffffffffu, hi = 0, mine = 0;
    for (int c = tid; c < chunks; c += 64 * kWaves) {
        const uint4 v = ((const uint4 *)p.chunk)[c];
        if (c < (int)blockIdx.x) { gt += v.x; eq += v.y; }
        mine += v.y;
        lo = min(lo, v.z);
        hi = max(hi, v.w);
    }
    const uint32_t sum4[4] = {wave_total(gt), wave_total(eq), wave_min_u32(lo), wave_max_u32(hi)};
    if (lane == 0) sums[wave] = make_uint4(sum4[0], sum4[1], sum4[2], sum4[3]);
    uint32_t total;
    const uint32_t in = block_scan<kWaves>(mine, wave_tot, total);   // (meets twice)
    upto[tid] = in;   // candidates of chunks 0 .. tid (of no use beyond kListedChunks)
    static_assert(kWaves == 4, "sums of four wavefronts");
    gt = sums[0].x + sums[1].x + sums[2].x + sums[3].x;
    eq = sums[0].y + sums[1].y + sums[2].y + sums[3].y;
    lo = min(min(sums[0].z, sums[1].z), min(sums[2].z, sums[3].z));
    hi = max(max(sums[0].w, sums[1].w), max(sums[2].w, sums[3].w));
    uint32_t limit = 0xffffffffu, ties = 0;
    if (k.a.k) {
        ties = p.state[1];
        limit = hi;
        if (lo != hi) {   // (else all are equal)
            const bool listed = total <= (uint32_t)kListed && chunks <= kListedChunks;
            uint32_t own[kListEach];
            __syncthreads();
            if (listed) {
                // a wavefront brings every fourth chunk's into LDS, one behind the other; then each thread takes its own
                for (int c0 = wave; c0 < chunks; c0 += 4 * kWaves) {
                    uint32_t from[4], n[4], x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int c = min(c0 + u * kWaves, chunks - 1);
                        from[u] = c ? upto[c - 1] : 0u;
                        n[u] = c0 + u * kWaves < chunks ? upto[c] - from[u] : 0u;
                        x[u] = (uint32_t)lane < n[u] ? p.cand[(int64_t)c * kChunk + lane] : 0u;
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        if ((uint32_t)lane < n[u]) list[from[u] + lane] = (int)x[u];
                        for (uint32_t i = lane + 64; i < n[u]; i += 64) list[from[u] + i] = (int)p.cand[(int64_t)(c0 + u * kWaves) * kChunk + i];
                    }
                }
                __syncthreads();
#pragma unroll
                for (int x = 0; x < kListEach; ++x) own[x] = (uint32_t)list[tid + x * 64 * kWaves];   // (behind the last: of no use)
                __syncthreads();   // (the list's place is wanted again)
            }
            // every candidate (all lanes of a wavefront come along): f(its key, whether it is one, whether its chunk lies in front)
            auto each = [&](auto f) __attribute__((always_inline)) {
                if (listed) {
#pragma unroll
                    for (int x = 0; x < kListEach; ++x) {
                        if (x * 64 * kWaves >= (int)total) break;
                        const uint32_t i = (uint32_t)tid + x * 64 * kWaves;
                        f(own[x], i < total, i < eq);
                    }
                } else {
                    for (int c = 0; c < chunks; ++c) {
                        const uint32_t n = p.chunk[4 * c + 1];
                        for (uint32_t i = tid; i < ((n + 63u) & ~63u); i += 64 * kWaves)
                            f(i < n ? p.cand[(int64_t)c * kChunk + i] : 0u, i < n, c < (int)blockIdx.x);
                    }
                }
            };
            limit = p.state[0];
#pragma unroll
            for (int shift = 10; shift >= 0; shift -= 10) {   // eleven bits, then ten
                const int width = shift ? 11 : 10;
                for (int i = tid; i < 2048; i += 64 * kWaves) hist[i] = 0;
                __syncthreads();
                each([&](uint32_t x, bool is, bool) { count_digit(hist, (x >> shift) & ((1u << width) - 1u), is && (x >> (shift + width)) == limit); });
                __syncthreads();
                find_digit<2048, kWaves>(hist, ties, wave_tot, found);
                limit = limit << width | found[0];
                ties -= found[1];
                __syncthreads();
            }
            uint32_t more = 0, same = 0;
            each([&](uint32_t x, bool is, bool front) {
                more += is && front && x > limit ? 1u : 0u;
                same += is && front && x == limit ? 1u : 0u;
            });
            more = wave_total(more);
            same = wave_total(same);
            if (lane == 0) sums[wave] = make_uint4(more, same, 0, 0);
            __syncthreads();
            gt += sums[0].x + sums[1].x + sums[2].x + sums[3].x;
            eq = sums[0].y + sums[1].y + sums[2].y + sums[3].y;
        }
    }
    place_kept<kKeys, kWaves>(s, t0, key, limit, ties, gt, eq, tots, list);
}

// Rows i, i + 1, ... of the new cache from rows keep_idx[i], ...; the weights with them, zeros behind.
// STREAM: past the caches, for moves that are larger than those: 134 MB 31.0 / 26.7 us (5.3 TB/s), 11 MB 4.2 / 4.9.
template <int ROW, bool STREAM>   // bytes of a row
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
            kk[u] = load_keys<STREAM>((const uint4 *)(sk + (int64_t)t[u] * k.s.st * elem));
            vv[u] = load_keys<STREAM>((const uint4 *)(sv + (int64_t)t[u] * k.s.st * elem));
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = r0 + u * RPP + rsub;
        if (t[u] >= 0) {
            store16<STREAM>(dk + (int64_t)r * k.d.st * elem, kk[u]);
            store16<STREAM>(dv + (int64_t)r * k.d.st * elem, vv[u]);
        }
    }
}

size_t evict_scratch_bytes(int64_t pairs, int64_t cap) { return cap > kPickMost ? (size_t)(pairs * pick_words(pick_chunks(cap))) * sizeof(uint32_t) : 0; }

hipError_t launch_evict(const Shape &s, const Shape &d, int dtype, const EvictArgs &a, hipStream_t st)
{
    const int64_t cap = (int64_t)s.max_blocks * s.B;
    const EvictKernelArgs k{s, d, a, cap, (int64_t)d.max_blocks * d.B, pick_chunks(cap)};
    const dim3 one(s.Hkv, s.batch), hists((unsigned)(k.chunks * kChunk / kHistTokens), s.Hkv, s.batch), chunks((unsigned)k.chunks, s.Hkv, s.batch), threads(64 * kPickWaves);
    // (us, whole call, 8 heads, a quarter kept: 4K with four keys a thread / sixteen / by many workgroups 10.8 / 14.8 / 21.3; 8K, sixteen / many
    // 17.0 / 24.3, 16K 21.5 / 26.8; 64 heads, 16K 64.6 / 70.1)
    if (cap <= 4096) {
        hipLaunchKernelGGL(pick_kernel<4>, one, threads, 0, st, k);
    } else if (cap <= kPickMost) {
        hipLaunchKernelGGL(pick_kernel<16>, one, threads, 0, st, k);
    } else {
        hipLaunchKernelGGL(first_digits_kernel, hists, threads, 0, st, k);
        hipLaunchKernelGGL(collect_kernel, chunks, dim3(64 * kWaves), 0, st, k);
        hipLaunchKernelGGL(resolve_kernel, chunks, dim3(64 * kWaves), 0, st, k);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int elem = dtype == SPECPV_BF16 ? 2 : 4, row = s.D * elem, per = 4 * 256 / (row / 16);
    const int64_t rows = a.new_weights ? k.dcap : (int64_t)a.ns + a.k + a.nr;
    const dim3 grid((unsigned)((rows + per - 1) / per), s.Hkv, s.batch);
    // Past the caches where the rows would only push each other out of them (bytes read and written; plain / past them, whole call, us: 64 MB 35.7 /
    // 36.4, 96 MB 43.6 / 42.8, 128 MB 54.6 / 49.9, 256 MB 79.5 / 72.1)
    const bool stream = (int64_t)s.batch * s.Hkv * rows * row * 4 > ((int64_t)64 << 20);
#define SPECPV_MOVE(ROW)                                                                                     \
    do {                                                                                                     \
        if (stream) hipLaunchKernelGGL((move_kernel<ROW, true>), grid, dim3(256), 0, st, k, elem);           \
        else hipLaunchKernelGGL((move_kernel<ROW, false>), grid, dim3(256), 0, st, k, elem);                 \
    } while (0)
    if (row == 512) SPECPV_MOVE(512);
    else if (row == 256) SPECPV_MOVE(256);
    else SPECPV_MOVE(128);
#undef SPECPV_MOVE
    return hipGetLastError();
}

}  // namespace specpv
