// Choice of pages: every kv head of a sequence ranks the pages by their mean keys,
//     score_j = max over the head's query heads h of q_h . mean_j,
// and keeps the first ones, the last ones and the best of the others.  The mean of a
// page's keys is what the chunk summaries use as a chunk's key; here it only decides
// which pages are attended exactly.
//
// The scores are 64-bit sums (of products that are exact for bf16 queries): which of two
// pages is kept must not depend on the order of a sum, and two pages of the same keys
// tie exactly, for the lower one.
#include "paged.hpp"

namespace eva {

namespace {

constexpr int kScoreWaves = 4;
constexpr int kChooseThreads = 512;
// Scores held in LDS by the choosing workgroup; longer rows are read again from memory.
constexpr int kChooseLds = kSelectAlone;
constexpr int kBins = 2048;  // 11 bits a pass
// Scores of the bin in which the choice ends that are ranked one against the other.
constexpr int kMaxTied = 256;

// Order of the scores as whole numbers: -0 and 0 alike, NaN above all (so that what it
// stands for reaches the output).
__device__ __forceinline__ unsigned long long ordered(double x) {
    if (x != x) return ~0ull;
    x = x + 0.0;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// The score again, in 32 bits; a NaN stays one.
__device__ __forceinline__ float score_of(unsigned long long k) {
    return (float)__builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k);
}

// Largest over the wave, in every lane.
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, __builtin_bit_cast(float, dpp<0xb1>(__builtin_bit_cast(int, x))));   // lanes 1 0 3 2 of a quad
    x = fmaxf(x, __builtin_bit_cast(float, dpp<0x4e>(__builtin_bit_cast(int, x))));   // 2 3 0 1
    x = fmaxf(x, __builtin_bit_cast(float, dpp<0x124>(__builtin_bit_cast(int, x))));  // a row of 16 turned by four
    x = fmaxf(x, __builtin_bit_cast(float, dpp<0x128>(__builtin_bit_cast(int, x))));  // by eight
    return xgroup_max(x);
}

__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
}
__device__ __forceinline__ void load4(const bf16* p, float (&x)[4]) {
    const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)v[i];
}

// How many pages of a sequence are ranked, those from a.first on; none where all are
// kept.
__device__ __forceinline__ int ranked(const SelectParams& a, int held) {
    return held > a.S ? held - a.first - a.last : 0;
}

// A wave scores 16 pages for four query heads at a time, with the matrix core's four
// products of 4 x 4 x 4: block c / 4 holds pages 4 (c / 4) + 0 .. 3 and all four the same heads,
//     A lane (g, c): page c, B: head c % 4, both contraction index g, which is feature
//     16 i + 4 g + e in step (i, e), so that the mean keys are 16-byte loads;
//     D lane (g, c): page 4 (c / 4) + g, head c % 4.
// (The 16 x 16 x 4 product, at the same rate, would spend three quarters of its columns on
// heads that there are not: 22 us against 11 for 256 rows of 513 pages, d = 128.)
// Scores 16 (tile + k tiles) + 0 .. 15 of the row go to put(index, score).  Returns how many
// pages are ranked.
template <int D, typename T, typename Put>
__device__ __forceinline__ int score_pages(const SelectParams& a, int b, int kvh, int tile, int tiles, Put put) {
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const T* heads = static_cast<const T*>(a.q) + ((size_t)b * a.H + (size_t)kvh * a.G) * D + 4 * g;
    // the heads h0 .. h0 + 3; past the last they repeat it, which changes no maximum
    double q[D / 4];
    auto load_heads = [&](int h0) {
        const T* row = heads + (size_t)min(h0 + (c & 3), a.G - 1) * D;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            float x[4];
            load4(row + 16 * i, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) q[4 * i + e] = (double)x[e];
        }
    };
    // a tile's pages are looked up one tile ahead, the first before the sequence's length is
    // known (any entry of its row may be read; what it names is checked below)
    const int* row = a.t.table + (size_t)b * a.t.max_pages;
    auto look_up = [&](int j) { return row[min(a.first + j + c, a.t.max_pages - 1)]; };
    int j0 = tile * 16, next = look_up(j0);
    load_heads(0);
    const int n = ranked(a, pages_of(held_tokens(a.t, b), a.t.shift));
    for (; j0 < n; j0 += tiles * 16) {
        const int page = next;  // past the last ranked page: others, whose scores are not used
        const bool lost = (unsigned)page >= (unsigned)a.t.n_pages;
        const float* mean = a.mean + ((size_t)(lost ? 0 : page) * a.Hkv + kvh) * D + 4 * g;
        floatx4 m[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) m[i] = *reinterpret_cast<const floatx4*>(mean + 16 * i);
        if (j0 + tiles * 16 < n) next = look_up(j0 + tiles * 16);
        const unsigned long long lost_rows = __builtin_amdgcn_ballot_w64(lost);
        unsigned long long best = 0;
        for (int h0 = 0; h0 < a.G; h0 += 4) {
            if (a.G > 4) load_heads(h0);
            double acc[4] = {0., 0., 0., 0.};  // four chains of products that wait for each other
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[e] = __builtin_amdgcn_mfma_f64_4x4x4f64((double)m[i][e], q[4 * i + e], acc[e], 0, 0, 0);
            const unsigned long long k = ordered((acc[0] + acc[1]) + (acc[2] + acc[3]));
            best = k > best ? k : best;
        }
        unsigned long long other = (unsigned long long)dpp<0xb1>((long long)best);  // lanes 1 0 3 2 of a quad
        best = other > best ? other : best;
        other = (unsigned long long)dpp<0x4e>((long long)best);                     // 2 3 0 1
        best = other > best ? other : best;
        const int j = (c & 12) + g;
        // a page that the pool does not have ranks first: its row becomes NaN
        if ((c & 3) == 0 && j0 + j < n) put(j0 + j, lost_rows >> j & 1 ? ~0ull : best);
    }
    return n;
}

// Bound by the mean keys' read and the chain table -> mean.
template <int D, typename T>
__global__ __launch_bounds__(kScoreWaves * 64) void paged_score_kernel(SelectParams a) {
    const int b = (int)blockIdx.y / a.Hkv, kvh = (int)blockIdx.y % a.Hkv;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    unsigned long long* keys = a.keys + (size_t)blockIdx.y * a.t.max_pages;
    score_pages<D, T>(a, b, kvh, (int)blockIdx.x * kScoreWaves + wave, (int)gridDim.x * kScoreWaves,
                      [&](int j, unsigned long long k) { keys[j] = k; });
}

// Of a workgroup's bins, the one in which the `want`-th highest score lies: each thread
// sums neighbouring bins from the top.
struct Found {
    int bin, above, count;  // scores in higher bins, and in this one
};
__device__ __forceinline__ void find_bin(const int* bins, int want, int* sums, Found* found) {
    constexpr int EACH = kBins / kChooseThreads;
    const int top = kBins - 1 - (int)threadIdx.x * EACH;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) mine += bins[top - i];
    int total;
    const int upto = block_scan(mine, sums, total);
    if (upto >= want && upto - mine < want) {
        int above = upto - mine;
        for (int i = 0; i < EACH; ++i) {
            if (above + bins[top - i] >= want) {
                *found = Found{top - i, above, bins[top - i]};
                break;
            }
            above += bins[top - i];
        }
    }
    __syncthreads();
}

// A workgroup per (sequence, kv head).  The scores are counted in bins of equal width
// between the lowest and the highest (a map that keeps their order, in 32 bits), which
// spreads them; the `want`-th highest lies in one bin, whose few scores are ranked one
// against the other.  Where it holds many (scores that tie, or one far from all others), a
// radix search over the bits finds it instead, 11 a pass.  Then the pages in their order.
// Bound by the passes' barriers.  SCORE: the workgroup makes the scores first, in LDS.
template <int D, typename T, bool SCORE>
__global__ __launch_bounds__(kChooseThreads) void paged_choose_kernel(SelectParams a) {
    __shared__ unsigned long long sh_keys[kChooseLds];
    __shared__ int bins[kBins];
    __shared__ long long sums[kChooseThreads / 64];
    __shared__ float sh_lo[kChooseThreads / 64], sh_hi[kChooseThreads / 64];
    __shared__ unsigned long long tied[kMaxTied];
    __shared__ int tied_at[kMaxTied];
    __shared__ Found found;
    __shared__ int sh_n, sh_want;
    __shared__ unsigned long long sh_key;
    int* isums = reinterpret_cast<int*>(sums);
    const int b = (int)blockIdx.x / a.Hkv, tid = threadIdx.x;
    const unsigned long long* gkeys = a.keys + (size_t)blockIdx.x * a.t.max_pages;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < kBins; i += kChooseThreads) bins[i] = 0;
    if (tid == 0) sh_n = 0;
    if constexpr (SCORE) {
        score_pages<D, T>(a, b, (int)blockIdx.x % a.Hkv, wave, kChooseThreads / 64,
                          [&](int j, unsigned long long k) { sh_keys[j] = k; });
        __syncthreads();
    }
    // the first scores, before the sequence's length is known (what lies past it is not used)
    constexpr int EARLY = 4;
    unsigned long long early[EARLY] = {};
    if constexpr (!SCORE) {
#pragma unroll
        for (int i = 0; i < EARLY; ++i)
            if (tid + i * kChooseThreads < a.t.max_pages) early[i] = gkeys[tid + i * kChooseThreads];
    }
    const int held = pages_of(held_tokens(a.t, b), a.t.shift);
    int* out = a.pages + (size_t)blockIdx.x * a.S;
    if (held <= a.S) {  // all of them
        for (int i = tid; i < a.S; i += kChooseThreads) out[i] = i < held ? i : -1;
        return;
    }
    for (int i = tid; i < a.first; i += kChooseThreads) out[i] = i;
    for (int i = tid; i < a.last; i += kChooseThreads) out[a.S - a.last + i] = held - a.last + i;
    const int n = ranked(a, held);
    int want = a.S - a.first - a.last;
    if (want == 0) return;
    const bool in_lds = SCORE || n <= kChooseLds;
    auto key = [&](int i) { return in_lds ? sh_keys[i] : gkeys[i]; };

    // the finite scores' range
    float low = INFINITY, high = -INFINITY;
    auto count = [&](int i, unsigned long long k) {
        if (!SCORE && in_lds) sh_keys[i] = k;
        const float x = score_of(k);
        if (fabsf(x) < INFINITY) {
            low = fminf(low, x);
            high = fmaxf(high, x);
        }
    };
    if constexpr (SCORE) {
        for (int i = tid; i < n; i += kChooseThreads) count(i, sh_keys[i]);
    } else {
#pragma unroll
        for (int i = 0; i < EARLY; ++i)
            if (tid + i * kChooseThreads < n) count(tid + i * kChooseThreads, early[i]);
        for (int i = tid + EARLY * kChooseThreads; i < n; i += kChooseThreads) count(i, gkeys[i]);
    }
    low = -wave_max(-low);
    high = wave_max(high);
    if ((tid & 63) == 0) {
        sh_lo[wave] = low;
        sh_hi[wave] = high;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kChooseThreads / 64; ++w) {
        low = fminf(low, sh_lo[w]);
        high = fmaxf(high, sh_hi[w]);
    }
    const float scale = high > low ? (kBins - 1) / (high - low) : 0.f;
    // (a range beyond the type's gives scale 0; infinities and NaN lie in the outer bins)
    auto bin_of = [&](unsigned long long k) {
        const float x = score_of(k);
        if (!(x < INFINITY)) return kBins - 1;
        const float at = (x - low) * scale;
        return at > 0.f ? at < kBins - 1 ? (int)at : kBins - 1 : 0;
    };
    for (int i = tid; i < n; i += kChooseThreads) atomicAdd(&bins[bin_of(key(i))], 1);  // whole numbers: any order
    __syncthreads();
    find_bin(bins, want, isums, &found);
    const Found f = found;
    unsigned long long prefix = 0;
    int shift = 64;
    if (f.count <= kMaxTied) {
        for (int i = tid; i < n; i += kChooseThreads) {
            const unsigned long long k = key(i);
            if (bin_of(k) == f.bin) {
                const int at = atomicAdd(&sh_n, 1);
                tied[at] = k;
                tied_at[at] = i;
            }
        }
        __syncthreads();
        if (tid < f.count) {
            const unsigned long long k = tied[tid];
            const int at = tied_at[tid];
            int above = 0, before = 0;  // of the bin: higher ones, and equal ones of lower pages
            for (int i = 0; i < f.count; ++i) {
                above += tied[i] > k;
                before += tied[i] == k && tied_at[i] < at;
            }
            if (f.above + above + before == want - 1) {  // the last one taken
                sh_key = k;
                sh_want = before + 1;
            }
        }
        __syncthreads();
        prefix = sh_key;
        want = sh_want;
        shift = 0;
    }
    // scores whose bits from `shift` on are `prefix` are still open; all above it are taken
    while (shift > 0) {
        const int next = max(shift - 11, 0), width = shift - next;
        __syncthreads();  // the last use of bins and found is over
        for (int i = tid; i < kBins; i += kChooseThreads) bins[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kChooseThreads) {
            const unsigned long long k = key(i);
            if (shift == 64 || k >> shift == prefix) atomicAdd(&bins[(int)(k >> next) & ((1 << width) - 1)], 1);
        }
        __syncthreads();
        find_bin(bins, want, isums, &found);
        prefix = shift == 64 ? (unsigned long long)found.bin : prefix << width | (unsigned)found.bin;
        want -= found.above;
        shift = next;
        if (found.count == want) break;
    }
    // taken: above the prefix; of those at it, the first `want`.  One scan of both counts.
    const int each = (n + kChooseThreads - 1) / kChooseThreads;
    const int i0 = min(tid * each, n), i1 = min(i0 + each, n);
    long long mine = 0;  // above: low half, at: high half
    for (int i = i0; i < i1; ++i) {
        const unsigned long long k = key(i) >> shift;
        mine += k > prefix ? 1 : k == prefix ? 1ll << 32 : 0;
    }
    long long total;
    const long long before = block_scan(mine, sums, total) - mine;
    int at = (int)(before >> 32);
    int to = (int)before + min(at, want);
    for (int i = i0; i < i1; ++i) {
        const unsigned long long k = key(i) >> shift;
        if (k > prefix || (k == prefix && at++ < want)) out[a.first + to++] = a.first + i;
    }
}

}  // namespace

template <int D, typename T>
hipError_t launch_paged_select(const SelectParams& p, hipStream_t stream) {
    const int rows = p.t.B * p.Hkv;
    if (!p.keys) {
        paged_choose_kernel<D, T, true><<<rows, kChooseThreads, 0, stream>>>(p);
        return hipGetLastError();
    }
    const int tiles = (p.t.max_pages + kScoreWaves * 16 - 1) / (kScoreWaves * 16);
    const int most = (768 + rows - 1) / rows;  // as many as the CUs hold at once
    paged_score_kernel<D, T><<<dim3(tiles < most ? tiles : most, rows), kScoreWaves * 64, 0, stream>>>(p);
    paged_choose_kernel<D, T, false><<<rows, kChooseThreads, 0, stream>>>(p);
    return hipGetLastError();
}
template hipError_t launch_paged_select<64, bf16>(const SelectParams&, hipStream_t);
template hipError_t launch_paged_select<128, bf16>(const SelectParams&, hipStream_t);
template hipError_t launch_paged_select<64, float>(const SelectParams&, hipStream_t);
template hipError_t launch_paged_select<128, float>(const SelectParams&, hipStream_t);

}  // namespace eva
