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

typedef double doublex4 __attribute__((ext_vector_type(4)));

constexpr int kScoreWaves = 4;
constexpr int kChooseThreads = 512;
// Scores held in LDS by the choosing workgroup; longer rows are read again from memory.
constexpr int kChooseLds = 4096;
constexpr int kBins = 2048;  // 11 bits a pass

// Order of the scores as whole numbers: -0 and 0 alike, NaN above all (so that what it
// stands for reaches the output).
__device__ __forceinline__ unsigned long long ordered(double x) {
    if (x != x) return ~0ull;
    x = x + 0.0;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// Pages of sequence b that are ranked: [lo, hi).  None where all are kept.
__device__ __forceinline__ void ranked(const SelectParams& a, int held, int& lo, int& hi) {
    lo = hi = 0;
    if (held > a.S) {
        lo = a.first;
        hi = held - a.last;
    }
}

// One wave scores 16 pages: A = their mean keys, B = 16 query heads, contraction step (i, e)
// of lane group g feature 16 i + 4 g + e, so that both are 16-byte loads.  D: lane (g, c)
// holds pages 4 r + g (r = 0 .. 3) for head c.  Bound by the mean keys' read.
template <int D, typename T>
__global__ __launch_bounds__(kScoreWaves * 64) void paged_score_kernel(SelectParams a) {
    const int b = (int)blockIdx.y / a.Hkv, kvh = (int)blockIdx.y % a.Hkv;
    const int held = pages_of(held_tokens(a.t, b), a.t.shift);
    int lo, hi;
    ranked(a, held, lo, hi);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, c = lane & 15;
    const int step = gridDim.x * kScoreWaves * 16;
    for (int j0 = lo + ((int)blockIdx.x * kScoreWaves + wave) * 16; j0 < hi; j0 += step) {
        // rows past the last repeat it
        const int page = a.t.table[(size_t)b * a.t.max_pages + min(j0 + c, hi - 1)];
        const bool lost = (unsigned)page >= (unsigned)a.t.n_pages;
        const float* mean = a.mean + ((size_t)(lost ? 0 : page) * a.Hkv + kvh) * D + 4 * g;
        floatx4 m[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) m[i] = *reinterpret_cast<const floatx4*>(mean + 16 * i);
        const unsigned long long lost_rows = __builtin_amdgcn_ballot_w64(lost);
        unsigned long long best[4] = {0, 0, 0, 0};
        for (int h0 = 0; h0 < a.G; h0 += 16) {
            const T* q = static_cast<const T*>(a.q) + ((size_t)b * a.H + kvh * a.G + min(h0 + c, a.G - 1)) * D + 4 * g;
            doublex4 acc = {0., 0., 0., 0.};
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)m[i][e], (double)to_f32(q[16 * i + e]), acc, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const unsigned long long k = ordered(acc[r]);
                best[r] = k > best[r] ? k : best[r];
            }
        }
        unsigned long long* out = a.keys + (size_t)blockIdx.y * a.t.max_pages;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) {
                const unsigned long long k = __shfl_xor(best[r], s);
                best[r] = k > best[r] ? k : best[r];
            }
            const int j = 4 * r + g;
            // a page that the pool does not have ranks first: its row becomes NaN
            if (c == 0 && j0 + j < hi) out[j0 + j] = lost_rows >> j & 1 ? ~0ull : best[r];
        }
    }
}

// Inclusive sum over the workgroup's threads, and the whole sum.
__device__ __forceinline__ int scan(int x, int* sums, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int y = __shfl_up(x, i);
        if (lane >= i) x += y;
    }
    __syncthreads();  // the last use of sums is over
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < kChooseThreads / 64; ++w) {
        const int s = sums[w];
        if (w < wave) before += s;
        total += s;
    }
    return x + before;
}

// A workgroup per (sequence, kv head): the k-th largest score by a radix search, 11 bits
// a pass, which ends as soon as a bin holds as many scores as are still wanted (two or
// three passes for scores that differ); then the pages in their order.
__global__ __launch_bounds__(kChooseThreads) void paged_choose_kernel(SelectParams a) {
    __shared__ unsigned long long sh_keys[kChooseLds];
    __shared__ int bins[kBins];
    __shared__ int sums[kChooseThreads / 64];
    __shared__ int sh_bin, sh_above, sh_count;
    const int b = (int)blockIdx.x / a.Hkv, tid = threadIdx.x;
    const int held = pages_of(held_tokens(a.t, b), a.t.shift);
    int lo, hi;
    ranked(a, held, lo, hi);
    int* out = a.pages + (size_t)blockIdx.x * a.S;
    if (hi == lo && held <= a.S) {  // all of them
        for (int i = tid; i < a.S; i += kChooseThreads) out[i] = i < held ? i : -1;
        return;
    }
    for (int i = tid; i < a.first; i += kChooseThreads) out[i] = i;
    for (int i = tid; i < a.last; i += kChooseThreads) out[a.S - a.last + i] = held - a.last + i;
    const int n = hi - lo;
    int want = a.S - a.first - a.last;
    if (want == 0) return;
    const unsigned long long* gkeys = a.keys + (size_t)blockIdx.x * a.t.max_pages + lo;
    const bool in_lds = n <= kChooseLds;
    if (in_lds)
        for (int i = tid; i < n; i += kChooseThreads) sh_keys[i] = gkeys[i];
    auto key = [&](int i) { return in_lds ? sh_keys[i] : gkeys[i]; };
    // scores whose bits from `shift` on are `prefix` are still open; all above it are taken
    unsigned long long prefix = 0;
    int shift = 64;
    while (shift > 0) {
        const int next = max(shift - 11, 0), width = shift - next;
        for (int i = tid; i < kBins; i += kChooseThreads) bins[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kChooseThreads) {
            const unsigned long long k = key(i);
            if (shift == 64 || k >> shift == prefix) atomicAdd(&bins[(int)(k >> next) & ((1 << width) - 1)], 1);
        }
        __syncthreads();
        // the highest bin with `want` scores in it and above it: four bins a thread, from the top
        constexpr int EACH = kBins / kChooseThreads;
        int mine = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) mine += bins[kBins - 1 - (tid * EACH + i)];
        int total;
        int upto = scan(mine, sums, total);
        if (upto >= want && upto - mine < want) {
            int above = upto - mine;
            for (int i = 0; i < EACH; ++i) {
                const int bin = kBins - 1 - (tid * EACH + i);
                if (above + bins[bin] >= want) {
                    sh_bin = bin;
                    sh_above = above;
                    sh_count = bins[bin];
                    break;
                }
                above += bins[bin];
            }
        }
        __syncthreads();
        prefix = shift == 64 ? (unsigned long long)sh_bin : prefix << width | (unsigned)sh_bin;
        want -= sh_above;
        shift = next;
        if (sh_count == want) break;
    }
    // taken: above the prefix; of those at it, the first `want` (all, unless 64 bits tie)
    const int each = (n + kChooseThreads - 1) / kChooseThreads;
    const int i0 = min(tid * each, n), i1 = min(i0 + each, n);
    int above = 0, at = 0;
    for (int i = i0; i < i1; ++i) {
        const unsigned long long k = key(i) >> shift;
        above += k > prefix;
        at += k == prefix;
    }
    int total;
    const int at_before = scan(at, sums, total) - at;
    const int taken_at = min(max(want - at_before, 0), at);
    int to = scan(above + taken_at, sums, total) - (above + taken_at);
    int left = taken_at;
    for (int i = i0; i < i1; ++i) {
        const unsigned long long k = key(i) >> shift;
        if (k > prefix || (k == prefix && left-- > 0)) out[a.first + to++] = lo + i;
    }
}

}  // namespace

template <int D, typename T>
hipError_t launch_paged_select(const SelectParams& p, hipStream_t stream) {
    const int rows = p.t.B * p.Hkv;
    if (p.t.max_pages > p.S) {
        const int tiles = (p.t.max_pages + kScoreWaves * 16 - 1) / (kScoreWaves * 16);
        const int most = (2048 + rows - 1) / rows;
        paged_score_kernel<D, T><<<dim3(tiles < most ? tiles : most, rows), kScoreWaves * 64, 0, stream>>>(p);
    }
    paged_choose_kernel<<<rows, kChooseThreads, 0, stream>>>(p);
    return hipGetLastError();
}
template hipError_t launch_paged_select<64, bf16>(const SelectParams&, hipStream_t);
template hipError_t launch_paged_select<128, bf16>(const SelectParams&, hipStream_t);
template hipError_t launch_paged_select<64, float>(const SelectParams&, hipStream_t);
template hipError_t launch_paged_select<128, float>(const SelectParams&, hipStream_t);

}  // namespace eva
