// Pages and places of a paged cache: which pages a sequence has, where its new
// tokens go, and the append that writes them there.
#include "paged.hpp"

namespace eva {

namespace {

// ---------------------------------------------------------------------------
// table
// ---------------------------------------------------------------------------
// The free pages are a stack.  Both calls are exclusive prefix sums over the
// sequences' numbers of pages: the r-th new page, in the order of (sequence, page),
// is the r-th from the top, and pages given back are laid down in the reverse
// order, so that a rollback restores the stack it started from.  One workgroup
// walks all sequences, a thread each, since every sequence's pages depend on the
// sum before it.  Bound by latency (a scan and a handful of dependent loads).
constexpr int kTableThreads = 1024;
// Tokens of a sequence whose slots the scanning thread writes by itself (a page holds 16 at
// least, so they need one new page at most); more go through a launch of their own.
constexpr int kFewTokens = 16;
// Slots that a workgroup of that launch writes.
constexpr int kSlotTile = 1024;

__global__ __launch_bounds__(kTableThreads) void page_extend_kernel(PageTableView t, const int* __restrict__ counts, int T,
                                                                    int* __restrict__ slots, int* __restrict__ start,
                                                                    int* __restrict__ granted) {
    __shared__ long long sums[kTableThreads / 64];
    const int tid = threadIdx.x;
    const int mask = (1 << t.shift) - 1;
    const int n_free = min(max(t.n_free[0], 0), t.n_pages);
    long long carry = 0;
    for (int b0 = 0; b0 < t.B; b0 += (int)blockDim.x) {
        const int b = b0 + tid;
        int n = 0, c = 0, held = 0;
        if (b < t.B) {
            n = held_tokens(t, b);
            c = counts ? min(max(counts[b], 0), T) : T;
            if (c > (t.max_pages << t.shift) - n) c = 0;
            held = pages_of(n, t.shift);
        }
        int need = pages_of(n + c, t.shift) - held;
        long long total;
        const long long upto = carry + block_scan((long long)need, sums, total);  // may pass 2^31
        carry += total;
        // a sequence that the stack does not suffice for gets nothing; what it asked
        // for still counts, so that later ones do not overtake it
        if (need > 0 && upto > n_free) c = need = 0;
        if (b < t.B) {
            start[b] = n;
            granted[b] = c;
            t.n_tok[b] = n + c;
            const int top = n_free - 1 - (int)(need > 0 ? upto - need : 0);  // its first new page
            int* row = slots + (size_t)b * T;
            if (T <= kFewTokens) {
                int* pages = t.table + (size_t)b * t.max_pages;
                const int last = c > 0 && (n & mask) ? pages[held - 1] : 0;
                const int fresh = need > 0 ? t.free_pages[top] : 0;
                if (need > 0) pages[held] = fresh;
                for (int i = 0; i < T; ++i) {
                    const int p = n + i;
                    row[i] = i < c ? ((p >> t.shift) < held ? last : fresh) << t.shift | (p & mask) : -1;
                }
            } else {
                // the tiles of the second launch find it in their first slot
                for (int i = 0; i < T; i += kSlotTile) row[i] = top;
            }
        }
    }
    __shared__ int taken;  // pages
    if (tid == 0) taken = 0;
    __syncthreads();
    int mine = 0;
    for (int b = tid; b < t.B; b += (int)blockDim.x)
        mine += pages_of(start[b] + granted[b], t.shift) - pages_of(start[b], t.shift);
    if (mine) atomicAdd(&taken, mine);  // whole numbers: any order
    __syncthreads();
    if (tid == 0) t.n_free[0] = n_free - taken;
}

// Slots and new pages of many tokens a sequence: a workgroup per kSlotTile tokens.
// Pages that the sequence had are read from its row, new ones from the stack, so that no
// workgroup reads what another writes.  Bound by the slots' write.
__global__ __launch_bounds__(256) void page_slots_kernel(PageTableView t, int T, int* __restrict__ slots,
                                                         const int* __restrict__ start, const int* __restrict__ granted) {
    const int b = blockIdx.y, t0 = (int)blockIdx.x * kSlotTile;
    const int n = start[b], c = granted[b];
    int* row = slots + (size_t)b * T;
    const int top = row[t0];
    __syncthreads();  // read before the first slot is written
    const int held = pages_of(n, t.shift), mask = (1 << t.shift) - 1;
    int* pages = t.table + (size_t)b * t.max_pages;
    for (int i = t0 + (int)threadIdx.x; i < min(T, t0 + kSlotTile); i += 256) {
        int s = -1;
        if (i < c) {
            const int p = n + i, lp = p >> t.shift;
            const int page = lp < held ? pages[lp] : t.free_pages[top - (lp - held)];
            s = page << t.shift | (p & mask);
            if (lp >= held && (p & mask) == 0) pages[lp] = page;
        }
        row[i] = s;
    }
}

__global__ __launch_bounds__(kTableThreads) void page_truncate_kernel(PageTableView t, const int* __restrict__ lens) {
    __shared__ long long sums[kTableThreads / 64];
    __shared__ int last[kTableThreads];   // pages dropped up to and with a sequence of the batch
    __shared__ int first[kTableThreads];  // a sequence's first dropped page
    const int tid = threadIdx.x;
    const int n_free = min(max(t.n_free[0], 0), t.n_pages);
    // the number of all dropped pages comes first: the stack's new top
    int mine = 0;
    for (int b = tid; b < t.B; b += (int)blockDim.x) {
        const int n = held_tokens(t, b);
        mine += pages_of(n, t.shift) - pages_of(min(n, max(lens[b], 0)), t.shift);
    }
    long long all;
    block_scan((long long)mine, sums, all);
    const int dropped = (int)min(all, (long long)t.n_pages);
    int base = 0;
    for (int b0 = 0; b0 < t.B; b0 += (int)blockDim.x) {
        const int b = b0 + tid;
        int drop = 0, keep = 0;
        if (b < t.B) {
            const int n = held_tokens(t, b);
            const int m = min(n, max(lens[b], 0));
            keep = pages_of(m, t.shift);
            drop = pages_of(n, t.shift) - keep;
            t.n_tok[b] = m;
        }
        long long total;
        const long long upto = block_scan((long long)drop, sums, total);
        if (total == 0) continue;  // the same for the whole workgroup
        last[tid] = (int)upto;
        first[tid] = keep;
        __syncthreads();
        // dropped pages in turn over all threads: rank r lies in the first sequence whose
        // running sum passes it
        for (int r = tid; r < (int)total; r += (int)blockDim.x) {
            int lo = 0, hi = (int)blockDim.x - 1;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (last[mid] > r) hi = mid;
                else lo = mid + 1;
            }
            int* entry = t.table + (size_t)(b0 + lo) * t.max_pages + first[lo] + (r - (lo ? last[lo - 1] : 0));
            const int at = n_free + dropped - 1 - (base + r);
            if (at >= 0 && at < t.n_pages) t.free_pages[at] = *entry;
            *entry = -1;
        }
        base += (int)total;
        __syncthreads();
    }
    if (tid == 0) t.n_free[0] = min(n_free + dropped, t.n_pages);
}

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
// One workgroup per (run of tokens that share a page, kv head, sequence): run j
// holds the tokens i with (o + i) / P = j, where o is the first token's place in
// its page.  Rows go to their slots; the last row of a page brings the mean of
// the page's keys, summed in fp32 in one fixed order over the rows as the cache
// holds them, so that it has the same bits however the tokens came in.
constexpr int kAppendThreads = 256;

template <int D, typename T>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(PagedAppendParams a) {
    constexpr int EPC = 16 / (int)sizeof(T);  // elements of a 16-byte piece
    constexpr int CH = D / EPC;               // pieces of a row
    constexpr int ROWS = 32;                  // rows of values staged at a time
    __shared__ T tile[ROWS][D + 16 / sizeof(T)];
    __shared__ int sh_slot[256];
    __shared__ float part[kAppendThreads / (D / 4)][D];
    const int P = 1 << a.shift, mask = P - 1;
    const int kvh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const int* srow = a.slots + (size_t)b * a.T;
    const int n_slots = a.n_pages << a.shift;
    const int o = srow[0] >= 0 ? srow[0] & mask : 0;
    const int i0 = max((int)blockIdx.x * P - o, 0), i1 = min((int)blockIdx.x * P - o + P, a.T);
    const int rows = i1 - i0;
    if (rows <= 0) return;
    // slots of the run (P <= 256), -1 for what does not lie in the pool
    if (tid < rows) {
        const int s = srow[i0 + tid];
        sh_slot[tid] = s < n_slots ? s : -1;
    }
    __syncthreads();
    const size_t src = (((size_t)b * a.Hkv + kvh) * a.T + i0) * D;
    const T* kn = static_cast<const T*>(a.k_new) + src;
    const T* vn = static_cast<const T*>(a.v_new) + src;
    T* kp = static_cast<T*>(a.k);
    T* vp = static_cast<T*>(a.vt);
    auto page_at = [&](int slot) { return ((size_t)(slot >> a.shift) * a.Hkv + kvh) * ((size_t)P * D); };

    for (int e = tid; e < rows * CH; e += kAppendThreads) {
        const int r = e / CH, ch = e % CH, s = sh_slot[r];
        if (s < 0) continue;
        *reinterpret_cast<u32x4*>(kp + page_at(s) + (size_t)(s & mask) * D + ch * EPC) =
            *reinterpret_cast<const u32x4*>(kn + (size_t)r * D + ch * EPC);
    }
    // values: 32 rows through LDS, then the slots of a feature that share a tile of
    // eight in one or two 16-byte pieces where all eight are here, else one by one
    for (int r0 = 0; r0 < rows; r0 += ROWS) {
        const int nr = min(ROWS, rows - r0);
        for (int e = tid; e < nr * CH; e += kAppendThreads) {
            const int r = e / CH, ch = e % CH;
            *reinterpret_cast<u32x4*>(&tile[r][ch * EPC]) =
                *reinterpret_cast<const u32x4*>(vn + (size_t)(r0 + r) * D + ch * EPC);
        }
        __syncthreads();
        // rows by tile of eight: the first and the last may be short
        const int s0 = sh_slot[r0];
        const int skew = s0 >= 0 ? s0 & 7 : 0;
        const int groups = (nr + skew + 7) / 8;
        for (int e = tid; e < groups * D; e += kAppendThreads) {
            const int f = e % D, gr = e / D;
            const int ra = max(gr * 8 - skew, 0), rb = min(gr * 8 - skew + 8, nr);
            const int sa = sh_slot[r0 + ra];
            const bool whole = rb - ra == 8 && sa >= 0 && (sa & 7) == 0 && sh_slot[r0 + rb - 1] == sa + 7;
            if (whole) {
                T w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = tile[ra + i][f];
                u32x4* dst = reinterpret_cast<u32x4*>(vp + page_at(sa) + vt_index<D>(f, sa & mask));
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) dst[i] = reinterpret_cast<const u32x4*>(w)[i];
            } else {
                for (int r = ra; r < rb; ++r) {
                    const int s = sh_slot[r0 + r];
                    if (s >= 0) vp[page_at(s) + vt_index<D>(f, s & mask)] = tile[r][f];
                }
            }
        }
        __syncthreads();
    }

    const int end = sh_slot[rows - 1];
    if (!a.mean || end < 0 || (end & mask) != mask) return;
    // row r of the page is token r - (P - rows) of the run, or already there
    constexpr int NP = kAppendThreads / (D / 4);  // partial sums of a feature
    const int f = tid % (D / 4) * 4, part_i = tid / (D / 4);
    const int have = P - rows;
    const T* page = kp + page_at(end);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int r = part_i; r < P; r += NP) {
        const T* x = (r < have ? page + (size_t)r * D : kn + (size_t)(r - have) * D) + f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += to_f32(x[i]);
    }
    *reinterpret_cast<floatx4*>(&part[part_i][f]) = sum;
    __syncthreads();
    if (tid < D) {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) m += part[i][tid];
        a.mean[((size_t)(end >> a.shift) * a.Hkv + kvh) * D + tid] = m / (float)P;
    }
}

}  // namespace

// A thread per sequence (a barrier of 16 waves costs more than one of four).
static int table_threads(int B) { return B <= 64 ? 64 : B <= 256 ? 256 : kTableThreads; }

hipError_t launch_page_truncate(const PageTableView& t, const int* lens, hipStream_t stream) {
    page_truncate_kernel<<<1, table_threads(t.B), 0, stream>>>(t, lens);
    return hipGetLastError();
}

hipError_t launch_page_extend(const PageTableView& t, const int* counts, int T, int* slots, int* start, int* granted,
                              hipStream_t stream) {
    page_extend_kernel<<<1, table_threads(t.B), 0, stream>>>(t, counts, T, slots, start, granted);
    if (T > kFewTokens)
        page_slots_kernel<<<dim3((T + kSlotTile - 1) / kSlotTile, t.B), 256, 0, stream>>>(t, T, slots, start, granted);
    return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_paged_append(const PagedAppendParams& p, hipStream_t stream) {
    const int P = 1 << p.shift;
    const int runs = p.T == 1 ? 1 : (p.T + P - 1 + P - 1) / P;  // the first may begin at a page's last place
    paged_append_kernel<D, T><<<dim3(runs, p.Hkv, p.B), kAppendThreads, 0, stream>>>(p);
    return hipGetLastError();
}
template hipError_t launch_paged_append<64, bf16>(const PagedAppendParams&, hipStream_t);
template hipError_t launch_paged_append<128, bf16>(const PagedAppendParams&, hipStream_t);
template hipError_t launch_paged_append<64, float>(const PagedAppendParams&, hipStream_t);
template hipError_t launch_paged_append<128, float>(const PagedAppendParams&, hipStream_t);

}  // namespace eva
