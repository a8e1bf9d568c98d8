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

// Slot of place `off` of a page.  Where the pool does not have it: a negative one, from which the
// append still learns the place (page << shift could pass 2^32 and come back inside).
__device__ __forceinline__ int slot_of(const PageTableView& t, int page, int off) {
    return ((unsigned)page < (unsigned)t.n_pages ? page << t.shift : -(1 << t.shift)) | off;
}

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
                    row[i] = i < c ? slot_of(t, (p >> t.shift) < held ? last : fresh, p & mask) : -1;
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
            s = slot_of(t, page, p & mask);
            if (lp >= held && (p & mask) == 0) pages[lp] = page;
        }
        row[i] = s;
    }
}

__global__ __launch_bounds__(kTableThreads) void page_truncate_kernel(PageTableView t, const int* __restrict__ lens) {
    __shared__ long long sums[kTableThreads / 64];
    __shared__ int last[kTableThreads];   // pages dropped up to and with a sequence of the batch
    __shared__ int first[kTableThreads];  // a sequence's first dropped page
    constexpr int EACH = 4;
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
        for (int r0 = tid; r0 < (int)total; r0 += EACH * (int)blockDim.x) {
            // EACH searches side by side, since each is a chain of LDS reads
            int at[EACH];
#pragma unroll
            for (int k = 0; k < EACH; ++k) at[k] = 0;
            for (int half = (int)blockDim.x / 2; half; half /= 2)
#pragma unroll
                for (int k = 0; k < EACH; ++k)
                    if (last[at[k] + half - 1] <= r0 + k * (int)blockDim.x) at[k] += half;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int r = r0 + k * (int)blockDim.x, l = at[k];
                if (r >= (int)total) break;
                int* entry = t.table + (size_t)(b0 + l) * t.max_pages + first[l] + (r - (l ? last[l - 1] : 0));
                const int to = n_free + dropped - 1 - (base + r);
                if (to >= 0 && to < t.n_pages) t.free_pages[to] = *entry;
                *entry = -1;
            }
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
//
// Threads hold 16-byte pieces of the rows, a piece's thread by the row's place in the page:
// keys go from registers to their rows and into the sums; values pass through LDS,
// from which a lane takes the eight slots of a feature, the tiles' 16 bytes.  Rows
// without a slot (a shorter sequence's padding) are not read.  Bound by memory for prompts
// (three prompts of up to 4096 tokens, 8 kv heads, d = 128: 80 MB in 15 us, 5.3 TB/s, in fp32
// 159 MB in 34 us, 4.6 TB/s; in bf16 18 with
// stores that keep their lines in the L2, 19 with 64 rows at a time, whose reads and
// writes overlap less), by the chain slot -> row -> store for single tokens (64
// sequences 3.5 us).
constexpr int kAppendThreads = 256;

template <int D, typename T>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(PagedAppendParams a) {
    constexpr int EPC = 16 / (int)sizeof(T);       // elements of a piece
    constexpr int CH = D / EPC;                    // pieces of a row
    constexpr int RPT = kAppendThreads / CH;       // rows that the threads hold at a time
    constexpr int ROWS = 2 * RPT;                  // rows staged at a time
    constexpr int NP = ROWS / RPT;
    constexpr int PAD = 16 / (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) T tile[ROWS][D + PAD];
    __shared__ int sh_slots[2 * 256];
    static_assert(sizeof(tile) >= RPT * D * sizeof(float), "the sums lie over the tile");
    const int P = 1 << a.shift, mask = P - 1;
    const int kvh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const int* srow = a.slots + (size_t)b * a.T;
    const int n_slots = a.n_pages << a.shift;
    // slots of all tokens that the run may have, whatever the first one's place is (P <= 256)
    const int at = (int)blockIdx.x * P - P + tid;
    const int s0 = srow[0];
    if (tid < P) {
        const int lo = at >= 0 && at < a.T ? srow[at] : -1, hi = at + P < a.T ? srow[at + P] : -1;
        sh_slots[tid] = lo < n_slots ? lo : -1;  // -1: none in the pool
        sh_slots[P + tid] = hi < n_slots ? hi : -1;
    }
    const int o = s0 & mask;  // (of a page that there is not as well; a row without tokens has no place)
    const int have = blockIdx.x == 0 ? o : 0;  // rows of the page that there are already
    const int i0 = blockIdx.x == 0 ? 0 : (int)blockIdx.x * P - o;
    const int end = min(P, have + a.T - i0);   // places [have, end) are the run's
    if (end <= have) return;
    const int* sh_slot = sh_slots + P - o;     // by place in the page
    __syncthreads();
    const size_t src = (((size_t)b * a.Hkv + kvh) * a.T + i0) * D;
    const T* kn = static_cast<const T*>(a.k_new) + src;
    const T* vn = static_cast<const T*>(a.v_new) + src;
    T* kp = static_cast<T*>(a.k);
    T* vp = static_cast<T*>(a.vt);
    auto page_at = [&](int s) { return ((size_t)(s >> a.shift) * a.Hkv + kvh) * ((size_t)P * D); };
    const int my_row = tid / CH, piece = tid % CH * EPC;

    float sum[EPC];
#pragma unroll
    for (int i = 0; i < EPC; ++i) sum[i] = 0.f;
    auto add = [&](const u32x4& x) {
        const T* e = reinterpret_cast<const T*>(&x);
#pragma unroll
        for (int i = 0; i < EPC; ++i) sum[i] += to_f32(e[i]);
    };
    const int last = sh_slot[end - 1];
    const bool complete = a.mean && end == P && last >= 0 && (last & mask) == mask;
    if (complete)  // the page's other rows come first
        for (int r = my_row; r < have; r += RPT)
            add(*reinterpret_cast<const u32x4*>(kp + page_at(last) + (size_t)r * D + piece));
    for (int r0 = have / ROWS * ROWS; r0 < end; r0 += ROWS) {
        if (sh_slot[max(r0, have)] < 0) break;  // the sequence's tokens end here
        u32x4 kx[NP], vx[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int r = r0 + p * RPT + my_row;
            if (r >= have && r < end && sh_slot[r] >= 0) {
                kx[p] = *reinterpret_cast<const u32x4*>(kn + (size_t)(r - have) * D + piece);
                vx[p] = *reinterpret_cast<const u32x4*>(vn + (size_t)(r - have) * D + piece);
            }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int r = r0 + p * RPT + my_row;
            if (r >= have && r < end && sh_slot[r] >= 0) {
                const int s = sh_slot[r];
                __builtin_nontemporal_store(kx[p], reinterpret_cast<u32x4*>(kp + page_at(s) + (size_t)(s & mask) * D + piece));
                add(kx[p]);
                *reinterpret_cast<u32x4*>(&tile[r - r0][piece]) = vx[p];
            }
        }
        __syncthreads();
        // 16 lanes take 16 features of a tile of eight places
        const int g0 = max(have - r0, 0) / 8, g1 = (min(end - r0, ROWS) + 7) / 8;
        for (int u = tid / 16 + g0 * (D / 16); u < g1 * (D / 16); u += kAppendThreads / 16) {
            const int t0 = u / (D / 16) * 8, f0 = u % (D / 16) * 16, f = f0 + tid % 16;
            const int sa = sh_slot[r0 + t0];
            const bool whole = r0 + t0 >= have && r0 + t0 + 8 <= end && sa >= 0 && (sa & 7) == 0 && sh_slot[r0 + t0 + 7] == sa + 7;
            if (whole) {
                T* dst = vp + page_at(sa) + vt_index<D>(f, sa & mask);
                if constexpr (sizeof(T) == 2) {
                    const bf16* from = &tile[t0 + tid % 16 / 4][f0 + tid % 4 * 4];
                    typedef short shortx8 __attribute__((ext_vector_type(8)));
                    const shortx4 lo = lds_read_tr16(from), hi = lds_read_tr16(from + 4 * (D + PAD));
                    __builtin_nontemporal_store(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7),
                                                reinterpret_cast<shortx8*>(dst));
                } else {
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = tile[t0 + i][f];
                    __builtin_nontemporal_store(floatx4{w[0], w[1], w[2], w[3]}, reinterpret_cast<floatx4*>(dst));
                    __builtin_nontemporal_store(floatx4{w[4], w[5], w[6], w[7]}, reinterpret_cast<floatx4*>(dst + 4));
                }
            } else {
                for (int r = max(t0, have - r0); r < min(t0 + 8, end - r0); ++r) {
                    const int s = sh_slot[r0 + r];
                    if (s >= 0) vp[page_at(s) + vt_index<D>(f, s & mask)] = tile[r][f];
                }
            }
        }
        __syncthreads();
    }
    if (!complete) return;
    float* part = reinterpret_cast<float*>(&tile[0][0]);
#pragma unroll
    for (int i = 0; i < EPC; ++i) part[my_row * D + piece + i] = sum[i];
    __syncthreads();
    if (tid < D) {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < RPT; ++i) m += part[i * D + tid];
        a.mean[((size_t)(last >> a.shift) * a.Hkv + kvh) * D + tid] = m / (float)P;
    }
}

}  // namespace

// Threads, a power of two: a wave for up to 64 sequences (a barrier of 16 waves costs 1 us more),
// four where pages are moved.
static int table_threads(int B, int least) { return B > 64 ? kTableThreads : least; }

hipError_t launch_page_truncate(const PageTableView& t, const int* lens, hipStream_t stream) {
    page_truncate_kernel<<<1, table_threads(t.B, 256), 0, stream>>>(t, lens);
    return hipGetLastError();
}

hipError_t launch_page_extend(const PageTableView& t, const int* counts, int T, int* slots, int* start, int* granted,
                              hipStream_t stream) {
    page_extend_kernel<<<1, table_threads(t.B, 64), 0, stream>>>(t, counts, T, slots, start, granted);
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
