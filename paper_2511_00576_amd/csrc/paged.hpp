// Paged cache: parameters and launches of pages.hip (table, append), paged.hip
// (decode) and paged_select.hip (choice of pages).
//
// A pool of n_pages pages of P = 2^shift tokens holds the rows of every sequence:
// keys k [n_pages][Hkv][P][d], values vt [n_pages][Hkv][P / 8][d][8] (the decode
// cache's 8-slot tiles: vt_index), mean keys [n_pages][Hkv][d] in fp32.  Position p
// of sequence b lies in page table[b][p / P], place p mod P.
#pragma once

#include "eva_device.hpp"
#include "eva_kernels.hpp"

namespace eva {

struct PageTableView {
    int B, shift, n_pages, max_pages;
    int* n_tok;   // [B]
    int* table;   // [B][max_pages], -1: no page
    int* free_pages;  // [n_pages], a stack of n_free[0] pages
    int* n_free;
};

// Token counts are only ever used within what the table's row has room for.
__device__ __forceinline__ int held_tokens(const PageTableView& t, int b) {
    return min(max(t.n_tok[b], 0), t.max_pages << t.shift);
}
__host__ __device__ __forceinline__ int pages_of(int tokens, int shift) {
    return (int)(((unsigned)tokens + (1u << shift) - 1) >> shift);
}

// Data movement between lanes in one VALU instruction (a shuffle goes through LDS, 100
// cycles and more); lanes that have no source get 0.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int dpp(int x) {
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ long long dpp(long long x) {
    const unsigned lo = (unsigned)dpp<CTRL, ROWS>((int)x);
    return (long long)((unsigned long long)(unsigned)dpp<CTRL, ROWS>((int)(x >> 32)) << 32 | lo);
}
// Inclusive sum over the wave: within rows of 16 lanes, then from row to row.
template <typename I>
__device__ __forceinline__ I wave_scan(I x) {
    x += dpp<0x111>(x);       // one lane up
    x += dpp<0x112>(x);       // two
    x += dpp<0x114>(x);       // four
    x += dpp<0x118>(x);       // eight
    x += dpp<0x142, 0xa>(x);  // rows 0 and 2 to the next
    x += dpp<0x143, 0xc>(x);  // the first two rows to the others
    return x;
}

// Inclusive sum over the workgroup's threads, and the whole sum; sums has room for
// every wave's.
template <typename I>
__device__ __forceinline__ I block_scan(I x, I* sums, I& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    x = wave_scan(x);
    __syncthreads();  // the last use of sums is over
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    I before = 0;
    total = 0;
    for (int w = 0; w < waves; ++w) {
        const I s = sums[w];
        if (w < wave) before += s;
        total += s;
    }
    return x + before;
}

hipError_t launch_page_truncate(const PageTableView& t, const int* lens, hipStream_t stream);
// slots [B][T], start [B], granted [B]
hipError_t launch_page_extend(const PageTableView& t, const int* counts, int T, int* slots, int* start, int* granted,
                              hipStream_t stream);

struct PagedAppendParams {
    void* k;
    void* vt;
    float* mean;       // or nullptr
    const void* k_new; // [B][Hkv][T][d]
    const void* v_new;
    const int* slots;  // [B][T]
    int B, Hkv, T, shift, n_pages;
};
template <int D, typename T>
hipError_t launch_paged_append(const PagedAppendParams& p, hipStream_t stream);

struct PagedParams {
    PageTableView t;
    const void* k;
    const void* vt;
    const int* pages;   // [B][Hkv][S] pages that a kv head's queries attend, or nullptr: all
    const int* active;  // [B] or nullptr
    const void* q;      // [B][H][d]
    void* o;
    float* ws;          // partials of split rows, nullptr: a workgroup per row
    int S, H, Hkv, G;
    int n_hg;           // groups of 16 paged_tiles(G) query heads of a kv head
    int rows;           // B Hkv n_hg
    int wgs;            // workgroups of the launch (with ws)
    FastDiv f_wgs;      // divisor of wgs
    int alone;          // without ws: a wave per row, not a workgroup
    FastDiv f_unit, f_hg;  // divisors of Hkv n_hg and of n_hg
    FastDiv f_H, f_G;      // of H and of G
    float scale_log2;
};
// Blocks of 16 tokens in a chunk, what a wave requests at once: 16 KB of keys and
// values, 64 registers a lane (two blocks of fp32 rows of 128 features would take 128).
constexpr int paged_blocks(int d, int bytes) { return bytes == 4 && d == 128 ? 1 : 2; }
// The fewest chunks a workgroup takes: one for each of its four waves.
constexpr int kPagedMinPart = 4;
// Rows of up to kPagedShortest chunks go to one wave each, and of up to kPagedShort where
// there are kPagedMany and more.  us in a replayed graph, a wave / a workgroup (which takes
// kPagedMinPart chunks and more, however many rows that is), by the rows' chunks:
//     rows   1 chunk      2            4            8
//   bf16, d = 128: 32 tokens, 16 KB
//      256   7.0 / 7.0    7.9 / 7.2    10.1 / 7.8   18.1 / 11.9
//      512   7.1 / 7.6    8.2 / 8.2    12.9 / 9.9   20.9 / 14.8
//     1024   8.2 / 14.1   10.7 / 12.7  16.0 / 16.2  25.7 / 27.2
//     4096   24 / 36      33 / 42      53 / 59      93 / 100
//   bf16, d = 64: 32 tokens, 8 KB
//      256   6.4 / 6.6    6.9 / 6.8    8.1 / 7.1    10.4 / 9.7
//      512   6.7 / 7.2    7.2 / 7.5    8.5 / 8.2    13.6 / 9.8
//     1024   8.2 / 13.4   8.8 / 11.0   11.7 / 12.7  17.0 / 17.6
//     4096   20 / 33      25 / 35      34 / 41      53 / 61
//   fp32, d = 128: 16 tokens, 16 KB (d = 64, 32 tokens, within 7% of it)
//      256   7.6 / 7.6    8.8 / 7.8    11.7 / 8.4   19.5 / 13.3
//      512   7.8 / 8.3    9.1 / 9.3    13.6 / 11.5  22.0 / 15.9
//     1024   9.1 / 17.3   11.3 / 15.3  16.6 / 19.3  27.3 / 28.9
//     4096   27 / 42      37 / 53      57 / 72      99 / 114
// Where rows can have no more than kPagedShort chunks at all and paged_whole() gives each
// its workgroup, a wave takes it from kPagedMany on (1 chunk: 512 rows 4.8 / 4.8, 1024 4.9 /
// 7.2, 4096 14.7 / 22.7).
constexpr int kPagedShortest = 2, kPagedShort = 8, kPagedMany = 1024;
// Tiles of 16 query heads that a workgroup has at once: with two, what a kv head's more than
// 16 heads read is read once for 32 of them (20 heads, 256 sequences of up to 4096 tokens, 2 kv
// heads, 720 MB: 139 us against 236).
constexpr int paged_tiles(int G) { return G > 16 ? 2 : 1; }
// Workgroups that share a decode's chunks: two a CU saturate the memory (64 sequences at 8k
// 218 us; 257 with one and a half, 220 with three), and parts that end with their rows.
constexpr int kPagedWgs = 512, kPagedWithin = 64;
// Whether every row, of `bytes` of keys and values at most, is left to one workgroup, which
// saves the second launch.  us in a replayed graph, shared / one each, rows of the same length
// in chunks of 16 KB:
//     rows   8 chunks     12           16           24           48
//        8   8.7 / 6.0    8.9 / 7.1    8.8 / 8.2    8.9 / 10.3   8.9 / 17.2
//       64   8.9 / 6.7    9.4 / 8.9    9.5 / 11.2   11.1 / 15.2  14.4 / 27.2
//      192                                          20.7 / 19.8  31.2 / 31.3
//      256   11.9 / 8.0   14.6 / 10.6  16.6 / 13.1  21.7 / 18.3  36.7 / 33.5
//     1024   26.2 / 22.1  37.0 / 31.9  46.6 / 41.9  67.7 / 61.4  124 / 120
// (300 rows of 96 chunks 80 / 104: from 48 on it is a matter of how rows fit the CUs.)
inline bool paged_whole(long long rows, long long bytes) { return bytes <= (rows >= 192 ? 24 : 12) * 16384; }
// Floats of a column of a share (paged.hip).
__host__ __device__ constexpr int share_col(int d) { return d + 4; }
// Bytes of the workspace: a pair of ints per row, then two shares per workgroup.
inline size_t paged_ws_bytes(long long rows, long long wgs, int d, int G) {
    return ((size_t)(rows + 1) / 2 * 4 + (size_t)wgs * 2 * 16 * paged_tiles(G) * share_col(d)) * sizeof(float);
}
template <int D, typename T>
hipError_t launch_paged_decode(const PagedParams& p, hipStream_t stream);

struct SelectParams {
    PageTableView t;
    const float* mean;  // [n_pages][Hkv][d]
    const void* q;      // [B][H][d]
    int* pages;         // [B][Hkv][S]
    unsigned long long* keys;  // [B Hkv][max_pages]: scores as ordered whole numbers; nullptr: in LDS
    int S, first, last, H, Hkv, G;
};
// Whether the workgroup that chooses makes its row's scores itself, in LDS, or a launch before
// spreads them over the chip: one CU reads 35 GB/s of mean keys, so many pages of few rows
// want more of them.  us in a replayed graph, alone / spread, d = 128 (a call that is not
// captured pays 2.6 us of host time for the second launch, so the bound is 256 and not 128):
//     rows   128 pages   256          512          1024         2048
//        8   8.4 / 8.8   10.2 / 8.8   13.9 / 9.0   21 / 10      36 / 12
//      128   8.6 / 9.0   10.5 / 10.7  14.9 / 15.2  22 / 22      37 / 34
//      256   8.6 / 10.7  11.0 / 15.1  18 / 21      29 / 33      50 / 57
//      512   16 / 16     21 / 22      33 / 35      53 / 63      113 / 143
constexpr int kSelectAlone = 4096;  // scores that LDS holds
inline bool select_alone(long long rows, int max_pages) {
    return max_pages <= 256 || (rows >= 256 && max_pages <= kSelectAlone);
}
template <int D, typename T>
hipError_t launch_paged_select(const SelectParams& p, hipStream_t stream);

}  // namespace eva
