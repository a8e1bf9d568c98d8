// Drafted trees with many query columns (G heads times T nodes of a kv head):
// workgroups of four waves whose blocks of keys and values pass through LDS,
// so that they are fetched once for 32 WC columns.  The decode's direct reads
// (tree.hip) would fetch them from the L1 for every 16.
//
// Bound by the instructions between the products.  On MI355X, d = 128, 512
// positions and 61 summaries: bf16, 32 x 8 heads of 256 columns 38 us (515 TFLOP/s, 3.0
// TB/s; 25.5 without the arithmetic, 35.5 without the requests), e4m3, 64 x 8 heads
// of 48 columns 28.8 us.
//
// Weights are rounded to bf16 for their products, their sums are fp32: see tree.hip.
//
// Blocks: summaries first, then the window, then the drafted tokens (32 rows,
// bf16).  They are requested ahead by LDS DMA into a ring of stages.  A wave
// holds 32 columns; S^T = K Q^T, then O^T += V^T P^T on 32x32x16 products.  With
// WC = 4 column waves every wave takes a whole block (32 rows, or 64 of an 8-bit
// cache: the same bytes); with WC = 2 blocks are 64 rows, the two key waves of
// a column wave take 32 each and are joined at the end.
//
// The cache's values lie transposed, 8 (16) keys of a feature in 16 bytes: their
// fragments are plain 16-byte reads, and the rows of S^T are permuted so that a
// lane's weights are of the keys it reads: element 8 kc + e of half h is key 16
// kc + 8 h + e (8-bit: element i of sub-block j is key 32 j + 16 h + i).  A
// 16-byte read of an 8-bit row or value column is two contraction steps, whose
// features (keys) are those of both.  Drafted values are rows, read transposed
// as the prefill reads them, in its key order.
#include "tile32.hpp"
#include "tree.hpp"

namespace eva {

namespace {

// A block of the cache in LDS: rows in groups of 1 KB, one DMA instruction each.
// The skew between groups and the swizzle of a row's 16-byte chunks spread the
// 16 rows of a fragment read over the banks.
template <int D, bool Q8, int WC>
struct CacheTile {
    static constexpr int KEYS = Q8 || WC == 2 ? 64 : 32;
    static constexpr int ROWB = Q8 ? D : 2 * D;
    static constexpr int RPI = 1024 / ROWB;
    static constexpr int GRP = 1024 + (Q8 ? 32 : 64);
    static constexpr int GROUPS = KEYS * ROWB / 1024;
    static constexpr int NI = GROUPS / 4;  // requests per wave
    // A bf16 ring and its summaries are a multiple of 32 rows: of a block of 64 each
    // half has its own place.  (An 8-bit cache's are a multiple of 64.)
    static constexpr int PARTS = !Q8 && KEYS == 64 ? 2 : 1;
    static constexpr int SUB = KEYS / 32 / (4 / WC);  // 32-key sub-blocks of a wave
    static __device__ __forceinline__ int row_at(int r) { return r / RPI * GRP + r % RPI * ROWB; }
    static __device__ __forceinline__ int swz(int r) { return (ROWB == 256 ? r : ROWB == 128 ? r >> 1 : r >> 2) & 3; }
    // key, within a 32-key sub-block, of product row m = 8 q + 4 h + i
    static __device__ __forceinline__ int key_of_row(int m) {
        const int q = m >> 3, h = (m >> 2) & 1, i = m & 3;
        return Q8 ? 16 * h + 4 * q + i : 16 * (q >> 1) + 8 * h + 4 * (q & 1) + i;
    }
    // and of score element i of half h
    static __device__ __forceinline__ int key_of(int i, int h) { return Q8 ? 16 * h + i : 16 * (i >> 3) + 8 * h + (i & 7); }
};

template <int D, bool Q8, int WC>
struct WideStage {
    typedef CacheTile<D, Q8, WC> T;
    static constexpr int BLK = T::GROUPS * T::GRP > Tile<D>::BLK ? T::GROUPS * T::GRP : Tile<D>::BLK;
    static constexpr int EXP = Q8 ? 4 * 512 : 0;  // exponent bytes, a copy per wave: 64 of the keys, 64 of the values
    static constexpr int BYTES = 2 * BLK + EXP;
    static constexpr int NS = BYTES > 24 * 1024 ? 2 : 3;  // stages: two workgroups a CU at least
};

// Buffer descriptor of `bytes` bytes at p, wave-uniform also where the compiler
// computed it in vector registers.
__device__ __forceinline__ u32x4 scalar_desc(uintptr_t p, unsigned bytes) {
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) & 0xffffu,
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// Two of a raw 16-byte read's contraction steps: the low or high eight codes.
__device__ __forceinline__ bf16x8 half_codes(const u32x4& w, int e) { return q_bf16x8(w[2 * e], w[2 * e + 1]); }

// N 16-byte LDS reads, requested kFragAhead before their use; the fences keep that
// distance, and the registers it takes, fixed.
template <int N, typename Load, typename Use>
__device__ __forceinline__ void stream_reads(Load&& load, Use&& use) {
    u32x4 op[kFragAhead + 1];
#pragma unroll
    for (int k = 0; k < kFragAhead && k < N; ++k) op[k] = load(k);
    __builtin_amdgcn_s_setprio(1);  // the products first
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (k + kFragAhead < N) op[(k + kFragAhead) % (kFragAhead + 1)] = load(k + kFragAhead);
        use(k, op[k % (kFragAhead + 1)]);
        __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
}

template <int D, bool Q8, int WC>
__global__ __launch_bounds__(256, 2) void tree_wide_kernel(TreeParams a) {
    typedef CacheTile<D, Q8, WC> T;
    typedef Tile<D> DT;
    typedef WideStage<D, Q8, WC> Stage;
    constexpr int WK = 4 / WC, SUB = T::SUB, NS = Stage::NS;
    constexpr int NDC = D / 16, NDB = D / 32;
    constexpr int NIT = 2 * T::NI + (Q8 ? 2 : 0);  // requests per wave and block
    static_assert(DT::NI <= T::NI, "drafted blocks take no more requests");
    extern __shared__ __attribute__((aligned(1024))) unsigned char wide_smem[];

    const TreePlace place(a);
    const int unit = place.unit, cb = place.cb;
    if (unit >= a.units) return;
    const CacheView& c = a.c;
    const size_t bg = (size_t)unit;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = wave % WC, wk = wave / WC;
    const int c32 = lane & 31, h2 = lane >> 5;

    // ---- the wave's columns (their loads are in flight while the tree is read) ----
    const int col0 = (cb * WC + wc) * 32;
    const int col = min(col0 + c32, a.cols - 1);  // past the last: the last again, not stored
    bf16x8 qf[NDC];  // features 16 dc + 8 h2 ..; 8-bit: step 2p + e has 32 p + 16 h2 + 8 e ..
    {
        const bf16* q = static_cast<const bf16*>(a.q) + (bg * a.cols + col) * D;
#pragma unroll
        for (int dc = 0; dc < NDC; ++dc)
            qf[dc] = *reinterpret_cast<const bf16x8*>(q + (Q8 ? 32 * (dc >> 1) + 16 * h2 + 8 * (dc & 1) : 16 * dc + 8 * h2));
    }
    const TreeRows rows(a, unit / a.fHkv, true);
    if (!rows.any) return;  // uniform across the workgroup
    const int n = rows.n, nodes = rows.nodes, split = blockIdx.y;

    // ---- the blocks ----
    const int sum_blocks = (rows.sum_last + T::KEYS - 1) / T::KEYS;
    const int win0 = rows.lo_first / T::KEYS;
    const int win_blocks = rows.lo_first < n ? (n - 1) / T::KEYS - win0 + 1 : 0;
    const int cache_blocks = sum_blocks + win_blocks;
    const int all_blocks = cache_blocks + (nodes + 31) / 32;
    // this workgroup's share, a range
    const int j0 = (int)((long long)all_blocks * split / a.splits), j1 = (int)((long long)all_blocks * (split + 1) / a.splits);

    const unsigned lds0 = lds_addr(wide_smem);
    const unsigned k_off = [&] {
        const int row = lane * 16 / T::ROWB, pos = (lane * 16 % T::ROWB) / 16;
        return (unsigned)((wave * T::RPI + row) * T::ROWB + ((pos ^ T::swz(row)) << 4));
    }();
    const unsigned v_off = wave * 1024 + lane * 16;
    const unsigned dk_off = dma_lane_off<D, true>(wave, lane), dv_off = dma_lane_off<D, false>(wave, lane);
    // ring slot of the next window block that is requested (blocks are requested in
    // their order: a division once)
    int slot = (win0 + max(j0 - sum_blocks, 0)) * T::KEYS % c.R;
    auto request = [&](int j, int stage) {
        const unsigned base = lds0 + stage * Stage::BYTES;
        if (j < cache_blocks || j >= j1) {
            const bool sum = j < sum_blocks;
            const size_t at = bg * (size_t)(sum ? c.S_max : c.R);  // the array's first row
            uintptr_t k, v;
            if constexpr (Q8) {
                k = (uintptr_t)(sum ? a.qc.k_sum : a.qc.k_ring);
                v = (uintptr_t)(sum ? a.qc.vt_sum : a.qc.vt_ring);
            } else {
                k = (uintptr_t)(sum ? c.k_sum : c.k_ring);
                v = (uintptr_t)(sum ? c.vt_sum : c.vt_ring);
            }
            int row = __builtin_amdgcn_readfirstlane(sum ? j * T::KEYS : slot);  // (descriptors lie in scalar registers)
#pragma unroll
            for (int p = 0; p < T::PARTS; ++p) {
                // past the last block, or the last summary there is room for: zeros,
                // no access
                const unsigned bytes = j < j1 && (!sum || row < c.S_max) ? T::KEYS / T::PARTS * T::ROWB : 0;
                const u32x4 dk = scalar_desc(k + (at + row) * T::ROWB, bytes), dv = scalar_desc(v + (at + row) * T::ROWB, bytes);
                constexpr int NP = T::NI / T::PARTS;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const unsigned to = base + (4 * (p * NP + i) + wave) * T::GRP;
                    dma16(dk, k_off, i * 4096, to);
                    dma16(dv, v_off, i * 4096, to + Stage::BLK);
                }
                if constexpr (Q8) {
                    const unsigned to = base + 2 * Stage::BLK + wave * 512;
                    dma4(scalar_desc((uintptr_t)(sum ? a.qc.k_sum_e : a.qc.k_ring_e) + at + row, bytes ? 64 : 0), lane * 4, to);
                    dma4(scalar_desc((uintptr_t)(sum ? a.qc.v_sum_e : a.qc.v_ring_e) + at + row, bytes ? 64 : 0), lane * 4,
                         to + 256);
                }
                row += T::KEYS / T::PARTS;
                if (!sum && row == c.R) row = 0;
            }
            if (!sum && j < j1) slot = row;
        } else {
            const int k0 = (j - cache_blocks) * 32;
            const size_t at = (bg * (size_t)a.T + k0) * DT::ROWB;
            const int there = min(nodes - k0, 32);  // rows past the last node: zeros
            const u32x4 dk = rows_desc<D>((uintptr_t)a.k + at, there), dv = rows_desc<D>((uintptr_t)a.v + at, there);
            dma_block<D>(dk, dk_off, base + wave * DT::GRP);
            dma_block<D>(dv, dv_off, base + Stage::BLK + wave * DT::GRP);
            // as many requests as any block has: zeros to places of no use now
            const u32x4 none{0, 0, 0, 0x00020000u};
#pragma unroll
            for (int i = DT::NI; i < T::NI; ++i) {
                dma16(none, v_off, 0, base + (4 * i + wave) * T::GRP);
                dma16(none, v_off, 0, base + Stage::BLK + (4 * i + wave) * T::GRP);
            }
            if constexpr (Q8) {
                const unsigned to = base + 2 * Stage::BLK + wave * 512;
                dma4(none, lane * 4, to);
                dma4(none, lane * 4, to + 256);
            }
        }
    };
    if (j0 < j1) {
#pragma unroll
        for (int i = 0; i < NS - 1; ++i) request(j0 + i, i);
    }

    unsigned long long line;
    int lo, n_sum;
    rows.node(a, col % a.fT, line, lo, n_sum);
    floatx16 acc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[db] = floatx16{};
    float m_run = -INFINITY, l_run = 0.f;  // l_run: this lane's share

    // fragment places in a stage
    const int krow = T::key_of_row(c32);
    const int kr0 = T::row_at(krow) + ((h2 ^ T::swz(krow)) << 4), kr1 = T::row_at(krow) + ((h2 ^ 2 ^ T::swz(krow)) << 4);
    const Frags<D> fr(lane, false);
    // 8-bit features of a drafted row: chunks 4 p + 2 h2 + e
    const int drow = DT::key_of(c32 >> 3, c32 & 3) + ((c32 >> 2) & 1) * DT::KH;

    auto raise_max = [&](float mx, float bias) {
        mx = xhalf_max(mx) * a.scale_log2 + bias;  // -inf: no key of the block is in the row
        const bool up = mx > m_run + kTreeTau;
        if (__builtin_amdgcn_ballot_w64(up)) {
            const float alpha = up ? fast_exp2(m_run - mx) : 1.f;  // first keys: exp2(-inf) = 0
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < NDB; ++db) acc[db] *= alpha;
            m_run = up ? mx : m_run;
        }
    };
    auto offset = [&](float bias) { return m_run == -INFINITY ? 0.f : bias - m_run; };  // no key yet: every score is -inf

    uint32_t special[NDB] = {};  // not_finite_outputs of each feature block
    auto add = [&](const bf16x8& v, const u32x4& w, int db, bool edge) {
        add_values(v, __builtin_bit_cast(bf16x8, w), acc[db], edge, special[db], 0, mfma32_bf16);
    };
    auto cache_block = [&](int j, const unsigned char* st) {
        const unsigned char *ks = st, *vs = st + Stage::BLK;
        const bool is_sum = j < sum_blocks;
        const int pos0 = (is_sum ? j : win0 + j - sum_blocks) * T::KEYS;
        int key_lo = 0, key_hi;  // keys that some column sees
        bool full;               // every column sees every key
        if (is_sum) {
            key_hi = min(T::KEYS, rows.sum_last - pos0) - 1;
            full = pos0 + T::KEYS <= rows.sum_first;
        } else {
            key_lo = max(0, rows.lo_first - pos0);
            key_hi = min(T::KEYS - 1, n - 1 - pos0);
            full = pos0 >= rows.lo_last && key_hi == T::KEYS - 1;
        }
        const float bias = is_sum ? a.log2C : 0.f;
        const int sub0 = WK == 2 ? wk : 0;  // the wave's first sub-block
        floatx16 s[SUB];
        u32x4 vx[SUB];
#pragma unroll
        for (int sb = 0; sb < SUB; ++sb) s[sb] = floatx16{};
        constexpr int KR = T::ROWB / 32;  // reads of a sub-block's rows
        stream_reads<SUB * KR>(
            [&](int k) {
                const int p = k % KR;
                return *reinterpret_cast<const u32x4*>(ks + (sub0 + k / KR) * (32 / T::RPI * T::GRP) + ((p & 1) ? kr1 : kr0) + (p >> 1) * 64);
            },
            [&](int k, const u32x4& w) {
                floatx16& o = s[k / KR];
                const int p = k % KR;
                if constexpr (Q8) {
                    o = mfma32_bf16(half_codes(w, 0), qf[2 * p], o);
                    o = mfma32_bf16(half_codes(w, 1), qf[2 * p + 1], o);
                } else {
                    o = mfma32_bf16(__builtin_bit_cast(bf16x8, w), qf[p], o);
                }
            });
        if constexpr (Q8) {
#pragma unroll
            for (int sb = 0; sb < SUB; ++sb) {
                const unsigned char* ex = st + 2 * Stage::BLK + wave * 512 + 32 * (sub0 + sb) + 16 * h2;
                const u32x4 kx = *reinterpret_cast<const u32x4*>(ex);
                vx[sb] = *reinterpret_cast<const u32x4*>(ex + 256);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[sb][i] *= q_scale(kx[i >> 2] >> (8 * (i & 3)) & 255);
            }
        }
        if (!full) {
            const int half = T::key_of(0, lane_here() >> 5) + 32 * sub0;
            const int first = (is_sum ? 0 : max(lo - pos0, key_lo)) - half;
            const int last = (is_sum ? min(n_sum - pos0 - 1, key_hi) : key_hi) - half;
#pragma unroll
            for (int sb = 0; sb < SUB; ++sb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = 32 * sb + T::key_of(i, 0);
                    s[sb][i] = key >= first && key <= last ? s[sb][i] : -INFINITY;
                }
            if constexpr (Q8) {
#pragma unroll
                for (int sb = 0; sb < SUB; ++sb) vx[sb] = q_finite_scales(vx[sb]);
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int sb = 0; sb < SUB; ++sb)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[sb][i]);
        raise_max(mx, bias);
        const float off = offset(bias);
        u32x4 pf[SUB][2];  // weights of 8 keys: element 8 kc ..
#pragma unroll
        for (int sb = 0; sb < SUB; ++sb)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float p0 = fast_exp2(fmaf(s[sb][i], a.scale_log2, off)), p1 = fast_exp2(fmaf(s[sb][i + 1], a.scale_log2, off));
                l_run += p0 + p1;
                if constexpr (Q8) {
                    const uint32_t x = vx[sb][i >> 2] >> (8 * (i & 3));
                    p0 *= q_scale(x & 255);
                    p1 *= q_scale(x >> 8 & 255);
                }
                pf[sb][i >> 3][(i & 7) >> 1] = pack_bf16x2(p0, p1);
            }
        // values: 16 bytes a feature are 8 keys, tile 4 sub + 2 kc + h2, or 16
        // codes, tile 2 sub + h2
        constexpr int TILEB = D * 16, VR = Q8 ? SUB : 2;  // tiles read by a lane
        auto vfrag = [&](int x, int db) {
            const int byte = ((Q8 ? 2 * (sub0 + x) : 4 * sub0 + 2 * x) + h2) * TILEB + (32 * db + c32) * 16;
            return *reinterpret_cast<const u32x4*>(vs + (byte >> 10) * T::GRP + (byte & 1023));
        };
        // Of a block with an edge a column may not see what others see, and slots
        // may be stale: whatever bits they hold, their weights are 0
        stream_reads<VR * NDB>([&](int k) { return vfrag(k / NDB, k % NDB); },
                              [&](int k, const u32x4& w) {
                                  const int x = k / NDB;
                                  if constexpr (Q8) {
                                      const bool nan = !full && __builtin_amdgcn_ballot_w64(q_has_nan(w));
                                      add(half_codes(w, 0), pf[x][0], k % NDB, nan);
                                      add(half_codes(w, 1), pf[x][1], k % NDB, nan);
                                  } else {
                                      add(__builtin_bit_cast(bf16x8, w), pf[0][x], k % NDB, !full);
                                  }
                              });
    };
    auto draft_block = [&](int j, const unsigned char* st) {
        if (WK == 2 && ((j - cache_blocks) & 1) != wk) return;  // the key waves take turns
        const unsigned char *ks = st, *vs = st + Stage::BLK;
        const int k0 = (j - cache_blocks) * 32;
        floatx16 s = floatx16{};
#pragma unroll
        for (int dc = 0; dc < NDC; ++dc) {
            bf16x8 k;
            if constexpr (Q8)
                k = *reinterpret_cast<const bf16x8*>(ks + DT::row_at(drow) + (((4 * (dc >> 1) + 2 * h2 + (dc & 1)) ^ DT::swz(drow)) << 4));
            else
                k = fr.row(ks, dc);
            s = mfma32_bf16(k, qf[dc], s);
        }
        const uint32_t seen = (uint32_t)(line >> k0) >> (h2 * DT::KH);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = seen >> DT::key_of(i / 4, i % 4) & 1 ? s[i] : -INFINITY;
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        raise_max(mx, 0.f);
        const float off = offset(0.f);
        u32x4 pf[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float p0 = fast_exp2(fmaf(s[i], a.scale_log2, off)), p1 = fast_exp2(fmaf(s[i + 1], a.scale_log2, off));
            l_run += p0 + p1;
            pf[i >> 3][(i & 7) >> 1] = pack_bf16x2(p0, p1);
        }
#pragma unroll
        for (int kc = 0; kc < 2; ++kc)
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
                add(fr.tr(vs, db, kc), pf[kc], db, true);
                __builtin_amdgcn_sched_barrier(0);
            }
    };

    int stage = 0;
    auto steps = [&](int from, int to, auto&& block) {
        for (int j = from; j < to; ++j) {
            // block j landed (of three stages the next may stay in flight); the block
            // requested now refills the stage whose last reads were before this barrier
            asm volatile("" ::: "memory");
            wait_vm_lgkm0<(NS - 2) * NIT>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            request(j + NS - 1, stage == 0 ? NS - 1 : stage - 1);
            const unsigned char* st = wide_smem + stage * Stage::BYTES;
            stage = stage == NS - 1 ? 0 : stage + 1;
            block(j, st);
        }
    };
    steps(j0, min(j1, cache_blocks), cache_block);
    steps(max(j0, cache_blocks), j1, draft_block);
#pragma unroll
    for (int db = 0; db < NDB; ++db)
        if (__builtin_amdgcn_ballot_w64(special[db] != 0)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] = with_not_finite(acc[db][i], special[db] >> (2 * i) & 3);
        }
    // no request may still be writing LDS: it is used again
    wait_vm_lgkm0<0>();
    __syncthreads();

    float l = xhalf_sum(l_run);
    if constexpr (WK == 2) {
        // the second key wave's sums to the first
        constexpr int STRIDE = D + 4;
        float* part = reinterpret_cast<float*>(wide_smem) + wc * 32 * (STRIDE + 2);
        float* po = part + 64 + c32 * STRIDE + 4 * h2;
        if (wk == 1) {
            if (h2 == 0) {
                part[c32] = m_run;
                part[32 + c32] = l;
            }
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<floatx4*>(po + 32 * db + 8 * q) =
                        floatx4{acc[db][4 * q], acc[db][4 * q + 1], acc[db][4 * q + 2], acc[db][4 * q + 3]};
        }
        __syncthreads();
        if (wk == 1) return;
        const float m2 = part[c32], l2 = part[32 + c32];
        const float M = fmaxf(m_run, m2);
        const float w1 = m_run == -INFINITY ? 0.f : fast_exp2(m_run - M), w2 = m2 == -INFINITY ? 0.f : fast_exp2(m2 - M);
        l = w1 * l + w2 * l2;  // (no key: a sum of 0, or NaN, which stays)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const floatx4 x = *reinterpret_cast<const floatx4*>(po + 32 * db + 8 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[db][4 * q + i] = w1 * acc[db][4 * q + i] + w2 * x[i];
            }
        m_run = M;
    }
    if (a.splits > 1) {
        // partial: [m, l, o[D]] per (unit, split, column)
        if (col0 + c32 >= a.cols || col % a.fT >= nodes) return;
        float* p = a.ws + ((bg * a.splits + split) * a.cols + col) * (D + 2);
        if (h2 == 0) {
            p[0] = m_run;
            p[1] = l;
        }
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) p[2 + 32 * db + 8 * (i >> 2) + 4 * h2 + (i & 3)] = acc[db][i];
        return;
    }
    // whole rows through LDS, the wave's own place
    const float inv = 1.f / l;
    unsigned char* stg = wide_smem + (WK == 2 ? wc * 32 * (D + 6) * 4 : wave * 32 * kStageRow<D>);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<u32x2*>(stg + c32 * kStageRow<D> + (db * 32 + 8 * q + 4 * h2) * 2) =
                u32x2{pack_bf16x2(acc[db][4 * q] * inv, acc[db][4 * q + 1] * inv), pack_bf16x2(acc[db][4 * q + 2] * inv, acc[db][4 * q + 3] * inv)};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    constexpr int LPR = 2 * D / 16, RPS = 64 / LPR;  // lanes a row, rows an instruction
    bf16* out = static_cast<bf16*>(a.o) + (bg * a.cols + col0) * D;
#pragma unroll
    for (int i = 0; i < 32 / RPS; ++i) {
        const int r = i * RPS + lane / LPR;
        const u32x4 x = *reinterpret_cast<const u32x4*>(stg + r * kStageRow<D> + (lane % LPR) * 16);
        if (col0 + r < a.cols && (col0 + r) % a.fT < nodes)
            *reinterpret_cast<u32x4*>(out + (size_t)r * D + (lane % LPR) * 8) = x;
    }
}

template <int D, bool Q8, int WC>
constexpr size_t wide_lds() {
    typedef WideStage<D, Q8, WC> Stage;
    const size_t ring = (size_t)Stage::NS * Stage::BYTES;
    const size_t end = WC == 2 ? 2 * 32 * (size_t)(D + 6) * 4 : 4 * 32 * (size_t)kStageRow<D>;
    return ring > end ? ring : end;
}

}  // namespace

template <int D, bool Q8>
hipError_t launch_tree_wide(const TreeParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.units + 7) / 8 * 8 * p.col_blocks), (unsigned)p.splits);
    if (p.shape == kTree64)
        hipLaunchKernelGGL((tree_wide_kernel<D, Q8, 2>), grid, dim3(256), (wide_lds<D, Q8, 2>()), stream, p);
    else
        hipLaunchKernelGGL((tree_wide_kernel<D, Q8, 4>), grid, dim3(256), (wide_lds<D, Q8, 4>()), stream, p);
    return hipGetLastError();
}
template hipError_t launch_tree_wide<64, false>(const TreeParams&, hipStream_t);
template hipError_t launch_tree_wide<128, false>(const TreeParams&, hipStream_t);
template hipError_t launch_tree_wide<64, true>(const TreeParams&, hipStream_t);
template hipError_t launch_tree_wide<128, true>(const TreeParams&, hipStream_t);

}  // namespace eva
