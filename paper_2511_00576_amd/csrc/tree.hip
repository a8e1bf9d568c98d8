// Attention of drafted tokens (a tree for each sequence) over a ragged cache of
// bf16, e4m3 or fp32 rows, and the decode of the 8-bit cache (a single query of
// the last position, no drafted token).
//
// Node t of sequence b is a token at position p = n + depth(t), n the tokens
// that the cache holds.  Its row is the softmax over
//   the summaries c < s(p)                    logit q . khat_c / sqrt(d) + ln C
//   the ring's positions win_lo(p) .. n - 1
//   its line: itself and its forerunners among the drafted tokens
// (trees are no deeper than the window: see eva_rtree_attention), and its
// neighbours on other branches are hidden by its line's bit mask.
//
// The query columns of a kv head are its G heads times the T nodes.  Here a
// workgroup holds 16 of them, as many as a 16x16x32 product has, and its waves
// take turns with the 32-key chunks (64-key for e4m3: the same bytes), as the
// decode kernel does: S^T = K Q^T, then O^T += V^T P^T, both operands of the cache
// read straight from memory into the matrix cores' layouts, 16 bytes a lane.
// Bound by memory for one block of 16 columns (8-bit decode of 64 x 8 heads, 560
// rows of 128: 16.6 us, 4.4 TB/s; of one sequence 8.1 us, latency); more columns
// fetch the rows again from the L2, and once their workgroups would be more than two
// a CU tree_wide.hip's kernel takes them.
//
// The weights of bf16 and 8-bit rows are rounded to bf16 (2^-8 of a weight at most), as
// the decode and the prefill round theirs: they are an operand of the bf16 products (fp32 ones
// run at an eighth of their rate: 153 and 1225 TFLOP/s for 8192^3).  The denominators sum them
// unrounded in fp32.  Measured against 64 bits: 0.0020 - 0.0023 of the output's norm,
// of which the output's own rounding is 0.0017.  No weight of fp32 rows is rounded.
//
// The codes of an 8-bit cache become bf16 in registers, exactly, and a row's
// power of two is put on its logit and on its softmax weight instead of its d
// features: as exact, for one product a key.
#include "tree.hpp"

namespace eva {

namespace {

template <int D>
constexpr int draft_stride() { return D + 8; }  // bf16 elements: rows of a transposing read on distinct banks
template <int D>
__host__ __device__ constexpr int col_floats() { return D + 4; }  // 16 columns on distinct banks

// Dynamic LDS of a workgroup: the drafted values' rows, then (in the same
// place) the waves' maxima, sums and accumulators.
template <int D>
inline size_t tree_lds(int waves, bool drafted) {
    const size_t draft = drafted ? (size_t)kMaxNodes * draft_stride<D>() * 2 : 0;
    const size_t merge = (size_t)waves * 16 * (col_floats<D>() + 2) * sizeof(float);
    return draft > merge ? draft : merge;
}

// Joins the NW waves' parts of a workgroup's 16 columns and stores the rows
// of the columns that there are, or their partials where rows are split.
template <int D, int NW, typename T>
__device__ __forceinline__ void join_waves(const TreeParams& a, const float* red_m, const float* red_l, const float* red_o,
                                           int unit, int cb, int split, int nodes) {
    constexpr int FPC = D / 4;  // threads per column
    for (int e = threadIdx.x; e < 16 * FPC; e += blockDim.x) {
        const int col = e / FPC, f0 = e % FPC * 4;
        const int at = cb * 16 + col;
        if (at >= a.cols || at % a.fT >= nodes) continue;
        float M = -INFINITY, lsum = 0.f;
        floatx4 out{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NW; ++i) M = fmaxf(M, red_m[i * 16 + col]);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float m = red_m[i * 16 + col];
            const float wt = m == -INFINITY ? 0.f : fast_exp2(m - M);  // no key: no weight, and sums of 0 (or NaN)
            lsum += wt * red_l[i * 16 + col];
            out += wt * *reinterpret_cast<const floatx4*>(red_o + (size_t)(i * 16 + col) * col_floats<D>() + f0);
        }
        if (a.splits == 1) {
            out *= 1.f / lsum;
            T* row = static_cast<T*>(a.o) + ((size_t)unit * a.cols + at) * D + f0;
            if constexpr (sizeof(T) == 2)
                *reinterpret_cast<u32x2*>(row) = u32x2{pack_bf16x2(out[0], out[1]), pack_bf16x2(out[2], out[3])};
            else
                *reinterpret_cast<floatx4*>(row) = out;
        } else {
            // partial: [m, l, o[D]] per (unit, split, column)
            float* p = a.ws + (((size_t)unit * a.splits + split) * a.cols + at) * (D + 2);
            if (f0 == 0) {
                p[0] = M;
                p[1] = lsum;
            }
#pragma unroll
            for (int f = 0; f < 4; ++f) p[2 + f0 + f] = out[f];
        }
    }
}

// Q8: the cache's rows are e4m3.  DRAFT: there are drafted tokens.
template <int D, bool Q8, bool DRAFT, int NW>
__global__ __launch_bounds__(NW * 64, NW == 12 ? 3 : 2) void tree_kernel(TreeParams a) {
    constexpr int NDC = D / 32, NDB = D / 16;
    constexpr int KB = Q8 ? 4 : 2, KC = 16 * KB;  // 16-key blocks, and keys, of a cache chunk
    extern __shared__ __attribute__((aligned(16))) float tree_smem[];

    const TreePlace place(a);
    const int unit = place.unit, cb = place.cb;
    if (unit >= a.units) return;
    const int split = blockIdx.y;
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c16 = lane & 15;
    const size_t bg = (size_t)unit;

    // Column c16 (past the last: the last again; a column's results depend on it
    // alone, and theirs are not stored), its query's features 32 dc + 8 g ..
    // (8-bit: 64 (dc / 2) + 16 g + 8 (dc % 2) .., both halves of a 16-byte read).
    const int col = min(cb * 16 + c16, a.cols - 1);
    auto feature = [&](int dc) { return Q8 ? 64 * (dc >> 1) + 16 * g + 8 * (dc & 1) : 32 * dc + 8 * g; };
    bf16x8 qf[NDC];
#pragma unroll
    for (int dc = 0; dc < NDC; ++dc)
        qf[dc] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16*>(a.q) + (bg * a.cols + col) * D + feature(dc));
    const TreeRows rows(a, unit / a.fHkv, DRAFT);  // (the queries' loads are in flight meanwhile)
    if (!rows.any) {  // uniform across the workgroup
        // a row over nothing, of an active sequence without a token, is zero
        if (!DRAFT && split == 0 && !(a.active && a.active[unit / a.fHkv] == 0))
            for (int e = threadIdx.x; e < min(16, a.cols - cb * 16) * D; e += NW * 64)
                static_cast<bf16*>(a.o)[((size_t)unit * a.cols + cb * 16) * D + e] = to_bf16(0.f);
        return;
    }
    const int n = rows.n, nodes = rows.nodes;

    // drafted values: rows into LDS
    bf16* vdraft = reinterpret_cast<bf16*>(tree_smem);
    if constexpr (DRAFT) {
        const bf16* v = static_cast<const bf16*>(a.v) + bg * (size_t)a.T * D;
        const int n_rows = (nodes + 31) & ~31;
        for (int e = tid; e < n_rows * (D / 8); e += NW * 64) {
            const int r = e / (D / 8), f = e % (D / 8) * 8;
            u32x4 x{0, 0, 0, 0};
            if (r < nodes) x = *reinterpret_cast<const u32x4*>(v + (size_t)r * D + f);
            *reinterpret_cast<u32x4*>(vdraft + r * draft_stride<D>() + f) = x;
        }
    }

    unsigned long long line;
    int lo, n_sum;
    rows.node(a, DRAFT ? col % a.fT : 0, line, lo, n_sum);
    floatx4 acc[NDB];  // features db*16 + 4g .. +3
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};
    uint32_t special[D / 64] = {};  // not_finite_outputs, four feature blocks each
    float m_run = -INFINITY, l_run = 0.f;
    if constexpr (DRAFT) __syncthreads();

    // Scores (score i of block kb is key 4 KB g + 4 kb + i) become weights; bias
    // in log2 units.  The reference moves only when a chunk exceeds it by more
    // than kTreeTau.
    auto weights = [&](auto& s, float bias) {
        constexpr int N = sizeof(s) / sizeof(s[0]);
        float mx = s[0][0];
#pragma unroll
        for (int kb = 0; kb < N; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[kb][i]);
        mx = xgroup_max(mx) * a.scale_log2 + bias;  // -inf: no key of the chunk is in the row
        const bool raise = mx > m_run + kTreeTau;
        if (__builtin_amdgcn_ballot_w64(raise)) {
            const float alpha = raise ? fast_exp2(m_run - mx) : 1.f;  // first keys: exp2(-inf) = 0
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < NDB; ++db) acc[db] *= alpha;
            m_run = raise ? mx : m_run;
        }
        const float off = m_run == -INFINITY ? 0.f : bias - m_run;  // no key yet: every score is -inf
#pragma unroll
        for (int kb = 0; kb < N; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[kb][i] = fast_exp2(fmaf(s[kb][i], a.scale_log2, off));
                l_run += s[kb][i];
            }
    };
    auto pack8 = [](const floatx4& x, const floatx4& y) {
        return __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]),
                                                pack_bf16x2(y[2], y[3])});
    };
    auto add = [&](const bf16x8& v, const bf16x8& p, int db, bool edge) {
        add_values(v, p, acc[db], edge, special[db / 4], 8 * (db % 4), mfma_bf16);
    };

    // ---- the cache's chunks ----
    const int sum_chunks = (rows.sum_last + KC - 1) / KC;
    const int win_chunk0 = rows.lo_first / KC;
    const int win_chunks = rows.lo_first < n ? (n - 1) / KC - win_chunk0 + 1 : 0;
    const int cache_chunks = sum_chunks + win_chunks;
    constexpr int kSkip = 0x40000000;  // past any tile: zeros, no access
    constexpr int kNt = 2;             // non-temporal: one block of columns reads a row once
    const int aux = a.col_blocks == 1 ? kNt : 0;
    int ch = split * NW + wave;
    for (; ch < cache_chunks; ch += a.splits * NW) {
        const bool is_sum = ch < sum_chunks;
        // key of row c16 of block kb: krow0 + 4 kb, so that a lane group's keys
        // are consecutive: 4 KB g ..
        const int krow0 = (c16 >> 2) * (4 * KB) + (c16 & 3);
        int row0, pos0;          // first row of the chunk, its position (or summary)
        int key_lo = 0, key_hi;  // keys that some column sees
        bool full;               // every column sees every key
        if (is_sum) {
            pos0 = row0 = ch * KC;
            key_hi = min(KC, rows.sum_last - pos0) - 1;
            full = pos0 + KC <= rows.sum_first;
        } else {
            pos0 = (win_chunk0 + ch - sum_chunks) * KC;
            row0 = pos0 % c.R;
            key_lo = max(0, rows.lo_first - pos0);
            key_hi = min(KC - 1, n - 1 - pos0);
            full = pos0 >= rows.lo_last && key_hi == KC - 1;
        }
        const unsigned span = (unsigned)(key_hi - key_lo);
        const float bias = is_sum ? a.log2C : 0.f;
        const size_t base = bg * (size_t)(is_sum ? c.S_max : c.R) + row0;
        floatx4 s[KB];
        // a column's keys: positions from lo, or summaries below n_sum
        auto hide = [&]() {
            const int first = (is_sum ? 0 : max(lo - pos0, key_lo)) - g * 4 * KB;
            const int last = (is_sum ? min(n_sum - pos0 - 1, key_hi) : key_hi) - g * 4 * KB;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kb][i] = kb * 4 + i >= first && kb * 4 + i <= last ? s[kb][i] : -INFINITY;
        };
        constexpr int ROWB = Q8 ? D : 2 * D;
        const void *kt, *vt;
        if constexpr (Q8) {
            kt = (is_sum ? a.qc.k_sum : a.qc.k_ring) + base * ROWB;
            vt = (is_sum ? a.qc.vt_sum : a.qc.vt_ring) + base * ROWB;
        } else {
            kt = static_cast<const char*>(is_sum ? c.k_sum : c.k_ring) + base * ROWB;
            vt = static_cast<const char*>(is_sum ? c.vt_sum : c.vt_ring) + base * ROWB;
        }
        const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(kt), 0, KC * ROWB, 0x00020000);
        const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(vt), 0, KC * ROWB, 0x00020000);
        auto ld = [&](__amdgpu_buffer_rsrc_t r, int at) {
            return aux ? __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kNt) : __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
        };
        // all loads of the chunk before any wait; rows and 16-byte pieces that no
        // column needs are not fetched
        u32x4 ka[KB][ROWB / 64], va[NDB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int key = krow0 + 4 * kb;
            const int at = (unsigned)(key - key_lo) <= span ? key * ROWB + 16 * g : kSkip;
#pragma unroll
            for (int h = 0; h < ROWB / 64; ++h) ka[kb][h] = ld(krs, at + 64 * h);
        }
        u32x4 kx, vx;
        if constexpr (Q8) {
            kx = *reinterpret_cast<const u32x4*>((is_sum ? a.qc.k_sum_e : a.qc.k_ring_e) + base + 16 * g);
            vx = *reinterpret_cast<const u32x4*>((is_sum ? a.qc.v_sum_e : a.qc.v_ring_e) + base + 16 * g);
        }
        {
            constexpr int K8 = 4 * KB;  // keys, and slots of a value tile, of a lane group
            const bool use = g * K8 <= key_hi && g * K8 + K8 - 1 >= key_lo;
            const int at = use ? (g * D + c16) * 16 : kSkip;
#pragma unroll
            for (int db = 0; db < NDB; ++db) va[db] = ld(vrs, at + db * 256);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int dc = 0; dc < NDC; ++dc) {
                bf16x8 k;
                if constexpr (Q8)
                    k = q_bf16x8(ka[kb][dc >> 1][2 * (dc & 1)], ka[kb][dc >> 1][2 * (dc & 1) + 1]);
                else
                    k = __builtin_bit_cast(bf16x8, ka[kb][dc]);
                s[kb] = mfma_bf16(k, qf[dc], s[kb]);
            }
            if constexpr (Q8) {  // this lane's keys 16g + 4kb + i
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kb][i] *= q_scale(kx[kb] >> (8 * i) & 255);
                __builtin_amdgcn_sched_barrier(0);  // one block's codes in bf16 at a time
            }
        }
        if (!full) {
            hide();
            if constexpr (!DRAFT) {
                // one position: what it does not see no column sees, and stale
                // slots may hold any bits: no value
                uint32_t keep[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    keep[i] = 0;
                    constexpr int PD = KB;  // keys of a dword
#pragma unroll
                    for (int y = 0; y < PD; ++y)
                        if ((unsigned)(g * 4 * KB + PD * i + y - key_lo) <= span) keep[i] |= (Q8 ? 255u : 0xffffu) << (32 / PD * y);
                }
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) va[db][i] &= keep[i];
            }
        }
        weights(s, bias);
        if constexpr (Q8) {
            if (!full) vx = q_finite_scales(vx);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kb][i] *= q_scale(vx[kb] >> (8 * i) & 255);
            const bf16x8 p0 = pack8(s[0], s[1]), p1 = pack8(s[2], s[3]);  // keys 16g .., 16g + 8 ..
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
                const bool nan = DRAFT && !full && __builtin_amdgcn_ballot_w64(q_has_nan(va[db]));
                add(q_bf16x8(va[db][0], va[db][1]), p0, db, nan);
                add(q_bf16x8(va[db][2], va[db][3]), p1, db, nan);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const bf16x8 p = pack8(s[0], s[1]);
#pragma unroll
            for (int db = 0; db < NDB; ++db) add(__builtin_bit_cast(bf16x8, va[db]), p, db, DRAFT && !full);
        }
    }

    // ---- the drafted tokens' chunks, 32 each; lane group g's keys are k0 + 8g .. ----
    if constexpr (DRAFT) {
        for (; ch < cache_chunks + (nodes + 31) / 32; ch += a.splits * NW) {
            const int k0 = (ch - cache_chunks) * 32;
            const bf16* kt = static_cast<const bf16*>(a.k) + (bg * a.T + k0) * D;
            const __amdgpu_buffer_rsrc_t krs =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(kt), 0, (nodes - k0) * D * 2, 0x00020000);
            const int krow0 = (c16 >> 2) * 8 + (c16 & 3);
            floatx4 s[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int key = krow0 + 4 * kb;
                s[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int dc = 0; dc < NDC; ++dc) {
                    const int at = k0 + key < nodes ? (key * D + feature(dc)) * 2 : kSkip;
                    s[kb] = mfma_bf16(__builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(krs, at, 0, 0)), qf[dc], s[kb]);
                }
                const uint32_t seen = (uint32_t)(line >> (k0 + 8 * g + 4 * kb));
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kb][i] = seen >> i & 1 ? s[kb][i] : -INFINITY;
            }
            weights(s, 0.f);
            const bf16x8 p = pack8(s[0], s[1]);
            // lane 4j + i names features 4i .. of row j, and receives feature
            // c16 of four rows
            const bf16* vrow = vdraft + (k0 + 8 * g + (c16 >> 2)) * draft_stride<D>() + 4 * (c16 & 3);
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
                const u32x2 x = __builtin_bit_cast(u32x2, lds_read_tr16(vrow + db * 16));
                const u32x2 y = __builtin_bit_cast(u32x2, lds_read_tr16(vrow + 4 * draft_stride<D>() + db * 16));
                add(__builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]}), p, db, true);
            }
        }
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                acc[db][i] = with_not_finite(acc[db][i], special[db / 4] >> (8 * (db % 4) + 2 * i) & 3);
        __syncthreads();  // the drafted values' place is free
    }

    // ---- join the waves ----
    float* red_m = tree_smem;
    float* red_l = red_m + NW * 16;
    float* red_o = red_l + NW * 16;
    {
        const int at = wave * 16 + c16;
        const float l = xgroup_sum(l_run);
        if (g == 0) {
            red_m[at] = m_run;
            red_l[at] = l;
        }
        float* o = red_o + (size_t)at * col_floats<D>() + 4 * g;
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<floatx4*>(o + db * 16) = acc[db];
    }
    __syncthreads();
    join_waves<D, NW, bf16>(a, red_m, red_l, red_o, unit, cb, split, nodes);
}

// fp32 caches: the same on fp32 matrix cores (16x16x4), 16 columns a workgroup
// whose NW waves take turns with the 32-key chunks, laid out as the fp32 decode:
// lane (g, c16) holds key 16 kb + 4g + i of column c16; contraction step (j, e)
// of S^T pairs feature 16j + 4g + e.  Bound by memory with two workgroups a CU (500
// heads of 16 columns, 690 rows of 128: 68 us, 5.5 TB/s), by latency below
// that (264 heads 55 us).
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void tree_f32_kernel(TreeParams a) {
    constexpr int NJ = D / 16;
    extern __shared__ __attribute__((aligned(16))) float tree_smem[];
    const TreePlace place(a);
    const int unit = place.unit, cb = place.cb;
    if (unit >= a.units) return;
    const int split = blockIdx.y;
    const CacheView& c = a.c;
    const TreeRows rows(a, unit / a.fHkv, true);
    if (!rows.any) return;
    const int n = rows.n, nodes = rows.nodes;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c16 = lane & 15;
    const size_t bg = (size_t)unit;
    const float* kring = static_cast<const float*>(c.k_ring) + bg * (size_t)c.R * D;
    const float* vring = static_cast<const float*>(c.vt_ring) + bg * (size_t)c.R * D;
    const float* ksum = static_cast<const float*>(c.k_sum) + bg * (size_t)c.S_max * D;
    const float* vsum = static_cast<const float*>(c.vt_sum) + bg * (size_t)c.S_max * D;
    const float* kdraft = static_cast<const float*>(a.k) + bg * (size_t)a.T * D;
    const float* vdraft = static_cast<const float*>(a.v) + bg * (size_t)a.T * D;

    const int lo_first = rows.lo_first, lo_last = rows.lo_last, sum_first = rows.sum_first, sum_last = rows.sum_last;
    // column c16 (past the last: the last again, not stored)
    const int col = min(cb * 16 + c16, a.cols - 1);
    unsigned long long line;
    int lo, n_sum;
    rows.node(a, col % a.fT, line, lo, n_sum);
    floatx4 qf[NJ], acc[NJ];
    const float* qrow = static_cast<const float*>(a.q) + (bg * a.cols + col) * D;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        qf[j] = *reinterpret_cast<const floatx4*>(qrow + 16 * j + 4 * g);
        acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    uint32_t special[D / 64] = {};  // not_finite_outputs, four feature blocks each
    float m_run = -INFINITY, l_run = 0.f;

    const int sum_chunks = (sum_last + 31) / 32;
    const int win_chunk0 = lo_first / 32;
    const int win_chunks = lo_first < n ? (n - 1) / 32 - win_chunk0 + 1 : 0;
    const int cache_chunks = sum_chunks + win_chunks;
    const int n_chunks = cache_chunks + (nodes + 31) / 32;
    for (int ch = split * NW + wave; ch < n_chunks; ch += a.splits * NW) {
        const bool draft = ch >= cache_chunks, is_sum = ch < sum_chunks;
        const float *kt, *vt;
        int key_lo = 0, key_hi, pos0;
        bool full = false;
        if (draft) {
            pos0 = (ch - cache_chunks) * 32;
            kt = kdraft + (size_t)pos0 * D;
            vt = vdraft + (size_t)pos0 * D;
            key_hi = min(31, nodes - 1 - pos0);
        } else if (is_sum) {
            pos0 = ch * 32;
            kt = ksum + (size_t)pos0 * D;
            vt = vsum + (size_t)pos0 * D;
            key_hi = min(32, sum_last - pos0) - 1;
            full = pos0 + 32 <= sum_first;
        } else {
            pos0 = (win_chunk0 + ch - sum_chunks) * 32;
            const int slot0 = pos0 % c.R;
            kt = kring + (size_t)slot0 * D;
            vt = vring + (size_t)slot0 * D;
            key_lo = max(0, lo_first - pos0);
            key_hi = min(31, n - 1 - pos0);
            full = pos0 >= lo_last && key_hi == 31;
        }
        // keys of this lane's column: first .. last, or its line
        const int first = draft || is_sum ? 0 : max(lo - pos0, key_lo);
        const int last = is_sum ? min(n_sum - pos0 - 1, key_hi) : key_hi;
        const uint32_t seen = draft ? (uint32_t)(line >> pos0) : 0xffffffffu;
        // all keys of the chunk before any wait (a drafted row past the last node:
        // the last one's), all values before the softmax
        floatx4 kf[2][NJ];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const float* krow = kt + (size_t)(draft ? min(16 * kb + c16, key_hi) : 16 * kb + c16) * D + 4 * g;
#pragma unroll
            for (int j = 0; j < NJ; ++j) kf[kb][j] = *reinterpret_cast<const floatx4*>(krow + 16 * j);
        }
        __builtin_amdgcn_sched_barrier(0);
        floatx4 s[2];
        float pw[2][4];
        // (four sums in turn: a product waits for the one before on the same sum)
        floatx4 s2[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[kb] = s2[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 4; e += 2)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    s[kb] = mfma_f32(kf[kb][j][e], qf[j][e], s[kb]);
                    s2[kb] = mfma_f32(kf[kb][j][e + 1], qf[j][e + 1], s2[kb]);
                }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            s[kb] += s2[kb];
            if (!full) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = 16 * kb + 4 * g + i;
                    s[kb][i] = k >= first && k <= last && (seen >> k & 1) ? s[kb][i] : -INFINITY;
                }
            }
        }
        floatx4 vf[2][NJ];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const float* vtile = vt + (size_t)(2 * kb + (g >> 1)) * (kVtTile * D) + 4 * (g & 1);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (draft) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        vf[kb][j][i] = vt[(size_t)min(16 * kb + 4 * g + i, key_hi) * D + 16 * j + c16];
                } else {
                    vf[kb][j] = *reinterpret_cast<const floatx4*>(vtile + (16 * j + c16) * kVtTile);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const float bias = is_sum ? a.log2C : 0.f;
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                         fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = xgroup_max(mx) * a.scale_log2 + bias;
        if (mx > m_run) {
            const float alpha = fast_exp2(m_run - mx);  // first keys: exp2(-inf) = 0
            l_run *= alpha;
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
            m_run = mx;
        }
        const float off = m_run == -INFINITY ? 0.f : bias - m_run;  // no key yet: every score is -inf
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pw[kb][i] = fast_exp2(fmaf(s[kb][i], a.scale_log2, off));
                l_run += pw[kb][i];
            }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if (!full) {
                // stale slots (no weight, whatever bits they hold), and values that
                // some columns do not see: see not_finite_outputs
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    floatx4& v = vf[kb][j];
                    bool bad = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) bad |= !is_finite(v[i]);
                    if (__builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            special[j / 4] |= not_finite_outputs_f32(v[i], pw[kb][i]) << (8 * (j % 4));
                            v[i] = is_finite(v[i]) ? v[i] : 0.f;
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[j] = mfma_f32(vf[kb][j][i], pw[kb][i], acc[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = with_not_finite(acc[j][i], special[j / 4] >> (8 * (j % 4) + 2 * i) & 3);

    // ---- join the waves ----
    float* red_m = tree_smem;
    float* red_l = red_m + NW * 16;
    float* red_o = red_l + NW * 16;
    {
        const int at = wave * 16 + c16;
        const float l = xgroup_sum(l_run);
        if (g == 0) {
            red_m[at] = m_run;
            red_l[at] = l;
        }
        float* o = red_o + (size_t)at * col_floats<D>() + 4 * g;
#pragma unroll
        for (int j = 0; j < NJ; ++j) *reinterpret_cast<floatx4*>(o + 16 * j) = acc[j];
    }
    __syncthreads();
    join_waves<D, NW, float>(a, red_m, red_l, red_o, unit, cb, split, nodes);
}

// Joins the splits of a column: one thread a feature, one workgroup of 256 / D
// columns, loads of eight splits in flight together.
template <int D, typename T>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeParams a) {
    const int col = blockIdx.x * (256 / D) + threadIdx.x / D, f = threadIdx.x % D;
    const int unit = blockIdx.y;
    if (col >= a.cols) return;
    const int b = unit / a.fHkv;
    if (a.active && a.active[b] == 0) return;
    if (a.k) {
        const int nodes = a.n_nodes ? min(a.n_nodes[b], a.T) : a.T;
        if (col % a.fT >= nodes) return;
    } else if (a.n_tok[b] <= 0) {
        return;
    }
    const float* base = a.ws + ((size_t)unit * a.splits * a.cols + col) * (D + 2);
    const size_t step = (size_t)a.cols * (D + 2);
    float M = -INFINITY, num = 0.f, den = 0.f;
    constexpr int NB = 8;
    for (int s0 = 0; s0 < a.splits; s0 += NB) {
        float m[NB], l[NB], o[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const float* w = base + min(s0 + i, a.splits - 1) * step;  // past the last: the last one's address
            m[i] = w[0];
            l[i] = w[1];
            o[i] = w[2 + f];
        }
        float mx = M;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            // no weight, and no sums either: infinite ones times no weight are NaN
            if (s0 + i >= a.splits) {
                m[i] = -INFINITY;
                l[i] = o[i] = 0.f;
            }
            mx = fmaxf(mx, m[i]);
        }
        // no maximum yet: no weight either, but a sum of NaN (all its keys were) stays one
        const float keep = M == -INFINITY ? 0.f : fast_exp2(M - mx);
        num *= keep;
        den *= keep;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const float wt = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - mx);
            den += wt * l[i];
            num += wt * o[i];
        }
        M = mx;
    }
    static_cast<T*>(a.o)[((size_t)unit * a.cols + col) * D + f] = from_f32<T>(num / den);
}

template <int D, bool Q8, bool DRAFT, int NW>
hipError_t launch_narrow(const TreeParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.units + 7) / 8 * 8 * p.col_blocks), (unsigned)p.splits);
    hipLaunchKernelGGL((tree_kernel<D, Q8, DRAFT, NW>), grid, dim3(NW * 64), tree_lds<D>(NW, DRAFT), stream, p);
    return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_join(const TreeParams& p, hipStream_t stream) {
    constexpr int per = 256 / D;
    hipLaunchKernelGGL((tree_join_kernel<D, T>), dim3((p.cols + per - 1) / per, p.units), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

template <int D, bool Q8>
hipError_t launch_tree(const TreeParams& p, hipStream_t stream) {
    hipError_t e;
    if (p.shape >= kTree64) {
        e = launch_tree_wide<D, Q8>(p, stream);
    } else if (p.k) {
        e = p.shape == kTreeNarrow ? launch_narrow<D, Q8, true, 4>(p, stream) : launch_narrow<D, Q8, true, 12>(p, stream);
    } else if constexpr (Q8) {
        e = p.shape == kTreeNarrow ? launch_narrow<D, Q8, false, 4>(p, stream) : launch_narrow<D, Q8, false, 12>(p, stream);
    } else {
        return hipErrorInvalidValue;  // the decode of a bf16 cache is decode.hip's
    }
    return e == hipSuccess && p.splits > 1 ? launch_join<D, bf16>(p, stream) : e;
}
template hipError_t launch_tree<64, false>(const TreeParams&, hipStream_t);
template hipError_t launch_tree<128, false>(const TreeParams&, hipStream_t);
template hipError_t launch_tree<64, true>(const TreeParams&, hipStream_t);
template hipError_t launch_tree<128, true>(const TreeParams&, hipStream_t);

template <int D>
hipError_t launch_tree_f32(const TreeParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.units + 7) / 8 * 8 * p.col_blocks), (unsigned)p.splits);
    if (p.shape == kTreeNarrow12)
        hipLaunchKernelGGL((tree_f32_kernel<D, 12>), grid, dim3(12 * 64), tree_lds<D>(12, false), stream, p);
    else
        hipLaunchKernelGGL((tree_f32_kernel<D, 4>), grid, dim3(4 * 64), tree_lds<D>(4, false), stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && p.splits > 1 ? launch_join<D, float>(p, stream) : e;
}
template hipError_t launch_tree_f32<64>(const TreeParams&, hipStream_t);
template hipError_t launch_tree_f32<128>(const TreeParams&, hipStream_t);

}  // namespace eva
