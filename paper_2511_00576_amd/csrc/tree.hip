// Attention of drafted tokens (a tree for each sequence) over a ragged cache of
// bf16 or e4m3 rows, and the decode of the 8-bit cache (a single query of the
// last position, no drafted token).
//
// Node t of sequence b is a token at position p = n + depth(t), n the tokens
// that the cache holds.  Its row is the softmax over
//   the summaries c < s(p)                    logit q . khat_c / sqrt(d) + ln C
//   the ring's positions win_lo(p) .. n - 1
//   its line: itself and its forerunners among the drafted tokens
// (trees are no deeper than the window: see eva_rtree_attention), and its
// neighbours on other branches are hidden by its line's bit mask.
//
// The query columns of a kv head are its G heads times the T nodes.  A wave
// holds NC tiles of 16 columns and works through 32-key chunks (64-key for
// e4m3: the same bytes) as the decode kernel does: S^T = K Q^T, then O^T += V^T
// P^T, with both operands of the cache read straight from memory into the
// matrix cores' layouts, 16 bytes a lane.  Keys are shared by all of the wave's
// columns; the WC column waves of a workgroup read the same chunk at about the
// same time (the L1 serves all but the first), and its WK key waves take
// turns with the chunks and are joined through LDS.
//
// The codes of an 8-bit cache become bf16 in registers, exactly, and a row's
// power of two is put on its logit and on its softmax weight instead of its d
// features: as exact, for one product a key.
#include "qrows.hpp"

namespace eva {

namespace {

constexpr float kLazyTau = 8.f;  // log2 units: unscaled weights stay <= 256
constexpr int kMaxNodes = 64;

// Lines of the tree's nodes: lane t holds the set of node t's forerunners and
// itself.  Parents name an earlier node; any other value makes a root.  Six
// rounds of doubling reach 64 nodes back.
__device__ __forceinline__ unsigned long long tree_lines(const int* parents, int nodes) {
    const int lane = threadIdx.x & 63;
    int up = lane < nodes ? parents[lane] : -1;
    if (up < 0 || up >= lane) up = -1;
    unsigned long long line = 1ull << lane;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
        const int from = max(up, 0);
        const unsigned long long l = __shfl(line, from, 64);
        const int u = __shfl(up, from, 64);
        if (up >= 0) {
            line |= l;
            up = u;
        }
    }
    return line;
}

// A wave's columns and their running softmax.
template <int D, int NC>
struct Columns {
    bf16x8 q[NC][D / 32];
    floatx4 acc[NC][D / 16];  // features db*16 + 4g .. +3
    float m[NC], l[NC];
    int lo[NC], n_sum[NC];    // first ring position, visible summaries
    unsigned long long line[NC];
};

// Scores of KB 16-key blocks (key of row 4g + i of block kb: base + 4 kb + i of
// lane group g's 4 KB keys) become weights, in place.  bias in log2 units.
template <int D, int NC, int KB>
__device__ __forceinline__ void weights(Columns<D, NC>& w, floatx4 (&s)[NC][KB], float scale_log2, float bias) {
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        float mx = s[nc][0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[nc][kb][i]);
        mx = xgroup_max(mx) * scale_log2 + bias;  // -inf: no key of the chunk is in the row
        // the reference moves only when a chunk exceeds it by more than kLazyTau
        const bool raise = mx > w.m[nc] + kLazyTau;
        if (__builtin_amdgcn_ballot_w64(raise)) {
            const float m_new = raise ? mx : w.m[nc];
            const float alpha = raise ? fast_exp2(w.m[nc] - m_new) : 1.f;  // first keys: exp2(-inf) = 0
            w.l[nc] *= alpha;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) w.acc[nc][db] *= alpha;
            w.m[nc] = m_new;
        }
        const float off = w.m[nc] == -INFINITY ? 0.f : bias - w.m[nc];  // no key yet: every score is -inf
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = fast_exp2(fmaf(s[nc][kb][i], scale_log2, off));
                sum += p;
                s[nc][kb][i] = p;
            }
        w.l[nc] += sum;
    }
}

__device__ __forceinline__ bf16x8 pack8(const floatx4& a, const floatx4& b) {
    return __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]),
                                            pack_bf16x2(b[2], b[3])});
}

// Whether a fragment holds an infinity or NaN.
__device__ __forceinline__ bool not_finite(const bf16x8& v) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}

// acc += V^T P^T of one 16-feature block where some column does not see a key
// whose value is infinite or NaN: a weight of 0 times it would be NaN.  The
// finite values are added as they are; a column with weight on others becomes
// the infinity that they all are, or NaN: the weights' sum over all of them
// equals the one over infinities with their sign.
template <int NC, typename Acc>
__device__ __forceinline__ void add_not_finite(const bf16x8& v, const bf16x8 (&p)[NC], Acc&& acc) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    u32x4 fin, any, inf;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = (w[i] & 0x7f80u) == 0x7f80u, hi = (w[i] & 0x7f800000u) == 0x7f800000u;
        fin[i] = w[i] & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
        any[i] = (lo ? 0x3f80u : 0u) | (hi ? 0x3f800000u : 0u);
        inf[i] = ((w[i] & 0x7fffu) == 0x7f80u ? 0x3f80u | (w[i] & 0x8000u) : 0u) |
                 ((w[i] & 0x7fff0000u) == 0x7f800000u ? 0x3f800000u | (w[i] & 0x80000000u) : 0u);
    }
    const floatx4 zero{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        floatx4& o = acc(nc);
        const floatx4 all = mfma_bf16(__builtin_bit_cast(bf16x8, any), p[nc], zero);
        const floatx4 sgn = mfma_bf16(__builtin_bit_cast(bf16x8, inf), p[nc], zero);
        o = mfma_bf16(__builtin_bit_cast(bf16x8, fin), p[nc], o);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (all[i] != 0.f) o[i] += sgn[i] == all[i] ? INFINITY : sgn[i] == -all[i] ? -INFINITY : NAN;
    }
}

// O^T += V^T P^T of one 32-key step.  `part`: some column may not see some key
// that others see.
template <int D, int NC>
__device__ __forceinline__ void add_values(Columns<D, NC>& w, const bf16x8 (&va)[D / 16], const bf16x8 (&pf)[NC], bool part) {
    if (part) {
        bool bad = false;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) bad |= not_finite(va[db]);
        if (__builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
                add_not_finite<NC>(va[db], pf, [&](int nc) -> floatx4& { return w.acc[nc][db]; });
            return;
        }
    }
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) w.acc[nc][db] = mfma_bf16(va[db], pf[nc], w.acc[nc][db]);
}

template <int D>
constexpr int draft_stride() { return D + 8; }  // bf16 elements: rows of a transposing read on distinct banks
template <int D>
__host__ __device__ constexpr int col_floats() { return D + 4; }  // 16 columns on distinct banks

// Dynamic LDS of a workgroup: the drafted values' rows, then (in the same
// place) the key waves' maxima, sums and accumulators.
template <int D>
inline size_t tree_lds(int NC, int WC, int WK, bool drafted) {
    const size_t draft = drafted ? (size_t)kMaxNodes * draft_stride<D>() * 2 : 0;
    const size_t merge = (size_t)WK * WC * NC * 16 * (col_floats<D>() + 2) * sizeof(float);
    return draft > merge ? draft : merge;
}

// Joins the WK key waves' parts of a workgroup's kCols columns and stores the rows
// of the columns that there are, or their partials where rows are split.
template <int D, int kCols, int WK, typename T>
__device__ __forceinline__ void join_waves(const TreeParams& a, const float* red_m, const float* red_l, const float* red_o,
                                           int unit, int cb, int split, int nodes) {
    constexpr int FPC = D / 4;  // threads per column
    for (int e = threadIdx.x; e < kCols * FPC; e += blockDim.x) {
        const int col = e / FPC, f0 = e % FPC * 4;
        const int at = cb * kCols + col;
        if (at >= a.cols || at % a.fT >= nodes) continue;
        float M = -INFINITY, lsum = 0.f;
        floatx4 out{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WK; ++i) M = fmaxf(M, red_m[i * kCols + col]);
#pragma unroll
        for (int i = 0; i < WK; ++i) {
            const float m = red_m[i * kCols + col];
            const float wt = m == -INFINITY ? 0.f : fast_exp2(m - M);  // no key: no weight, and sums of 0 (or NaN)
            lsum += wt * red_l[i * kCols + col];
            out += wt * *reinterpret_cast<const floatx4*>(red_o + (size_t)(i * kCols + col) * col_floats<D>() + f0);
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
template <int D, bool Q8, bool DRAFT, int NC, int WC, int WK>
__global__ __launch_bounds__(WC * WK * 64) void tree_kernel(TreeParams a) {
    constexpr int NDC = D / 32, NDB = D / 16;
    constexpr int KB = Q8 ? 4 : 2, KC = 16 * KB;  // keys of a cache chunk
    constexpr int kCols = 16 * NC * WC;
    extern __shared__ __attribute__((aligned(16))) float tree_smem[];

    // Workgroups of a unit are 8 apart, so that one XCD's L2 has its rows.
    const int id = blockIdx.x;
    const int group = id / a.f8cb, r8 = id - group * a.f8cb.d;
    const int unit = group * 8 + (r8 & 7), cb = r8 >> 3;
    if (unit >= a.units) return;
    const int split = blockIdx.y;
    const int b = unit / a.fHkv;
    if (a.active && a.active[b] == 0) return;
    const CacheView& c = a.c;
    const int n = min(max(a.n_tok[b], 0), a.max_tok);
    int nodes = 1;
    if constexpr (DRAFT) {
        nodes = a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
        if (nodes == 0) return;
    } else {
        if (n == 0) return;
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wc = wave % WC, wk = wave / WC;
    const int g = lane >> 4, c16 = lane & 15;
    const size_t bg = (size_t)unit;

    // drafted values: rows into LDS
    bf16* vdraft = reinterpret_cast<bf16*>(tree_smem);
    if constexpr (DRAFT) {
        const bf16* v = static_cast<const bf16*>(a.v) + bg * (size_t)a.T * D;
        const int rows = (nodes + 31) & ~31;
        for (int e = tid; e < rows * (D / 8); e += WC * WK * 64) {
            const int r = e / (D / 8), f = e % (D / 8) * 8;
            u32x4 x{0, 0, 0, 0};
            if (r < nodes) x = *reinterpret_cast<const u32x4*>(v + (size_t)r * D + f);
            *reinterpret_cast<u32x4*>(vdraft + r * draft_stride<D>() + f) = x;
        }
    }

    // the wave's columns
    Columns<D, NC> w;
    const int col0 = (cb * WC + wc) * 16 * NC;
    int lo_first, lo_last, sum_first, sum_last;  // over the tree's nodes
    {
        unsigned long long line = 0;
        int deepest = 0;
        if constexpr (DRAFT) {
            line = tree_lines(a.parents + (size_t)b * a.T, nodes);
            deepest = lane < nodes ? __builtin_popcountll(line) - 1 : 0;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) deepest = max(deepest, __shfl_xor(deepest, off, 64));
            deepest = __builtin_amdgcn_readfirstlane(deepest);
        }
        const int p0 = DRAFT ? n : n - 1;
        lo_first = win_lo_rt(c.window, p0, c.W, c.C);
        lo_last = win_lo_rt(c.window, p0 + deepest, c.W, c.C);
        sum_first = min(lo_first / c.C, c.S_max);
        sum_last = min(lo_last / c.C, c.S_max);
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            // columns past the last repeat it: a column's results depend on it
            // alone, and theirs are not stored
            const int col = min(col0 + 16 * nc + c16, a.cols - 1);
            const int t = DRAFT ? col % a.fT : 0;
            w.line[nc] = DRAFT ? __shfl(line, t, 64) : 0;
            const int p = p0 + (DRAFT ? __builtin_popcountll(w.line[nc]) - 1 : 0);
            w.lo[nc] = win_lo_rt(c.window, p, c.W, c.C);
            w.n_sum[nc] = min(w.lo[nc] / c.C, c.S_max);
            if (DRAFT && t >= nodes) w.line[nc] = 0;  // no such node: not stored either
            const bf16* row = static_cast<const bf16*>(a.q) + (bg * a.cols + col) * D;
#pragma unroll
            for (int dc = 0; dc < NDC; ++dc)
                w.q[nc][dc] = *reinterpret_cast<const bf16x8*>(row + (Q8 ? 64 * (dc >> 1) + 16 * g + 8 * (dc & 1) : 32 * dc + 8 * g));
#pragma unroll
            for (int db = 0; db < NDB; ++db) w.acc[nc][db] = floatx4{0.f, 0.f, 0.f, 0.f};
            w.m[nc] = -INFINITY;
            w.l[nc] = 0.f;
        }
    }
    if constexpr (DRAFT) __syncthreads();

    const int sum_chunks = (sum_last + KC - 1) / KC;
    const int win_chunk0 = lo_first / KC;
    const int win_chunks = lo_first < n ? (n - 1) / KC - win_chunk0 + 1 : 0;
    const int cache_chunks = sum_chunks + win_chunks;
    const int draft_chunks = DRAFT ? (nodes + 31) / 32 : 0;
    const int n_chunks = cache_chunks + draft_chunks;
    // key of row c16 of block kb: krow0 + 4 kb, so that a lane group's keys are
    // consecutive: 4 KB g ..
    constexpr int kSkip = 0x40000000;  // past any tile: zeros, no access
    constexpr int kNt = NC * WC == 1 ? 2 : 0;  // rows that one wave reads stay out of the caches

    for (int ch = split * WK + wk; ch < n_chunks; ch += a.splits * WK) {
        if (!DRAFT || ch < cache_chunks) {
            const bool is_sum = ch < sum_chunks;
            const int krow0 = (c16 >> 2) * (4 * KB) + (c16 & 3);
            int row0, key_lo, key_hi;  // first row of the chunk, its keys that some column sees
            int pos0;                  // position (or summary) of the first row
            bool full;                 // every column sees every key
            if (is_sum) {
                pos0 = row0 = ch * KC;
                key_lo = 0;
                key_hi = min(KC, sum_last - pos0) - 1;
                full = pos0 + KC <= sum_first;
            } else {
                pos0 = (win_chunk0 + ch - sum_chunks) * KC;
                row0 = pos0 % c.R;
                key_lo = max(0, lo_first - pos0);
                key_hi = min(KC - 1, n - 1 - pos0);
                full = pos0 >= lo_last && key_hi == KC - 1;
            }
            const unsigned span = (unsigned)(key_hi - key_lo);
            floatx4 s[NC][KB];
            const float bias = is_sum ? a.log2C : 0.f;
            // valid keys of a column: positions from lo, or summaries below n_sum
            auto hide = [&]() {
#pragma unroll
                for (int nc = 0; nc < NC; ++nc) {
                    const int first = is_sum ? 0 : max(w.lo[nc] - pos0, key_lo);
                    const int last = is_sum ? min(w.n_sum[nc] - pos0 - 1, key_hi) : key_hi;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = g * 4 * KB + kb * 4 + i;
                            s[nc][kb][i] = key >= first && key <= last ? s[nc][kb][i] : -INFINITY;
                        }
                }
            };
            if constexpr (Q8) {
                const QCacheView& qc = a.qc;
                const size_t base = is_sum ? bg * (size_t)qc.S_max : bg * (size_t)qc.R;
                const uint8_t* kt = (is_sum ? qc.k_sum : qc.k_ring) + (base + row0) * D;
                const uint8_t* vt = (is_sum ? qc.vt_sum : qc.vt_ring) + (base + row0) * D;
                const uint8_t* ke = (is_sum ? qc.k_sum_e : qc.k_ring_e) + base + row0;
                const uint8_t* ve = (is_sum ? qc.v_sum_e : qc.v_ring_e) + base + row0;
                constexpr int kBytes = KC * D;
                const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(kt), 0, kBytes, 0x00020000);
                const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(vt), 0, kBytes, 0x00020000);
                u32x4 ka[KB][D / 64], va[NDB];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const int key = krow0 + 4 * kb;
                    const int at = (unsigned)(key - key_lo) <= span ? key * D + 16 * g : kSkip;
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) ka[kb][h] = __builtin_amdgcn_raw_buffer_load_b128(krs, at + 64 * h, 0, kNt);
                }
                const u32x4 kx = *reinterpret_cast<const u32x4*>(ke + 16 * g), vx = *reinterpret_cast<const u32x4*>(ve + 16 * g);
                {
                    const bool use = g * 16 <= key_hi && g * 16 + 15 >= key_lo;
                    const int at = use ? (int)qt_index<D>(c16, 16 * g) : kSkip;
#pragma unroll
                    for (int db = 0; db < NDB; ++db) va[db] = __builtin_amdgcn_raw_buffer_load_b128(vrs, at + db * 16 * kQTile, 0, kNt);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    bf16x8 kf[NDC];
#pragma unroll
                    for (int dc = 0; dc < NDC; ++dc) kf[dc] = q_bf16x8(ka[kb][dc >> 1][2 * (dc & 1)], ka[kb][dc >> 1][2 * (dc & 1) + 1]);
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc) {
                        s[nc][kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int dc = 0; dc < NDC; ++dc) s[nc][kb] = mfma_bf16(kf[dc], w.q[nc][dc], s[nc][kb]);
                    }
                    // this lane's keys 16g + 4kb + i
                    floatx4 sc;
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[i] = q_scale(kx[kb] >> (8 * i) & 255);
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc) s[nc][kb] *= sc;
                }
                if (!full) {
                    hide();
                    // stale slots may hold any byte: no value, no exponent
                    uint32_t keep[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        keep[i] = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if ((unsigned)(16 * g + 4 * i + j - key_lo) <= span) keep[i] |= 255u << (8 * j);
                    }
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
#pragma unroll
                        for (int i = 0; i < 4; ++i) va[db][i] &= keep[i];
                    weights<D, NC, KB>(w, s, a.scale_log2, bias);
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float sc = q_scale(vx[kb] >> (8 * i) & keep[kb] >> (8 * i) & 255);
#pragma unroll
                            for (int nc = 0; nc < NC; ++nc) s[nc][kb][i] *= sc;
                        }
                } else {
                    weights<D, NC, KB>(w, s, a.scale_log2, bias);
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float sc = q_scale(vx[kb] >> (8 * i) & 255);
#pragma unroll
                            for (int nc = 0; nc < NC; ++nc) s[nc][kb][i] *= sc;
                        }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // keys 16g + 8h ..
                    bf16x8 vf[NDB], pf[NC];
#pragma unroll
                    for (int db = 0; db < NDB; ++db) vf[db] = q_bf16x8(va[db][2 * h], va[db][2 * h + 1]);
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc) pf[nc] = pack8(s[nc][2 * h], s[nc][2 * h + 1]);
                    add_values<D, NC>(w, vf, pf, DRAFT && !full);
                }
            } else {
                const size_t base = is_sum ? bg * (size_t)c.S_max : bg * (size_t)c.R;
                const bf16* kt = static_cast<const bf16*>(is_sum ? c.k_sum : c.k_ring) + (base + row0) * D;
                const bf16* vt = static_cast<const bf16*>(is_sum ? c.vt_sum : c.vt_ring) + (base + row0) * D;
                constexpr int kBytes = KC * D * 2;
                const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(kt), 0, kBytes, 0x00020000);
                const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(vt), 0, kBytes, 0x00020000);
                bf16x8 ka[KB][NDC], va[NDB];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const int key = krow0 + 4 * kb;
                    const int at = (unsigned)(key - key_lo) <= span ? (key * D + 8 * g) * 2 : kSkip;
#pragma unroll
                    for (int dc = 0; dc < NDC; ++dc)
                        ka[kb][dc] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(krs, at + dc * 64, 0, kNt));
                }
                {
                    const bool use = g * 8 <= key_hi && g * 8 + 7 >= key_lo;
                    const int at = use ? (int)vt_index<D>(c16, 8 * g) * 2 : kSkip;
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
                        va[db] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(vrs, at + db * 16 * kVtTile * 2, 0, kNt));
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc) {
                        s[nc][kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int dc = 0; dc < NDC; ++dc) s[nc][kb] = mfma_bf16(ka[kb][dc], w.q[nc][dc], s[nc][kb]);
                    }
                if (!full) {
                    hide();
                    // stale slots may hold any bit pattern: zero their values
                    uint32_t keep[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned rel = (unsigned)(g * 8 + 2 * i - key_lo);
                        keep[i] = (rel <= span ? 0x0000ffffu : 0u) | (rel + 1 <= span ? 0xffff0000u : 0u);
                    }
#pragma unroll
                    for (int db = 0; db < NDB; ++db) {
                        u32x4 x = __builtin_bit_cast(u32x4, va[db]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] &= keep[i];
                        va[db] = __builtin_bit_cast(bf16x8, x);
                    }
                }
                weights<D, NC, KB>(w, s, a.scale_log2, bias);
                bf16x8 pf[NC];
#pragma unroll
                for (int nc = 0; nc < NC; ++nc) pf[nc] = pack8(s[nc][0], s[nc][1]);
                add_values<D, NC>(w, va, pf, DRAFT && !full);
            }
        } else if constexpr (DRAFT) {
            // 32 drafted tokens; lane group g's keys are k0 + 8g ..
            const int k0 = (ch - cache_chunks) * 32;
            const bf16* kt = static_cast<const bf16*>(a.k) + (bg * a.T + k0) * D;
            const __amdgpu_buffer_rsrc_t krs =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(kt), 0, (nodes - k0) * D * 2, 0x00020000);
            const int krow0 = (c16 >> 2) * 8 + (c16 & 3);
            floatx4 s[NC][2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int key = krow0 + 4 * kb;
                bf16x8 ka[NDC];
#pragma unroll
                for (int dc = 0; dc < NDC; ++dc) {
                    const int f = Q8 ? 64 * (dc >> 1) + 16 * g + 8 * (dc & 1) : 32 * dc + 8 * g;
                    const int at = k0 + key < nodes ? (key * D + f) * 2 : kSkip;
                    ka[dc] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(krs, at, 0, 0));
                }
#pragma unroll
                for (int nc = 0; nc < NC; ++nc) {
                    s[nc][kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int dc = 0; dc < NDC; ++dc) s[nc][kb] = mfma_bf16(ka[dc], w.q[nc][dc], s[nc][kb]);
                    const uint32_t seen = (uint32_t)(w.line[nc] >> (k0 + 8 * g + 4 * kb));
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nc][kb][i] = seen >> i & 1 ? s[nc][kb][i] : -INFINITY;
                }
            }
            weights<D, NC, 2>(w, s, a.scale_log2, 0.f);
            bf16x8 va[NDB], pf[NC];
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) pf[nc] = pack8(s[nc][0], s[nc][1]);
            // lane 4j + i names features 4i .. of row j, and receives feature
            // c16 of four rows
            const bf16* vrow = vdraft + (k0 + 8 * g + (c16 >> 2)) * draft_stride<D>() + 4 * (c16 & 3);
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
                const u32x2 x = __builtin_bit_cast(u32x2, lds_read_tr16(vrow + db * 16));
                const u32x2 y = __builtin_bit_cast(u32x2, lds_read_tr16(vrow + 4 * draft_stride<D>() + db * 16));
                va[db] = __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
            }
            add_values<D, NC>(w, va, pf, true);
        }
    }

    // ---- join the key waves ----
    if constexpr (DRAFT) __syncthreads();  // the drafted values' place is free
    float* red_m = tree_smem;
    float* red_l = red_m + WK * kCols;
    float* red_o = red_l + WK * kCols;
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        const int col = (wc * NC + nc) * 16 + c16, at = wk * kCols + col;
        const float l = xgroup_sum(w.l[nc]);
        if (g == 0) {
            red_m[at] = w.m[nc];
            red_l[at] = l;
        }
        float* o = red_o + (size_t)at * col_floats<D>() + 4 * g;
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<floatx4*>(o + db * 16) = w.acc[nc][db];
    }
    __syncthreads();
    join_waves<D, kCols, WK, bf16>(a, red_m, red_l, red_o, unit, cb, split, nodes);
}

// fp32 caches: the same on fp32 matrix cores (16x16x4), 16 columns a workgroup
// whose NW waves take turns with the 32-key chunks, laid out as the fp32 decode:
// lane (g, c16) holds key 16 kb + 4g + i of column c16; contraction step (j, e)
// of S^T pairs feature 16j + 4g + e.
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void tree_f32_kernel(TreeParams a) {
    constexpr int NJ = D / 16;
    extern __shared__ __attribute__((aligned(16))) float tree_smem[];
    const int id = blockIdx.x;
    const int group = id / a.f8cb, r8 = id - group * a.f8cb.d;
    const int unit = group * 8 + (r8 & 7), cb = r8 >> 3;
    if (unit >= a.units) return;
    const int split = blockIdx.y;
    const int b = unit / a.fHkv;
    if (a.active && a.active[b] == 0) return;
    const CacheView& c = a.c;
    const int n = min(max(a.n_tok[b], 0), a.max_tok);
    const int nodes = a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
    if (nodes == 0) return;
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

    const unsigned long long lines = tree_lines(a.parents + (size_t)b * a.T, nodes);
    int deepest = lane < nodes ? __builtin_popcountll(lines) - 1 : 0;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) deepest = max(deepest, __shfl_xor(deepest, off, 64));
    deepest = __builtin_amdgcn_readfirstlane(deepest);
    const int lo_first = win_lo_rt(c.window, n, c.W, c.C);
    const int lo_last = win_lo_rt(c.window, n + deepest, c.W, c.C);
    const int sum_first = min(lo_first / c.C, c.S_max), sum_last = min(lo_last / c.C, c.S_max);

    // column c16 (past the last: the last again, not stored)
    const int col = min(cb * 16 + c16, a.cols - 1);
    const int t = col % a.fT;
    unsigned long long line = __shfl(lines, t, 64);
    const int lo = win_lo_rt(c.window, n + __builtin_popcountll(line) - 1, c.W, c.C);
    const int n_sum = min(lo / c.C, c.S_max);
    if (t >= nodes) line = 0;
    floatx4 qf[NJ], acc[NJ];
    const float* qrow = static_cast<const float*>(a.q) + (bg * a.cols + col) * D;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        qf[j] = *reinterpret_cast<const floatx4*>(qrow + 16 * j + 4 * g);
        acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
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
        const unsigned span = (unsigned)(key_hi - key_lo);
        // keys of this lane's column: first .. last, or its line
        const int first = draft || is_sum ? 0 : max(lo - pos0, key_lo);
        const int last = is_sum ? min(n_sum - pos0 - 1, key_hi) : key_hi;
        const uint32_t seen = draft ? (uint32_t)(line >> pos0) : 0xffffffffu;
        floatx4 s[2];
        float pw[2][4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            s[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
            // a drafted row past the last node is not there: the last one's
            const int key = draft ? min(16 * kb + c16, key_hi) : 16 * kb + c16;
            const float* krow = kt + (size_t)key * D + 4 * g;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const floatx4 kf = *reinterpret_cast<const floatx4*>(krow + 16 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[kb] = mfma_f32(kf[e], qf[j][e], s[kb]);
            }
            if (!full) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = 16 * kb + 4 * g + i;
                    s[kb][i] = k >= first && k <= last && (seen >> k & 1) ? s[kb][i] : -INFINITY;
                }
            }
        }
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
            const float* vtile = vt + (size_t)(2 * kb + (g >> 1)) * (kVtTile * D) + 4 * (g & 1);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                floatx4 vf;
                if (draft) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        vf[i] = vt[(size_t)min(16 * kb + 4 * g + i, key_hi) * D + 16 * j + c16];
                } else {
                    vf = *reinterpret_cast<const floatx4*>(vtile + (16 * j + c16) * kVtTile);
                }
                if (!full) {
                    bool bad = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned rel = (unsigned)(16 * kb + 4 * g + i - key_lo);
                        vf[i] = rel <= span ? vf[i] : 0.f;
                        bad |= !is_finite(vf[i]);
                    }
                    if (__builtin_amdgcn_ballot_w64(bad)) {
                        // a weight of 0 times it would be NaN: finite values as
                        // they are, of the others what their weights make of them
                        const floatx4 zero{0.f, 0.f, 0.f, 0.f};
                        floatx4 cn = zero, ci = zero, cm = zero;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = vf[i];
                            cn = mfma_f32(x != x ? 1.f : 0.f, pw[kb][i], cn);
                            ci = mfma_f32(x == INFINITY ? 1.f : 0.f, pw[kb][i], ci);
                            cm = mfma_f32(x == -INFINITY ? 1.f : 0.f, pw[kb][i], cm);
                            vf[i] = is_finite(x) ? x : 0.f;
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (cn[i] > 0.f) acc[j][i] = NAN;
                            if (ci[i] > 0.f) acc[j][i] += INFINITY;
                            if (cm[i] > 0.f) acc[j][i] -= INFINITY;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j] = mfma_f32(vf[i], pw[kb][i], acc[j]);
            }
        }
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
        for (int j = 0; j < NJ; ++j) *reinterpret_cast<floatx4*>(o + 16 * j) = acc[j];
    }
    __syncthreads();
    join_waves<D, 16, NW, float>(a, red_m, red_l, red_o, unit, cb, split, nodes);
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
        if (mx == -INFINITY) continue;
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

template <int D, bool Q8, bool DRAFT, int NC, int WC, int WK>
hipError_t launch_shape(const TreeParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.units + 7) / 8 * 8 * p.col_blocks), (unsigned)p.splits);
    hipLaunchKernelGGL((tree_kernel<D, Q8, DRAFT, NC, WC, WK>), grid, dim3(WC * WK * 64), tree_lds<D>(NC, WC, WK, DRAFT), stream, p);
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
    switch (p.shape) {
        case kTreeNarrow:
            e = p.k ? launch_shape<D, Q8, true, 1, 1, 4>(p, stream) : launch_shape<D, Q8, false, 1, 1, 4>(p, stream);
            break;
        case kTreeNarrowWide:
            e = p.k ? launch_shape<D, Q8, true, 1, 1, 12>(p, stream) : launch_shape<D, Q8, false, 1, 1, 12>(p, stream);
            break;
        case kTree32: e = launch_shape<D, Q8, true, 2, 1, 4>(p, stream); break;
        case kTree64: e = launch_shape<D, Q8, true, 2, 2, 2>(p, stream); break;
        default: e = launch_shape<D, Q8, true, 2, 4, 1>(p, stream); break;
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
    if (p.shape == kTreeNarrowWide)
        hipLaunchKernelGGL((tree_f32_kernel<D, 12>), grid, dim3(12 * 64), tree_lds<D>(1, 1, 12, false), stream, p);
    else
        hipLaunchKernelGGL((tree_f32_kernel<D, 4>), grid, dim3(4 * 64), tree_lds<D>(1, 1, 4, false), stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && p.splits > 1 ? launch_join<D, float>(p, stream) : e;
}
template hipError_t launch_tree_f32<64>(const TreeParams&, hipStream_t);
template hipError_t launch_tree_f32<128>(const TreeParams&, hipStream_t);

}  // namespace eva
