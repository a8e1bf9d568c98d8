// Decode over a paged cache: one query per sequence attends all its tokens, or
// those of a list of pages.
//
// A row is (sequence, kv head, group of up to 16 query heads, or 32 where a kv head has more
// than 16: NC = 2 tiles of columns share the operands); its keys go by
// chunks of one or two blocks of 16 tokens, each of which lies in one page.  Per
// chunk a wave computes S^T = K Q^T and O^T += V^T P^T on the matrix cores with
// the operands read straight from memory, 16 bytes a lane, the softmax's maximum
// and sum running: every key and value is read once for the heads that share it, past
// the caches (with loads that keep them, 64 sequences at 8k take 249 us instead of 218.8,
// 6.5 TB/s).  Bound by memory; calls of few tokens by the chain counts -> table -> keys ->
// softmax -> join, 14 us for one sequence of 8000 (32 MB).
//
// The batch's rows may differ in length by any factor, and their lengths are on
// the device.  So the launch has a fixed number of workgroups, and they share the
// chunks of all rows in equal parts, each within a row where the workgroups suffice for that,
// else one row after the other: a workgroup finds its part from the sequences' token counts
// (a scan, half a microsecond), and rows in more than one part are joined by a second launch.  Where rows are
// short and many, every wave takes rows of its own, whole ones: no barrier, no joining.
#include "paged.hpp"

namespace eva {

namespace {

constexpr float kPagedTau = 8.f;  // log2 units: unscaled weights stay <= 256
constexpr int kPagedWaves = 4;

// Pages that a row's query attends, of a sequence of n tokens: all it has, or the
// first so many of its list.
__device__ __forceinline__ int row_pages(const PagedParams& a, int n) {
    const int held = pages_of(n, a.t.shift);
    return a.pages ? min(a.S, held) : held;
}
// Chunks of a row; at least one, which writes the zeros of a sequence without tokens;
// none for an inactive one.
template <int TOKENS>
__device__ __forceinline__ int row_chunks(const PagedParams& a, int b, int n) {
    if (a.active && a.active[b] == 0) return 0;
    const int len = a.pages ? row_pages(a, n) << a.t.shift : n;
    return max((len + TOKENS - 1) / TOKENS, 1);
}

// A word that every lane wants and that nothing writes during the launch: through the
// scalar cache, so that waiting for it does not wait for the vector loads before it.
__device__ __forceinline__ int scalar_load(const int* p) {
    return *(const __attribute__((address_space(4))) int*)p;
}

// 16 tokens of a page.
struct Block {
    size_t at;  // elements from the pool's start to their rows (keys and values alike)
    int left;   // tokens of the sequence from the first of them on
    int valid;  // of the block's, the first so many are attended
    bool lost;  // the table names no page of the pool
};

// Chunk `chunk` of NB blocks of the row (b, kvh).  Pages hold whole chunks, but for
// those of 16 tokens where NB is 2.
template <int D, int NB>
__device__ __forceinline__ void locate(Block (&x)[NB], const PagedParams& a, int b, int kvh, int n, int n_pages, int chunk) {
    const int shift = a.t.shift;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        if (i > 0 && shift > 4) {
            x[i].at = x[0].at + 16 * i * D;
            x[i].valid = max(min(x[0].left - 16 * i, 16), 0);
            x[i].lost = x[0].lost;
            continue;
        }
        const int v = (chunk * NB + i) * 16, e = v >> shift, off = v & ((1 << shift) - 1);
        x[i] = Block{};
        if (e < n_pages) {
            int lp = e;
            if (a.pages) lp = scalar_load(a.pages + ((size_t)b * a.Hkv + kvh) * a.S + e);
            const int left = (unsigned)lp < (unsigned)pages_of(n, shift) ? n - ((lp << shift) + off) : 0;
            if (left > 0) {
                const int page = scalar_load(a.t.table + (size_t)b * a.t.max_pages + lp);
                x[i].left = left;
                x[i].valid = min(left, 16);
                x[i].lost = (unsigned)page >= (unsigned)a.t.n_pages;
                x[i].at = ((((size_t)(x[i].lost ? 0 : page) * a.Hkv + kvh) << shift) + off) * D;
            }
        }
    }
}

// The running state of a wave: 16 columns, per lane (g, c16) the features
// 16 db + 4 g .. + 3 of column c16.
template <int D>
struct RowState {
    float m, l;
    floatx4 acc[D / 16];
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    // Scores of a chunk (two blocks of four per lane) become weights; the reference
    // maximum moves only when the chunk's exceeds it by more than kPagedTau.  The maximum is one of
    // the scores as they are and is taken off before they are scaled, so that it weighs 1 exactly:
    // scaled and rounded first it would be off by half a step, 128 from 2^31 on, and the weights
    // infinite or 0.  (One instruction a score more than a fused scaling: 64 sequences at 8k 218.8
    // us against 218.7, 1024 rows of 64 to 512 tokens 0 to 1%.)
    template <int NB>
    __device__ __forceinline__ void weigh(floatx4 (&s)[NB], float scale) {
        float mx = s[0][0];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[kb][i]);
        mx = xgroup_max(mx);
        const bool raise = (mx - m) * scale > kPagedTau;
        if (__builtin_amdgcn_ballot_w64(raise)) {
            const float next = raise ? mx : m;
            const float alpha = raise ? fast_exp2((m - next) * scale) : 1.f;  // the first time: exp2(-inf) = 0
            l *= alpha;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) acc[i] *= alpha;
            m = next;
        }
        // no maximum yet (scores of -inf alone): their weights are 0
        const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[kb][i] = fast_exp2((s[kb][i] - off) * scale);
                l += s[kb][i];
            }
    }
};

// Query fragments, and one chunk's products, by type.  `valid` has a bit for each
// of the chunk's tokens that is attended, `lost` for each whose page there is not.
template <int D, typename T>
struct Chunk;

template <int D>
struct Chunk<D, bf16> {
    static constexpr int kBlocks = 2;
    bf16x8 k[2][D / 32], v[D / 16];
    // Rows are permuted so that the eight scores of a lane are keys 8g .. 8g + 7 (block kb:
    // + 4 kb + i), the slots of its 16 bytes of a feature's values.
    static __device__ __forceinline__ void query(bf16x8 (&q)[D / 32], const bf16* row, int g) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) q[i] = *reinterpret_cast<const bf16x8*>(row + 32 * i + 8 * g);
    }
    static __device__ __forceinline__ int mask_of(uint32_t bits, int g, int kb) { return (int)(bits >> (8 * g + 4 * kb)) & 15; }
    __device__ __forceinline__ void load_keys(const bf16* kp, const Block (&x)[2], int g, int c) {
        const bf16* kr = kp + (c >= 8 ? x[1].at : x[0].at) + ((c >> 2 & 1) * 8 + (c & 3)) * D + 8 * g;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                k[kb][i] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(kr + 4 * kb * D + 32 * i));
    }
    __device__ __forceinline__ void load_values(const bf16* vp, const Block (&x)[2], int g, int c) {
        const bf16* vr = vp + (g >= 2 ? x[1].at : x[0].at) + vt_index<D>(c, 8 * (g & 1));
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            v[i] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(vr + 16 * i * kVtTile));
    }
    __device__ __forceinline__ void scores(const bf16x8 (&q)[D / 32], floatx4 (&s)[2]) const {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            s[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) s[kb] = mfma_bf16(k[kb][i], q[i], s[kb]);
        }
    }
    // values of tokens that are not attended may be any bits: they become zeros
    __device__ __forceinline__ void keep_values(uint32_t valid, int g) {
        uint32_t keep[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t two = valid >> (8 * g + 2 * i);
            keep[i] = (two & 1 ? 0x0000ffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            u32x4 w = __builtin_bit_cast(u32x4, v[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] &= keep[j];
            v[i] = __builtin_bit_cast(bf16x8, w);
        }
    }
    // Weights as the products' operand: two bf16 numbers each, the weight cut off after 8
    // bits and what that left, 16 bits in all (one rounded number would double the square of
    // the output's error, 0.0017 -> 0.0023 of its norm with the output's own rounding).  The
    // second product is hidden behind memory: 217.8 us for 64 sequences at 8k either way.  (A third
    // number, which holds all 24 bits, changes 0.4% of the outputs by one step, leaves their error as it
    // is, 0.0017, and takes 219.3 us against 218.7, and 0.1 to 0.2 us of calls of few or short rows.)
    //
    // What is left is not 0 under a weight that is not, since an infinite value times 0 is NaN: it is
    // 2^-126 at least, bf16's smallest normal number and the smallest weight that exp2 gives
    // (those below are 0), or the weight itself if that is less.
    static __device__ __forceinline__ float rest(float x, uint32_t xu) {
        return fmaxf(x - __uint_as_float(xu & 0xffff0000u), fminf(x, 0x1p-126f));
    }
    __device__ __forceinline__ void add(const floatx4 (&p)[2], floatx4 (&acc)[D / 16]) const {
        u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = p[i / 2][i % 2 * 2], y = p[i / 2][i % 2 * 2 + 1];
            const uint32_t xu = __float_as_uint(x), yu = __float_as_uint(y);
            hi[i] = __builtin_amdgcn_perm(yu, xu, 0x07060302);
            lo[i] = pack_bf16x2(rest(x, xu), rest(y, yu));
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            acc[i] = mfma_bf16(v[i], __builtin_bit_cast(bf16x8, lo), mfma_bf16(v[i], __builtin_bit_cast(bf16x8, hi), acc[i]));
    }
};

template <int D>
struct Chunk<D, float> {
    static constexpr int NB = paged_blocks(D, sizeof(float));
    static constexpr int kBlocks = NB;
    floatx4 k[NB][D / 16], v[NB][D / 16];
    // Contraction step (i, e) of the scores: feature 16 i + 4 g + e; of the values: key
    // 16 kb + 4 g + e, whose weight the lane holds already.
    static __device__ __forceinline__ void query(floatx4 (&q)[D / 16], const float* row, int g) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const floatx4*>(row + 16 * i + 4 * g);
    }
    static __device__ __forceinline__ int mask_of(uint32_t bits, int g, int kb) { return (int)(bits >> (16 * kb + 4 * g)) & 15; }
    __device__ __forceinline__ void load_keys(const float* kp, const Block (&x)[NB], int g, int c) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const float* kr = kp + x[kb].at + c * D + 4 * g;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                k[kb][i] = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(kr + 16 * i));
        }
    }
    __device__ __forceinline__ void load_values(const float* vp, const Block (&x)[NB], int g, int c) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const float* vr = vp + x[kb].at + vt_index<D>(c, 4 * g);
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                v[kb][i] = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(vr + 16 * i * kVtTile));
        }
    }
    __device__ __forceinline__ void scores(const floatx4 (&q)[D / 16], floatx4 (&s)[NB]) const {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            s[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[kb] = mfma_f32(k[kb][i][e], q[i][e], s[kb]);
        }
    }
    __device__ __forceinline__ void keep_values(uint32_t valid, int g) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const int m = mask_of(valid, g, kb);
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[kb][i][e] = m >> e & 1 ? v[kb][i][e] : 0.f;
        }
    }
    __device__ __forceinline__ void add(const floatx4 (&p)[NB], floatx4 (&acc)[D / 16]) const {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i] = mfma_f32(v[kb][i][e], p[kb][e], acc[i]);
    }
};

template <typename T>
struct QueryFragment;
template <>
struct QueryFragment<bf16> {
    typedef bf16x8 type;
    static constexpr int kFeatures = 32;
};
template <>
struct QueryFragment<float> {
    typedef floatx4 type;
    static constexpr int kFeatures = 16;
};

__device__ __forceinline__ void store4(bf16* o, const floatx4& x) {
    *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
}
__device__ __forceinline__ void store4(float* o, const floatx4& x) { *reinterpret_cast<floatx4*>(o) = x; }

// What a row's sums come to.  m = -inf: no key had a score above -inf; l tells
// why: 0 no keys (zeros), else the formula has no value (-1: scores of -inf alone,
// NaN: of NaN).
__device__ __forceinline__ floatx4 finish(float m, float l, const floatx4& o) {
    if (m == -INFINITY) {
        const float x = l == 0.f ? 0.f : NAN;
        return floatx4{x, x, x, x};
    }
    return o * (1.f / l);
}

// Workspace: an int2 for each row (x: -1, or 2 w + s for a row whose first part is share
// s of workgroup w; y: how many workgroups after w hold the rest), then [wgs][2] shares
// of 16 NC columns: maximum, sum, two floats unused, [D] weighted values.  Share 0 is that of a part's first row,
// share 1 that of its last one.
template <int D, int NC>
__host__ __device__ constexpr int share_floats() { return 16 * NC * share_col(D); }
__device__ __forceinline__ float* shares_of(const PagedParams& a) { return a.ws + (a.rows + 1) / 2 * 4; }

template <int D, typename T, int NC>
__global__ __launch_bounds__(kPagedWaves * 64) __attribute__((amdgpu_waves_per_eu(NC == 1 ? 3 : 2, 8)))
void paged_decode_kernel(PagedParams a) {
    constexpr int NW = kPagedWaves;
    constexpr int COL = D + 4;  // 16 columns on distinct banks
    typedef typename QueryFragment<T>::type Frag;
    constexpr int NQ = D / QueryFragment<T>::kFeatures;
    constexpr int NB = Chunk<D, T>::kBlocks;
    __shared__ float red_m[NW][16 * NC], red_l[NW][16 * NC];
    __shared__ __attribute__((aligned(16))) float red_o[NW][16 * NC][COL];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c16 = lane & 15;
    const int unit = a.f_unit;  // rows of a sequence
    const T* kp = static_cast<const T*>(a.k);
    const T* vp = static_cast<const T*>(a.vt);

    // This workgroup's part: `todo` chunks from chunk c0 of row `row` of sequence b on; or,
    // where rows are short and many (`alone`), this wave's: `todo` rows.  The lanes hold 64
    // sequences' counts at a time, w0 the first of them.
    int b, row, c0 = 0, todo, part = 0, w0, tokens, chunk_of;
    bool alone;
    auto window = [&](int from) {
        w0 = from;
        const int i = min(from + lane, a.t.B - 1);
        tokens = held_tokens(a.t, i);
        chunk_of = from + lane < a.t.B ? row_chunks<16 * NB>(a, i, tokens) : 0;
    };
    if (a.ws) {
        // all sequences: chunks, how many take part, whether a row is longer than a wave takes alone
        int chunks = 0, active = 0, i = 0;
        unsigned long long longer = 0, longest = 0;
        do {
            window(i);
            chunks += chunk_of;
            active += __builtin_popcountll(__builtin_amdgcn_ballot_w64(chunk_of > 0));
            longer |= __builtin_amdgcn_ballot_w64(chunk_of > kPagedShortest);
            longest |= __builtin_amdgcn_ballot_w64(chunk_of > kPagedShort);
            i += 64;
        } while (i < a.t.B);
        int total = __builtin_amdgcn_readlane(wave_scan(chunks), 63) * unit;
        alone = (active * unit >= kPagedMany ? longest : longer) == 0;
        // What the workers are given in their order: rows (alone); parts of `part` chunks, each
        // within one row (within), if that takes no more workgroups than there are; else
        // chunks, whatever their row.  (A second row costs a workgroup 4 us: one sequence of 8000
        // tokens 15.1 us against 13.8, so it is looked at for parts of up to kPagedWithin.)
        bool within = false;
        float inv = 0.f;
        auto parts_of = [&](int x) {  // exact: x stays below 2^24 / kPagedWithin where it is asked
            const int q = (int)((float)(x + part - 1) * inv);
            return q - (q * part > x + part - 1) + ((q + 1) * part <= x + part - 1);
        };
        int workers = a.wgs, me = blockIdx.x;
        if (alone) {
            total = active * unit;
            workers = a.wgs * NW;
            me = me * NW + wave;
        } else {
            part = max((total + a.wgs - 1) / a.f_wgs, kPagedMinPart);
            if (part <= kPagedWithin) {
                inv = 1.f / (float)part;
                int parts = 0;
                if (a.t.B <= 64) {
                    parts = parts_of(chunk_of);
                } else {
                    for (i = 0; i < a.t.B; i += 64) {
                        window(i);
                        parts += parts_of(chunk_of);
                    }
                }
                parts = __builtin_amdgcn_readlane(wave_scan(parts), 63) * unit;
                within = parts <= a.wgs;
                if (within) total = parts;
            }
        }
        const int share = within ? 1 : alone ? (total + workers - 1) / workers : part;
        const long long from = (long long)me * share;
        if (from >= total) return;
        todo = min(share, total - (int)from);
        // the sequence that holds `from`
        if (a.t.B > 64) window(0);
        int before = 0, at, each;
        while (true) {
            const int mine = alone ? chunk_of > 0 : within ? parts_of(chunk_of) : chunk_of;
            const int upto = before + wave_scan(mine * unit);
            const unsigned long long past = __builtin_amdgcn_ballot_w64(upto > (int)from);
            if (past) {
                const int l = __builtin_ctzll(past);
                b = w0 + l;
                each = __builtin_amdgcn_readlane(mine, l);
                at = (int)from - (__builtin_amdgcn_readlane(upto, l) - each * unit);
                break;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
            if (w0 + 64 >= a.t.B) return;  // only where the counts change during the call
            window(w0 + 64);
        }
        row = at / each;
        c0 = at - row * each;
        if (within) {
            c0 *= part;
            todo = min(part, __builtin_amdgcn_readlane(chunk_of, b - w0) - c0);
        }
    } else {
        alone = a.alone;
        const int r = alone ? (int)blockIdx.x * NW + wave : (int)blockIdx.x;
        if (r >= a.rows) return;
        b = r / a.f_unit;
        row = r % a.f_unit;
        window(b / 64 * 64);
        const int chunks = __builtin_amdgcn_readlane(chunk_of, b - w0);
        if (chunks == 0) return;
        todo = alone ? 1 : chunks;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    row = __builtin_amdgcn_readfirstlane(row);
    c0 = __builtin_amdgcn_readfirstlane(c0);
    todo = __builtin_amdgcn_readfirstlane(todo);
    const int step = alone ? 1 : NW;

    for (bool first = true;; first = false) {
        const int n = __builtin_amdgcn_readlane(tokens, b - w0);
        const int n_pages = row_pages(a, n);
        const int chunks = __builtin_amdgcn_readlane(chunk_of, b - w0);
        const int c1 = alone ? chunks : min(chunks, c0 + todo);
        const int kvh = row / a.f_hg, hg = row % a.f_hg;
        const int h0 = kvh * a.G + hg * 16 * NC;
        const int ncols = min(16 * NC, a.G - hg * 16 * NC);
        // columns past ncols repeat the last head; their outputs are not stored
        Frag q[NC][NQ];
        RowState<D> st[NC];
#pragma unroll
        for (int t = 0; t < NC; ++t) {
            Chunk<D, T>::query(q[t], static_cast<const T*>(a.q) + ((size_t)b * a.H + h0 + min(16 * t + c16, ncols - 1)) * D, g);
            st[t].clear();
        }
        bool any = false;
        // a chunk's keys are requested while the one before is weighed, its values once
        // that one's have been used: the wave always has half a chunk in flight
        Chunk<D, T> rows;
        Block x[NB];
        int ch = alone ? 0 : c0 + wave;
        if (ch < c1) {
            locate<D, NB>(x, a, b, kvh, n, n_pages, ch);
            rows.load_keys(kp, x, g, c16);
            rows.load_values(vp, x, g, c16);
        }
        while (ch < c1) {
            // a bit for each token that is attended, and for each whose page there is not
            uint32_t valid = 0, lost = 0;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                valid |= ((1u << x[i].valid) - 1) << (16 * i);
                lost |= (x[i].lost ? 0xffffu : 0u) << (16 * i);
            }
            any = any || valid != 0;
            ch += step;
            const bool more = ch < c1;
            if (more) locate<D, NB>(x, a, b, kvh, n, n_pages, ch);
            floatx4 s[NC][NB];
#pragma unroll
            for (int t = 0; t < NC; ++t) rows.scores(q[t], s[t]);
            __builtin_amdgcn_sched_barrier(0);
            if (more) rows.load_keys(kp, x, g, c16);
            if (valid != 0xffffffffu >> (32 - 16 * NB) || lost) {
#pragma unroll
                for (int kb = 0; kb < NB; ++kb) {
                    const int in = Chunk<D, T>::mask_of(valid, g, kb), no = Chunk<D, T>::mask_of(lost, g, kb);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int t = 0; t < NC; ++t)
                            s[t][kb][i] = in >> i & 1 ? no >> i & 1 ? NAN : s[t][kb][i] : -INFINITY;
                }
                rows.keep_values(valid, g);
            }
#pragma unroll
            for (int t = 0; t < NC; ++t) {
                st[t].weigh(s[t], a.scale_log2);
                rows.add(s[t], st[t].acc);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) rows.load_values(vp, x, g, c16);
        }

        // ---- the waves' parts of the row ----
        bool whole = true;
#pragma unroll
        for (int t = 0; t < NC; ++t) {
            const int col = 16 * t + c16;
            float l = xgroup_sum(st[t].l);
            if (any && st[t].m == -INFINITY && l == 0.f) l = -1.f;  // see finish()
            if (alone) {
                if (col < ncols) {
                    T* o = static_cast<T*>(a.o) + ((size_t)b * a.H + h0 + col) * D + 4 * g;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) store4(o + 16 * i, finish(st[t].m, l, st[t].acc[i]));
                }
                continue;
            }
            if (g == 0) {
                red_m[wave][col] = st[t].m;
                red_l[wave][col] = l;
            }
            if (col < ncols) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    *reinterpret_cast<floatx4*>(&red_o[wave][col][16 * i + 4 * g]) = st[t].acc[i];
            }
        }
        const int share = first ? 0 : 1;
        if (!alone) {
            __syncthreads();
            whole = c0 == 0 && c1 == chunks;
            float* part_ws = a.ws ? shares_of(a) + ((size_t)blockIdx.x * 2 + share) * share_floats<D, NC>() : nullptr;
            for (int t = tid; t < ncols * (D / 4); t += NW * 64) {
                const int col = t / (D / 4), f = t % (D / 4) * 4;
                float m = -INFINITY, sum = 0.f;
                floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < NW; ++w) m = fmaxf(m, red_m[w][col]);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    // without a maximum there is no weight; sums of NaN stay, and where there is none at
                    // all the waves' reasons are summed as they are
                    const float mw = red_m[w][col];
                    const float wt = m == -INFINITY ? 1.f : mw == -INFINITY ? 0.f : fast_exp2((mw - m) * a.scale_log2);
                    sum += wt * red_l[w][col];
                    o += wt * *reinterpret_cast<const floatx4*>(&red_o[w][col][f]);
                }
                if (whole) {
                    store4(static_cast<T*>(a.o) + ((size_t)b * a.H + h0 + col) * D + f, finish(m, sum, o));
                } else {
                    float* to = part_ws + col * share_col(D);
                    if (f == 0) *reinterpret_cast<floatx2*>(to) = floatx2{m, sum};
                    *reinterpret_cast<floatx4*>(to + 4 + f) = o;
                }
            }
        }
        if (!a.ws) return;
        if (c0 == 0 && (alone ? lane : tid) == 0) {
            int2 info = {-1, 0};
            if (!whole) info = int2{2 * (int)blockIdx.x + share, (chunks - c1 + part - 1) / part};
            reinterpret_cast<int2*>(a.ws)[b * unit + row] = info;
        }
        todo -= alone ? 1 : c1 - c0;
        if (todo == 0) return;
        c0 = 0;
        if (++row == unit) {
            row = 0;
            do {  // todo > 0: there is one (unless the counts change during the call)
                if (++b == a.t.B) return;
                if (b == w0 + 64) window(b);
            } while (__builtin_amdgcn_readlane(chunk_of, b - w0) == 0);
        }
        if (!alone) __syncthreads();  // the parts have been read
    }
}

// Joins the shares of rows that more than one workgroup held: a workgroup per query
// head, whose threads, four features each, divide the shares and meet in LDS (one sequence
// of 8000 tokens, 63 shares a row: 13.8 us the whole decode, 15.3 with a workgroup per row that
// reads all its columns through one CU).
constexpr int kJoinThreads = 256;
template <int D>
struct Joined {
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    template <int N>
    __device__ __forceinline__ void add(const float (&mx)[N], const float (&lx)[N], const floatx4 (&ox)[N], float scale) {
        float top = m;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, mx[i]);
        // without a maximum there is no weight; sums of NaN stay, and where there is none at
        // all the reasons (finish()) are summed as they are
        const float keep = top == -INFINITY ? 1.f : m == -INFINITY ? 0.f : fast_exp2((m - top) * scale);
        l *= keep;
        o *= keep;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float wt = top == -INFINITY ? 1.f : mx[i] == -INFINITY ? 0.f : fast_exp2((mx[i] - top) * scale);
            l += wt * lx[i];
            o += wt * ox[i];
        }
        m = top;
    }
};

template <int D, typename T, int NC>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedParams a) {
    constexpr int ITEMS = D / 4, GROUPS = kJoinThreads / ITEMS;
    constexpr int NB = 4;  // shares whose loads are in flight together
    __shared__ float red_m[GROUPS], red_l[GROUPS];
    __shared__ __attribute__((aligned(16))) floatx4 red_o[GROUPS][ITEMS];
    const int b = (int)blockIdx.x / a.f_H, h = (int)blockIdx.x % a.f_H;
    if (a.active && a.active[b] == 0) return;  // no one has written its entry
    const int kvh = h / a.f_G, hg = h % a.f_G / (16 * NC), col = h % a.f_G % (16 * NC);
    const int2 info = reinterpret_cast<const int2*>(a.ws)[b * a.f_unit.d + kvh * a.n_hg + hg];
    if (info.x < 0) return;
    // (what no one has written, where counts change during the call, is no place of a share)
    if ((unsigned)(info.x >> 1) >= (unsigned)a.wgs || (unsigned)info.y >= (unsigned)(a.wgs - (info.x >> 1))) return;
    const int shares = 1 + info.y;
    const float* first = shares_of(a) + (size_t)info.x * share_floats<D, NC>();
    const float* rest = shares_of(a) + (size_t)((info.x >> 1) + 1) * 2 * share_floats<D, NC>();
    const int grp = threadIdx.x / ITEMS, f = threadIdx.x % ITEMS * 4;
    Joined<D> j;
    for (int s0 = grp; s0 < shares; s0 += GROUPS * NB) {
        float m[NB], l[NB];
        floatx4 o[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int s = min(s0 + i * GROUPS, shares - 1);
            const float* w = (s == 0 ? first : rest + (size_t)(s - 1) * 2 * share_floats<D, NC>()) + col * share_col(D);
            const floatx2 ml = *reinterpret_cast<const floatx2*>(w);
            m[i] = ml[0];
            l[i] = ml[1];
            o[i] = *reinterpret_cast<const floatx4*>(w + 4 + f);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
            if (s0 + i * GROUPS >= shares) {  // past the last
                m[i] = -INFINITY;
                l[i] = 0.f;
                o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
            }
        j.add(m, l, o, a.scale_log2);
    }
    if (f == 0) {
        red_m[grp] = j.m;
        red_l[grp] = j.l;
    }
    red_o[grp][f / 4] = j.o;
    __syncthreads();
    if (grp != 0) return;
    float m[GROUPS], l[GROUPS];
    floatx4 o[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        m[i] = red_m[i];
        l[i] = red_l[i];
        o[i] = red_o[i][f / 4];
    }
    Joined<D> all;
    all.add(m, l, o, a.scale_log2);
    store4(static_cast<T*>(a.o) + (size_t)blockIdx.x * D + f, finish(all.m, all.l, all.o));
}

}  // namespace

template <int D, typename T, int NC>
static hipError_t launch_columns(const PagedParams& p, hipStream_t stream) {
    const int wgs = p.ws ? p.wgs : p.alone ? (p.rows + kPagedWaves - 1) / kPagedWaves : p.rows;
    paged_decode_kernel<D, T, NC><<<wgs, kPagedWaves * 64, 0, stream>>>(p);
    if (p.ws) paged_join_kernel<D, T, NC><<<p.t.B * p.H, kJoinThreads, 0, stream>>>(p);
    return hipGetLastError();
}
template <int D, typename T>
hipError_t launch_paged_decode(const PagedParams& p, hipStream_t stream) {
    return paged_tiles(p.G) == 1 ? launch_columns<D, T, 1>(p, stream) : launch_columns<D, T, 2>(p, stream);
}
template hipError_t launch_paged_decode<64, bf16>(const PagedParams&, hipStream_t);
template hipError_t launch_paged_decode<128, bf16>(const PagedParams&, hipStream_t);
template hipError_t launch_paged_decode<64, float>(const PagedParams&, hipStream_t);
template hipError_t launch_paged_decode<128, float>(const PagedParams&, hipStream_t);

}  // namespace eva
