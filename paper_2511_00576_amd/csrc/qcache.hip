// The 8-bit cache's writes and its read-back: fill after a prefill, the append
// of a path of tokens (one token is a path of one; bf16 and fp32 caches take
// paths here too), and the copy into a bf16 cache.  All bound by memory: each
// row is read and written once, one exponent byte beside its codes.  On MI355X, d128:
// fill of 256 heads, 576 rows each 24.5 us, 4.6 TB/s; read back of 512 heads, 352
// rows each 25.7 us, 5.4 TB/s; paths of 8 tokens to 512 heads 14 us, the latency of
// a completed chunk's rows.
#include <type_traits>

#include "qrows.hpp"
#include "summary.hpp"

namespace eva {

namespace {

// ---------------------------------------------------------------------------
// fill
// ---------------------------------------------------------------------------
// One workgroup quantises 64 rows: 64 ring positions (64-aligned, so they are
// 64 consecutive slots) or 64 summaries.  A row is D / 8 lanes of eight
// features, keys go out as whole rows; the values' codes pass through LDS and
// leave as 16-byte pieces, one feature's 16 slots.
constexpr int kQFillRows = 64;
template <int D>
__global__ __launch_bounds__(256) void qcache_fill_kernel(QCacheView c, const bf16* __restrict__ K,
                                                          const bf16* __restrict__ V, const bf16* __restrict__ Ks,
                                                          const bf16* __restrict__ Vs, int L, int n_chunks, int ring_tiles,
                                                          const int* __restrict__ lens, RaggedState rs) {
    constexpr int TPR = D / 8, RPS = 256 / TPR;
    constexpr int kStride = D + 4;  // bytes: rows of a column's reads on distinct banks
    __shared__ __attribute__((aligned(16))) uint8_t vcodes[kQFillRows * kStride];
    const size_t bg = blockIdx.y;
    const int b = (int)blockIdx.y / c.Hkv;
    const int len = min(max(lens[b], 0), min(L, rs.max_tok));
    if (blockIdx.x == 0 && (int)blockIdx.y % c.Hkv == 0 && threadIdx.x == 0) {
        rs.n_tok[b] = len;
        rs.arrive[b] = 0;
    }
    const int first = max(0, len - c.R);
    const bool ring = (int)blockIdx.x < ring_tiles;
    int t0, r0, r1, slot0;  // the tile's first row, its valid rows, the slot of t0
    const bf16 *src_k, *src_v;
    uint8_t *dst_k, *dst_vt, *dst_ke, *dst_ve;
    if (ring) {
        t0 = (first / kQFillRows + (int)blockIdx.x) * kQFillRows;
        r0 = max(t0, first);
        r1 = min(t0 + kQFillRows, len);
        slot0 = t0 % c.R;
        src_k = K + bg * (size_t)L * D;
        src_v = V + bg * (size_t)L * D;
        dst_k = c.k_ring + bg * (size_t)c.R * D;
        dst_vt = c.vt_ring + bg * (size_t)c.R * D;
        dst_ke = c.k_ring_e + bg * (size_t)c.R;
        dst_ve = c.v_ring_e + bg * (size_t)c.R;
    } else {
        t0 = ((int)blockIdx.x - ring_tiles) * kQFillRows;
        r0 = t0;
        r1 = min(t0 + kQFillRows, len / c.C);
        slot0 = t0;
        src_k = Ks + bg * (size_t)n_chunks * D;
        src_v = Vs + bg * (size_t)n_chunks * D;
        dst_k = c.k_sum + bg * (size_t)c.S_max * D;
        dst_vt = c.vt_sum + bg * (size_t)c.S_max * D;
        dst_ke = c.k_sum_e + bg * (size_t)c.S_max;
        dst_ve = c.v_sum_e + bg * (size_t)c.S_max;
    }
    if (r0 >= r1) return;  // the same for the whole workgroup
    const int cc = threadIdx.x % TPR;
    // all of the thread's pieces before any wait (rows that are not the tile's:
    // its first again)
    constexpr int NS = kQFillRows / RPS;
    u32x4 kw[NS], vw[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int row = t0 + s * RPS + (int)threadIdx.x / TPR;
        const size_t at = (size_t)(row < r0 || row >= r1 ? r0 : row) * D + cc * 8;
        kw[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src_k + at));
        vw[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src_v + at));
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int i = s * RPS + (int)threadIdx.x / TPR;
        const int row = t0 + i;
        if (row < r0 || row >= r1) continue;  // a row's lanes stay together
        float x[8];
        u32x2 codes;
        unpack8(kw[s], x);
        const uint32_t ke = q_row<D>(x, codes);
        *reinterpret_cast<u32x2*>(dst_k + (size_t)(slot0 + i) * D + cc * 8) = codes;
        unpack8(vw[s], x);
        const uint32_t ve = q_row<D>(x, codes);
        *reinterpret_cast<uint32_t*>(vcodes + i * kStride + cc * 8) = codes[0];
        *reinterpret_cast<uint32_t*>(vcodes + i * kStride + cc * 8 + 4) = codes[1];
        if (cc == 0) {
            dst_ke[slot0 + i] = (uint8_t)ke;
            dst_ve[slot0 + i] = (uint8_t)ve;
        }
    }
    __syncthreads();
    // 16 slots x 4 features a thread: 16 words in, four 16-byte pieces out
    for (int e = threadIdx.x; e < kQFillRows / kQTile * (D / 4); e += 256) {
        const int f = e % (D / 4) * 4, g = e / (D / 4) * kQTile;
        const bool whole = t0 + g >= r0 && t0 + g + kQTile <= r1;
        uint8_t* out = dst_vt + qt_index<D>(f, slot0 + g);
        if (whole) {
            uint32_t t[4][4];  // [feature][four slots]
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint32_t*>(vcodes + (g + 4 * q + i) * kStride + f);
                // bytes of rows 0, 1 and of rows 2, 3 side by side, then both
                const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b2 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
                const uint32_t c2 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d2 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
                t[0][q] = __builtin_amdgcn_perm(c2, a, 0x05040100);
                t[1][q] = __builtin_amdgcn_perm(c2, a, 0x07060302);
                t[2][q] = __builtin_amdgcn_perm(d2, b2, 0x05040100);
                t[3][q] = __builtin_amdgcn_perm(d2, b2, 0x07060302);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<u32x4*>(out + j * kQTile) = u32x4{t[j][0], t[j][1], t[j][2], t[j][3]};
        } else {
            for (int i = max(r0 - t0, g); i < min(r1 - t0, g + kQTile); ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) out[j * kQTile + i - g] = vcodes[i * kStride + f + j];
        }
    }
}

// ---------------------------------------------------------------------------
// append of a path
// ---------------------------------------------------------------------------
// The summary of a chunk of the 8-bit ring, chunk_summary's in its own layout:
// keys in batches of four rows a thread (requested together: one after the
// other, each sweep waits for memory), values by 16 slots of a feature a load.
// Threads t < D / 8 are left with features 8t .. of both rows.
template <int D>
__device__ void q_chunk_summary(const QRingChunk<D>& src, int C, float* logits, float* red, float khat[8], float vhat[8]) {
    constexpr int TPR = D / 8, RPS = kSummaryThreads / TPR, NB = 4;
    const int t = threadIdx.x, cc = t % TPR, r0 = t / TPR;
    // rows r, r + RPS, ..: their features cc 8 .. times their scale
    auto keys = [&](int r, float (&k)[NB][8]) {
        u32x2 w[NB];
        uint32_t x[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int s = src.slot(min(r + i * RPS, C - 1));
            w[i] = *reinterpret_cast<const u32x2*>(src.k + (size_t)s * D + cc * 8);
            x[i] = src.ke[s];
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) k[i][e] = q_value(w[i][e >> 2] >> (8 * (e & 3)), q_scale(x[i]));
    };
    float ks[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int r = r0; r < C; r += NB * RPS) {
        float k[NB][8];
        keys(r, k);
#pragma unroll
        for (int i = 0; i < NB; ++i)
            if (r + i * RPS < C)
#pragma unroll
                for (int e = 0; e < 8; ++e) ks[e] += k[i][e];
    }
    reduce_rows8<TPR>(ks, red);
#pragma unroll
    for (int e = 0; e < 8; ++e) khat[e] = ks[e] * (1.0f / (float)C);

    const float sc = kLog2e * rsqrtf((float)D);
    float amax = -INFINITY;
    for (int r = r0; r < C; r += NB * RPS) {
        float k[NB][8];
        keys(r, k);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += khat[e] * k[i][e];
#pragma unroll
            for (int off = 1; off < TPR; off <<= 1) s += __shfl_xor(s, off, 64);
            s *= sc;
            if (r + i * RPS < C) {
                if (cc == 0) logits[r + i * RPS] = s;
                amax = fmaxf(amax, s);
            }
        }
    }
    amax = block_max(amax, red);  // also orders the logits' writes before their reads

    // thread's feature and its share of the 16-slot tiles that the chunk touches
    constexpr int TG = kSummaryThreads / D;
    const int f = t % D;
    const long long p16 = src.pos0 & ~15ll;
    const int tiles = (int)((src.pos0 + C - 1 - p16) / 16) + 1;
    float acc = 0.f, den = 0.f;
    for (int i = t / D; i < tiles; i += TG) {
        const int s = (int)((p16 + 16 * i) % src.R);
        const u32x4 w = *reinterpret_cast<const u32x4*>(src.vt + qt_index<D>(f, s));
        const u32x4 x = *reinterpret_cast<const u32x4*>(src.ve + s);
        const int row = (int)(p16 - src.pos0) + 16 * i;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if ((unsigned)(row + j) >= (unsigned)C) continue;  // another chunk's row
            const float p = fast_exp2(logits[row + j] - amax);
            den += p;
            acc += p * q_value(w[j >> 2] >> (8 * (j & 3)), q_scale(x[j >> 2] >> (8 * (j & 3)) & 255));
        }
    }
    __syncthreads();  // block_max's reads of red are done
    red[t] = acc;
    red[kSummaryThreads + t] = den;
    __syncthreads();
    if (t < TPR) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a = 0.f, d = 0.f;
#pragma unroll
            for (int g = 0; g < TG; ++g) {
                a += red[g * D + 8 * t + e];
                d += red[kSummaryThreads + g * D + 8 * t + e];
            }
            vhat[e] = a / d;
        }
    }
}

// One workgroup per (b, kv head).  The path's tokens take positions n, n + 1,
// ... : all their rows are written first, then the chunks they complete are
// summarised from the ring (which holds every position of such a chunk: R >=
// W + C - 1, and a path is at most W long).  The last of the sequence's H_kv
// workgroups advances n_tok[b].

// Tokens that the path of sequence b appends: its count, up to the first entry
// that names no token, and as many as the sequence may still hold.  Called by
// every thread of a workgroup.
__device__ inline int path_length(const PathParams& a, int b, int n) {
    int count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    count = min(count, max(a.max_tok - n, 0));
    if (a.path) {
        const int lane = threadIdx.x & 63;  // T <= 64
        const bool bad = lane < count && (unsigned)a.path[(size_t)b * a.T + lane] >= (unsigned)a.T;
        const unsigned long long m = __builtin_amdgcn_ballot_w64(bad);
        if (m) count = min(count, (int)__builtin_ctzll(m));
    }
    return __builtin_amdgcn_readfirstlane(count);
}

// Rows of a cache of T (bf16 or fp32).
template <int D, typename T>
struct PlainStore {
    CacheView c;
    T *kr, *vr;
    __device__ PlainStore(const CacheView& c_, size_t bg)
        : c(c_), kr(static_cast<T*>(c_.k_ring) + bg * (size_t)c_.R * D), vr(static_cast<T*>(c_.vt_ring) + bg * (size_t)c_.R * D) {}
    __device__ void rows(const T* k, const T* v, const int* path, int n, int count) const {
        for (int e = threadIdx.x; e < count * D; e += kSummaryThreads) {
            const int i = e / D, f = e % D;
            const size_t src = (size_t)(path ? path[i] : i) * D + f;
            const int slot = (n + i) % c.R;
            kr[(size_t)slot * D + f] = k[src];
            vr[vt_index<D>(f, slot)] = v[src];
        }
    }
    __device__ RingChunk<D, T> chunk(int s) const { return RingChunk<D, T>{kr, vr, (long long)s * c.C, c.R}; }
    __device__ void summary(size_t bg, int s, const float kh[8], const float vh[8]) const {
        const int t = threadIdx.x;
        if (t >= D / 8) return;
        T* ks = static_cast<T*>(c.k_sum) + (bg * c.S_max + s) * D + t * 8;
        T* vs = static_cast<T*>(c.vt_sum) + bg * (size_t)c.S_max * D;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ks[i] = from_f32<T>(kh[i]);
            vs[vt_index<D>(t * 8 + i, s)] = from_f32<T>(vh[i]);
        }
    }
};

// Rows of the 8-bit cache.
template <int D>
struct QuantStore {
    QCacheView c;
    uint8_t *k, *vt, *ke, *ve;
    __device__ QuantStore(const QCacheView& c_, size_t bg)
        : c(c_),
          k(c_.k_ring + bg * (size_t)c_.R * D),
          vt(c_.vt_ring + bg * (size_t)c_.R * D),
          ke(c_.k_ring_e + bg * (size_t)c_.R),
          ve(c_.v_ring_e + bg * (size_t)c_.R) {}
    __device__ void rows(const bf16* kn, const bf16* vn, const int* path, int n, int count) const {
        constexpr int TPR = D / 8;
        const int cc = threadIdx.x % TPR;
        // keys and values are rows of one list
        for (int r = threadIdx.x / TPR; r < 2 * count; r += kSummaryThreads / TPR) {
            const bool value = r >= count;
            const int i = value ? r - count : r;
            const int slot = (n + i) % c.R;
            float x[8];
            u32x2 codes;
            row8((value ? vn : kn) + (size_t)(path ? path[i] : i) * D + cc * 8, x);
            const uint32_t byte = q_row<D>(x, codes);
            if (value) {
#pragma unroll
                for (int j = 0; j < 8; ++j) vt[qt_index<D>(cc * 8 + j, slot)] = (uint8_t)(codes[j >> 2] >> (8 * (j & 3)));
            } else {
                *reinterpret_cast<u32x2*>(k + (size_t)slot * D + cc * 8) = codes;
            }
            if (cc == 0) (value ? ve : ke)[slot] = (uint8_t)byte;
        }
    }
    __device__ QRingChunk<D> chunk(int s) const { return QRingChunk<D>{k, vt, ke, ve, (long long)s * c.C, c.R}; }
    __device__ void summary(size_t bg, int s, const float kh[8], const float vh[8]) const {
        const int t = threadIdx.x;
        if (t >= D / 8) return;  // one row of lanes is left
        u32x2 codes;
        uint32_t byte = q_row<D>(kh, codes);
        *reinterpret_cast<u32x2*>(c.k_sum + (bg * c.S_max + s) * D + t * 8) = codes;
        if (t == 0) c.k_sum_e[bg * c.S_max + s] = (uint8_t)byte;
        byte = q_row<D>(vh, codes);
        uint8_t* vs = c.vt_sum + bg * (size_t)c.S_max * D;
#pragma unroll
        for (int j = 0; j < 8; ++j) vs[qt_index<D>(t * 8 + j, s)] = (uint8_t)(codes[j >> 2] >> (8 * (j & 3)));
        if (t == 0) c.v_sum_e[bg * c.S_max + s] = (uint8_t)byte;
    }
};

template <int D, typename T, typename Store, typename View>
__global__ __launch_bounds__(kSummaryThreads) void append_path_kernel(View c, PathParams a) {
    extern __shared__ float smem[];
    __shared__ int sh_n;
    const size_t bg = blockIdx.x;
    const int b = (int)blockIdx.x / c.Hkv;
    if (a.active && a.active[b] == 0) return;
    if (threadIdx.x == 0) sh_n = min(max(a.n_tok[b], 0), a.max_tok);
    __syncthreads();
    const int n = sh_n;
    const int count = path_length(a, b, n);
    if (count == 0) return;  // every workgroup of the sequence agrees
    const Store store(c, bg);
    const size_t in = bg * (size_t)a.T * D;
    store.rows(static_cast<const T*>(a.k) + in, static_cast<const T*>(a.v) + in, a.path ? a.path + (size_t)b * a.T : nullptr,
               n, count);
    const int s1 = min((n + count) / c.C, c.S_max);
    for (int s = n / c.C; s < s1; ++s) {
        __syncthreads();  // the rows are written, the last chunk's LDS is free
        float kh[8], vh[8];
        if constexpr (std::is_same<View, CacheView>::value) {
            if (c.rf) {
                const int cc = threadIdx.x % (D / 8);
                float e[8];
                rf_normals4(c.rf_seed, (uint32_t)(2 * cc), (uint32_t)s, (uint32_t)bg, e);
                rf_normals4(c.rf_seed, (uint32_t)(2 * cc + 1), (uint32_t)s, (uint32_t)bg, e + 4);
                chunk_summary<D, true>(store.chunk(s), c.C, smem, smem + c.C, kh, vh, RfNoise{e, c.rf_scale});
                store.summary(bg, s, kh, vh);
                continue;
            }
        }
        if constexpr (std::is_same<View, QCacheView>::value)
            q_chunk_summary<D>(store.chunk(s), c.C, smem, smem + c.C, kh, vh);
        else
            chunk_summary<D>(store.chunk(s), c.C, smem, smem + c.C, kh, vh);
        store.summary(bg, s, kh, vh);
    }
    if (threadIdx.x == 0) {
        if (atomicAdd(&a.arrive[b], 1) == c.Hkv - 1) {
            a.arrive[b] = 0;
            a.n_tok[b] = n + count;
        }
    }
}

// ---------------------------------------------------------------------------
// read back
// ---------------------------------------------------------------------------
// One workgroup per 32 rows (32 ring positions, 32-aligned, or 32 summaries):
// keys row by row, values feature by feature (16 slots in, two of the bf16
// cache's 8-slot pieces out), all in registers.  Non-temporal stores: 25.8 us for
// 137 MB instead of 29.3 (64 x 8 heads x 352 rows of 128 features; 64 rows a
// workgroup 27.6).
constexpr int kQReadRows = 32;
template <int D>
__global__ __launch_bounds__(256) void qcache_read_kernel(QCacheView c, CacheView to, const int* __restrict__ n_tok,
                                                          int max_tok, RaggedState rs, int ring_tiles) {
    const size_t bg = blockIdx.y;
    const int b = (int)blockIdx.y / c.Hkv;
    const int n = min(max(n_tok[b], 0), min(max_tok, rs.max_tok));
    if (blockIdx.x == 0 && (int)blockIdx.y % c.Hkv == 0 && threadIdx.x == 0) {
        rs.n_tok[b] = n;
        rs.arrive[b] = 0;
    }
    const bool ring = (int)blockIdx.x < ring_tiles;
    int t0, r0, r1, src0, dst0;
    const uint8_t *k, *vt, *ke, *ve;
    bf16 *ok, *ovt;
    if (ring) {
        const int first = max(0, n - min(c.R, to.R));
        t0 = (first / 32 + (int)blockIdx.x) * 32;
        r0 = max(t0, first);
        r1 = min(t0 + 32, n);
        src0 = t0 % c.R;
        dst0 = t0 % to.R;
        k = c.k_ring + bg * (size_t)c.R * D;
        vt = c.vt_ring + bg * (size_t)c.R * D;
        ke = c.k_ring_e + bg * (size_t)c.R;
        ve = c.v_ring_e + bg * (size_t)c.R;
        ok = static_cast<bf16*>(to.k_ring) + bg * (size_t)to.R * D;
        ovt = static_cast<bf16*>(to.vt_ring) + bg * (size_t)to.R * D;
    } else {
        t0 = ((int)blockIdx.x - ring_tiles) * 32;
        r0 = t0;
        r1 = min(t0 + 32, min(n / c.C, min(c.S_max, to.S_max)));
        src0 = dst0 = t0;
        k = c.k_sum + bg * (size_t)c.S_max * D;
        vt = c.vt_sum + bg * (size_t)c.S_max * D;
        ke = c.k_sum_e + bg * (size_t)c.S_max;
        ve = c.v_sum_e + bg * (size_t)c.S_max;
        ok = static_cast<bf16*>(to.k_sum) + bg * (size_t)to.S_max * D;
        ovt = static_cast<bf16*>(to.vt_sum) + bg * (size_t)to.S_max * D;
    }
    if (r0 >= r1) return;
    for (int e = threadIdx.x; e < 32 * (D / 16); e += 256) {
        const int i = e / (D / 16), f = e % (D / 16) * 16;
        if (t0 + i < r0 || t0 + i >= r1) continue;
        const u32x4 w = *reinterpret_cast<const u32x4*>(k + (size_t)(src0 + i) * D + f);
        const float sc = q_scale(ke[src0 + i]);
        uint32_t out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            out[j] = pack_bf16x2(q_value(w[j >> 1] >> (16 * (j & 1)), sc), q_value(w[j >> 1] >> (16 * (j & 1) + 8), sc));
        u32x4* dst = reinterpret_cast<u32x4*>(ok + (size_t)(dst0 + i) * D + f);
        __builtin_nontemporal_store(u32x4{out[0], out[1], out[2], out[3]}, dst);
        __builtin_nontemporal_store(u32x4{out[4], out[5], out[6], out[7]}, dst + 1);
    }
    for (int e = threadIdx.x; e < 2 * D; e += 256) {
        const int f = e % D, g = e / D * kQTile;
        const u32x4 w = *reinterpret_cast<const u32x4*>(vt + qt_index<D>(f, src0 + g));
        const u32x4 x = *reinterpret_cast<const u32x4*>(ve + src0 + g);
        uint32_t out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c2 = w[j >> 1] >> (16 * (j & 1)), e2 = x[j >> 1] >> (16 * (j & 1));
            out[j] = pack_bf16x2(q_value(c2, q_scale(e2 & 255)), q_value(c2 >> 8, q_scale(e2 >> 8 & 255)));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i0 = g + 8 * h;
            bf16* dst = ovt + vt_index<D>(f, dst0 + i0);
            if (t0 + i0 >= r0 && t0 + i0 + 8 <= r1) {
                __builtin_nontemporal_store(u32x4{out[4 * h], out[4 * h + 1], out[4 * h + 2], out[4 * h + 3]}, reinterpret_cast<u32x4*>(dst));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (t0 + i0 + j >= r0 && t0 + i0 + j < r1)
                        reinterpret_cast<uint16_t*>(dst)[j] = (uint16_t)(out[4 * h + (j >> 1)] >> (16 * (j & 1)));
            }
        }
    }
}

}  // namespace

template <int D>
hipError_t launch_qcache_fill(const QCacheView& c, const void* K, const void* V, const void* Ks, const void* Vs, int L,
                              const int* lens, const RaggedState& r, hipStream_t stream) {
    const int n_chunks = L / c.C;
    // min(L, R) positions from any start touch one more 64-aligned tile at most
    const int ring_tiles = (min(L, c.R) + kQFillRows - 1) / kQFillRows + 1;
    const int sum_tiles = (n_chunks + kQFillRows - 1) / kQFillRows;
    hipLaunchKernelGGL((qcache_fill_kernel<D>), dim3(ring_tiles + sum_tiles, c.B * c.Hkv), dim3(256), 0, stream, c,
                       static_cast<const bf16*>(K), static_cast<const bf16*>(V), static_cast<const bf16*>(Ks),
                       static_cast<const bf16*>(Vs), L, n_chunks, ring_tiles, lens, r);
    return hipGetLastError();
}

template <int D>
hipError_t launch_qcache_read(const QCacheView& c, const CacheView& to, const int* n_tok, int max_tok,
                              const RaggedState& r, hipStream_t stream) {
    const int most = min(max_tok, r.max_tok);
    const int ring_tiles = (min(most, min(c.R, to.R)) + kQReadRows - 1) / kQReadRows + 1;
    const int sum_tiles = (min(most / c.C, min(c.S_max, to.S_max)) + kQReadRows - 1) / kQReadRows;
    hipLaunchKernelGGL((qcache_read_kernel<D>), dim3(ring_tiles + sum_tiles, c.B * c.Hkv), dim3(256), 0, stream, c, to,
                       n_tok, max_tok, r, ring_tiles);
    return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_append_path(const CacheView& c, const PathParams& a, hipStream_t stream) {
    const size_t lds = (size_t)(c.C + summary_red_floats<D>()) * sizeof(float);
    hipLaunchKernelGGL((append_path_kernel<D, T, PlainStore<D, T>, CacheView>), dim3(c.B * c.Hkv), dim3(kSummaryThreads), lds,
                       stream, c, a);
    return hipGetLastError();
}
template <int D>
hipError_t launch_qappend_path(const QCacheView& c, const PathParams& a, hipStream_t stream) {
    constexpr int red = summary_red_floats<D>() > 2 * kSummaryThreads ? summary_red_floats<D>() : 2 * kSummaryThreads;
    const size_t lds = (size_t)(c.C + red) * sizeof(float);
    hipLaunchKernelGGL((append_path_kernel<D, bf16, QuantStore<D>, QCacheView>), dim3(c.B * c.Hkv), dim3(kSummaryThreads), lds,
                       stream, c, a);
    return hipGetLastError();
}

#define EVA_QCACHE(D)                                                                                                   \
    template hipError_t launch_qcache_fill<D>(const QCacheView&, const void*, const void*, const void*, const void*, int, \
                                              const int*, const RaggedState&, hipStream_t);                              \
    template hipError_t launch_qcache_read<D>(const QCacheView&, const CacheView&, const int*, int, const RaggedState&,  \
                                              hipStream_t);                                                              \
    template hipError_t launch_append_path<D, bf16>(const CacheView&, const PathParams&, hipStream_t);                   \
    template hipError_t launch_append_path<D, float>(const CacheView&, const PathParams&, hipStream_t);                  \
    template hipError_t launch_qappend_path<D>(const QCacheView&, const PathParams&, hipStream_t);
EVA_QCACHE(64)
EVA_QCACHE(128)
#undef EVA_QCACHE

}  // namespace eva
