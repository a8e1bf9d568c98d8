// Norms of queries and keys per head with the position rotation, and the split
// of the projection's output into head-major Q, K and V, in one pass; and its
// backward.  For a token's head row x (d features) at position p:
//
//   n = x g / sqrt(mean(x^2) + eps)            (rows without a weight: n = x)
//   y = n with pair i < rot / 2 turned by p turns_i:
//       (a cos - b sin, a sin + b cos)
//
//   dn = the turn back of dy;  dg = sum over rows of dn x^;  x^ = x rstd
//   dx = rstd (dn g - x^ mean(dn g x^))
//
// Both are bound by memory: every element is read once and written once (the
// backward reads x and the gradients), about ten operations each.  On MI355X,
// bf16, H32/8 d128: 32768 tokens in 152 us, 5.3 TB/s; 16384 tokens forward and
// backward 72 + 121 + 4.7 us, 5.1 TB/s (a copy of 1 GB runs at 5.1).
//
// A row is held by D / 16 lanes of 16 features, in pieces of 16 bytes that hold
// both members of the lane's eight pairs, so a turn stays in the lane;
// a wave works on 1024 / D rows of one token at a time and computes the
// token's angles once for all its heads.  Where the heads of every kind would leave
// half of the lanes idle or more, a wave holds several tokens.  Angles are whole numbers: p times
// the frequency in 2^-64 turns, modulo 2^64, is exact to 2^-64 p turns at any
// position, where a product in fp32 is off by radians from 2^24 on.
#include "eva_device.hpp"
#include "eva_kernels.hpp"

namespace eva {

namespace {

constexpr int kNormRopeWaves = 4;

// A lane's 16 features of a row as they lie in memory, in 16-byte pieces.
template <typename T>
struct RawRow {
    static constexpr int N = (int)sizeof(T);
    u32x4 w[N];
    template <typename Row>
    __device__ __forceinline__ void load(const T* row, const Row& r) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const u32x4*>(row + r.piece(i));
    }
    __device__ __forceinline__ void values(float (&x)[16]) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (sizeof(T) == 2)
                x[i] = (i & 1) ? bf16_hi(w[i / 8][i % 8 / 2]) : bf16_lo(w[i / 8][i % 8 / 2]);
            else
                x[i] = __uint_as_float(w[i / 4][i % 4]);
        }
    }
};
__device__ __forceinline__ void store_piece(bf16* p, const float* x) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                         pack_bf16x2(x[6], x[7])};
}
__device__ __forceinline__ void store_piece(float* p, const float* x) {
    *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]};
}

// Where a lane's pieces lie and how its pairs are formed.  fp32 pieces lie side by
// side across the lanes that are turned, and across the others, so that an
// instruction reads whole lines: 8192 tokens of H32/8 d128 90 us, with a lane's 16
// features side by side 117 (forward and backward 215 / 252; H16/2 d64 191 / 187).
// (bf16 with adjacent pairs, and what is not turned, two pieces side by side in a
// lane: half of a line each.)
// ADJ: pairs are adjacent features.  PACK: a wave holds 1 << a.pack tokens, each
// with all its heads of a kind in one sweep; else one token.
template <int D, typename T, bool ADJ, bool PACK>
struct LaneRow {
    static constexpr int kLanes = D / 16;           // lanes per row
    static constexpr int kRows = 64 / kLanes;       // rows per wave
    int c, sub;                                     // place in the row, row in the wave
    int h, t;                                       // its head in a sweep, its token in the wave
    int f0, f1;                                     // bf16: first feature of the pieces; fp32: and their distance
    bool turned;                                    // its pairs are turned
    __device__ LaneRow(const NormRopeParams& a) {
        const int lane = threadIdx.x & 63;
        c = lane % kLanes;
        sub = lane / kLanes;
        h = sub;
        t = 0;
        if constexpr (PACK) {
            h = sub & ((kRows >> a.pack) - 1);
            t = sub / (kRows >> a.pack);
        }
        turned = 16 * c < a.rot;
        // halves: pair i is (i, i + rot / 2), whose members lie in pieces half of the
        // lane's pieces apart
        if constexpr (sizeof(T) == 2) {
            const bool halves = turned && !ADJ;
            f0 = 8 * (halves ? c : 2 * c);
            f1 = 8 * (halves ? c + a.rot / 16 : 2 * c + 1);
        } else {
            f0 = turned ? 4 * c : a.rot + 4 * (c - a.rot / 16);
            f1 = 4 * (turned ? a.rot / 16 : kLanes - a.rot / 16);
        }
    }
    // First feature of piece i.
    __device__ __forceinline__ int piece(int i) const {
        if constexpr (sizeof(T) == 2) return i ? f1 : f0;
        return f0 + i * f1;
    }
    // The lane's element i is this feature; its pair j has this frequency.
    __device__ __forceinline__ int feature(int i) const { return piece(i / (16 / (int)sizeof(T))) + i % (16 / (int)sizeof(T)); }
    __device__ __forceinline__ int frequency(int j) const {
        if constexpr (sizeof(T) == 2) return 8 * c + j;
        return ADJ ? (f0 + (j >> 1) * f1) / 2 + (j & 1) : f0 + (j >> 2) * f1 + (j & 3);
    }
    __device__ float sum(float x) const {
#pragma unroll
        for (int off = 1; off < kLanes; off <<= 1) x += __shfl_xor(x, off, 64);
        return x;
    }
    __device__ void load(const T* row, float (&x)[16]) const {
        RawRow<T> w;
        w.load(row, *this);
        w.values(x);
    }
    __device__ void store(T* row, const float (&x)[16]) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) store_piece(row + piece(i), x + i * (16 / (int)sizeof(T)));
    }
    // SIGN 1: by the angles, -1: back
    template <int SIGN>
    __device__ void turn(float (&y)[16], const float (&cs)[8], const float (&sn)[8]) const {
        if (!turned) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float &lo = y[ADJ ? 2 * j : j], &hi = y[ADJ ? 2 * j + 1 : 8 + j];
            const float p = lo, q = hi, t = SIGN * sn[j];
            lo = p * cs[j] - q * t;
            hi = p * t + q * cs[j];
        }
    }
};

// cos and sin of t 2^-64 turns.  The nearest quarter turn is taken off the whole
// number, exactly; what is left, at most pi / 4, goes into the Taylor series to
// x^9 and x^10, whose next terms are below 2^-29 and 2^-33.  Beside the series'
// own roundings x is off by the turns below 2^-32 (2 pi 2^-32 = 0.03 of 2^-24), the
// rounding of a whole number of 30 bits and that of the product, 2^-24 of pi / 4 each: sine
// and cosine within 4 x 2^-24.
__device__ __forceinline__ void cos_sin(unsigned long long t, float& c, float& s) {
    const uint32_t hi = (uint32_t)(t >> 32);
    const uint32_t quarter = (hi + 0x20000000u) >> 30;
    const float x = (float)(int)(hi - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi 2^-32
    const float z = x * x;
    const float sn = fmaf(fmaf(fmaf(fmaf(2.7557319e-6f, z, -1.9841270e-4f), z, 8.3333333e-3f), z, -1.6666667e-1f) * z, x, x);
    const float cs = fmaf(fmaf(fmaf(fmaf(fmaf(-2.7557319e-7f, z, 2.4801587e-5f), z, -1.3888889e-3f), z, 4.1666667e-2f), z, -0.5f), z, 1.f);
    const float u = (quarter & 1) ? sn : cs, v = (quarter & 1) ? cs : sn;
    c = ((quarter + 1) & 2) ? -u : u;
    s = (quarter & 2) ? -v : v;
}

// cos and sin of the lane's eight pairs at a token's position.
template <typename Row>
__device__ __forceinline__ void angles(const NormRopeParams& a, const Row& r, int tok, float (&cs)[8], float (&sn)[8]) {
    if (!r.turned) return;
    const int b = tok / a.fL, l = tok - b * a.fL.d;
    const long long pos = (long long)(a.start ? a.start[b] : 0) + (a.offsets ? a.offsets[tok] : l);
#pragma unroll
    for (int j = 0; j < 8; ++j) cos_sin((unsigned long long)pos * a.turns[r.frequency(j)], cs[j], sn[j]);
}

// Sweeps of a token: kRows heads each, queries first, then keys, then values.
struct Sweeps {
    int q, k, all;
    __device__ Sweeps(const NormRopeParams& a, int rows) {
        q = (a.H + rows - 1) / rows;
        const int kv = (a.Hkv + rows - 1) / rows;
        k = q + kv;
        all = k + kv;
    }
};

// One wave per token (and part of its heads where there are few tokens), or per
// 1 << a.pack tokens.
template <int D, typename T, bool ADJ, bool PACK>
__global__ __launch_bounds__(kNormRopeWaves * 64) void norm_rope_kernel(NormRopeParams a) {
    const LaneRow<D, T, ADJ, PACK> r(a);
    int tok = blockIdx.x * kNormRopeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (PACK) tok = (tok << a.pack) + r.t;
    if (tok >= a.tokens) return;  // (all lanes of a row together)
    const int b = tok / a.fL, l = tok - b * a.fL.d;
    const Sweeps sw(a, r.kRows);
    const T* xt = static_cast<const T*>(a.x) + b * a.stride_b + l * a.stride_l;
    // sweep s: its heads are `heads` from the row's `first` on, this lane's is h
    struct Sweep {
        int kind, first, heads, h;  // kind 0 queries, 1 keys, 2 values
    };
    auto sweep = [&](int s) {
        const int kind = s < sw.q ? 0 : s < sw.k ? 1 : 2;
        return Sweep{kind, kind == 0 ? 0 : kind == 1 ? a.H : a.H + a.Hkv, kind == 0 ? a.H : a.Hkv,
                     (s - (kind == 0 ? 0 : kind == 1 ? sw.q : sw.k)) * r.kRows + r.h};
    };
    RawRow<T> raw;
    auto request = [&](const Sweep& w) { raw.load(xt + (size_t)(w.first + min(w.h, w.heads - 1)) * D, r); };
    // rows are requested a sweep ahead, the first before the angles
    Sweep w = sweep(blockIdx.y);
    request(w);
    float cs[8], sn[8];
    angles(a, r, tok, cs, sn);
    for (int s = blockIdx.y; s < sw.all; s += gridDim.y) {
        float y[16];
        raw.values(y);
        const Sweep now = w;
        if (s + (int)gridDim.y < sw.all) {
            w = sweep(s + gridDim.y);
            request(w);
        }
        T* out = static_cast<T*>(now.kind == 0 ? a.Q : now.kind == 1 ? a.K : a.V);
        if (now.kind < 2) {
            const T* g = static_cast<const T*>(now.kind ? a.gk : a.gq);
            if (g) {
                float wt[16], ss = 0.f;
                r.load(g, wt);
#pragma unroll
                for (int i = 0; i < 16; ++i) ss += y[i] * y[i];
                const float inv = rsqrtf(r.sum(ss) * (1.f / D) + a.eps);
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = y[i] * inv * wt[i];
            }
            r.template turn<1>(y, cs, sn);
        }
        if (now.h < now.heads) r.store(out + (((size_t)b * now.heads + now.h) * a.fL.d + l) * D, y);
    }
}

// Tokens are dealt round to the waves; each wave's share of the weights'
// gradients stays in registers, its workgroup's sum goes to its own place of
// the workspace, and a second launch adds those up in their order: the same
// bits every time.
template <int D, typename T, bool ADJ, bool PACK>
__global__ __launch_bounds__(kNormRopeWaves * 64, 3) void norm_rope_bwd_kernel(NormRopeParams a) {
    const LaneRow<D, T, ADJ, PACK> r(a);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Sweeps sw(a, r.kRows);
    float dg[2][16] = {};
    const int pack = PACK ? a.pack : 0;
    for (int tok = ((blockIdx.x * kNormRopeWaves + wave) << pack) + r.t; tok < a.tokens; tok += gridDim.x * kNormRopeWaves << pack) {
        const int b = tok / a.fL, l = tok - b * a.fL.d;
        const T* xt = static_cast<const T*>(a.x) + b * a.stride_b + l * a.stride_l;
        T* dxt = static_cast<T*>(a.dx) + (size_t)tok * (a.H + 2 * a.Hkv) * D;
        float cs[8], sn[8];
        angles(a, r, tok, cs, sn);
        auto rows = [&](int s, int heads, int head0, const void* grad, const void* weight, float (&acc)[16]) {
            const int h = s * r.kRows + r.h;
            const bool on = h < heads;
            const size_t row = (size_t)(head0 + min(h, heads - 1)) * D;
            float dy[16];
            r.load(static_cast<const T*>(grad) + (((size_t)b * heads + min(h, heads - 1)) * a.fL.d + l) * D, dy);
            r.template turn<-1>(dy, cs, sn);
            if (weight) {
                float x[16], w[16], ss = 0.f;
                r.load(xt + row, x);
                r.load(static_cast<const T*>(weight), w);
#pragma unroll
                for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
                const float inv = rsqrtf(r.sum(ss) * (1.f / D) + a.eps);
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[i] *= inv;
                    const float t = dy[i] * x[i];
                    acc[i] += on ? t : 0.f;
                    dot += t * w[i];
                }
                dot = r.sum(dot) * (1.f / D);
#pragma unroll
                for (int i = 0; i < 16; ++i) dy[i] = inv * (dy[i] * w[i] - x[i] * dot);
            }
            if (on) r.store(dxt + row, dy);
        };
        for (int s = 0; s < sw.q; ++s) rows(s, a.H, 0, a.dQ, a.gq, dg[0]);
        for (int s = sw.q; s < sw.k; ++s) rows(s - sw.q, a.Hkv, a.H, a.dK, a.gk, dg[1]);
        for (int s = sw.k; s < sw.all; ++s) {
            const int h = (s - sw.k) * r.kRows + r.h;
            if (h >= a.Hkv) continue;
            float y[16];
            r.load(static_cast<const T*>(a.dV) + (((size_t)b * a.Hkv + h) * a.fL.d + l) * D, y);
            r.store(dxt + (size_t)(a.H + a.Hkv + h) * D, y);
        }
    }
    if (!a.gq && !a.gk) return;
    __shared__ float part[kNormRopeWaves][2][D];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float x = dg[n][i];
#pragma unroll
            for (int off = r.kLanes; off < 64; off <<= 1) x += __shfl_xor(x, off, 64);
            if (r.sub == 0) part[wave][n][r.feature(i)] = x;
        }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * D; e += blockDim.x) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kNormRopeWaves; ++w) x += part[w][e / D][e % D];
        a.ws[(size_t)blockIdx.x * 2 * D + e] = x;
    }
}

// Sums the n workgroups' shares of 8 features: 128 threads a feature, each with
// its loads of eight shares in flight together, then their sums in a fixed
// order.  (16 threads a feature, one load after the other, took 20 us for 1024
// shares.)
constexpr int kSumFeatures = 8;
template <int D>
__global__ __launch_bounds__(1024) void norm_rope_sum_kernel(const float* __restrict__ ws, int n, float* dgq, float* dgk) {
    constexpr int R = 1024 / kSumFeatures;
    __shared__ float part[R][kSumFeatures + 1];
    const int f = threadIdx.x % kSumFeatures, r = threadIdx.x / kSumFeatures;
    const int e = blockIdx.x * kSumFeatures + f;
    float x = 0.f;
    for (int i0 = r; i0 < n; i0 += 8 * R) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = i0 + i * R < n ? ws[(size_t)(i0 + i * R) * 2 * D + e] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x += y[i];
    }
    part[r][f] = x;
    __syncthreads();
    for (int half = R / 2; half > 0; half /= 2) {
        if (r < half) part[r][f] += part[r + half][f];
        __syncthreads();
    }
    float* out = e < D ? dgq : dgk;
    if (r == 0 && out) out[e % D] = part[0][f];
}

}  // namespace

// log2 of the tokens a wave holds: as many as fit with all their heads of the kind
// that has more (a sweep of a packed wave holds all of a kind).
// (us a launch on MI355X, several tokens a wave / one: bf16 d64 H1 B28 L1300 8.6 /
// 36.5 and backward 14.7 / 44.8, d128 H4/1 B16 L1300 17.1 / 23.8 and 28 / 44, fp32
// d64 H8/2 B16 L1300 32.0 / 36.5 and 42.7 / 67.)
template <int D>
int tokens_log2(int H, int Hkv) {
    const int heads = H > Hkv ? H : Hkv;
    int n = 0;
    while (heads << (n + 1) <= 1024 / D) ++n;
    return n;
}

template <int D, typename T>
hipError_t launch_norm_rope(NormRopeParams p, hipStream_t stream) {
    constexpr int rows = 1024 / D;
    p.pack = tokens_log2<D>(p.H, p.Hkv);
    const int sweeps = (p.H + rows - 1) / rows + 2 * ((p.Hkv + rows - 1) / rows);
    const int per = kNormRopeWaves << p.pack, wgs = (p.tokens + per - 1) / per;
    // few tokens: their heads over workgroups, until there are four waves a CU
    int split = (256 + wgs - 1) / wgs;
    if (split > sweeps) split = sweeps;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(wgs, split), dim3(kNormRopeWaves * 64), 0, stream, p); };
    if (p.interleaved)
        p.pack ? go(norm_rope_kernel<D, T, true, true>) : go(norm_rope_kernel<D, T, true, false>);
    else
        p.pack ? go(norm_rope_kernel<D, T, false, true>) : go(norm_rope_kernel<D, T, false, false>);
    return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_norm_rope_backward(NormRopeParams p, hipStream_t stream) {
    p.pack = tokens_log2<D>(p.H, p.Hkv);
    const int wgs = norm_rope_bwd_wgs((p.tokens + (1 << p.pack) - 1) >> p.pack);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(wgs), dim3(kNormRopeWaves * 64), 0, stream, p); };
    if (p.interleaved)
        p.pack ? go(norm_rope_bwd_kernel<D, T, true, true>) : go(norm_rope_bwd_kernel<D, T, true, false>);
    else
        p.pack ? go(norm_rope_bwd_kernel<D, T, false, true>) : go(norm_rope_bwd_kernel<D, T, false, false>);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!p.gq && !p.gk)) return e;
    hipLaunchKernelGGL((norm_rope_sum_kernel<D>), dim3(2 * D / kSumFeatures), dim3(1024), 0, stream, p.ws, wgs, p.dgq, p.dgk);
    return hipGetLastError();
}

#define EVA_NORM_ROPE(D, T)                                                             \
    template hipError_t launch_norm_rope<D, T>(NormRopeParams, hipStream_t);            \
    template hipError_t launch_norm_rope_backward<D, T>(NormRopeParams, hipStream_t);
EVA_NORM_ROPE(64, bf16)
EVA_NORM_ROPE(128, bf16)
EVA_NORM_ROPE(64, float)
EVA_NORM_ROPE(128, float)
#undef EVA_NORM_ROPE

}  // namespace eva
