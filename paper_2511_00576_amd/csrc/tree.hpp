// What the kernels of drafted trees share: the nodes' lines, the rows' geometry
// and the sums that infinite and NaN values need.
#pragma once

#include "qrows.hpp"

namespace eva {

constexpr float kTreeTau = 8.f;  // log2 units: unscaled weights stay <= 256
constexpr int kMaxNodes = 64;

// Lines of the tree's nodes: lane t holds the set of node t's forerunners and
// itself.  parent: lane t's entry of the parents; they name an earlier node, any
// other value makes a root.  Each round doubles the reach, until every line has
// its root: `deepest` is a bound on the nodes' depths, below twice the largest.
__device__ __forceinline__ unsigned long long tree_lines(int parent, int nodes, int& deepest) {
    const int lane = threadIdx.x & 63;
    int up = lane < nodes && parent >= 0 && parent < lane ? parent : -1;
    unsigned long long line = 1ull << lane;
    int reach = 1;
#pragma unroll 1
    while (__builtin_amdgcn_ballot_w64(up >= 0)) {  // six rounds at most: up < lane
        const int from = max(up, 0);
        const unsigned long long l = __shfl(line, from, 64);
        const int u = __shfl(up, from, 64);
        if (up >= 0) {
            line |= l;
            up = u;
        }
        reach *= 2;
    }
    deepest = min(reach, nodes) - 1;
    return line;
}

// A sequence's rows: the first ring position and the visible summaries of the
// shallowest and of the deepest node there may be, and of single nodes.  A plain decode
// (drafted false) is one node at the last position.
struct TreeRows {
    int n, nodes;              // tokens held, nodes there are
    int p0;                    // position of a root
    unsigned long long lines;  // lane t: node t's line
    int lo_first, lo_last, sum_first, sum_last;
    bool any;                  // there is a row to compute
    __device__ __forceinline__ TreeRows(const TreeParams& a, int b, bool drafted) {
        // (all of the sequence's words requested at once)
        const int lane = threadIdx.x & 63;
        const int parent = drafted ? a.parents[(size_t)b * a.T + min(lane, a.T - 1)] : 0;
        n = min(max(a.n_tok[b], 0), a.max_tok);
        nodes = !drafted ? 1 : a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
        any = !(a.active && a.active[b] == 0) && (drafted ? nodes : n) > 0;
        p0 = drafted ? n : n - 1;
        lines = 0;
        lo_first = lo_last = sum_first = sum_last = 0;
        if (!any) return;
        int deepest = 0;
        if (drafted) {
            lines = tree_lines(parent, nodes, deepest);
        }
        lo_first = win_lo_rt(a.c.window, p0, a.c.W, a.c.C);
        lo_last = win_lo_rt(a.c.window, p0 + deepest, a.c.W, a.c.C);
        sum_first = min(lo_first / a.c.C, a.c.S_max);
        sum_last = min(lo_last / a.c.C, a.c.S_max);
    }
    // Node t: its line (no node: nothing), first ring position and summaries.
    __device__ __forceinline__ void node(const TreeParams& a, int t, unsigned long long& line, int& lo, int& n_sum) const {
        line = __shfl(lines, t, 64);
        lo = win_lo_rt(a.c.window, p0 + max(__builtin_popcountll(line) - 1, 0), a.c.W, a.c.C);
        n_sum = min(lo / a.c.C, a.c.S_max);
        if (t >= nodes) line = 0;
    }
};

// Unit (b, kv head) and column block of a workgroup.  Workgroups of a unit are 8
// apart, so that one XCD's L2 has its rows.
struct TreePlace {
    int unit, cb;
    __device__ __forceinline__ TreePlace(const TreeParams& a) {
        const int id = blockIdx.x;
        const int group = id / a.f8cb, r = id - group * a.f8cb.d;
        unit = group * 8 + (r & 7);
        cb = r >> 3;
    }
};

// Whether a fragment holds an infinity or NaN.
__device__ __forceinline__ bool not_finite(const bf16x8& v) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}

// The finite values of a fragment, zeros in the place of others.
__device__ __forceinline__ bf16x8 finite_values(const bf16x8& v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] &= ((w[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
    return __builtin_bit_cast(bf16x8, w);
}

// What the infinite and NaN values of a fragment, which are rare, make of the N
// outputs of a lane: two bits each, 1: some column weight meets +inf (or NaN), 2:
// -inf (or NaN).  They are kept apart from the accumulators, whose sums take the
// finite values alone: a weight of 0 times an infinity would be NaN, and adding
// them in the loop of the products would cost it twice its accumulators'
// registers.
template <int N>
__device__ __forceinline__ uint32_t not_finite_outputs(const bf16x8& v, const bf16x8& p) {
    constexpr int COLS = N == 16 ? 32 : 16;  // columns, and features, of the product
    const u32x4 w = __builtin_bit_cast(u32x4, v), pw = __builtin_bit_cast(u32x4, p);
    const int lane = lane_here(), col = lane % COLS, g = lane / COLS;
    uint32_t bits = 0;
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {
        // this lane's key e: its value and its column's weight
        const uint32_t vw = (e >> 1) == 0 ? w[0] : (e >> 1) == 1 ? w[1] : (e >> 1) == 2 ? w[2] : w[3];
        const uint32_t qw = (e >> 1) == 0 ? pw[0] : (e >> 1) == 1 ? pw[1] : (e >> 1) == 2 ? pw[2] : pw[3];
        const float ve = (e & 1) ? bf16_hi(vw) : bf16_lo(vw), pe = (e & 1) ? bf16_hi(qw) : bf16_lo(qw);
#pragma unroll 1
        for (int from = 0; from < 64; from += COLS) {
            const float pk = __shfl(pe, from + col, 64);
#pragma unroll 1
            for (int i = 0; i < N; ++i) {
                const float x = __shfl(ve, from + (N == 16 ? 8 * (i >> 2) + 4 * g + (i & 3) : 4 * g + i), 64);
                const uint32_t kind = x != x ? 3 : x == INFINITY ? 1 : x == -INFINITY ? 2 : 0;
                if (pk != 0.f) bits |= kind << (2 * i);
            }
        }
    }
    return bits;
}
// The same of one step of four fp32 keys (16x16x4): v is the lane's feature of its
// group's key, p its column's weight on it.
__device__ __forceinline__ uint32_t not_finite_outputs_f32(float v, float p) {
    const int lane = lane_here(), col = lane % 16, g = lane / 16;
    uint32_t bits = 0;
#pragma unroll 1
    for (int from = 0; from < 64; from += 16) {
        const float pk = __shfl(p, from + col, 64);
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            const float x = __shfl(v, from + 4 * g + i, 64);
            const uint32_t kind = x != x ? 3 : x == INFINITY ? 1 : x == -INFINITY ? 2 : 0;
            if (pk != 0.f) bits |= kind << (2 * i);
        }
    }
    return bits;
}
__device__ __forceinline__ float with_not_finite(float o, uint32_t kind) {
    return kind == 0 ? o : kind == 1 ? o + INFINITY : kind == 2 ? o - INFINITY : NAN;
}

// O^T += V^T P^T of one product.  edge: some columns may not see keys that others
// see, or slots may be stale (their weights are 0, whatever bits they hold).
// bits <<: what infinite and NaN values make of the outputs.
template <typename Acc, typename Mfma>
__device__ __forceinline__ void add_values(const bf16x8& v, const bf16x8& p, Acc& o, bool edge, uint32_t& bits, int shift,
                                           Mfma&& mfma) {
    bf16x8 x = v;
    if (edge && __builtin_amdgcn_ballot_w64(not_finite(v))) {
        x = finite_values(v);
        bits |= not_finite_outputs<sizeof(Acc) / 4>(v, p) << shift;
    }
    o = mfma(x, p, o);
}

}  // namespace eva
