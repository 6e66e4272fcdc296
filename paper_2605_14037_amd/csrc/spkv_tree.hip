// Attention of trees of drafted tokens over the cache on gfx950.
#include <type_traits>

#include "spkv_lists.h"

// The mathematics.  Draft i of a sequence that holds T tokens hangs behind draft parent(i) < i or behind the newest
// token; the drafts from there to it are its path, and with d(i) drafts before it on the path it stands at position
// T + d(i).  It sees a cached key at position s if T + d(i) - s < w or that key's gate is on, and draft a if a is on its
// path and d(i) - d(a) < w or a's gate is on (Eq. 3-5 for the tokens of the path alone).  All drafts of a sequence
// and all heads of a group are columns of one product with the list, as the rows of sequences that share a prompt are
// (spkv_lists.h), with d(i) for the place behind the list's newest token; the drafts themselves, at most 64
// keys, are one unit of work more, whose mask is a word of 64 bits a draft.  Lists of a few half-pages, or lists enough to fill
// the chip, are taken whole: one workgroup a list, the drafts with it, its results final (32 sequences of 300 tokens, 16 drafts, 25 -> 19
// us, 64 drafts 53 -> 29; 64 of 1k-16k, 64 drafts, 201 -> 155).
//
// A lane of a wave stands for a draft: paths are words of bits, joined along the parents by doubling (log2 of the deepest
// path's length rounds of three lane exchanges), depths their counts of bits.
//
// Bound: the lists are read once, 4 D bytes a key for 4 D flops a key and column: past about 180 columns a list the matrix
// units, below the read; few columns or short lists by the start of a workgroup and the join.  Measured, 16 sequences of 32k tokens
// (484 MB, 32 heads over 8 of 128), a call: 4 drafts 83 us (5.8 TB/s), 8: 91, 16: 98, 32: 119, 64: 165 (2.9 TB/s, 0.75 PF/s); one
// sequence of 128k, 16 drafts 34; of 2k, 14.

// ------------------------------------------------------------------------------- paths
struct TreePath {
    unsigned long long path;     // of lane's draft: itself and what it hangs behind
    int up, depth;
};
// Any value but 0 .. i - 1 for a parent means that the draft hangs behind the newest token.
__device__ __forceinline__ int tree_parent(const int32_t* __restrict__ parents, int n) {      // of lane's draft
    const int lane = threadIdx.x & 63;
    return lane < n ? parents[lane] : -1;
}
__device__ __forceinline__ TreePath tree_path(int p) {
    const int lane = threadIdx.x & 63;
    TreePath t;
    t.up = p >= 0 && p < lane ? p : -1;
    t.path = 1ull << lane;
    int up = t.up;
    while (__ballot(up >= 0) != 0ull) {                       // at most six rounds
        const int at = max(up, 0);
        const unsigned long long more = lane_word(t.path, at);
        const int next = __shfl(up, at);
        if (up >= 0) {
            t.path |= more;
            up = next;
        }
    }
    t.depth = __popcll(t.path) - 1;
    return t;
}
// The drafts that lane's draft sees: its path within the window, and past it where the gate is on.
__device__ __forceinline__ unsigned long long tree_seen(const SpkvView& v, const TreePath& t, const float* __restrict__ f, int h,
                                                        int row0, int n, int T) {
    const int lane = threadIdx.x & 63;
    if (__ballot(lane < n && t.depth >= v.w) == 0ull) return t.path;
    // the draft w places up, by the bits of w
    int at = lane, jump = t.up;
    for (int k = 0; k < 6; ++k) {
        const int step = __shfl(jump, max(at, 0)), twice = __shfl(jump, max(jump, 0));
        if (at >= 0 && ((v.w >> k) & 1)) at = step;
        jump = jump >= 0 ? twice : -1;
    }
    const unsigned long long far = lane_word(t.path, max(at, 0));
    const bool on = lane < n && f != nullptr && gate_passes(v, f[(size_t)(row0 + lane) * v.Hkv + h], T + t.depth);
    const unsigned long long gates = __ballot(on);
    return at >= 0 ? t.path & (~far | gates) : t.path;
}

// Sums of one column over the drafts that it sees, key by key, where an infinity or NaN among the values of a draft that it
// does not see has reached it (a weight of zero times it).  The whole wave.
template <int D>
__device__ __attribute__((noinline)) void careful_tree_sums(const uint16_t* k, const uint16_t* vv, int stride, const uint16_t* qrow,
                                                            unsigned long long seen, float scale_log2e, float m, bool add, float* sums) {
    const int lane = threadIdx.x & 63;
    float q[D / 64], acc[D / 64];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
        q[e] = bf16_at(qrow + e * 64 + lane);
        acc[e] = 0.f;
    }
    for (; seen != 0ull; seen &= seen - 1) {
        const size_t at = (size_t)__builtin_ctzll(seen) * stride;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) x += q[e] * bf16_at(k + at + e * 64 + lane);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale_log2e, -m));
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] += p * bf16_at(vv + at + e * 64 + lane);
    }
#pragma unroll
    for (int e = 0; e < D / 64; ++e) sums[e * 64 + lane] = acc[e] + (add ? sums[e * 64 + lane] : 0.f);
}
// Is there a value that is not finite, in a draft that others need not see?  (The whole wave.)
template <int D>
__device__ __attribute__((noinline)) bool careful_tree_needed(const uint16_t* vv, int stride, int n) {
    bool odd = false;
    for (int i = 0; n > 1 && i < n; ++i)
        for (int d = threadIdx.x & 63; d < D; d += 64) {
            const float x = bf16_at(vv + (size_t)i * stride + d);
            odd = odd || !(x - x == 0.f);
        }
    return __ballot(odd) != 0ull;
}

__device__ __forceinline__ void store_result(uint16_t* to, f32x4 x) {
    uint2 packed;
    packed.x = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[0]) | ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[1]) << 16);
    packed.y = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[2]) | ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[3]) << 16);
    *reinterpret_cast<uint2*>(to) = packed;
}
__device__ __forceinline__ float log_of_sum(float m, float l) { return l == 0.f ? SPKV_NEG_INF : (m + log2f(l)) * 0.6931471805599453f; }

// ---------------------------------------------------------------------------- the work
// Workgroup id -> unit: the ranges of the lists, by the host's table, the ranges of a pair's block of columns next to each
// other.  W: every list is one range, whose unit writes the results, and there is no join.  With: the drafts go with a list's first range,
// where they count for `weight` half-pages (of a short list it has little else); without, they are units of their own, behind the lists'.
template <bool W, bool With>
struct TreeWork {
    static constexpr bool kTree = With, kPaths = true, kWhole = W;
    const SpkvTree& tree;
    const SpkvTreeTable& table;
    int pair, h, range, ranges, block, n, row0, unit, width, weight;
    __device__ __forceinline__ TreeWork(const SpkvView& v, const SpkvTree& t, const SpkvTreeTable& tab, int id, SpkvTreeKernel kernel)
        : tree(t), table(tab), width(spkv_tree_width(kernel)) {
        int local = 0;
        if (!With && id >= t.n_units) {
            local = id - t.n_units;
            ranges = 1;
            block = 0;
            range = -1;
        } else {
            const uint4 raw = reinterpret_cast<const uint4*>(tab.end)[threadIdx.x & 63];      // eight pairs a lane
            const unsigned e[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                local += __popcll(__ballot((int)(e[i] & 0xffffu) <= id));
                local += __popcll(__ballot((int)(e[i] >> 16) <= id));
            }
            const int start = local > 0 ? tab.end[local - 1] : 0;
            ranges = tab.ranges[local];
            block = (id - start) / ranges;
            range = id - start - block * ranges;
        }
        unit = id;
        pair = t.pair0 + tab.pair[local];
        const int b = pair / v.Hkv, at = b - t.seq0;
        h = pair - b * v.Hkv;
        row0 = t.row0 + tab.cu[at];
        n = tab.cu[at + 1] - tab.cu[at];
        weight = spkv_tree_draft_weight(kernel, n);
    }
    __device__ __forceinline__ bool drafts() const { return With && (W || range == 0); }
    __device__ __forceinline__ int draft_weight() const { return weight; }
    __device__ __forceinline__ int begin(const ShareList& list, int j) const {
        if (!With) return list.begin(j, ranges);
        const int x = (int)((int64_t)j * (2 * list.n_hp - list.nA + weight) / ranges) - weight;
        return x <= 0 ? 0 : x <= list.nA ? x : list.nA + (x - list.nA + 1) / 2;
    }
    __device__ __forceinline__ int columns(const SpkvView& v) const { return n * v.G; }
    __device__ __forceinline__ ShareRow row(const SpkvView& v, int c, bool ring) const {
        ShareRow r;
        const int i = c / v.G;
        r.head = c - i * v.G;
        r.row = row0 + i;
        r.place = ring ? place(v, c, tree_path(parent())) : 0;
        return r;
    }
    __device__ __forceinline__ int parent() const { return tree_parent(tree.parents + row0, n); }
    __device__ __forceinline__ TreePath path(int p) const { return tree_path(p); }
    __device__ __forceinline__ int place(const SpkvView& v, int c, const TreePath& path) const { return __shfl(path.depth, c / v.G); }
    __device__ __forceinline__ float* part(const SpkvView& v) const { return v.part_acc; }
    template <int D>
    __device__ __forceinline__ float2* part_ml(const SpkvView& v) const { return reinterpret_cast<float2*>(v.part_ml); }
    __device__ __forceinline__ size_t part0(const SpkvView&) const { return (size_t)(unit - block) * width; }

    // ---- the drafts
    __device__ __forceinline__ int stride(const SpkvView& v) const { return v.Hkv * v.D; }
    __device__ __forceinline__ const uint16_t* keys(const SpkvView& v) const { return tree.k + ((size_t)row0 * v.Hkv + h) * v.D; }
    __device__ __forceinline__ const uint16_t* values(const SpkvView& v) const { return tree.v + ((size_t)row0 * v.Hkv + h) * v.D; }
    __device__ __forceinline__ unsigned long long seen(const SpkvView& v, int T) const { return seen(v, T, tree_path(parent())); }
    __device__ __forceinline__ unsigned long long seen(const SpkvView& v, int T, const TreePath& path) const {
        return tree_seen(v, path, tree.f, h, row0, n, T);
    }
    // Operands of attend_list_few, N groups of 16 of the values' elements from group first on.  Keys straight from their rows;
    // values, of which an operand wants eight keys of one element, by 2-byte loads.
    template <int D, int N>
    __device__ __forceinline__ void load_few(const SpkvView& v, bf16x8 (&k)[2][D / 32], bf16x8 (&va)[N], int first = 0) const {
        const int lane = threadIdx.x & 63, kc = lane >> 4, col = lane & 15, step = v.Hkv * D;
        const uint16_t *kr = keys(v), *vr = values(v);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int sl = 0; sl < D / 32; ++sl) {            // (rows that are not there: the last one's; no column sees them)
                const int key = min(8 * (col >> 2) + 4 * t + (col & 3), n - 1);
                k[t][sl] = *reinterpret_cast<const bf16x8*>(kr + (size_t)key * step + sl * 32 + kc * 8);
            }
        uint16_t raw[N][8];
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) raw[i][e] = vr[(size_t)min(8 * kc + e, n - 1) * step + (first + i) * 16 + col];
        const unsigned there = bits_below(n - 8 * kc);       // (a weight of zero would make a NaN of an infinity)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint4 u;
            u.x = raw[i][0] | ((unsigned)raw[i][1] << 16);
            u.y = raw[i][2] | ((unsigned)raw[i][3] << 16);
            u.z = raw[i][4] | ((unsigned)raw[i][5] << 16);
            u.w = raw[i][6] | ((unsigned)raw[i][7] << 16);
            va[i] = keep_keys(__builtin_bit_cast(bf16x8, u), there);
        }
    }
    // Keys and values in LDS, in the operand order of attend_list_split, a half-page of them to a tile: rows of 1 KB, D / 16 of keys
    // and as many of values.  Four rows of each are in flight at once: one after the other they were most of the unit's time.
    template <int D, int NW>
    __device__ __forceinline__ void stage_split(const SpkvView& v, uint16_t* s_tile) const {
        constexpr int NS = D / 16, NB = D / 32, kAtOnce = 4;
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31, wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const int rows = ((n + kHalfTokens - 1) >> 5) * NS, step = v.Hkv * D;
        const uint16_t *kr = keys(v) + 8 * half, *vr = values(v) + col;
        const int k_key = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
        for (int r0 = wv; r0 < rows; r0 += kAtOnce * NW) {
            uint4 k[kAtOnce];
            unsigned x[kAtOnce][8];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {              // (rows of drafts that are not there: the last one's)
                const int r = min(r0 + j * NW, rows - 1), t = r / NS, row = r - t * NS;
                k[j] = *reinterpret_cast<const uint4*>(kr + (size_t)min(32 * t + k_key, n - 1) * step + 16 * row);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[j][e] = vr[(size_t)min(32 * t + 16 * (row / NB) + 8 * half + e, n - 1) * step + 32 * (row % NB)];
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if (r0 + j * NW >= rows) break;
                const int r = r0 + j * NW, t = r / NS, row = r - t * NS;
                uint16_t* to = s_tile + (size_t)t * (2 * kHalfTokens * D) + row * 512 + lane * 8;
                *reinterpret_cast<uint4*>(to) = k[j];
                const uint4 u = make_uint4(x[j][0] | (x[j][1] << 16), x[j][2] | (x[j][3] << 16), x[j][4] | (x[j][5] << 16), x[j][6] | (x[j][7] << 16));
                *reinterpret_cast<bf16x8*>(to + kHalfTokens * D) =          // (a weight of zero would make a NaN of an infinity)
                    keep_keys(__builtin_bit_cast(bf16x8, u), bits_below(n - (32 * t + 16 * (row / NB) + 8 * half)));
            }
        }
    }
    template <int D>
    __device__ __forceinline__ bool careful_needed(const SpkvView& v) const {
        return careful_tree_needed<D>(values(v), stride(v), n);
    }
    template <int D>
    __device__ __forceinline__ void add_careful(const SpkvView& v, const uint16_t* qrow, unsigned long long word, float scale_log2e, float m,
                                                float* sums) const {
        __builtin_amdgcn_wave_barrier();
        careful_tree_sums<D>(keys(v), values(v), stride(v), qrow, word, scale_log2e, m, true, sums);
    }

    // ---- results
    __device__ __forceinline__ size_t result(const SpkvView& v, int c) const {
        const int draft = c / v.G;
        return (size_t)(row0 + draft) * v.Hq + (size_t)h * v.G + (c - draft * v.G);
    }
    // four elements of column c; m, l of its sums
    template <int D>
    __device__ __forceinline__ void store(const SpkvView& v, int c, int d, f32x4 a, float m, float l) const {
        const size_t id = result(v, c);
        store_result(tree.out + id * D + d, a * (l == 0.f ? 0.f : 1.0f / l));
        if (tree.lse != nullptr && d == 0) tree.lse[id] = log_of_sum(m, l);
    }
    // attend_list_split's: a wave's sums of columns c0 .. + n_here - 1, or, again, each worked out by careful; sums: room in LDS
    template <int D, class Careful>
    __device__ __forceinline__ void finish_split(const SpkvView& v, f32x16 (&acc)[D / 32], float m, float l, float* sums, int c0, int n_here,
                                                 bool again, Careful&& careful) const {
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        if (tree.lse != nullptr && half == 0 && col < n_here) tree.lse[result(v, c0 + col)] = log_of_sum(m, l);
        if (__builtin_expect(again, 0)) {
            for (int i = 0; i < n_here; ++i) {
                const float scale = __shfl(inv, i);
                careful(i, sums);
                for (int d = lane; d < D; d += 64) tree.out[result(v, c0 + i) * D + d] = __builtin_bit_cast(uint16_t, (__bf16)(sums[d] * scale));
            }
            return;
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] *= inv;
        column_sums_to_lds<D>(acc, sums);
        constexpr int kUnits = D / 4, kColsPerPass = 64 / kUnits;
        const int unit = lane % kUnits;
#pragma unroll 4
        for (int i = lane / kUnits; i < n_here; i += kColsPerPass)
            store_result(tree.out + result(v, c0 + i) * D + unit * 4, column_sum_at<D>(sums, i, unit));
    }
};

// The drafts as keys, up to 16 NQ columns (so at most 32 drafts: one half-page): every wave has all scores and a
// quarter of the values' elements.
template <int D, int NQ>
__device__ __forceinline__ void attend_drafts_few(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e,
                                                  const TreeWork<false, false>& work) {
    constexpr int NS = D / 32, NB = D / 16, kMine = NB / 4;
    const int lane = threadIdx.x & 63, kc = lane >> 4, col = lane & 15, wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = work.n, h = work.h, n_cols = work.columns(v);
    if (n == 0) return;
    bf16x8 k[2][NS], va[kMine];
    work.load_few<D>(v, k, va, wv * kMine);
    const unsigned long long word = work.seen(v, v.t_pair[work.pair]);
    const size_t pc0 = work.part0(v);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int c = i * 16 + col;
        const bool valid = c < n_cols;
        const int draft = (valid ? c : 0) / v.G;
        const uint16_t* qrow = q + ((size_t)(work.row0 + draft) * v.Hq + (size_t)h * v.G + ((valid ? c : 0) - draft * v.G)) * D;
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) {
            const bf16x8 qb = *reinterpret_cast<const bf16x8*>(qrow + sl * 32 + kc * 8);
            s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[0][sl], qb, s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[1][sl], qb, s1, 0, 0, 0);
        }
        const unsigned long long seen = lane_word(word, draft);
        const unsigned mine = (unsigned)(seen >> (8 * kc)) & 0xffu;
        f32x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = ((mine >> e) & 1u) ? (e < 4 ? s0[e & 3] : s1[e & 3]) * scale_log2e : SPKV_NEG_INF;
        float m = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float ref = m == SPKV_NEG_INF ? 0.f : m;
        f32x8 p;
        float l = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(x[e] - ref);
            l += p[e];
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const bf16x8 hi = __builtin_convertvector(p, bf16x8);
        const bf16x8 lo = __builtin_convertvector(p - __builtin_convertvector(hi, f32x8), bf16x8);
        f32x4 acc[kMine];
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            acc[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[j], hi, acc[j], 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[j], lo, acc[j], 0, 0, 0);
        }
        float* to = v.part_acc + (pc0 + c) * D;
        if (valid) {
#pragma unroll
            for (int j = 0; j < kMine; ++j) *reinterpret_cast<f32x4*>(to + (wv * kMine + j) * 16 + kc * 4) = acc[j];
            if (wv == 0 && kc == 0) work.part_ml<D>(v)[pc0 + c] = make_float2(m, l);
        }
        // every wave looks at its own elements, one of them writes the column again
        const bool odd = valid && odd_sums(acc, kMine, l);
        if (__builtin_expect(__syncthreads_or(odd) != 0, 0)) {
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0): the stores above come first
            __syncthreads();
            if (wv == 0)
                for (int x0 = 0; x0 < 16 && i * 16 + x0 < n_cols; ++x0) {
                    const int cc = i * 16 + x0, dd = cc / v.G;
                    careful_tree_sums<D>(work.keys(v), work.values(v), work.stride(v), q + work.result(v, cc) * D, lane_word(word, dd), scale_log2e,
                                         __shfl(ref, x0), false, v.part_acc + (pc0 + cc) * D);
                }
        }
    }
}

// 33 to 64 columns: every wave has all of them, two groups of MFMA 32x32x16, and an eighth of the workgroup's range to
// itself.  Its half-pages go from memory into 16 KB of LDS of its own (D = 128) in operand order, keys and values in turn: while
// the scores are weighed the next keys arrive, while these are multiplied the next values.  No wave waits for another.
// Read once, the half-pages are loaded as such (nt: 484 MB in 98 us, 114 without; 94 MB that the caches hold 30, 29 without).
// The queries are shared, in LDS.  The drafts are up to two half-pages more in the list's first range, for a wave each.
template <int D, bool W>
__device__ __forceinline__ void attend_own_copies(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e,
                                                  const TreeWork<W, true>& work) {
    constexpr int NS = D / 16, NB = D / 32, kRow = D + 4, kHalfElems = 2 * kHalfTokens * D;
    __shared__ __attribute__((aligned(16))) uint16_t s_q[2 * NS * 512];
    __shared__ __attribute__((aligned(16))) float s_acc[4][64 * kRow];         // (half-pages before)
    __shared__ float2 s_ml[4][64];
    static_assert(sizeof(s_acc) >= (size_t)8 * kHalfElems * 2, "the half-pages' room");
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pair = work.pair, h = work.h;
    const FirstPages first_ids = first_pages(v, pair);
    const ShareList list = share_list(v, pair);
    const int n_cols = work.columns(v), c0 = work.block * 64;
    if (c0 >= n_cols) return;
    const int tiles = (work.n + kHalfTokens - 1) >> 5, nA = list.nA;
    const int r_begin = work.begin(list, work.range), r_end = work.begin(list, work.range + 1);
    const int with_drafts = work.drafts() ? tiles : 0;       // the first waves take one half-page of them each
    auto cut_wave = [&](int w) -> int {
        const int all = r_end - r_begin + kOwnDrafts * with_drafts;
        return r_begin + max(0, all * w / 8 - kOwnDrafts * min(w, with_drafts));
    };
    const int x_begin = cut_wave(wv), x_end = cut_wave(wv + 1);
    const bool ring = x_end > nA, drafts = wv < with_drafts;
    SharePages pages = share_pages(v, pair, first_ids, x_begin >> 1);

    const unsigned k_lane = ((((col >> 3) & 1) * (D / 8) + half) * 16 + 8 * (col >> 4) + 4 * ((col >> 2) & 1) + (col & 3)) * 16;
    const unsigned v_lane = (((col >> 4) * 4 + half) * 16 + (col & 15)) * 16 + kHalfTokens * D * 2;
    uint16_t* const slot = reinterpret_cast<uint16_t*>(&s_acc[0][0]) + wv * kHalfElems;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)slot;
    auto page_of = [&](int x) -> const char* { return reinterpret_cast<const char*>(half_page_at(v, list, pages, x)); };
    auto send_k = [&](const char* base) {
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) load_row_to_lds_once(base + sl * 512, k_lane, lds0 + sl * 1024);
    };
    auto send_v = [&](const char* base) {
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) load_row_to_lds_once(base + (j / NB) * 512 + (j % NB) * 2048, v_lane, lds0 + (NS + j) * 1024);
    };
    // Loads into LDS and reads of it: the compiler does not know that they belong together.
    auto read_all = [&]() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); };           // what was read has arrived
    const char* base = nullptr;
    auto send_first = [&]() {
        if (x_begin >= x_end) return;
        base = page_of(x_begin);
        send_k(base);
        send_v(base);
    };
    if (!drafts) send_first();
    if (with_drafts > 0) work.template stage_split<D, 8>(v, reinterpret_cast<uint16_t*>(&s_acc[0][0]));     // into the first waves' slots
    int place[2], draft[2], least = 0, most = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = c0 + i * 32 + col;
        const ShareRow sr = work.row(v, c < n_cols ? c : 0, ring);
        place[i] = sr.place;
        draft[i] = sr.row - work.row0;
        const uint16_t* qrow = q + ((size_t)sr.row * v.Hq + (size_t)h * v.G + sr.head) * D + half * 8;
        if ((wv & 1) == i && wv < 4) {
#pragma unroll
            for (int j = 0; j < NS / 2; ++j) {
                const int sl = (wv >> 1) * (NS / 2) + j;
                *reinterpret_cast<bf16x8*>(&s_q[(i * NS + sl) * 512 + lane * 8]) = *reinterpret_cast<const bf16x8*>(qrow + sl * 16);
            }
        }
    }
    RingGates gates = {0, 0u};
    if (ring) {
        gates = ring_gates(v, list, x_begin, x_end);
        least = min(place[0], place[1]);
        most = max(place[0], place[1]);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            least = min(least, __shfl_xor(least, o));
            most = max(most, __shfl_xor(most, o));
        }
        least = __builtin_amdgcn_readfirstlane(least);
        most = __builtin_amdgcn_readfirstlane(most);
    }
    __syncthreads();
    f32x16 acc[2][NB];
    float m[2], l[2], neg_ref[2], limit[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        m[i] = SPKV_NEG_INF;
        l[i] = neg_ref[i] = 0.f;
        limit[i] = -1.f;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][db][e] = 0.f;
    }
    f32x16 s[2];
    auto scores = [&]() {
        f32x16 zero;
#pragma unroll
        for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) {
            const bf16x8 key = *reinterpret_cast<const bf16x8*>(slot + sl * 512 + lane * 8);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, *reinterpret_cast<const bf16x8*>(&s_q[(i * NS + sl) * 512 + lane * 8]),
                                                               sl == 0 ? zero : s[i], 0, 0, 0);
        }
    };
    // weights of group i against its reference as it stands; where one is too low or not set, it is raised first
    bf16x8 pb[2][2];
    auto weigh = [&](int i) {
        float psum;
        auto weights = [&]() -> bool {
            f32x8 p[2];
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e >> 3][e & 7] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], scale_log2e, neg_ref[i]));
            float s4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) s4[e] = (p[0][e] + p[0][4 + e]) + (p[1][e] + p[1][4 + e]);
            psum = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            pb[i][0] = __builtin_convertvector(p[0], bf16x8);
            pb[i][1] = __builtin_convertvector(p[1], bf16x8);
            return __builtin_amdgcn_ballot_w64(!(psum <= limit[i])) != 0ull;
        };
        if (__builtin_expect(weights(), 0)) {
            float cm = s[i][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) cm = fmaxf(cm, s[i][e]);
            cm *= scale_log2e;
            cm = fmaxf(cm, __shfl_xor(cm, 32));
            const float m_new = fmaxf(m[i], cm);
            const bool unset = m_new == SPKV_NEG_INF;         // every key so far excluded
            const float m_ref = unset ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m[i] - m_ref);
            l[i] *= alpha;
#pragma unroll
            for (int db = 0; db < NB; ++db) acc[i][db] *= alpha;
            m[i] = m_new;
            neg_ref[i] = -m_ref;
            limit[i] = unset ? -1.f : kSumLimit;
            (void)weights();
        }
        l[i] += psum;
    };
    auto accumulate = [&](unsigned seen) {                    // seen: keys that some column sees, 16 of the lane's half
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int db = 0; db < NB; ++db) {
                bf16x8 val = *reinterpret_cast<const bf16x8*>(slot + kHalfTokens * D + (g * NB + db) * 512 + lane * 8);
                if (seen != 0xffffu) val = keep_keys(val, seen >> (8 * g));
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(val, pb[i][g], acc[i][db], 0, 0, 0);
            }
    };
    const int full = min(list.L >> 5, x_end);
    auto seen_of = [&](int x) -> unsigned {
        asm volatile("" : "+s"(x));                           // (nothing of this is to be carried along from turn to turn)
        unsigned seen = 0u;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int k0 = 16 * g + 8 * half, at0 = (x - nA) * kHalfTokens + k0;
            unsigned ok[2], any;
            if (x < nA) {
                ok[0] = ok[1] = any = bits_below(list.L - x * kHalfTokens - k0);
            } else {
                const unsigned on = gates_of(v, list, gates, x - nA, k0);
                ok[0] = ring_seen(v, list, on, at0, place[0]);
                ok[1] = ring_seen(v, list, on, at0, place[1]);
                any = ring_seen(v, list, on, at0, least);
            }
            seen |= any << (8 * g);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[i][8 * g + e] = ((ok[i] >> e) & 1u) ? s[i][8 * g + e] : SPKV_NEG_INF;
        }
        return seen;
    };
    // Loads land in the order sent: keys, values, keys, values.
    auto turn = [&](int x, auto edge) {
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * NB) : "memory");       // the keys are here
        scores();
        const bool more = x + 1 < x_end;
        if (more) base = page_of(x + 1);
        read_all();
        if (more) send_k(base);
        unsigned seen = 0xffffu;
        if (decltype(edge)::value) seen = seen_of(x);
        weigh(0);
        weigh(1);
        if (more) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(NS) : "memory");  // the values are here
        else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        accumulate(decltype(edge)::value ? seen : 0xffffu);
        read_all();
        if (more) send_v(base);
    };
    unsigned long long word = 0ull;
    if (drafts) {
        word = work.seen(v, list.T);
        scores();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned mine = (unsigned)(lane_word(word, draft[i]) >> (32 * wv));
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = ((mine >> (16 * (e >> 3) + 8 * half + (e & 7))) & 1u) ? s[i][e] : SPKV_NEG_INF;
        }
        weigh(0);
        weigh(1);
        accumulate(0xffffu);
        read_all();
        send_first();
    }
    int x = x_begin;
#pragma unroll 1
    for (; x < full; ++x) turn(x, std::false_type());
#pragma unroll 1
    for (; x < x_end; ++x) turn(x, std::true_type());
#pragma unroll
    for (int i = 0; i < 2; ++i) l[i] += __shfl_xor(l[i], 32);
    const bool odd = odd_sums(acc[0], NB, l[0]) || odd_sums(acc[1], NB, l[1]);
    // Sums of one column, worked out again (see careful_sums): into `to`.
    auto careful = [&](int c, float ref, float* to) {
        const CarefulRange range = careful_range(v, list, scale_log2e, x_begin, x_end);
        const ShareRow sr = work.row(v, c0 + c, true);
        const uint16_t* qrow = q + ((size_t)sr.row * v.Hq + (size_t)h * v.G + sr.head) * D;
        careful_sums<D>(range, qrow, sr.place, ref, to);
        if (drafts) {                                         // (of this wave's half-page of them)
            const unsigned long long mine = lane_word(word, sr.row - work.row0) & (0xffffffffull << (32 * wv));
            work.template add_careful<D>(v, qrow, mine, scale_log2e, ref, to);
        }
        read_all();
    };
    bool again = false;
    if (__builtin_expect(__ballot(odd) != 0ull, 0))
        again = (ring && least != most && careful_needed<D>(careful_range(v, list, scale_log2e, x_begin, x_end), least, most)) ||
                (drafts && work.template careful_needed<D>(v));
    // Four waves leave their sums in LDS, the other four add theirs.
    __syncthreads();                                          // the half-pages are no longer read
    float* mine = s_acc[wv & 3];
    auto leave = [&]() {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* pa = mine + (i * 32 + col) * kRow + half * 4;
#pragma unroll
            for (int db = 0; db < NB; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4*>(pa + db * 32 + g * 8) =
                        (f32x4){acc[i][db][4 * g], acc[i][db][4 * g + 1], acc[i][db][4 * g + 2], acc[i][db][4 * g + 3]};
            if (half == 0) s_ml[wv & 3][i * 32 + col] = make_float2(m[i], l[i]);
        }
    };
    const int n_here = min(64, n_cols - c0);
    if (wv >= 4) {
        leave();
        if (__builtin_expect(again, 0)) {
            read_all();
            for (int c = 0; c < n_here; ++c) careful(c, s_ml[wv & 3][c].x, mine + c * kRow);
        }
    }
    __syncthreads();
    if (wv < 4) {
        if (__builtin_expect(again, 0)) {                     // column by column: what is there, scaled, and the sums worked out again
#pragma unroll 1
            for (int c = 0; c < n_here; ++c) {
                const float my_m = __shfl(c < 32 ? m[0] : m[1], c & 31), my_l = __shfl(c < 32 ? l[0] : l[1], c & 31);
                const float2 there = s_ml[wv][c];
                const float top = fmaxf(my_m, there.x), ref = top == SPKV_NEG_INF ? 0.f : top;
                const float a = __builtin_amdgcn_exp2f(there.x - ref), b = __builtin_amdgcn_exp2f(my_m - ref);
                float old[D / 64];
#pragma unroll
                for (int e = 0; e < D / 64; ++e) old[e] = mine[c * kRow + e * 64 + lane];
                read_all();
                careful(c, my_m, mine + c * kRow);
#pragma unroll
                for (int e = 0; e < D / 64; ++e) mine[c * kRow + e * 64 + lane] = old[e] * a + mine[c * kRow + e * 64 + lane] * b;
                if (lane == 0) s_ml[wv][c] = make_float2(top, there.y * a + my_l * b);
                read_all();
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 there = s_ml[wv][i * 32 + col];
                const float top = fmaxf(m[i], there.x), ref = top == SPKV_NEG_INF ? 0.f : top;
                const float a = __builtin_amdgcn_exp2f(there.x - ref), b = __builtin_amdgcn_exp2f(m[i] - ref);
                const float* pa = mine + (i * 32 + col) * kRow + half * 4;
#pragma unroll
                for (int db = 0; db < NB; ++db)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 y = *reinterpret_cast<const f32x4*>(pa + db * 32 + g * 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][db][4 * g + e] = acc[i][db][4 * g + e] * b + y[e] * a;
                    }
                l[i] = l[i] * b + there.y * a;
                m[i] = top;
            }
            read_all();
            leave();
        }
    }
    __syncthreads();
    const size_t pc0 = W ? 0 : work.part0(v);
    for (int e = tid; e < n_here * (D / 4); e += 512) {
        const int c = e / (D / 4), d = (e - c * (D / 4)) * 4;
        float M = SPKV_NEG_INF, sum = 0.f;
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, s_ml[w][c].x);
        const float m_ref = M == SPKV_NEG_INF ? 0.f : M;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 ml = s_ml[w][c];
            const float sc = __builtin_amdgcn_exp2f(ml.x - m_ref);
            a += *reinterpret_cast<const f32x4*>(s_acc[w] + c * kRow + d) * sc;
            sum += ml.y * sc;
        }
        if constexpr (W) {
            work.template store<D>(v, c0 + c, d, a, M, sum);
        } else {
            *reinterpret_cast<f32x4*>(v.part_acc + (pc0 + c0 + c) * D + d) = a;
            if (d == 0) work.template part_ml<D>(v)[pc0 + c0 + c] = make_float2(M, sum);
        }
    }
}

template <int D, int NQ, int NV, bool W>
__global__ __launch_bounds__(64 * NV) __attribute__((amdgpu_waves_per_eu(2, NQ == 1 && NV == 4 ? 3 : 2)))
void spkv_tree_few(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvTree tree, SpkvTreeTable table) {
    TreeWork<W, W> work(v, tree, table, (int)blockIdx.x, NQ == 1 ? kTreeFew16 : kTreeFew32);
    if constexpr (!W)
        if (work.range < 0) return attend_drafts_few<D, NQ>(v, q, scale_log2e, work);
    attend_list_few<D, NQ, NV>(v, q, scale_log2e, work);
}

template <int D, int NW, bool W>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 2 ? 1 : 2, 2)))
void spkv_tree_split(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvTree tree, SpkvTreeTable table) {
    __shared__ __attribute__((aligned(16))) uint16_t s_tile[kSplitSlots<NW>][2 * kHalfTokens * D];
    TreeWork<W, true> work(v, tree, table, (int)blockIdx.x, NW == 2 ? kTreeSplit64 : NW == 4 ? kTreeSplit128 : kTreeSplit256);
    attend_list_split<D, NW>(v, q, scale_log2e, work, s_tile);
}

template <int D, bool W>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void spkv_tree_own_copies(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvTree tree, SpkvTreeTable table) {
    TreeWork<W, true> work(v, tree, table, (int)blockIdx.x, kTreeOwnCopies);
    attend_own_copies<D, W>(v, q, scale_log2e, work);
}

// The join: D / 4 threads own a column, four consecutive elements each; S such groups share a column, each with every
// S-th of its partial results, and meet in LDS.
template <int D, int S>
__global__ __launch_bounds__(256, 8) void spkv_tree_merge(SpkvView v, SpkvTree tree, SpkvTreeTable table, int width) {
    constexpr int TPC = D / 4, CPB = 256 / TPC, kFold = S > 1 ? 5 : 2, kCols = CPB / S;
    __shared__ f32x4 s_num[S > 1 ? CPB : 1][S > 1 ? TPC : 1];
    __shared__ float2 s_ml[S > 1 ? CPB : 1];
    const int slice = (int)threadIdx.x / TPC, share = slice % S, d = ((int)threadIdx.x % TPC) * 4;
    const int local = blockIdx.y, pair = tree.pair0 + table.pair[local], b = pair / v.Hkv, h = pair - b * v.Hkv, at = b - tree.seq0;
    const int n_cols = (table.cu[at + 1] - table.cu[at]) * v.G, c0 = (int)blockIdx.x * kCols;
    if (c0 >= n_cols) return;
    const bool exists = c0 + slice / S < n_cols;
    const int c = exists ? c0 + slice / S : c0, block = c / width, in = c - block * width;
    const int ranges = table.ranges[local], start = local > 0 ? table.end[local - 1] : 0;
    const size_t lists = (size_t)(start + block * ranges) * width + in;
    const float2* ml = reinterpret_cast<const float2*>(v.part_ml);
    float M = SPKV_NEG_INF, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    const int parts = ranges + tree.alone;                   // (the drafts', where they are units of their own)
    for (int r0 = share; r0 < parts; r0 += kFold * S) {
        float2 x[kFold];
        f32x4 a[kFold];
#pragma unroll
        for (int u = 0; u < kFold; ++u) {
            const int r = min(r0 + u * S, parts - 1);        // past the end: re-read, ignored
            const size_t pc = r == ranges ? (size_t)(tree.n_units + local) * width + in : lists + (size_t)r * width;
            x[u] = ml[pc];
            a[u] = *reinterpret_cast<const f32x4*>(v.part_acc + pc * D + d);
        }
        float m_new = M;
#pragma unroll
        for (int u = 0; u < kFold; ++u)
            if (r0 + u * S < parts) m_new = fmaxf(m_new, x[u].x);
        const float m_ref = m_new == SPKV_NEG_INF ? 0.f : m_new, so = __builtin_amdgcn_exp2f(M - m_ref);
        den *= so;
        num *= so;
#pragma unroll
        for (int u = 0; u < kFold; ++u)
            if (r0 + u * S < parts && (x[u].x != SPKV_NEG_INF || x[u].y != 0.f)) {       // (a range without keys has written no sums)
                const float sc = __builtin_amdgcn_exp2f(x[u].x - m_ref);
                num += a[u] * sc;
                den += x[u].y * sc;
            }
        M = m_new;
    }
    if (S > 1) {
        s_num[slice][(int)threadIdx.x % TPC] = num;
        if (d == 0) s_ml[slice] = make_float2(M, den);
        __syncthreads();
        if (share != 0) return;
        float top = M;
#pragma unroll
        for (int i = 1; i < S; ++i) top = fmaxf(top, s_ml[slice + i].x);
        const float m_ref = top == SPKV_NEG_INF ? 0.f : top, so = __builtin_amdgcn_exp2f(M - m_ref);
        num *= so;
        den *= so;
#pragma unroll
        for (int i = 1; i < S; ++i) {
            const float2 y = s_ml[slice + i];
            const float sc = __builtin_amdgcn_exp2f(y.x - m_ref);
            num += s_num[slice + i][(int)threadIdx.x % TPC] * sc;
            den += y.y * sc;
        }
        M = top;
    }
    if (!exists) return;
    const float inv = den == 0.f ? 0.f : 1.0f / den;
    const int draft = c / v.G;
    const size_t id = (size_t)(tree.row0 + table.cu[at] + draft) * v.Hq + (size_t)h * v.G + (c - draft * v.G);
    store_result(tree.out + id * D + d, num * inv);
    if (tree.lse != nullptr && d == 0) tree.lse[id] = log_of_sum(M, den);
}

// The kernel of own copies has the higher rate on long lists and the longer start: 33 to 64 columns, split / own copies, us: 484 MB
// in 128 lists 116 / 98, 404 MB in 512 uneven ones 170 / 105, 120 MB in 8 38.3 / 36.5; D = 64, 94 MB 43 / 29; but 28 MB
// in 256 26 / 30, 17 MB in 32 19.5 / 22.6, 2 MB in 8 13.9 / 19.6.
// 129 columns and more: 256 to a workgroup, whose eight waves read a half-page once, or blocks of 128 on four waves, two workgroups to a
// compute unit.  256 / blocks of 128, us, 4 heads a group: 16 sequences of 32k, 33, 48, 64 drafts 158 / 180, 152 / 170, 155 / 176 (D = 64 88 / 104,
// 93 / 107 with 33, 64); 64 of 1k-16k 173 / 200, 174 / 199, 180 / 203; 32 of 300 25.4 / 30, 27.6 / 30, 28.2 / 30; one of 128k, 64 drafts
// 49.6 / 51; 16 heads a group, 16 of 8k, 1024 columns 56 / 58.  A few short lists alone are the other way: 4 of 4k 27.2 / 26.0, one of 2k 22.3 / 20.4.
constexpr int64_t kTreeOwnHalfPages = 4096;
SpkvTreeKernel spkv_tree_kernel(int n_cols, int64_t half_pages) {
    return n_cols <= 16 ? kTreeFew16 : n_cols <= 32 ? kTreeFew32 : n_cols <= 64 ? (half_pages >= kTreeOwnHalfPages ? kTreeOwnCopies : kTreeSplit64)
                        : n_cols <= 128 ? kTreeSplit128 : kTreeSplit256;
}
// Whole lists, one to a compute unit: eight waves to a list are better than two or four.  us, 16 drafts of 4 heads, split / own copies: 8
// sequences of 500 19.4 / 17.5, 32 of 1000 27 / 21.5, but 64 of 300 (512 lists) 25 / 36.6; D = 64, 8 drafts of 8 heads, 32 of 1000 18.5 / 13.4;
// 8 drafts of 4 heads, four / eight waves: 8 of 500 14.8 / 12.9, 32 of 1000 20.4 / 18.2; 4 drafts, one of 300 10 / 8.2.
SpkvTreeKernel spkv_tree_kernel_whole(SpkvTreeKernel k, int64_t lists, int64_t compute_units) {
    if (lists > compute_units) return k;
    return k == kTreeSplit64 ? kTreeOwnCopies : k == kTreeFew16 ? kTreeFew16Eight : k == kTreeFew32 ? kTreeFew32Eight : k;
}
int spkv_tree_resident(SpkvTreeKernel k) { return k == kTreeOwnCopies || k == kTreeSplit256 ? 1 : 2; }

constexpr int kTreeMergeRound = 2048;
template <int D, bool W>
static void launch_lists(const SpkvView& v, const uint16_t* q, float sl, SpkvTreeKernel kernel, const SpkvTree& tree, const SpkvTreeTable& table,
                         int n_pairs, hipStream_t s) {
    const dim3 grid((unsigned)(tree.n_units + tree.alone * n_pairs));
    switch (kernel) {
        case kTreeFew16: spkv_tree_few<D, 1, 4, W><<<grid, dim3(256), 0, s>>>(v, q, sl, tree, table); break;
        case kTreeFew32: spkv_tree_few<D, 2, 4, W><<<grid, dim3(256), 0, s>>>(v, q, sl, tree, table); break;
        case kTreeFew16Eight:
            if constexpr (W) spkv_tree_few<D, 1, 8, W><<<grid, dim3(512), 0, s>>>(v, q, sl, tree, table);
            break;
        case kTreeFew32Eight:
            if constexpr (W) spkv_tree_few<D, 2, 8, W><<<grid, dim3(512), 0, s>>>(v, q, sl, tree, table);
            break;
        case kTreeOwnCopies: spkv_tree_own_copies<D, W><<<grid, dim3(512), 0, s>>>(v, q, sl, tree, table); break;
        case kTreeSplit64: spkv_tree_split<D, 2, W><<<grid, dim3(128), 0, s>>>(v, q, sl, tree, table); break;
        case kTreeSplit128: spkv_tree_split<D, 4, W><<<grid, dim3(256), 0, s>>>(v, q, sl, tree, table); break;
        case kTreeSplit256: spkv_tree_split<D, 8, W><<<grid, dim3(512), 0, s>>>(v, q, sl, tree, table); break;
    }
}
template <int D>
static hipError_t launch_tree(const SpkvView& v, const uint16_t* q, float sl, SpkvTreeKernel kernel, const SpkvTree& tree,
                              const SpkvTreeTable& table, int n_pairs, int most_cols, int most_ranges, hipStream_t s) {
    const int width = spkv_tree_width(kernel);
    if (tree.whole) {
        launch_lists<D, true>(v, q, sl, kernel, tree, table, n_pairs, s);
        return hipGetLastError();
    }
    launch_lists<D, false>(v, q, sl, kernel, tree, table, n_pairs, s);
    constexpr int CPB = 256 / (D / 4);
    int share = std::min(8, CPB);
    while (share > 1 && (n_pairs * ((most_cols * share + CPB - 1) / CPB) > kTreeMergeRound || share > most_ranges + tree.alone)) share >>= 1;
    const dim3 merge((unsigned)((most_cols * share + CPB - 1) / CPB), (unsigned)n_pairs);
    if (share == 8) spkv_tree_merge<D, 8><<<merge, dim3(256), 0, s>>>(v, tree, table, width);
    else if (share == 4) spkv_tree_merge<D, 4><<<merge, dim3(256), 0, s>>>(v, tree, table, width);
    else if (share == 2) spkv_tree_merge<D, 2><<<merge, dim3(256), 0, s>>>(v, tree, table, width);
    else spkv_tree_merge<D, 1><<<merge, dim3(256), 0, s>>>(v, tree, table, width);
    return hipGetLastError();
}

hipError_t spkv_launch_tree(const SpkvView& v, const uint16_t* q, float sm_scale, SpkvTreeKernel kernel, const SpkvTree& tree,
                            const SpkvTreeTable& table, int n_pairs, int most_cols, int most_ranges, hipStream_t s) {
    const float sl = sm_scale * 1.4426950408889634f;
    return v.D == 128 ? launch_tree<128>(v, q, sl, kernel, tree, table, n_pairs, most_cols, most_ranges, s)
                      : launch_tree<64>(v, q, sl, kernel, tree, table, n_pairs, most_cols, most_ranges, s);
}
