// Attention of trees of drafted tokens over the cache on gfx950.
#include "spkv_lists.h"

// The mathematics.  Draft i of a sequence that holds T tokens hangs behind draft parent(i) < i or behind the newest
// token; the drafts from there to it are its path, and with d(i) drafts before it on the path it stands at position
// T + d(i).  It sees a cached key at position s if T + d(i) - s < w or that key's gate is on, and draft a if a is on its
// path and d(i) - d(a) < w or a's gate is on (Eq. 3-5 for the tokens of the path alone).  All drafts of a sequence
// and all heads of a group are columns of one product with the list, as the rows of sequences that share a prompt are
// (spkv_lists.h), with d(i) for the place behind the list's newest token; the drafts themselves, at most 64
// keys, are one unit of work more, whose mask is a word of 64 bits a draft.
//
// A lane of a wave stands for a draft: paths are words of bits, joined along the parents by doubling (log2 of the deepest
// path's length rounds of three lane exchanges), depths their counts of bits.
//
// Bound: the lists are read once, 4 D bytes a key for 4 D flops a key and column: past about 300 columns a list the matrix
// units, below the read; few columns or short lists by the start of a workgroup and the join.

// ------------------------------------------------------------------------------- paths
struct TreePath {
    unsigned long long path;     // of lane's draft: itself and what it hangs behind
    int up, depth;
};
__device__ __forceinline__ unsigned long long lane_word(unsigned long long x, int lane) {
    return (unsigned long long)(unsigned)__shfl((int)(unsigned)x, lane) | ((unsigned long long)(unsigned)__shfl((int)(x >> 32), lane) << 32);
}
// Any value but 0 .. i - 1 for a parent means that the draft hangs behind the newest token.
__device__ __forceinline__ TreePath tree_path(const int32_t* __restrict__ parents, int n) {
    const int lane = threadIdx.x & 63;
    TreePath t;
    const int p = lane < n ? parents[lane] : -1;
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

// ---------------------------------------------------------------------------- the work
// Workgroup id -> unit: the drafts of every pair's blocks of columns first, then the ranges of the lists, by the host's
// table, the ranges of a pair's block of columns next to each other.
struct TreeWork {
    const SpkvTree& tree;
    const SpkvTreeTable& table;
    int pair, h, range, ranges, block, n, row0, unit, width;
    __device__ __forceinline__ TreeWork(const SpkvView& v, const SpkvTree& t, const SpkvTreeTable& tab, int id, int w)
        : tree(t), table(tab), width(w) {
        int local;
        if (id < t.n_own) {
            local = id / t.n_blocks;
            block = id - local * t.n_blocks;
            range = -1;
            ranges = 1;
            unit = t.n_units + id;
        } else {
            id -= t.n_own;
            const uint4 raw = reinterpret_cast<const uint4*>(tab.end)[threadIdx.x & 63];      // eight pairs a lane
            const unsigned e[4] = {raw.x, raw.y, raw.z, raw.w};
            local = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                local += __popcll(__ballot((int)(e[i] & 0xffffu) <= id));
                local += __popcll(__ballot((int)(e[i] >> 16) <= id));
            }
            const int start = local > 0 ? tab.end[local - 1] : 0;
            ranges = tab.ranges[local];
            block = (id - start) / ranges;
            range = id - start - block * ranges;
            unit = id;
        }
        pair = t.pair0 + local;
        const int b = pair / v.Hkv, at = b - t.seq0;
        h = pair - b * v.Hkv;
        row0 = t.row0 + tab.cu[at];
        n = tab.cu[at + 1] - tab.cu[at];
    }
    __device__ __forceinline__ int columns(const SpkvView& v) const { return n * v.G; }
    __device__ __forceinline__ ShareRow row(const SpkvView& v, int c, bool ring) const {
        ShareRow r;
        const int i = c / v.G;
        r.head = c - i * v.G;
        r.row = row0 + i;
        r.place = ring ? __shfl(tree_path(tree.parents + row0, n).depth, i) : 0;
        return r;
    }
    __device__ __forceinline__ float* part(const SpkvView& v) const { return v.part_acc; }
    template <int D>
    __device__ __forceinline__ float2* part_ml(const SpkvView& v) const { return reinterpret_cast<float2*>(v.part_ml); }
    __device__ __forceinline__ size_t part0(const SpkvView&) const { return (size_t)(unit - block) * width; }
};

// Sums of one column over the drafts that it sees, key by key, where an infinity or NaN among the values of a draft that it
// does not see has reached it (a weight of zero times it).  The whole wave.
template <int D>
__device__ __attribute__((noinline)) void careful_tree_sums(const uint16_t* k, const uint16_t* vv, int stride, const uint16_t* qrow,
                                                            unsigned long long seen, float scale_log2e, float m, float* sums) {
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
    for (int e = 0; e < D / 64; ++e) sums[e * 64 + lane] = acc[e];
}

// The drafts as keys, up to 16 NQ columns (so at most 32 drafts: one half-page): every wave has all scores and a
// quarter of the values' elements.  Keys straight from their rows; values, of which an operand wants eight keys of one
// element, by 2-byte loads: a unit of a few microseconds beside those of the lists.
template <int D, int NQ>
__device__ __forceinline__ void attend_drafts_few(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e,
                                                  const TreeWork& work) {
    constexpr int NS = D / 32, NB = D / 16, kMine = NB / 4;
    const int lane = threadIdx.x & 63, kc = lane >> 4, col = lane & 15, wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = work.n, h = work.h, stride = v.Hkv * D, n_cols = work.columns(v);
    if (n == 0) return;
    const uint16_t* kr = work.tree.k + ((size_t)work.row0 * v.Hkv + h) * D;
    const uint16_t* vr = work.tree.v + ((size_t)work.row0 * v.Hkv + h) * D;
    const uint4 zero = {0u, 0u, 0u, 0u};
    bf16x8 k[2][NS];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) {
            const int key = 8 * (col >> 2) + 4 * t + (col & 3);
            k[t][sl] = __builtin_bit_cast(bf16x8, key < n ? *reinterpret_cast<const uint4*>(kr + (size_t)key * stride + sl * 32 + kc * 8) : zero);
        }
    uint16_t raw[kMine][8];
#pragma unroll
    for (int i = 0; i < kMine; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int key = 8 * kc + e;
            raw[i][e] = key < n ? vr[(size_t)key * stride + (wv * kMine + i) * 16 + col] : (uint16_t)0;
        }
    const int T = v.t_pair[work.pair];
    const TreePath path = tree_path(work.tree.parents + work.row0, n);
    const unsigned long long word = tree_seen(v, path, work.tree.f, h, work.row0, n, T);
    bf16x8 va[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        uint4 u;
        u.x = raw[i][0] | ((unsigned)raw[i][1] << 16);
        u.y = raw[i][2] | ((unsigned)raw[i][3] << 16);
        u.z = raw[i][4] | ((unsigned)raw[i][5] << 16);
        u.w = raw[i][6] | ((unsigned)raw[i][7] << 16);
        va[i] = __builtin_bit_cast(bf16x8, u);
    }
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
                    careful_tree_sums<D>(kr, vr, stride, q + ((size_t)(work.row0 + dd) * v.Hq + (size_t)h * v.G + (cc - dd * v.G)) * D,
                                         lane_word(word, dd), scale_log2e, __shfl(ref, x0), v.part_acc + (pc0 + cc) * D);
                }
        }
    }
}

// More columns: keys and values into LDS once, in the operand order of attend_list_split, then 32 columns a wave.
template <int D, int NW>
__device__ __forceinline__ void attend_drafts_split(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e,
                                                    const TreeWork& work, uint16_t (&s_tile)[kSplitSlots<NW>][2 * kHalfTokens * D]) {
    constexpr int NS = D / 16, NB = D / 32;
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31, wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = work.n, h = work.h, stride = v.Hkv * D, n_cols = work.columns(v), col0 = work.block * (32 * NW);
    if (col0 >= n_cols) return;
    const uint16_t* kr = work.tree.k + ((size_t)work.row0 * v.Hkv + h) * D;
    const uint16_t* vr = work.tree.v + ((size_t)work.row0 * v.Hkv + h) * D;
    const int tiles = (n + kHalfTokens - 1) >> 5;
    for (int r = wv; r < tiles * (D / 8); r += NW) {          // rows of 1 KB: D / 16 of keys, D / 16 of values
        const int t = r / (D / 8), row = r - t * (D / 8);
        uint4 u = {0u, 0u, 0u, 0u};
        if (row < NS) {
            const int key = 32 * t + 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
            if (key < n) u = *reinterpret_cast<const uint4*>(kr + (size_t)key * stride + 16 * row + 8 * half);
        } else {
            const int g = (row - NS) / NB, d = 32 * ((row - NS) % NB) + col, key0 = 32 * t + 16 * g + 8 * half;
            unsigned x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = key0 + e < n ? vr[(size_t)(key0 + e) * stride + d] : 0u;
            u = make_uint4(x[0] | (x[1] << 16), x[2] | (x[3] << 16), x[4] | (x[5] << 16), x[6] | (x[7] << 16));
        }
        *reinterpret_cast<uint4*>(&s_tile[t][row * 512 + lane * 8]) = u;
    }
    const int c = col0 + wv * 32 + col;
    const bool valid = c < n_cols;
    const int draft = (valid ? c : 0) / v.G;
    const uint16_t* qrow = q + ((size_t)(work.row0 + draft) * v.Hq + (size_t)h * v.G + ((valid ? c : 0) - draft * v.G)) * D;
    bf16x8 qb[NS];
#pragma unroll
    for (int sl = 0; sl < NS; ++sl) qb[sl] = *reinterpret_cast<const bf16x8*>(qrow + sl * 16 + half * 8);
    const int T = v.t_pair[work.pair];
    const TreePath path = tree_path(work.tree.parents + work.row0, n);
    const unsigned long long word = tree_seen(v, path, work.tree.f, h, work.row0, n, T), seen = lane_word(word, draft);
    __syncthreads();
    f32x16 s[2], acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
    float m = SPKV_NEG_INF;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
        if (t < tiles) {
#pragma unroll
            for (int sl = 0; sl < NS; ++sl)
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(&s_tile[t][sl * 512 + lane * 8]), qb[sl], s[t], 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int key = 32 * t + 16 * (e >> 3) + 8 * half + (e & 7);
            s[t][e] = ((seen >> key) & 1ull) ? s[t][e] * scale_log2e : SPKV_NEG_INF;
            m = fmaxf(m, s[t][e]);
        }
    }
    m = fmaxf(m, __shfl_xor(m, 32));
    const float ref = m == SPKV_NEG_INF ? 0.f : m;
    float l = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (t >= tiles) break;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            f32x8 p;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(s[t][8 * g + e] - ref);
                l += p[e];
            }
            const bf16x8 pb = __builtin_convertvector(p, bf16x8);
#pragma unroll
            for (int db = 0; db < NB; ++db)
                acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    *reinterpret_cast<const bf16x8*>(&s_tile[t][kHalfTokens * D + (g * NB + db) * 512 + lane * 8]), pb, acc[db], 0, 0, 0);
        }
    }
    l += __shfl_xor(l, 32);
    const size_t pc0 = work.part0(v);
    if (valid && half == 0) work.part_ml<D>(v)[pc0 + c] = make_float2(m, l);
    const bool odd = valid && odd_sums(acc, NB, l);
    __syncthreads();                                         // the tiles are no longer read
    const int n_here = min(32, n_cols - (col0 + wv * 32));
    float* to = v.part_acc + (pc0 + col0 + wv * 32) * D;
    store_column_sums<D>(acc, reinterpret_cast<float*>(&s_tile[0][0]) + wv * 32 * D, to, n_here);
    if (__builtin_expect(__ballot(odd) != 0ull, 0)) {
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): the stores above come first
        for (int i = 0; i < n_here; ++i) {
            const int cc = col0 + wv * 32 + i, dd = cc / v.G;
            careful_tree_sums<D>(kr, vr, stride, q + ((size_t)(work.row0 + dd) * v.Hq + (size_t)h * v.G + (cc - dd * v.G)) * D,
                                 lane_word(word, dd), scale_log2e, __shfl(ref, i), to + (size_t)i * D);
        }
    }
}

template <int D, int NQ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, NQ == 1 ? 3 : 2)))
void spkv_tree_few(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvTree tree, SpkvTreeTable table) {
    TreeWork work(v, tree, table, (int)blockIdx.x, 16 * NQ);
    if (work.range < 0) attend_drafts_few<D, NQ>(v, q, scale_log2e, work);
    else attend_list_few<D, NQ>(v, q, scale_log2e, work);
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 2 ? 1 : 2, 2)))
void spkv_tree_split(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvTree tree, SpkvTreeTable table) {
    __shared__ __attribute__((aligned(16))) uint16_t s_tile[kSplitSlots<NW>][2 * kHalfTokens * D];
    TreeWork work(v, tree, table, (int)blockIdx.x, 32 * NW);
    if (work.range < 0) attend_drafts_split<D, NW>(v, q, scale_log2e, work, s_tile);
    else attend_list_split<D, NW>(v, q, scale_log2e, work, s_tile);
}

// The join: D / 4 threads own a column, four consecutive elements each; S such groups share a column, each with every
// S-th of its partial results, and meet in LDS.
template <int D, int S>
__global__ __launch_bounds__(256, 8) void spkv_tree_merge(SpkvView v, SpkvTree tree, SpkvTreeTable table, int width, uint16_t* out, float* lse) {
    constexpr int TPC = D / 4, CPB = 256 / TPC, kFold = S > 1 ? 5 : 2, kCols = CPB / S;
    __shared__ f32x4 s_num[S > 1 ? CPB : 1][S > 1 ? TPC : 1];
    __shared__ float2 s_ml[S > 1 ? CPB : 1];
    const int slice = (int)threadIdx.x / TPC, share = slice % S, d = ((int)threadIdx.x % TPC) * 4;
    const int local = blockIdx.y, pair = tree.pair0 + local, b = pair / v.Hkv, h = pair - b * v.Hkv, at = b - tree.seq0;
    const int n_cols = (table.cu[at + 1] - table.cu[at]) * v.G, c0 = (int)blockIdx.x * kCols;
    if (c0 >= n_cols) return;
    const bool exists = c0 + slice / S < n_cols;
    const int c = exists ? c0 + slice / S : c0, block = c / width, in = c - block * width;
    const int ranges = table.ranges[local], start = local > 0 ? table.end[local - 1] : 0;
    const size_t own = (size_t)(tree.n_units + local * tree.n_blocks + block) * width + in;
    const size_t lists = (size_t)(start + block * ranges) * width + in;
    const float2* ml = reinterpret_cast<const float2*>(v.part_ml);
    float M = SPKV_NEG_INF, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    const int parts = ranges + 1;
    for (int r0 = share; r0 < parts; r0 += kFold * S) {
        float2 x[kFold];
        f32x4 a[kFold];
#pragma unroll
        for (int u = 0; u < kFold; ++u) {
            const int r = min(r0 + u * S, parts - 1);        // past the end: re-read, ignored
            const size_t pc = r == 0 ? own : lists + (size_t)(r - 1) * width;
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
    uint2 packed;
    packed.x = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[0] * inv)) |
               ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[1] * inv)) << 16);
    packed.y = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[2] * inv)) |
               ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[3] * inv)) << 16);
    const int draft = c / v.G;
    const size_t id = (size_t)(tree.row0 + table.cu[at] + draft) * v.Hq + (size_t)h * v.G + (c - draft * v.G);
    *reinterpret_cast<uint2*>(out + id * D + d) = packed;
    if (lse != nullptr && d == 0) lse[id] = den == 0.f ? SPKV_NEG_INF : (M + log2f(den)) * 0.6931471805599453f;
}

int spkv_tree_width(int n_cols) { return n_cols <= 16 ? 16 : n_cols <= 32 ? 32 : n_cols <= 64 ? 64 : n_cols <= 128 ? 128 : 256; }
int spkv_tree_waves(int width) { return width <= 32 ? 4 : width / 32; }

constexpr int kTreeMergeRound = 2048;
template <int D>
static hipError_t launch_tree(const SpkvView& v, const uint16_t* q, float sl, int width, const SpkvTree& tree, const SpkvTreeTable& table,
                              int n_pairs, int most_cols, int most_ranges, uint16_t* out, float* lse, hipStream_t s) {
    const dim3 grid((unsigned)(tree.n_own + tree.n_units)), block(64 * spkv_tree_waves(width));
    if (width == 16) spkv_tree_few<D, 1><<<grid, block, 0, s>>>(v, q, sl, tree, table);
    else if (width == 32) spkv_tree_few<D, 2><<<grid, block, 0, s>>>(v, q, sl, tree, table);
    else if (width == 64) spkv_tree_split<D, 2><<<grid, block, 0, s>>>(v, q, sl, tree, table);
    else if (width == 128) spkv_tree_split<D, 4><<<grid, block, 0, s>>>(v, q, sl, tree, table);
    else spkv_tree_split<D, 8><<<grid, block, 0, s>>>(v, q, sl, tree, table);
    constexpr int CPB = 256 / (D / 4);
    int share = std::min(8, CPB);
    while (share > 1 && (n_pairs * ((most_cols * share + CPB - 1) / CPB) > kTreeMergeRound || share > most_ranges + 1)) share >>= 1;
    const dim3 merge((unsigned)((most_cols * share + CPB - 1) / CPB), (unsigned)n_pairs);
    if (share == 8) spkv_tree_merge<D, 8><<<merge, dim3(256), 0, s>>>(v, tree, table, width, out, lse);
    else if (share == 4) spkv_tree_merge<D, 4><<<merge, dim3(256), 0, s>>>(v, tree, table, width, out, lse);
    else if (share == 2) spkv_tree_merge<D, 2><<<merge, dim3(256), 0, s>>>(v, tree, table, width, out, lse);
    else spkv_tree_merge<D, 1><<<merge, dim3(256), 0, s>>>(v, tree, table, width, out, lse);
    return hipGetLastError();
}

hipError_t spkv_launch_tree(const SpkvView& v, const uint16_t* q, float sm_scale, int width, const SpkvTree& tree,
                            const SpkvTreeTable& table, int n_pairs, int most_cols, int most_ranges, uint16_t* out, float* lse,
                            hipStream_t s) {
    const float sl = sm_scale * 1.4426950408889634f;
    return v.D == 128 ? launch_tree<128>(v, q, sl, width, tree, table, n_pairs, most_cols, most_ranges, out, lse, s)
                      : launch_tree<64>(v, q, sl, width, tree, table, n_pairs, most_cols, most_ranges, out, lse, s);
}
