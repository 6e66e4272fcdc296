// Attention over shared prompts on gfx950: sequences that continue the same prompt read its lists
// once for all of them, and the result is joined with what they attend to of their own.
#include "spkv_lists.h"

// The mathematics.  A token at place i of its sequence, which continues a prompt of P tokens, stands at
// position P + i: it sees the prompt's key at position s if P + i - s < w, and else if that key's gate is
// on (Eq. 3-4).  The prompt's long-term list holds keys that passed, so all tokens see all of it;
// its ring holds the last min(P, w) keys, and a ring key of age a (0 = position P - w) is seen by
// the tokens at places i < a and, with its gate on, by all.  What all query rows of all sequences of
// a prompt share is then one product of a list with a block of columns (row, head):
//   S[key][column] = K Q^T,  weights 2^(S - m),  O[d][column] += V^T weights
// with m and the sum l of every column kept along the list, and (m, l, O) of list ranges and of the
// sequence's own attention (m = lse, l = 1, O = out) joined at the end:
//   out = sum_r 2^(m_r - M) O_r / sum_r 2^(m_r - M) l_r,  M = max_r m_r.
//
// Bound: with few columns by the read of the lists (once, whatever the number of sequences); 4 D
// flops per key and column stand against 4 D bytes per key, so past about 300 columns by the matrix units;
// in between by what the ranges' results cost to write and read again, 4 (D + 2) bytes per column and range.
// Two kernels for the lists, by the columns of the prompt with the most rows:
//   spkv_prefix_few    up to 32 columns: every wave has all of them and a part of the range to itself, operands straight
//                      from memory to registers, the next half-page's loads out before this one's products
//   spkv_prefix_split  more: a workgroup of NW waves has 32 NW columns (32 a wave, one group of MFMA 32x32x16) and
//                      shares the range's half-pages through a ring of LDS buffers
// Measured, joins included: 16 sequences (64 columns) behind 30 MB of lists, with their own 8 MB, 22 us; 64 behind 45 MB, with their
// own 57, 45 us; 1632 rows of four heads behind 30 MB 230 us, 0.83 PFLOP/s.
// The sequences' cache as the helpers of spkv_device.h take it: its lists, the shape of the prompts' one.
__device__ __forceinline__ SpkvView own_view(const SpkvShareOwn& o, const SpkvView& prompts) {
    SpkvView v = prompts;
    v.n_pairs = o.n_pairs;
    v.pt_cap = o.pt_cap;
    v.ring = o.ring;
    v.page_table = o.page_table;
    v.pool = o.pool;
    v.t_pair = o.t_pair;
    v.kept_len = o.kept_len;
    return v;
}
// Items that a pair of them is cut into (pair_split).
__device__ __forceinline__ int own_ranges(const SpkvShareOwn& o, int pair) {
    const int n_hp = ((o.kept_len[pair] + kHalfTokens - 1) >> 5) + ((min(o.t_pair[pair], o.w) + kHalfTokens - 1) >> 5);
    return min((n_hp + o.split.hp_per_item - 1) / o.split.hp_per_item, o.split.slots);
}

// The sequences' own tokens in the same launch (spkv_decode_attention_shared, short lists): one wave per item of a
// (sequence, KV head), cut as for spkv_decode_split, 16 columns of which the group's heads are used;
// operands straight from memory, weights in two bf16 parts.
template <int D>
__device__ __forceinline__ void own_item(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e, SpkvSplit sp,
                                         float* part, int item) {
    constexpr int NS = D / 32, NB = D / 16;
    const int pair = item / sp.slots, j = item - pair * sp.slots;
    if (pair >= v.n_pairs) return;
    const int lane = threadIdx.x & 63, kc = lane >> 4, n = lane & 15;
    const int32_t* pt = v.page_table + (size_t)pair * v.pt_cap;
    int pbase = 0, my_page = pt[min(lane, v.pt_cap - 1)];
    const PairSplit ps = pair_split(v, pair, sp);
    if (j >= ps.groups) return;
    const int hp0 = (int)((int64_t)j * ps.nhp / ps.groups), hp1 = (int)((int64_t)(j + 1) * ps.nhp / ps.groups);
    const int b = pair / v.Hkv, h = pair - b * v.Hkv;
    bf16x8 qb[NS];
    const uint16_t* qrow = q + ((size_t)b * v.Hq + (size_t)h * v.G + n) * D + kc * 8;
#pragma unroll
    for (int sl = 0; sl < NS; ++sl) {
        uint4 raw = {0u, 0u, 0u, 0u};
        if (n < v.G) raw = *reinterpret_cast<const uint4*>(qrow + sl * 32);
        qb[sl] = __builtin_bit_cast(bf16x8, raw);
    }
    f32x4 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = SPKV_NEG_INF, l = 0.f;
    // two half-pages in flight: what limits an item is its round trips to memory
    bf16x8 ka[2][2][NS], va[2][NB];
    auto load = [&](int at, int hp) {
        const uint16_t* base;
        if (hp < ps.ghp) {
            const int lp = hp >> 1;
            if (lp >= pbase + 64) {
                pbase = lp;
                my_page = pt[min(pbase + lane, v.pt_cap - 1)];
            }
            base = pool_page(v, __builtin_amdgcn_readlane(my_page, lp - pbase)) + (hp & 1) * (2 * kHalfTokens * D);
        } else {
            const int r = hp - ps.ghp;
            base = ring_page(v, pair, r >> 1) + (r & 1) * (2 * kHalfTokens * D);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) ka[at][t][sl] = load_stream_b128(base + lane * 8 + (t * (D / 8) + sl * 4) * 128);
#pragma unroll
        for (int db = 0; db < NB; ++db) va[at][db] = load_stream_b128(base + kHalfTokens * D + lane * 8 + db * 512);
    };
    auto attend = [&](int at, int hp) {
        const int nvalid = hp < ps.ghp ? ps.L - hp * kHalfTokens : ps.Tw - (hp - ps.ghp) * kHalfTokens;
        const bool any_kill = nvalid < kHalfTokens;
        const unsigned kill = any_kill ? bits_from(nvalid - kc * 8) : 0u;
        attend_half_page<D, true>(ka[at], va[at], qb, kill, any_kill, scale_log2e, acc, m, l);
    };
    for (int hp = hp0; hp < hp1; hp += 2) {
        load(0, hp);
        if (hp + 1 < hp1) load(1, hp + 1);
        attend(0, hp);
        if (hp + 1 < hp1) attend(1, hp + 1);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (n >= v.G) return;
    const size_t pc = (size_t)item * v.G + n;
    float* pa = part + pc * D + kc * 4;
#pragma unroll
    for (int db = 0; db < NB; ++db) *reinterpret_cast<f32x4*>(pa + db * 16) = acc[db];
    if (kc == 0) reinterpret_cast<float2*>(part + (size_t)v.n_pairs * sp.slots * v.G * D)[pc] = make_float2(m, l);
}

// Which list, range and block of columns a workgroup has: id counts workgroups without gaps, the ranges of a list's
// block of columns next to each other (round-robin over the XCDs).  With up to kShareTablePairs lists the host's
// table says where each list's workgroups end -- ids with nothing to do in between would fill some
// XCDs' compute units and leave others idle; with more lists each is one range.
struct ShareUnit {
    int list, range, ranges, block;
};
__device__ __forceinline__ ShareUnit find_unit(const SpkvShareCut& cut, const SpkvShareTable& table, int id, int n_kv_heads) {
    ShareUnit u;
    if (cut.whole != 0) {
        u.list = id / cut.n_blocks;
        u.block = id - u.list * cut.n_blocks;
        u.range = 0;
        u.ranges = 1;
        return u;
    }
    const int lane = threadIdx.x & 63;
    const uint2 raw = reinterpret_cast<const uint2*>(table.end)[lane];           // four lists a lane
    const unsigned e[4] = {raw.x & 0xffffu, raw.x >> 16, raw.y & 0xffffu, raw.y >> 16};
    int before = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) before += __popcll(__ballot((int)e[i] <= id));
    u.list = before;
    const int start = before > 0 ? table.end[before - 1] : 0;
    u.ranges = table.ranges[before];
    u.block = (id - start) / u.ranges;
    u.range = id - start - u.block * u.ranges;
    return u;
}

// The query row of column c of an active prompt.  Columns past the last one repeat the first and are never stored.
__device__ __forceinline__ int share_first(const SpkvShareRows& rows, int act) {
    return rows.in_spans ? rows.spans.first[act] : rows.table != nullptr ? rows.first_row[act] : rows.first[act];
}
__device__ __forceinline__ ShareRow share_row(const SpkvShareRows& rows, int first, int c, int G, int n_kv_heads, bool ring) {
    ShareRow r;
    const int i = c / G;
    r.head = c - i * G;
    if (rows.in_spans) {                                     // lane k has span k; all lanes of the wave are here
        const SpkvShareSpans& sp = rows.spans;
        const int k = min((int)threadIdx.x & 63, sp.n - 1), start = sp.start[k], shift = sp.row[k] - start;
        int place = 0;
        if (ring) place = rows.t_own[(int)sp.seq[k] * n_kv_heads] - (rows.appended ? sp.start[k + 1] : start);
        r.row = r.place = 0;
        for (int x = 0; x < sp.n; ++x)
            if (first + i >= __builtin_amdgcn_readlane(start, x)) {
                r.row = first + i + __builtin_amdgcn_readlane(shift, x);
                r.place = first + i + __builtin_amdgcn_readlane(place, x);
            }
    } else if (rows.table != nullptr) {
        const int2 e = rows.table[first + i];
        r.row = e.x;
        r.place = e.y;
    } else {
        r.row = rows.seq[first + i];
        r.place = ring ? rows.t_own[r.row * n_kv_heads] - rows.appended : 0;
    }
    return r;
}

struct PromptWork {
    static constexpr bool kTree = false, kPaths = false, kWhole = false;
    static constexpr int parent() { return 0; }
    static constexpr bool drafts() { return false; }
    static constexpr int draft_weight() { return 0; }
    const SpkvShareCut& cut;
    const SpkvShareRows& rows;
    int act, h, pair, range, ranges, block, first;
    __device__ __forceinline__ PromptWork(const SpkvView& v, const SpkvShareCut& c, const SpkvShareTable& table,
                                          const SpkvShareRows& r, int id)
        : cut(c), rows(r) {
        const ShareUnit u = find_unit(cut, table, id, v.Hkv);
        act = u.list / v.Hkv;
        h = u.list - act * v.Hkv;
        range = u.range;
        ranges = u.ranges;
        block = u.block;
        pair = (int)rows.prefix[act] * v.Hkv + h;
    }
    __device__ __forceinline__ int begin(const ShareList& list, int i) const { return list.begin(i, ranges); }
    __device__ __forceinline__ int columns(const SpkvView& v) {
        first = share_first(rows, act);
        return (share_first(rows, act + 1) - first) * v.G;
    }
    __device__ __forceinline__ ShareRow row(const SpkvView& v, int c, bool ring) const {
        return share_row(rows, first, c, v.G, v.Hkv, ring);
    }
    __device__ __forceinline__ float* part(const SpkvView&) const { return cut.part; }
    template <int D>
    __device__ __forceinline__ float2* part_ml(const SpkvView& v) const {
        return reinterpret_cast<float2*>(cut.part + (size_t)v.Hkv * cut.slots * cut.n_cols * D);
    }
    __device__ __forceinline__ size_t part0(const SpkvView& v) const {
        return ((size_t)h * cut.slots + range) * cut.n_cols + (size_t)first * v.G;
    }
};

template <int D, int NQ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, NQ == 1 ? 3 : 2)))
void spkv_prefix_few(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvShareCut cut, SpkvShareTable table,
                     SpkvShareRows rows, SpkvShareOwn own) {
    if ((int)blockIdx.x < own.n_blocks) {
        own_item<D>(own_view(own, v), q, scale_log2e, own.split, own.part,
                    (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
        return;
    }
    PromptWork work(v, cut, table, rows, (int)blockIdx.x - own.n_blocks);
    attend_list_few<D, NQ, 4>(v, q, scale_log2e, work);
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 2 ? 1 : 2, 2)))
void spkv_prefix_split(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvShareCut cut, SpkvShareTable table,
                       SpkvShareRows rows, SpkvShareOwn own) {
    if ((int)blockIdx.x < own.n_blocks) {
        own_item<D>(own_view(own, v), q, scale_log2e, own.split, own.part,
                    (int)blockIdx.x * NW + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
        return;
    }
    __shared__ __attribute__((aligned(16))) uint16_t s_tile[kSplitSlots<NW>][2 * kHalfTokens * D];
    PromptWork work(v, cut, table, rows, (int)blockIdx.x - own.n_blocks);
    attend_list_split<D, NW>(v, q, scale_log2e, work, s_tile);
}

// The join: D / 4 threads own a column (row, head), four consecutive elements each; S such groups share a column,
// each with every S-th of its partial results, and meet in LDS (few columns of many ranges: 512 columns
// of 64 ranges in one group each took 14 us, a chain of eight round trips on a quarter of the chip).  kFold results are loaded
// before any is used.  Call, joins included, with 2 / 5 / 8: one sequence behind 32k (S = 8) 13.2 / 12.5 / 14.0 us, 16 21.4 / 21.4 /
// 25.6; four questions of 512 tokens behind 2k (S = 1, few ranges and many columns) 49.2 / 52.3 / 49.3.
// The sequence's own part is a set of partial results too (own.part), or comes as a call's bf16 output and fp32
// logarithm of its sum: half a step of bf16 more than from sums in 32 bits, on the share that the own tokens have.
template <int D, int S>
__global__ __launch_bounds__(256, 8) void spkv_prefix_merge(SpkvShareCut cut, SpkvShareMerge rows, SpkvShareOwn own, int n_q_heads,
                                                         int n_kv_heads, const uint16_t* own_out, const float* own_lse,
                                                         uint16_t* out, float* lse) {      // (out may be own_out, lse own_lse)
    constexpr int TPC = D / 4, CPB = 256 / TPC, kFold = S > 1 ? 5 : 2, kCols = CPB / S;
    __shared__ f32x4 s_num[S > 1 ? CPB : 1][S > 1 ? TPC : 1];
    __shared__ float2 s_ml[S > 1 ? CPB : 1];
    const int slice = (int)threadIdx.x / TPC, share = slice % S, d = ((int)threadIdx.x % TPC) * 4;
    // a workgroup's columns are heads of one row: what belongs to the row is looked up once, in scalar registers
    const int per_row = (n_q_heads + kCols - 1) / kCols, row = (int)blockIdx.x / per_row;
    const int head0 = ((int)blockIdx.x - row * per_row) * kCols;
    const bool exists = head0 + slice / S < n_q_heads;
    const int G = n_q_heads / n_kv_heads, head = exists ? head0 + slice / S : head0, h = head / G, g = head - h * G;
    const int64_t id = (int64_t)row * n_q_heads + head;
    int act, at;
    if (rows.in_spans) {                                     // the span that holds the row, if any
        const SpkvShareSpans& sp = rows.spans;
        const int lane = (int)threadIdx.x & 63, k = max(min(lane, sp.n - 1), 0), off = row - sp.row[k];
        const unsigned long long here = __ballot(lane < sp.n && off >= 0 && off < sp.start[k + 1] - sp.start[k]);
        const int x = here != 0ull ? __builtin_ctzll(here) : 0;
        act = here != 0ull ? (int)sp.act[x] : -1;
        at = sp.start[x] + row - sp.row[x];
    } else if (rows.by_row != nullptr) {
        const int2 e = rows.by_row[row];
        act = e.x;
        at = e.y;
    } else {
        act = rows.active[row];
        at = rows.place[row];
    }
    float M = SPKV_NEG_INF, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    const int h_first = head0 / G, h_last = (min(head0 + kCols, n_q_heads) - 1) / G;      // (one, or the table is asked per lane)
    const int ranges = act < 0 ? 0 : cut.whole != 0 ? 1
                     : h_first == h_last ? rows.ranges[act * n_kv_heads + h_first] : rows.ranges[act * n_kv_heads + h];
    const int pair = row * n_kv_heads + h, parts = ranges + (own.part != nullptr ? own_ranges(own, pair) : 0);
    if (own.part == nullptr && share == 0 && exists) {
        const uint2 ob = *reinterpret_cast<const uint2*>(own_out + id * D + d);
        const float z = own_lse[id];
        if (ranges == 0) {                                   // no prompt: the own part as it is
            *reinterpret_cast<uint2*>(out + id * D + d) = ob;
            if (lse != nullptr && d == 0) lse[id] = z;
        }
        if (z != SPKV_NEG_INF) {                             // (a NaN shows)
            M = z * 1.4426950408889634f;
            den = 1.f;
            num = (f32x4){__builtin_bit_cast(float, ob.x << 16), __builtin_bit_cast(float, ob.x & 0xffff0000u),
                          __builtin_bit_cast(float, ob.y << 16), __builtin_bit_cast(float, ob.y & 0xffff0000u)};
        }
    }
    // partial results, the prompt's and then the own ones, kFold at a time: their loads in flight together, only the
    // rescaling is chained
    const float2* ml = reinterpret_cast<const float2*>(cut.part + (size_t)n_kv_heads * cut.slots * cut.n_cols * D);
    const float2* own_ml = reinterpret_cast<const float2*>(own.part + own.n_floats);
    const size_t prompt0 = (size_t)h * cut.slots * cut.n_cols + (size_t)at * G + g, own0 = (size_t)pair * own.split.slots * G + g;
    for (int r0 = share; r0 < parts; r0 += kFold * S) {
        float2 x[kFold];
        f32x4 a[kFold];
#pragma unroll
        for (int u = 0; u < kFold; ++u) {
            const int r = min(r0 + u * S, parts - 1);        // past the end: re-read, ignored
            const bool mine = r >= ranges;
            const size_t pc = mine ? own0 + (size_t)(r - ranges) * G : prompt0 + (size_t)r * cut.n_cols;
            x[u] = (mine ? own_ml : ml)[pc];
            a[u] = *reinterpret_cast<const f32x4*>((mine ? own.part : cut.part) + pc * D + d);
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
    if (!exists || (ranges == 0 && own.part == nullptr)) return;
    const float inv = den == 0.f ? 0.f : 1.0f / den;         // (a row that sees no key at all: zeros; a NaN shows)
    uint2 packed;
    packed.x = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[0] * inv)) |
               ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[1] * inv)) << 16);
    packed.y = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[2] * inv)) |
               ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[3] * inv)) << 16);
    *reinterpret_cast<uint2*>(out + id * D + d) = packed;
    if (lse != nullptr && d == 0) lse[id] = den == 0.f ? SPKV_NEG_INF : (M + log2f(den)) * 0.6931471805599453f;
}

// Rows of a call with several tokens a sequence, grouped by prompt: one workgroup per sequence.
//   table[i]   (row, place of its token in the sequence) of the i-th row in the order of the prompts
//   by_row[r]  (active prompt or -1, i)
//   first_row  [n_active + 1]
__global__ __launch_bounds__(256) void spkv_prefix_rows(SpkvCu cu, SpkvShareActive a, const int32_t* __restrict__ t_own,
                                                        int n_seq, int n_kv_heads, int appended, int n_active,
                                                        int2* table, int2* by_row, int32_t* first_row) {
    __shared__ int s_sum[4];
    const int b = blockIdx.x, tid = threadIdx.x;
    auto sum = [&](int act, int until) -> int {              // rows of the prompts before act, and of act's sequences before `until`
        int s = 0;
        for (int i = tid; i < n_seq; i += 256) {
            const int x = a.active[i];
            if (x >= 0 && (x < act || (x == act && i < until))) s += cu.v[i + 1] - cu.v[i];
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
        __syncthreads();
        if ((tid & 63) == 0) s_sum[tid >> 6] = s;
        __syncthreads();
        return (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    };
    const int row0 = cu.v[b], n = cu.v[b + 1] - row0, act = a.active[b];
    const int at = sum(act, b);
    if (act < 0) {
        for (int i = tid; i < n; i += 256) by_row[row0 + i] = make_int2(-1, 0);
    } else {
        const int place0 = t_own[b * n_kv_heads] - (appended ? n : 0);
        for (int i = tid; i < n; i += 256) {
            table[at + i] = make_int2(row0 + i, place0 + i);
            by_row[row0 + i] = make_int2(act, at + i);
        }
    }
    if (b == 0)
        for (int x = 0; x <= n_active; ++x) {
            const int s = sum(x, 0);
            if (tid == 0) first_row[x] = s;
        }
}

int spkv_prefix_groups(int n_cols) { return n_cols <= 16 ? 1 : n_cols <= 32 ? 2 : n_cols <= 64 ? 4 : n_cols <= 128 ? 8 : 16; }

constexpr int kMergeRound = 2048;
int spkv_prefix_kernel_waves(int groups) { return groups == 16 ? 8 : groups == 4 ? 2 : 4; }

template <int D>
static hipError_t launch_prefix(const SpkvView& v, const uint16_t* q, float sl, int groups, const SpkvShareCut& cut,
                                const SpkvShareTable& table, const SpkvShareRows& rows, const SpkvShareMerge& merge,
                                SpkvShareOwn own, const uint16_t* own_out, const float* own_lse, uint16_t* out, float* lse,
                                hipStream_t s) {
    const int items = own.part != nullptr ? own.n_pairs * own.split.slots : 0, waves = spkv_prefix_kernel_waves(groups);
    own.n_blocks = (items + waves - 1) / waves;
    const dim3 grid((unsigned)(own.n_blocks + cut.n_units)), block(64 * waves);
    if (grid.x > 0) {
        if (groups == 16) spkv_prefix_split<D, 8><<<grid, block, 0, s>>>(v, q, sl, cut, table, rows, own);
        else if (groups == 8) spkv_prefix_split<D, 4><<<grid, block, 0, s>>>(v, q, sl, cut, table, rows, own);
        else if (groups == 4) spkv_prefix_split<D, 2><<<grid, block, 0, s>>>(v, q, sl, cut, table, rows, own);
        else if (groups == 2) spkv_prefix_few<D, 2><<<grid, block, 0, s>>>(v, q, sl, cut, table, rows, own);
        else spkv_prefix_few<D, 1><<<grid, block, 0, s>>>(v, q, sl, cut, table, rows, own);
    }
    // groups to a column: as many as one round of workgroups (eight on a compute unit) leaves room for, no more than
    // there are ranges
    constexpr int CPB = 256 / (D / 4);
    const int64_t rows_out = cut.n_out / v.Hq;
    int share = 8;
    while (share > 1 && (rows_out * ((v.Hq * share + CPB - 1) / CPB) > kMergeRound || share > cut.slots)) share >>= 1;
    const int cols = CPB / share;
    const dim3 merge_grid((unsigned)(rows_out * ((v.Hq + cols - 1) / cols)));
    if (share == 8) spkv_prefix_merge<D, 8><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    else if (share == 4) spkv_prefix_merge<D, 4><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    else if (share == 2) spkv_prefix_merge<D, 2><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    else spkv_prefix_merge<D, 1><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    return hipGetLastError();
}

hipError_t spkv_launch_prefix(const SpkvView& v, const uint16_t* q, float sm_scale, int groups, const SpkvShareCut& cut,
                              const SpkvShareTable& table, const SpkvShareRows& rows, const SpkvShareMerge& merge,
                              const SpkvShareOwn& own, const uint16_t* own_out, const float* own_lse, uint16_t* out,
                              float* lse, hipStream_t s) {
    const float sl = sm_scale * 1.4426950408889634f;
    return v.D == 128 ? launch_prefix<128>(v, q, sl, groups, cut, table, rows, merge, own, own_out, own_lse, out, lse, s)
                      : launch_prefix<64>(v, q, sl, groups, cut, table, rows, merge, own, own_out, own_lse, out, lse, s);
}

hipError_t spkv_launch_prefix_rows(const SpkvCu& cu, const SpkvShareActive& a, const int32_t* t_own, int n_seq,
                                   int n_kv_heads, bool appended, int n_active, int32_t* table, int32_t* by_row,
                                   int32_t* first_row, hipStream_t s) {
    spkv_prefix_rows<<<dim3((unsigned)n_seq), dim3(256), 0, s>>>(cu, a, t_own, n_seq, n_kv_heads, appended ? 1 : 0,
                                                                 n_active, reinterpret_cast<int2*>(table),
                                                                 reinterpret_cast<int2*>(by_row), first_row);
    return hipGetLastError();
}
