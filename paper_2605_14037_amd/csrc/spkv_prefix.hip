// Attention over shared prompts on gfx950: sequences that continue the same prompt read its lists
// once for all of them, and the result is joined with what they attend to of their own.
#include "spkv_device.h"

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
constexpr float kSumLimit = 2048.0f;         // a sum of 16 weights above it: the reference is too low

// Bits e = 0 .. 7 with e < n, with e >= n.
__device__ __forceinline__ unsigned bits_below(int n) { return 0xffu >> (8 - min(max(n, 0), 8)); }
__device__ __forceinline__ unsigned bits_from(int n) { return bits_below(n) ^ 0xffu; }

// One prompt's list and ring for a workgroup: half-pages 0 .. nA - 1 are the list's, then those of the ring.
struct ShareList {
    int pair, T, L, held, nA, n_hp;
    int slot0;                  // ring slot of age 0 (negative while the ring is not full)
    // Begin of the j-th of n ranges.  A half-page of the ring counts twice: its mask takes about as long as its
    // products (16 sequences behind 30 MB of lists: workgroups with the ring 3.5 us behind the others, of 16).
    __device__ __forceinline__ int begin(int j, int n) const {
        const int x = (int)((int64_t)j * (2 * n_hp - nA) / n);
        return x <= nA ? x : nA + (x - nA + 1) / 2;
    }
};
__device__ __forceinline__ ShareList share_list(const SpkvView& v, int pair) {
    ShareList s;
    s.pair = pair;
    s.T = v.t_pair[pair];
    s.L = v.kept_len[pair];
    s.held = min(s.T, v.w);
    s.nA = (s.L + kHalfTokens - 1) >> 5;
    s.n_hp = s.nA + ((s.held + kHalfTokens - 1) >> 5);
    s.slot0 = s.T >= v.w ? s.T % v.w : s.T - v.w;
    return s;
}
// Does the ring's slot hold a key that passes the gate?
__device__ __forceinline__ bool ring_gate(const SpkvView& v, const ShareList& s, int at) {
    const int age = at - s.slot0 + (at < s.slot0 ? v.w : 0);
    return gate_passes(v, v.ring_logit[(size_t)s.pair * v.w + at], s.T - v.w + age);
}
// Keys at0 .. at0 + 7 of the ring that a token at `place` sees: gate on, or of an age above its place (a run of
// slots from slot0 + place + 1 on, modulo w).
__device__ __forceinline__ unsigned ring_seen(const SpkvView& v, const ShareList& s, unsigned gates, int at0, int place) {
    const int from = s.slot0 + place + 1 - at0;
    return (gates | bits_from(from) | (bits_from(from - v.w) & bits_below(s.slot0 - at0))) & bits_below(s.held - at0);
}
// Gates of a wave's ring half-pages, lane t those of half-page ring0 + t; loads four at a time.
constexpr int kRingGateTiles = 64;
struct RingGates {
    int ring0;
    unsigned mine;
};
__device__ __forceinline__ RingGates ring_gates(const SpkvView& v, const ShareList& s, int x_begin, int x_end) {
    RingGates r = {max(x_begin - s.nA, 0), 0u};
    const int lane = threadIdx.x & 63, n = min(x_end - s.nA - r.ring0, kRingGateTiles);
    for (int t = 0; t < n; t += 8) {
        bool on[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) on[u] = ring_gate(v, s, min((r.ring0 + t + 2 * u) * kHalfTokens + lane, s.held - 1));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const unsigned long long gates = __ballot(on[u]);
            if (lane == t + 2 * u) r.mine = (unsigned)gates;
            if (lane == t + 2 * u + 1) r.mine = (unsigned)(gates >> 32);
        }
    }
    return r;
}
// Gates (bits 0 .. 7) of ring half-page t's keys k0 .. k0 + 7, t wave-uniform.
__device__ __forceinline__ unsigned gates_of(const SpkvView& v, const ShareList& s, const RingGates& r, int t, int k0) {
    if (t - r.ring0 < kRingGateTiles)
        return ((unsigned)__builtin_amdgcn_readlane((int)r.mine, t - r.ring0) >> k0) & 0xffu;
    unsigned g = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (ring_gate(v, s, min(t * kHalfTokens + k0 + e, s.held - 1))) g |= 1u << e;
    return g;
}
// Page ids of a list, 64 at a time, one a lane.  The first 256 of the list are sent for before its length is known
// (share_pages) and those from the range's begin on picked from them.
struct SharePages {
    const int32_t* pt;
    int cap, at, ids;           // ids: of pages at .. at + 63
};
__device__ __forceinline__ int page_at(SharePages& p, int lp) {               // lp wave-uniform, never decreasing
    if (lp >= p.at + 64) {
        p.at = lp;
        p.ids = p.pt[min(lp + ((int)threadIdx.x & 63), p.cap - 1)];
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0)
    }
    return __builtin_amdgcn_readlane(p.ids, lp - p.at);
}
struct FirstPages {
    int a, b, c, d;             // pages 0 .., 64 .., 128 .., 192 ..
};
__device__ __forceinline__ FirstPages first_pages(const SpkvView& v, int pair) {
    const int32_t* pt = v.page_table + (size_t)pair * v.pt_cap;
    const int lane = threadIdx.x & 63, end = v.pt_cap - 1;
    return FirstPages{pt[min(lane, end)], pt[min(64 + lane, end)], pt[min(128 + lane, end)], pt[min(192 + lane, end)]};
}
__device__ __forceinline__ SharePages share_pages(const SpkvView& v, int pair, FirstPages f, int from) {
    SharePages p = {v.page_table + (size_t)pair * v.pt_cap, v.pt_cap, from, 0};
    const int lp = from + ((int)threadIdx.x & 63), block = from >> 6;        // pages lp lie in two blocks of 64
    if (block >= 3) {
        p.ids = p.pt[min(lp, p.cap - 1)];
        return p;
    }
    const int x = block == 0 ? f.a : block == 1 ? f.b : f.c, y = block == 0 ? f.b : block == 1 ? f.c : f.d;
    const int xs = __shfl(x, lp & 63), ys = __shfl(y, lp & 63);
    p.ids = (lp >> 6) == block ? xs : ys;
    return p;
}
__device__ __forceinline__ const uint16_t* half_page_at(const SpkvView& v, const ShareList& s, SharePages& p, int x) {
    const int half = 2 * kHalfTokens * v.D;
    if (x < s.nA) return pool_page(v, min(max(page_at(p, x >> 1), 0), v.n_pages - 1)) + (x & 1) * half;
    return ring_page(v, s.pair, (x - s.nA) >> 1) + ((x - s.nA) & 1) * half;
}
// 16 bytes of V, eight consecutive keys: those whose bit is not set to zero -- no column sees them, and a weight of
// zero would turn an infinity among them into a NaN.
__device__ __forceinline__ bf16x8 keep_keys(bf16x8 x, unsigned seen) {
    uint4 u = __builtin_bit_cast(uint4, x);
    u.x &= (seen & 1u ? 0xffffu : 0u) | (seen & 2u ? 0xffff0000u : 0u);
    u.y &= (seen & 4u ? 0xffffu : 0u) | (seen & 8u ? 0xffff0000u : 0u);
    u.z &= (seen & 16u ? 0xffffu : 0u) | (seen & 32u ? 0xffff0000u : 0u);
    u.w &= (seen & 64u ? 0xffffu : 0u) | (seen & 128u ? 0xffff0000u : 0u);
    return __builtin_bit_cast(bf16x8, u);
}

// Where some columns of a wave see a ring key and others do not, an infinity or NaN among its values reaches the others
// too, with a weight of zero.  A column whose sums are not finite though its weights are, in a range with such keys, is
// summed up once more, key by key (careful_sums).  Calls, so that the loops keep their registers: with the
// values looked at and set aside on the way 64 sequences behind 128k took 50.7 us instead of 45.8.  (An infinity that all
// columns see may come out as a NaN: the second part of its weight may be negative.)
struct CarefulRange {
    const uint16_t *pool, *ring;        // pages: of the pool, of this list's ring
    const float* logit;                 // of the ring
    const int32_t* pages;               // of the list
    float theta, scale_log2e;
    int n_sink, w, n_pages, T, L, held, nA, slot0, x_begin, x_end;
};
__device__ __forceinline__ CarefulRange careful_range(const SpkvView& v, const ShareList& s, float scale_log2e, int x_begin,
                                                      int x_end) {
    return CarefulRange{v.pool, ring_page(v, s.pair, 0), v.ring_logit + (size_t)s.pair * v.w, v.page_table + (size_t)s.pair * v.pt_cap,
                        v.theta, scale_log2e, v.n_sink, v.w, v.n_pages, s.T, s.L, s.held, s.nA, s.slot0, x_begin, x_end};
}
__device__ __forceinline__ bool careful_seen(const CarefulRange& r, int at, int place) {          // the ring's slot, by a token there
    const int age = at - r.slot0 + (at < r.slot0 ? r.w : 0);
    return age > place || r.logit[at] >= r.theta || r.T - r.w + age < r.n_sink;
}
__device__ __forceinline__ float bf16_at(const uint16_t* p) { return __builtin_bit_cast(float, (unsigned)*p << 16); }
// Is there a key that a token at `least` sees and one at `most` does not, with a value that is not finite?  (The whole wave.)
template <int D>
__device__ __attribute__((noinline)) bool careful_needed(CarefulRange r, int least, int most) {
    bool odd = false;
    for (int at = max(r.x_begin - r.nA, 0) * kHalfTokens; at < min((r.x_end - r.nA) * kHalfTokens, r.held); ++at) {
        if (!careful_seen(r, at, least) || careful_seen(r, at, most)) continue;
        for (int d = threadIdx.x & 63; d < D; d += 64) {
            const float x = bf16_at(r.ring + (size_t)(at >> 6) * spkv_page_elems(D) + spkv_v_off(D, at & 63, d));
            odd = odd || !(x - x == 0.f);
        }
    }
    return __ballot(odd) != 0ull;
}
// Sums of the range for the column of a query row (in memory) and place, against its reference m.  (The whole wave.)
template <int D>
__device__ __attribute__((noinline)) void careful_sums(CarefulRange r, const uint16_t* qrow, int place, float m, float* sums) {
    const int lane = threadIdx.x & 63;
    float q[D / 64], acc[D / 64];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
        q[e] = bf16_at(qrow + e * 64 + lane);
        acc[e] = 0.f;
    }
    const int end = r.nA * kHalfTokens;                      // place of the ring's slots in the numbering of keys below
    for (int k = r.x_begin * kHalfTokens; k < r.x_end * kHalfTokens; ++k) {
        const uint16_t* page;
        if (k < end) {
            if (k >= r.L) continue;
            page = r.pool + (size_t)min(max(r.pages[k >> 6], 0), r.n_pages - 1) * spkv_page_elems(D);
        } else {
            if (k - end >= r.held || !careful_seen(r, k - end, place)) continue;
            page = r.ring + (size_t)((k - end) >> 6) * spkv_page_elems(D);
        }
        const int in = (k < end ? k : k - end) & 63;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) x += q[e] * bf16_at(page + spkv_k_off(D, in, e * 64 + lane));
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, r.scale_log2e, -m));
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] += p * bf16_at(page + spkv_v_off(D, in, e * 64 + lane));
    }
#pragma unroll
    for (int e = 0; e < D / 64; ++e) sums[e * 64 + lane] = acc[e];
}
// Are the weights' sum finite and the n sums not?  (0 * x is a NaN where x is not finite.)
template <class Acc>
__device__ __forceinline__ bool odd_sums(const Acc* acc, int n, float l) {
    Acc t = acc[0] * 0.f;
#pragma unroll
    for (int i = 1; i < n; ++i) t += acc[i] * 0.f;
    float sum = t[0];
#pragma unroll
    for (int e = 1; e < (int)(sizeof(Acc) / sizeof(float)); ++e) sum += t[e];
    return sum != 0.f && l - l == 0.f;
}

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

// The query row of column c of an active prompt, its head in the group, and its token's place in the sequence
// (looked for only where the ring is read).  Columns past the last one repeat the first and are never stored.
struct ShareRow {
    int row, head, place;
};
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

// Up to 16 NQ columns.  A half-page's operands come straight from memory (1 KB a load, as in spkv_decode_split) and are
// used for all NQ groups of 16 columns: scores of all groups -- the next half-page's keys are sent for -- then
// weights against the references as they stand -- raised, and sums and accumulators rescaled, only where some lane's
// eight weights add up to more than kSumLimit -- then the products with V, the weights as two bf16 parts (16 bits: the
// lists' read takes the time, not these products) -- and the next values are sent for.  One body for every half-page:
// two of them in turn on two sets of operands were slower where a wave has only a few (cold instructions).  The four
// waves take a quarter of the range each and meet in LDS.
template <int D, int NQ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, NQ == 1 ? 3 : 2)))
void spkv_prefix_few(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvShareCut cut, SpkvShareTable table,
                     SpkvShareRows rows, SpkvShareOwn own) {
    constexpr int NS = D / 32, NB = D / 16, kRow = D + 4;
    __shared__ __attribute__((aligned(16))) float s_acc[4][16 * NQ * kRow];
    __shared__ float2 s_ml[4][16 * NQ];
    __shared__ __attribute__((aligned(16))) uint16_t s_q[NQ == 1 ? 1 : NQ * NS][512];
    const int tid = threadIdx.x, lane = tid & 63, kc = lane >> 4, n = lane & 15;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    if ((int)blockIdx.x < own.n_blocks) {
        own_item<D>(own_view(own, v), q, scale_log2e, own.split, own.part, (int)blockIdx.x * 4 + wv);
        return;
    }
    const ShareUnit u = find_unit(cut, table, (int)blockIdx.x - own.n_blocks, v.Hkv);
    const int act = u.list / v.Hkv, h = u.list - act * v.Hkv, j = u.range, ranges = u.ranges;
    const int pair = (int)rows.prefix[act] * v.Hkv + h;
    const FirstPages first_ids = first_pages(v, pair);
    const ShareList list = share_list(v, pair);
    const int first = share_first(rows, act), n_cols = (share_first(rows, act + 1) - first) * v.G;
    if (n_cols <= 0) return;
    const int nA = list.nA;
    const int r_begin = list.begin(j, ranges), r_end = list.begin(j + 1, ranges);
    const int x_begin = r_begin + (r_end - r_begin) * wv / 4, x_end = r_begin + (r_end - r_begin) * (wv + 1) / 4;

    SharePages pages = share_pages(v, pair, first_ids, x_begin >> 1);
    bf16x8 k[2][NS], va[NB];
    auto load_k = [&](const uint16_t* page) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) k[i][sl] = load_stream_b128(page + lane * 8 + (i * (D / 8) + sl * 4) * 128);
    };
    auto load_v = [&](const uint16_t* page) {
#pragma unroll
        for (int db = 0; db < NB; ++db) va[db] = load_stream_b128(page + kHalfTokens * D + lane * 8 + db * 512);
    };
    bf16x8 q1[NQ == 1 ? NS : 1];                             // the query operands of one group; of several they lie in LDS
    int place[NQ], least = 0, most = 0;                      // of the wave's columns, the smallest sees most of the ring
    const bool ring = x_end > nA;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int c = i * 16 + n;
        const ShareRow sr = share_row(rows, first, c < n_cols ? c : 0, v.G, v.Hkv, ring);
        place[i] = sr.place;
        const uint16_t* qrow = q + ((size_t)sr.row * v.Hq + (size_t)h * v.G + sr.head) * D + kc * 8;
        if (NQ == 1) {
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) q1[NQ == 1 ? sl : 0] = *reinterpret_cast<const bf16x8*>(qrow + sl * 32);
        } else if (i % 4 == wv % NQ) {                       // a wave's share of the groups (NQ = 2: two waves the same)
#pragma unroll
            for (int sl = 0; sl < NS; ++sl)
                *reinterpret_cast<bf16x8*>(&s_q[NQ == 1 ? 0 : i * NS + sl][lane * 8]) = *reinterpret_cast<const bf16x8*>(qrow + sl * 32);
        }
    }
    if (x_begin < x_end) {
        const uint16_t* page = half_page_at(v, list, pages, x_begin);
        load_k(page);
        load_v(page);
    }
    if (NQ > 1) __syncthreads();
    RingGates gates = {0, 0u};
    if (ring) {
        gates = ring_gates(v, list, x_begin, x_end);
        least = most = place[0];
#pragma unroll
        for (int i = 1; i < NQ; ++i) {
            least = min(least, place[i]);
            most = max(most, place[i]);
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            least = min(least, __shfl_xor(least, o));
            most = max(most, __shfl_xor(most, o));
        }
        least = __builtin_amdgcn_readfirstlane(least);
        most = __builtin_amdgcn_readfirstlane(most);
    }
    f32x4 acc[NQ][NB];
    float m[NQ], l[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        m[i] = SPKV_NEG_INF;
        l[i] = 0.f;
#pragma unroll
        for (int db = 0; db < NB; ++db) acc[i][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const int full = list.L >> 5;                            // half-pages that need no mask
#pragma unroll 1
    for (int x = x_begin; x < x_end; ++x) {
        const bool more = x + 1 < x_end;
        const uint16_t* next = more ? half_page_at(v, list, pages, x + 1) : nullptr;
        f32x8 s[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) {
                const bf16x8 qb = NQ == 1 ? q1[NQ == 1 ? sl : 0]
                                          : *reinterpret_cast<const bf16x8*>(&s_q[NQ == 1 ? 0 : i * NS + sl][lane * 8]);
                s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[0][sl], qb, s0, 0, 0, 0);
                s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[1][sl], qb, s1, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[i][e] = s0[e];
                s[i][4 + e] = s1[e];
            }
        }
        if (more) load_k(next);
        if (x >= full) {
            unsigned any, on = 0u;
            const int at0 = (x - nA) * kHalfTokens + kc * 8;
            if (x < nA) any = bits_below(list.L - x * kHalfTokens - kc * 8);
            else any = ring_seen(v, list, on = gates_of(v, list, gates, x - nA, kc * 8), at0, least);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const unsigned ok = x < nA ? any : ring_seen(v, list, on, at0, place[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[i][e] = ((ok >> e) & 1u) ? s[i][e] : SPKV_NEG_INF;
            }
#pragma unroll
            for (int db = 0; db < NB; ++db) va[db] = keep_keys(va[db], any);
        }
        f32x8 p[NQ];
        float psum[NQ];
        auto weights = [&]() -> bool {
            bool low = false;
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const bool unset = m[i] == SPKV_NEG_INF;
                const float neg_ref = unset ? 0.f : -m[i];
#pragma unroll
                for (int e = 0; e < 8; ++e) p[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], scale_log2e, neg_ref));
                psum[i] = ((p[i][0] + p[i][1]) + (p[i][2] + p[i][3])) + ((p[i][4] + p[i][5]) + (p[i][6] + p[i][7]));
                low = low || unset || !(psum[i] <= kSumLimit);
            }
            return __ballot(low) != 0ull;
        };
#pragma unroll 1
        for (bool again = true; weights() && again; again = false) {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                float cm = fmaxf(fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3])),
                                 fmaxf(fmaxf(s[i][4], s[i][5]), fmaxf(s[i][6], s[i][7]))) * scale_log2e;
                cm = fmaxf(cm, __shfl_xor(cm, 16));
                cm = fmaxf(cm, __shfl_xor(cm, 32));
                const float m_new = fmaxf(m[i], cm);
                // (no key so far: the reference stays unset, sums and accumulators are zero)
                const float alpha = __builtin_amdgcn_exp2f(m[i] - (m_new == SPKV_NEG_INF ? 0.f : m_new));
                m[i] = m_new;
                l[i] *= alpha;
                if (x > x_begin) {
#pragma unroll
                    for (int db = 0; db < NB; ++db) acc[i][db] *= alpha;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            l[i] += psum[i];
            const bf16x8 hi = __builtin_convertvector(p[i], bf16x8);
            const bf16x8 lo = __builtin_convertvector(p[i] - __builtin_convertvector(hi, f32x8), bf16x8);
#pragma unroll
            for (int db = 0; db < NB; ++db) acc[i][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[db], hi, acc[i][db], 0, 0, 0);
#pragma unroll
            for (int db = 0; db < NB; ++db) acc[i][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[db], lo, acc[i][db], 0, 0, 0);
        }
        if (more) load_v(next);
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        l[i] += __shfl_xor(l[i], 16);
        l[i] += __shfl_xor(l[i], 32);
        float* pa = s_acc[wv] + (i * 16 + n) * kRow + kc * 4;
#pragma unroll
        for (int db = 0; db < NB; ++db) *reinterpret_cast<f32x4*>(pa + db * 16) = acc[i][db];
        if (kc == 0) s_ml[wv][i * 16 + n] = make_float2(m[i], l[i]);
    }
    if (ring && least != most) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NQ; ++i) odd = odd || odd_sums(acc[i], NB, l[i]);
        if (__builtin_expect(__ballot(odd) != 0ull, 0)) {
            const CarefulRange range = careful_range(v, list, scale_log2e, x_begin, x_end);
            if (careful_needed<D>(range, least, most))
                for (int c = 0; c < min(16 * NQ, n_cols); ++c) {
                    const ShareRow sr = share_row(rows, first, c, v.G, v.Hkv, true);
                    __builtin_amdgcn_wave_barrier();
                    careful_sums<D>(range, q + ((size_t)sr.row * v.Hq + (size_t)h * v.G + sr.head) * D, sr.place, s_ml[wv][c].x,
                                    s_acc[wv] + c * kRow);
                }
        }
    }
    __syncthreads();
    const size_t pc0 = ((size_t)h * cut.slots + j) * cut.n_cols + (size_t)first * v.G;
    float2* part_ml = reinterpret_cast<float2*>(cut.part + (size_t)v.Hkv * cut.slots * cut.n_cols * D);
    for (int e = tid; e < n_cols * (D / 4); e += 256) {
        const int c = e / (D / 4), d = (e - c * (D / 4)) * 4;
        float2 ml[4];
        float M = SPKV_NEG_INF;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            ml[w] = s_ml[w][c];
            M = fmaxf(M, ml[w].x);
        }
        const float m_ref = M == SPKV_NEG_INF ? 0.f : M;     // no key at all: every weight 0
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float sc = __builtin_amdgcn_exp2f(ml[w].x - m_ref);
            a += *reinterpret_cast<const f32x4*>(s_acc[w] + c * kRow + d) * sc;
            sum += ml[w].y * sc;
        }
        *reinterpret_cast<f32x4*>(cut.part + (pc0 + c) * D + d) = a;
        if (d == 0) part_ml[pc0 + c] = make_float2(M, sum);
    }
}

// More columns: the copies of the range's half-pages go from memory straight into LDS, in operand order, so that
// every wave reads its operands as 1 KB in lane order.  The products K Q^T of a half-page stand beside the
// weights of the one before.  Eight waves fetch two half-pages to a step (as spkv_prefill_attend32, whose
// pipeline this is); with fewer waves a step is one half-page and two workgroups share a compute unit.  The weights go
// into the second product as one bf16 part, half a step (2^-8) at most each, their sum in 32 bits: from 33 columns on the
// products count, and a second part would be half as many again (errors against 64 bits 2.3e-3 of the 2-norm instead of 1.7e-3).

template <int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 2 ? 1 : 2, 2)))
void spkv_prefix_split(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvShareCut cut, SpkvShareTable table,
                       SpkvShareRows rows, SpkvShareOwn own) {
    constexpr int NS = D / 16, NB = D / 32;
    constexpr int kHalfElems = 2 * kHalfTokens * D;
    constexpr int kHps = NW == 8 ? 2 : 1;                    // half-pages to a step
    constexpr int kSlots = NW == 8 ? 8 : 5;                  // half-pages in LDS
    constexpr int kRowsPerWave = kHps * (D / 8) / NW;        // 1 KB rows of a step that a wave copies
    __shared__ __attribute__((aligned(16))) uint16_t s_tile[kSlots][kHalfElems];
    if ((int)blockIdx.x < own.n_blocks) {
        own_item<D>(own_view(own, v), q, scale_log2e, own.split, own.part,
                    (int)blockIdx.x * NW + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
        return;
    }
    const ShareUnit u = find_unit(cut, table, (int)blockIdx.x - own.n_blocks, v.Hkv);
    const int act = u.list / v.Hkv, h = u.list - act * v.Hkv, j = u.range, ranges = u.ranges;
    const int pair = (int)rows.prefix[act] * v.Hkv + h;
    const FirstPages first_ids = first_pages(v, pair);
    const ShareList list = share_list(v, pair);
    const int first = share_first(rows, act), n_cols = (share_first(rows, act + 1) - first) * v.G;
    const int col0 = u.block * (32 * NW);
    if (col0 >= n_cols) return;
    const int nA = list.nA;
    const int x_begin = list.begin(j, ranges), x_end = list.begin(j + 1, ranges), last = x_end - 1;

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = col0 + wv * 32 + col;
    const bool valid = c < n_cols;
    const size_t pc = ((size_t)h * cut.slots + j) * cut.n_cols + (size_t)first * v.G + c;      // of the partial result
    float2* part_ml = reinterpret_cast<float2*>(cut.part + (size_t)v.Hkv * cut.slots * cut.n_cols * D);
    if (x_begin >= x_end) {                                  // fewer half-pages than ranges
        if (valid && half == 0) part_ml[pc] = make_float2(SPKV_NEG_INF, 0.f);
        return;
    }
    const ShareRow sr = share_row(rows, first, valid ? c : 0, v.G, v.Hkv, x_end > nA);
    SharePages pages = share_pages(v, pair, first_ids, x_begin >> 1);
    bf16x8 qb[NS];
    {
        const uint16_t* qrow = q + ((size_t)sr.row * v.Hq + (size_t)h * v.G + sr.head) * D + half * 8;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) qb[sl] = *reinterpret_cast<const bf16x8*>(qrow + sl * 16);
    }
    auto base_of = [&](int x) -> const uint16_t* { return half_page_at(v, list, pages, min(x, last)); };

    // A half-page's rows in LDS: K row sl holds, for lane (half, r), d = 16 sl + 8 half .. of key 16 (r >> 4) +
    // 8 ((r >> 2) & 1) + 4 ((r >> 3) & 1) + (r & 3) -- the score of row r of an MFMA then comes out in the
    // register and lane in which the product with V wants the weight of that key; V row (g, db) holds
    // keys 16 g + 8 half .. + 7 of d = 32 db + r.  Waves take consecutive rows, so all of K or all of V.
    const int wq = wv % (NW / kHps), wh = wv / (NW / kHps);  // share of a half-page, half-page of the step
    const unsigned k_lane = ((((col >> 3) & 1) * (D / 8) + half) * 16 + 8 * (col >> 4) + 4 * ((col >> 2) & 1) + (col & 3)) * 16;
    const unsigned v_lane = (((col >> 4) * 4 + half) * 16 + (col & 15)) * 16 + kHalfTokens * D * 2;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)&s_tile[0][0];
    auto stage_half_page_rows = [&](const uint16_t* base, int slot) {
        const unsigned dst = lds0 + (unsigned)slot * (kHalfElems * 2);
#pragma unroll
        for (int i = 0; i < kRowsPerWave; ++i) {
            const int row_id = wq * kRowsPerWave + i;
            const bool is_k = wq * kRowsPerWave < NS;
            const int vr = row_id - NS, off = is_k ? row_id * 512 : (vr / NB) * 512 + (vr % NB) * 2048;
            load_row_to_lds(reinterpret_cast<const char*>(base) + off, is_k ? k_lane : v_lane, dst + row_id * 1024);
        }
    };
    auto stage_step = [&](int k, int slot) {                 // half-page k of the range (and the one behind it)
        if (kHps == 2) stage_half_page_rows(base_of(x_begin + k + wh), slot + wh);
        else stage_half_page_rows(base_of(x_begin + k), slot);
    };

    // The tiles of the first steps travel with the queries.  Step s + kAhead is sent off in step s.
    constexpr int kAhead = NW == 8 ? 3 : 4;
#pragma unroll
    for (int s = 0; s < kAhead; ++s) stage_step(s * kHps, s * kHps);
    RingGates gates = {0, 0u};
    int least = 0, most = 0;                                 // places of the wave's columns: the smallest sees most of the ring
    if (x_end > nA) {
        gates = ring_gates(v, list, x_begin, x_end);
        least = most = sr.place;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            least = min(least, __shfl_xor(least, o));
            most = max(most, __shfl_xor(most, o));
        }
        least = __builtin_amdgcn_readfirstlane(least);
        most = __builtin_amdgcn_readfirstlane(most);
    }
    f32x16 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
    float m = SPKV_NEG_INF, l = 0.f;
    bf16x8 kf[NS];                                           // K operands of the half-page after the current one
    auto load_k = [&](const uint16_t* hp) {
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) kf[sl] = *reinterpret_cast<const bf16x8*>(hp + sl * 512 + lane * 8);
    };
    auto scores = [&](f32x16& s) {
        f32x16 zero;
#pragma unroll
        for (int e = 0; e < 16; ++e) zero[e] = 0.f;
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qb[0], zero, 0, 0, 0);
#pragma unroll
        for (int sl = 1; sl < NS; ++sl) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[sl], qb[sl], s, 0, 0, 0);
    };
    // Excluded keys to -inf: past the list's end, past the ring's, gate off and outside the column's window.
    // Returns the keys (bit 8 g + e: 16 g + 8 half + e) that some column of the wave sees.
    auto mask = [&](f32x16& s, int x) -> unsigned {
        unsigned seen = 0u;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int k0 = 16 * g + 8 * half;
            unsigned ok, any;
            if (x < nA) {
                ok = any = bits_below(list.L - x * kHalfTokens - k0);
            } else {
                const unsigned on = gates_of(v, list, gates, x - nA, k0);
                ok = ring_seen(v, list, on, (x - nA) * kHalfTokens + k0, sr.place);
                any = ring_seen(v, list, on, (x - nA) * kHalfTokens + k0, least);
            }
            seen |= any << (8 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[8 * g + e] = ((ok >> e) & 1u) ? s[8 * g + e] : SPKV_NEG_INF;
        }
        return seen;
    };
    // weights against the column's reference as it stands; true (wave-uniform) if one is too low or not set
    bf16x8 pb[2];
    float psum, neg_ref = 0.f, limit = -1.f;
    auto weights = [&](const f32x16& s) -> bool {
        f32x8 p[2];
#pragma unroll
        for (int e = 0; e < 16; ++e)
            p[e >> 3][e & 7] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale_log2e, neg_ref));
        float s4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) s4[e] = (p[0][e] + p[0][4 + e]) + (p[1][e] + p[1][4 + e]);
        psum = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        pb[0] = __builtin_convertvector(p[0], bf16x8);       // (the sum keeps 32 bits)
        pb[1] = __builtin_convertvector(p[1], bf16x8);
        return __builtin_amdgcn_ballot_w64(!(psum <= limit)) != 0ull;
    };
    auto rescale = [&](const f32x16& s) {
        float cm = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) cm = fmaxf(cm, s[e]);
        cm *= scale_log2e;
        cm = fmaxf(cm, __shfl_xor(cm, 32));
        const float m_new = fmaxf(m, cm);
        const bool unset = m_new == SPKV_NEG_INF;            // every key so far excluded
        const float m_ref = unset ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_ref);
        l *= alpha;
#pragma unroll
        for (int db = 0; db < NB; ++db) acc[db] *= alpha;
        m = m_new;
        neg_ref = -m_ref;
        limit = unset ? -1.f : kSumLimit;
        (void)weights(s);
    };
    bf16x8 va[2][NB];
    auto load_v = [&](const uint16_t* hp, int g) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
            va[g][db] = *reinterpret_cast<const bf16x8*>(hp + kHalfTokens * D + (g * NB + db) * 512 + lane * 8);
    };
    auto accumulate = [&](int g) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[g][db], pb[g], acc[db], 0, 0, 0);
    };
    // One half-page: its scores are in sc and its first V operands in va[0]; the scores of the next one (hp1)
    // go to sn from kf, which then holds the K operands of hp2.
    const int full = list.L >> 5;                                 // half-pages that need no mask
    auto process = [&](f32x16& sc, f32x16& sn, int x, const uint16_t* hp, const uint16_t* hp1, const uint16_t* hp2,
                       auto&& more) {
        const bool edge = x >= full;
        unsigned seen = 0xffffu;
        if (edge) seen = mask(sc, x);
        __builtin_amdgcn_sched_barrier(0);
        // (the waves that are here first: the matrix and vector work of this part side by side with the products of the
        // other waves' last one; questions of 1632 tokens behind 30 MB of lists 230 -> 224 us)
        __builtin_amdgcn_s_setprio(1);
        scores(sn);
        const bool low = weights(sc);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if (__builtin_expect(low, 0)) rescale(sc);
        load_v(hp, 1);
        load_k(hp2);
        __builtin_amdgcn_sched_barrier(0);
        if (edge) {
#pragma unroll
            for (int db = 0; db < NB; ++db) {
                va[0][db] = keep_keys(va[0][db], seen);
                va[1][db] = keep_keys(va[1][db], seen >> 8);
            }
        }
        l += psum;
        accumulate(0);
        load_v(hp1, 0);
        more();
        __builtin_amdgcn_sched_barrier(0);
        accumulate(1);
        __builtin_amdgcn_sched_barrier(0);
    };

    const int n = x_end - x_begin;
    __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0): queries, gates, the first tiles
    asm volatile("" : : "s"(scale_log2e));
    __syncthreads();
    f32x16 s0, s1;
    load_k(s_tile[0]);
    scores(s0);
    load_k(s_tile[1]);
    load_v(s_tile[0], 0);
    // The copies of a step have landed once at most those of the newest step are in flight; behind the last
    // step of the range nothing is sent off any more, and all are waited for.
    auto next_step = [&](bool sent) {
        if (sent) wait_loads_but<kRowsPerWave>();
        else wait_loads_but<0>();
        __syncthreads();
    };
    int at = 0;                                              // slot of half-page k
    auto up = [&](int a, int by) -> int { return a + by >= kSlots ? a + by - kSlots : a + by; };
    for (int k = 0; k < n; k += 2) {
        const uint16_t* t0 = s_tile[at];
        const uint16_t* t1 = s_tile[up(at, 1)];
        const uint16_t* t2 = s_tile[up(at, 2)];
        const uint16_t* t3 = s_tile[up(at, 3)];
        bool sent = k + kAhead * kHps < n;
        process(s0, s1, x_begin + k, t0, t1, t2, [&]() { if (sent) stage_step(k + kAhead * kHps, up(at, kAhead * kHps)); });
        if (k + 1 >= n) break;
        if (kHps == 1) {
            next_step(sent);
            sent = k + 1 + kAhead < n;
        }
        process(s1, s0, x_begin + k + 1, t1, t2, t3,
                [&]() { if (kHps == 1 && sent) stage_step(k + 1 + kAhead, up(at, 1 + kAhead >= kSlots ? 1 + kAhead - kSlots : 1 + kAhead)); });
        next_step(sent);
        at = up(at, 2);
    }
    wait_loads_but<0>();

    l += __shfl_xor(l, 32);
    if (valid && half == 0) part_ml[pc] = make_float2(m, l);
    const bool odd = x_end > nA && least != most && odd_sums(acc, NB, l);
    // The sums leave through LDS, a column's row at a time (straight from the registers every store touched 32 rows,
    // 32 bytes each).  16-byte unit x of column col lies at x ^ col: no bank conflicts either way.
    __syncthreads();                                         // the tiles are no longer read
    float* sums = reinterpret_cast<float*>(&s_tile[0][0]) + wv * 32 * D;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(sums + col * D + ((db * 8 + g * 2 + half) ^ (col & (D / 4 - 1))) * 4) =
                (f32x4){acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
    __builtin_amdgcn_wave_barrier();
    constexpr int kUnits = D / 4, kColsPerPass = 64 / kUnits;
    const int unit = lane % kUnits, n_here = min(32, n_cols - (col0 + wv * 32));
    float* to = cut.part + (((size_t)h * cut.slots + j) * cut.n_cols + (size_t)first * v.G + col0 + wv * 32) * D;
#pragma unroll 4
    for (int i = lane / kUnits; i < n_here; i += kColsPerPass)
        *reinterpret_cast<f32x4*>(to + (size_t)i * D + unit * 4) =
            *reinterpret_cast<const f32x4*>(sums + i * D + (unit ^ (i & (D / 4 - 1))) * 4);
    if (__builtin_expect(__ballot(odd) != 0ull, 0)) {
        const CarefulRange range = careful_range(v, list, scale_log2e, x_begin, x_end);
        if (careful_needed<D>(range, least, most)) {
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0): the stores above come first
            for (int i = 0; i < n_here; ++i) {
                const ShareRow at = share_row(rows, first, col0 + wv * 32 + i, v.G, v.Hkv, true);
                careful_sums<D>(range, q + ((size_t)at.row * v.Hq + (size_t)h * v.G + at.head) * D, at.place, __shfl(m, i),
                                to + (size_t)i * D);
            }
        }
    }
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
