// Attention of a block of columns (query row, head) over one list and its ring: what attention over shared prompts
// and of trees of drafts have in common.  A column stands at some place behind the list's newest token: it sees all of
// the list, which holds keys that passed the gate, and of the ring the keys inside its window or past the gate.
#pragma once
#include "spkv_device.h"

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

__device__ __forceinline__ unsigned long long lane_word(unsigned long long x, int lane) {
    return (unsigned long long)(unsigned)__shfl((int)(unsigned)x, lane) | ((unsigned long long)(unsigned)__shfl((int)(x >> 32), lane) << 32);
}

// The query row of a column, its head in the group, and its token's place behind the list's newest token (looked for
// only where the ring is read).
struct ShareRow {
    int row, head, place;
};

// What the two bodies below are told of a workgroup's work:
//   pair, h, range, ranges, block    list and KV head, which of the list's ranges, which block of columns
//   columns(v)                       columns of the list, asked once and before those that follow
//   row(v, c, ring)                  ShareRow of column c; ring: the place is wanted.  The whole wave asks.
//   part(v), part_ml<D>(v), part0(v) partial sums and (m, l), those of column c at part0 + c
//   begin(list, j)                   first half-page of the list's range j
//   kTree                            there are drafts, too: keys that every column sees some of, which the workgroup of a list's first
//                                    range takes (drafts()); see TreeWork in spkv_tree.hip for what is asked of it then
//   kPaths, parent(), place(v, c, path(parent()))            places by themselves, for who has other loads to send first
//   kWhole                           the range is the whole list, and what the workgroup has at the end is the columns' result

// Up to 16 NQ columns.  A half-page's operands come straight from memory (1 KB a load, as in spkv_decode_split) and are
// used for all NQ groups of 16 columns: scores of all groups -- the next half-page's keys are sent for -- then
// weights against the references as they stand -- raised, and sums and accumulators rescaled, only where some lane's
// eight weights add up to more than kSumLimit -- then the products with V, the weights as two bf16 parts (16 bits: the
// lists' read takes the time, not these products) -- and the next values are sent for.  One body for every half-page:
// two of them in turn on two sets of operands were slower where a wave has only a few (cold instructions).  The NV
// waves, four or eight, take an equal part of the range each and meet in LDS.
template <int D, int NQ, int NV, class Work>
__device__ __forceinline__ void attend_list_few(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e, Work& work) {
    constexpr int NS = D / 32, NB = D / 16, kRow = D + 4;
    __shared__ __attribute__((aligned(16))) float s_acc[NV][16 * NQ * kRow];
    __shared__ float2 s_ml[NV][16 * NQ];
    __shared__ __attribute__((aligned(16))) uint16_t s_q[NQ == 1 ? 1 : NQ * NS][512];
    const int tid = threadIdx.x, lane = tid & 63, kc = lane >> 4, n = lane & 15;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pair = work.pair, h = work.h, j = work.range;
    const FirstPages first_ids = first_pages(v, pair);
    const ShareList list = share_list(v, pair);
    const int n_cols = work.columns(v);
    if (n_cols <= 0) return;
    const int nA = list.nA;
    const int r_begin = work.begin(list, j), r_end = work.begin(list, j + 1);
    const bool drafts = work.drafts() && wv == 0;            // they are the first wave's, and count as some half-pages
    const int n_drafts = work.drafts() ? work.draft_weight() : 0;
    auto cut = [&](int w) -> int { return r_begin + max(0, (r_end - r_begin + n_drafts) * w / NV - n_drafts); };
    const int x_begin = wv == 0 ? r_begin : cut(wv), x_end = cut(wv + 1);
    const int x_first = drafts ? x_begin - 1 : x_begin;      // they come before the half-pages

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
    const int parent = work.parent();                        // (of trees; sent for before what waits longer)
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int c = i * 16 + n;
        const ShareRow sr = work.row(v, c < n_cols ? c : 0, ring && !Work::kPaths);
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
    unsigned long long word = 0ull;                          // drafts that lane's draft sees
    if (drafts) {
        if constexpr (Work::kTree) work.template load_few<D>(v, k, va);
    } else if (x_begin < x_end) {
        const uint16_t* page = half_page_at(v, list, pages, x_begin);
        load_k(page);
        load_v(page);
    }
    if constexpr (Work::kPaths) {
        if (ring || drafts) {
            const auto path = work.path(parent);
#pragma unroll
            for (int i = 0; i < NQ; ++i) place[i] = work.place(v, i * 16 + n < n_cols ? i * 16 + n : 0, path);
            if (drafts) word = work.seen(v, list.T, path);
        }
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
    for (int x = x_first; x < x_end; ++x) {
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
        if (Work::kTree && drafts && x == x_first) {          // a draft: a word of the drafts that it sees
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const int c = i * 16 + n;
                const unsigned mine = (unsigned)(lane_word(word, (c < n_cols ? c : 0) / v.G) >> (8 * kc));
#pragma unroll
                for (int e = 0; e < 8; ++e) s[i][e] = ((mine >> e) & 1u) ? s[i][e] : SPKV_NEG_INF;
            }
        } else if (x >= full) {
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
                if (x > x_first) {
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
    if ((ring && least != most) || drafts) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NQ; ++i) odd = odd || odd_sums(acc[i], NB, l[i]);
        if (__builtin_expect(__ballot(odd) != 0ull, 0)) {
            const CarefulRange range = careful_range(v, list, scale_log2e, x_begin, x_end);
            bool again = ring && least != most && careful_needed<D>(range, least, most);
            if constexpr (Work::kTree) again = again || (drafts && work.template careful_needed<D>(v));
            if (again)
                for (int c = 0; c < min(16 * NQ, n_cols); ++c) {
                    const ShareRow sr = work.row(v, c, true);
                    __builtin_amdgcn_wave_barrier();
                    const uint16_t* qrow = q + ((size_t)sr.row * v.Hq + (size_t)h * v.G + sr.head) * D;
                    careful_sums<D>(range, qrow, sr.place, s_ml[wv][c].x, s_acc[wv] + c * kRow);
                    if constexpr (Work::kTree)
                        if (drafts) work.template add_careful<D>(v, qrow, lane_word(word, sr.row - work.row0), scale_log2e, s_ml[wv][c].x, s_acc[wv] + c * kRow);
                }
        }
    }
    __syncthreads();
    const size_t pc0 = Work::kWhole ? 0 : work.part0(v);
    float* part = work.part(v);
    float2* part_ml = work.template part_ml<D>(v);
    for (int e = tid; e < n_cols * (D / 4); e += 64 * NV) {
        const int c = e / (D / 4), d = (e - c * (D / 4)) * 4;
        float2 ml[NV];
        float M = SPKV_NEG_INF;
#pragma unroll
        for (int w = 0; w < NV; ++w) {
            ml[w] = s_ml[w][c];
            M = fmaxf(M, ml[w].x);
        }
        const float m_ref = M == SPKV_NEG_INF ? 0.f : M;     // no key at all: every weight 0
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < NV; ++w) {
            const float sc = __builtin_amdgcn_exp2f(ml[w].x - m_ref);
            a += *reinterpret_cast<const f32x4*>(s_acc[w] + c * kRow + d) * sc;
            sum += ml[w].y * sc;
        }
        if constexpr (Work::kWhole) {
            work.template store<D>(v, c, d, a, M, sum);
        } else {
            *reinterpret_cast<f32x4*>(part + (pc0 + c) * D + d) = a;
            if (d == 0) part_ml[pc0 + c] = make_float2(M, sum);
        }
    }
}

// A wave's sums of 32 columns leave through LDS, a column's row at a time (straight from the registers every store touched 32 rows,
// 32 bytes each).  16-byte unit x of column col lies at x ^ col: no bank conflicts either way.
template <int D>
__device__ __forceinline__ void column_sums_to_lds(const f32x16 (&acc)[D / 32], float* sums) {
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(sums + col * D + ((db * 8 + g * 2 + half) ^ (col & (D / 4 - 1))) * 4) =
                (f32x4){acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
    __builtin_amdgcn_wave_barrier();
}
template <int D>
__device__ __forceinline__ f32x4 column_sum_at(const float* sums, int i, int unit) {
    return *reinterpret_cast<const f32x4*>(sums + i * D + (unit ^ (i & (D / 4 - 1))) * 4);
}
template <int D>
__device__ __forceinline__ void store_column_sums(const f32x16 (&acc)[D / 32], float* sums, float* to, int n_here) {
    column_sums_to_lds<D>(acc, sums);
    const int lane = threadIdx.x & 63;
    constexpr int kUnits = D / 4, kColsPerPass = 64 / kUnits;
    const int unit = lane % kUnits;
#pragma unroll 4
    for (int i = lane / kUnits; i < n_here; i += kColsPerPass)
        *reinterpret_cast<f32x4*>(to + (size_t)i * D + unit * 4) = column_sum_at<D>(sums, i, unit);
}

// More columns: the copies of the range's half-pages go from memory straight into LDS, in operand order, so that
// every wave reads its operands as 1 KB in lane order.  The products K Q^T of a half-page stand beside the
// weights of the one before.  Eight waves fetch two half-pages to a step (as spkv_prefill_attend32, whose
// pipeline this is); with fewer waves a step is one half-page and two workgroups share a compute unit.  The weights go
// into the second product as one bf16 part, half a step (2^-8) at most each, their sum in 32 bits: from 33 columns on the
// products count, and a second part would be half as many again (errors against 64 bits 2.3e-3 of the 2-norm instead of 1.7e-3).
template <int NW>
constexpr int kSplitSlots = NW == 8 ? 8 : 5;                 // half-pages in LDS
template <int D, int NW, class Work>
__device__ __forceinline__ void attend_list_split(const SpkvView& v, const uint16_t* __restrict__ q, float scale_log2e, Work& work,
                                                  uint16_t (&s_tile)[kSplitSlots<NW>][2 * kHalfTokens * D]) {
    constexpr int NS = D / 16, NB = D / 32;
    constexpr int kHalfElems = 2 * kHalfTokens * D;
    constexpr int kHps = NW == 8 ? 2 : 1;                    // half-pages to a step
    constexpr int kSlots = kSplitSlots<NW>;
    constexpr int kRowsPerWave = kHps * (D / 8) / NW;        // 1 KB rows of a step that a wave copies
    const int pair = work.pair, h = work.h, j = work.range;
    const FirstPages first_ids = first_pages(v, pair);
    const ShareList list = share_list(v, pair);
    const int n_cols = work.columns(v);
    const int col0 = work.block * (32 * NW);
    if (col0 >= n_cols) return;
    const int nA = list.nA;
    const int x_begin = work.begin(list, j), x_end = work.begin(list, j + 1), last = max(x_end - 1, x_begin);

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = col0 + wv * 32 + col;
    const bool valid = c < n_cols;
    const size_t pc = Work::kWhole ? 0 : work.part0(v) + c;  // of the partial result
    float2* part_ml = work.template part_ml<D>(v);
    if (x_begin >= x_end && !work.drafts()) {                // fewer half-pages than ranges
        if (valid && half == 0) part_ml[pc] = make_float2(SPKV_NEG_INF, 0.f);
        return;
    }
    const ShareRow sr = work.row(v, valid ? c : 0, x_end > nA);
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

    unsigned long long word = 0ull;                          // drafts that lane's draft sees
    if constexpr (Work::kTree) {
        if (work.drafts()) {
            __syncthreads();                                 // the tiles are no longer read
            work.template stage_split<D, NW>(v, s_tile[0]);
            word = work.seen(v, list.T);
            const unsigned long long mine = lane_word(word, sr.row - work.row0);
            __syncthreads();
#pragma unroll 1
            for (int t = 0; t < (work.n + kHalfTokens - 1) / kHalfTokens; ++t) {
                load_k(s_tile[t]);
                load_v(s_tile[t], 0);
                load_v(s_tile[t], 1);
                scores(s0);
                const unsigned ok = (unsigned)(mine >> (32 * t)) >> (8 * half);
#pragma unroll
                for (int e = 0; e < 16; ++e) s0[e] = ((ok >> (16 * (e >> 3) + (e & 7))) & 1u) ? s0[e] : SPKV_NEG_INF;
                if (weights(s0)) rescale(s0);
                l += psum;
                accumulate(0);
                accumulate(1);
            }
        }
    }
    l += __shfl_xor(l, 32);
    const bool ring = x_end > nA && least != most;
    const bool odd = (ring || work.drafts()) && odd_sums(acc, NB, l);
    __syncthreads();                                         // the tiles are no longer read
    const int n_here = min(32, n_cols - (col0 + wv * 32));
    float* sums = reinterpret_cast<float*>(&s_tile[0][0]) + wv * 32 * D;
    bool again = false;
    const CarefulRange range = careful_range(v, list, scale_log2e, x_begin, x_end);
    if (__builtin_expect(__ballot(odd) != 0ull, 0)) {
        again = ring && careful_needed<D>(range, least, most);
        if constexpr (Work::kTree) again = again || (work.drafts() && work.template careful_needed<D>(v));
    }
    auto careful = [&](int i, float* to) {                   // column i's sums, key by key
        const ShareRow at = work.row(v, col0 + wv * 32 + i, true);
        const uint16_t* qrow = q + ((size_t)at.row * v.Hq + (size_t)h * v.G + at.head) * D;
        const float ref = __shfl(m, i);
        careful_sums<D>(range, qrow, at.place, ref, to);
        if constexpr (Work::kTree)
            if (work.drafts()) work.template add_careful<D>(v, qrow, lane_word(word, at.row - work.row0), scale_log2e, ref, to);
    };
    if constexpr (Work::kWhole) {
        work.template finish_split<D>(v, acc, m, l, sums, col0 + wv * 32, n_here, again, careful);
    } else {
        if (valid && half == 0) part_ml[pc] = make_float2(m, l);
        float* to = work.part(v) + (work.part0(v) + col0 + wv * 32) * D;
        store_column_sums<D>(acc, sums, to, n_here);
        if (__builtin_expect(again, 0)) {
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0): the stores above come first
            for (int i = 0; i < n_here; ++i) careful(i, to + (size_t)i * D);
        }
    }
}
