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
//
// spkv_prefix_split: a workgroup of NW waves takes 32 NW columns (32 a wave, one group of MFMA 32x32x16)
// and a range of the list's half-pages, which it copies from memory straight into a ring of LDS
// buffers, in operand order, so that every wave reads its operands as 1 KB in lane order.  The products
// K Q^T of a half-page stand beside the weights of the one before.  Eight waves fetch two half-pages to
// a step (as spkv_prefill_attend32, whose pipeline this is); with fewer waves a step is one half-page and
// two workgroups share a compute unit.
constexpr float kSumLimit = 2048.0f;         // a sum of 16 weights above it: the reference is too low
constexpr int kRingGateTiles = 64;           // half-pages of the ring whose gates a wave looks up beforehand, one a lane

__device__ __forceinline__ unsigned bits_upto8(int n) { return n <= 0 ? 0u : n >= 8 ? 0xffu : (1u << n) - 1u; }

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
    for (int hp = hp0; hp < hp1; ++hp) {
        const uint16_t* base;
        int nvalid;
        if (hp < ps.ghp) {
            const int lp = hp >> 1;
            if (lp >= pbase + 64) {
                pbase = lp;
                my_page = pt[min(pbase + lane, v.pt_cap - 1)];
            }
            base = pool_page(v, __builtin_amdgcn_readlane(my_page, lp - pbase)) + (hp & 1) * (2 * kHalfTokens * D);
            nvalid = min(kHalfTokens, ps.L - hp * kHalfTokens);
        } else {
            const int r = hp - ps.ghp;
            base = ring_page(v, pair, r >> 1) + (r & 1) * (2 * kHalfTokens * D);
            nvalid = min(kHalfTokens, ps.Tw - r * kHalfTokens);
        }
        const bool any_kill = nvalid < kHalfTokens;
        const unsigned kill = any_kill ? 0xffu << min(max(nvalid - kc * 8, 0), 8) : 0u;
        const uint16_t* kp = base + lane * 8;
        const uint16_t* vp = base + kHalfTokens * D + lane * 8;
        bf16x8 ka[2][NS], va[NB];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) ka[t][sl] = load_stream_b128(kp + (t * (D / 8) + sl * 4) * 128);
#pragma unroll
        for (int db = 0; db < NB; ++db) va[db] = load_stream_b128(vp + db * 512);
        attend_half_page<D, true>(ka, va, qb, kill, any_kill, scale_log2e, acc, m, l);
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
// XCDs' compute units and leave others idle; with more lists each has as many.
struct ShareUnit {
    int list, range, ranges, block;
};
__device__ __forceinline__ ShareUnit find_unit(const SpkvShareCut& cut, const SpkvShareTable& table, int id, int n_kv_heads) {
    ShareUnit u;
    if (cut.uniform > 0) {
        const int each = cut.uniform * cut.n_blocks;
        u.list = id / each;
        const int rest = id - u.list * each;
        u.ranges = cut.uniform;
        u.block = rest / u.ranges;
        u.range = rest - u.block * u.ranges;
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

template <int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW >= 4 ? 2 : 1, NW >= 4 ? 2 : 1)))
void spkv_prefix_split(SpkvView v, const uint16_t* __restrict__ q, float scale_log2e, SpkvShareCut cut, SpkvShareTable table,
                       SpkvShareRows rows, SpkvShareOwn own) {
    constexpr int NS = D / 16, NB = D / 32;
    constexpr int kHalfElems = 2 * kHalfTokens * D;
    constexpr int kHps = NW == 8 ? 2 : 1;                    // half-pages to a step
    constexpr int kSlots = NW == 8 ? 8 : 5;                  // half-pages in LDS
    constexpr int kRowsPerWave = kHps * (D / 8) / NW;        // 1 KB rows of a step that a wave copies
    __shared__ __attribute__((aligned(16))) uint16_t s_tile[kSlots][kHalfElems];
    if ((int)blockIdx.x >= cut.n_units) {                    // behind the prompts': the sequences' own lists
        const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        own_item<D>(own_view(own, v), q, scale_log2e, own.split, own.part, ((int)blockIdx.x - cut.n_units) * NW + wave);
        return;
    }
    const ShareUnit u = find_unit(cut, table, blockIdx.x, v.Hkv);
    const int act = u.list / v.Hkv, h = u.list - act * v.Hkv, j = u.range, ranges = u.ranges;
    const int first = rows.table != nullptr ? rows.first_row[act] : rows.first[act];
    const int n_cols = ((rows.table != nullptr ? rows.first_row[act + 1] : rows.first[act + 1]) - first) * v.G;
    const int col0 = u.block * (32 * NW);
    if (col0 >= n_cols) return;
    const int pair = (int)rows.prefix[act] * v.Hkv + h;
    const int T = v.t_pair[pair], L = v.kept_len[pair], held = min(T, v.w);
    const int nA = (L + kHalfTokens - 1) >> 5, n_hp = nA + ((held + kHalfTokens - 1) >> 5);
    const int x_begin = (int)((int64_t)j * n_hp / ranges), x_end = (int)((int64_t)(j + 1) * n_hp / ranges), last = x_end - 1;

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wv = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = col0 + wv * 32 + col;
    const bool valid = c < n_cols;
    const int in_group = valid ? c / v.G : 0, g_head = valid ? c - in_group * v.G : 0;
    int row, place;                                          // this column's query row and its token's place
    if (rows.table != nullptr) {
        const int2 e = rows.table[first + in_group];
        row = e.x;
        place = e.y;
    } else {
        row = rows.seq[first + in_group];
        place = rows.t_own[row * v.Hkv] - 1;
    }
    const size_t pc = ((size_t)h * cut.slots + j) * cut.n_cols + (size_t)first * v.G + c;      // of the partial result
    float2* part_ml = reinterpret_cast<float2*>(cut.part + (size_t)v.Hkv * cut.slots * cut.n_cols * D);
    if (x_begin >= x_end) {                                  // fewer half-pages than ranges
        if (valid && half == 0) part_ml[pc] = make_float2(SPKV_NEG_INF, 0.f);
        return;
    }
    // page ids of 64 logical pages, one a lane
    const int32_t* pt = v.page_table + (size_t)pair * v.pt_cap;
    int page_lane0 = x_begin >> 1, my_page = pt[min(page_lane0 + lane, v.pt_cap - 1)];
    auto page_of = [&](int lp) -> int {                      // lp wave-uniform, never decreasing
        if (lp >= page_lane0 + 64) {
            page_lane0 = lp;
            my_page = pt[min(lp + lane, v.pt_cap - 1)];
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0)
        }
        return __builtin_amdgcn_readlane(my_page, lp - page_lane0);
    };
    auto base_of = [&](int x) -> const uint16_t* {
        x = min(x, last);
        if (x < nA) {
            const int page = min(max(page_of(x >> 1), 0), v.n_pages - 1);
            return pool_page(v, page) + (x & 1) * kHalfElems;
        }
        return ring_page(v, pair, (x - nA) >> 1) + ((x - nA) & 1) * kHalfElems;
    };
    bf16x8 qb[NS];
    {
        const uint16_t* qrow = q + ((size_t)row * v.Hq + (size_t)h * v.G + g_head) * D + half * 8;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) {
            uint4 raw = {0u, 0u, 0u, 0u};
            if (valid) raw = *reinterpret_cast<const uint4*>(qrow + sl * 16);
            qb[sl] = __builtin_bit_cast(bf16x8, raw);
        }
    }
    // ring: age of a slot's key, 0 = position T - w; does it pass the gate?
    const int slot0 = T >= v.w ? T % v.w : T - v.w;
    auto age_of = [&](int at) -> int { return at - slot0 + (at < slot0 ? v.w : 0); };
    auto ring_gate = [&](int at) -> bool {
        return gate_passes(v, v.ring_logit[(size_t)pair * v.w + at], T - v.w + age_of(at));
    };
    const int ring0 = max(x_begin - nA, 0);                  // this workgroup's first ring half-page
    unsigned my_gate = 0u;                                   // lane t: the gates of ring half-page ring0 + t
    for (int t = 0; t < min(x_end - nA - ring0, kRingGateTiles); t += 8) {                // two half-pages a load
        bool on[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) on[u] = ring_gate(min((ring0 + t + 2 * u) * kHalfTokens + lane, held - 1));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const unsigned long long gates = __ballot(on[u]);
            if (lane == t + 2 * u) my_gate = (unsigned)gates;
            if (lane == t + 2 * u + 1) my_gate = (unsigned)(gates >> 32);
        }
    }

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
            const int row_id = NW == 1 ? i : wq * kRowsPerWave + i;
            const bool is_k = NW == 1 ? i < NS : wq * kRowsPerWave < NS;
            const int vr = row_id - NS, off = is_k ? row_id * 512 : (vr / NB) * 512 + (vr % NB) * 2048;
            load_row_to_lds(reinterpret_cast<const char*>(base) + off, is_k ? k_lane : v_lane, dst + row_id * 1024);
        }
    };
    auto stage_step = [&](int k, int slot) {                 // half-page k of the range (and the one behind it)
        if (kHps == 2) stage_half_page_rows(base_of(x_begin + k + wh), slot + wh);
        else stage_half_page_rows(base_of(x_begin + k), slot);
    };

    f32x16 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
    float m = valid ? SPKV_NEG_INF : 0.f, l = 0.f;
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
            unsigned ok;
            if (x < nA) {
                ok = bits_upto8(L - x * kHalfTokens - k0);
            } else {
                const int at0 = (x - nA) * kHalfTokens + k0, t = x - nA - ring0;
                ok = 0u;
                if (t < kRingGateTiles) {
                    ok = ((unsigned)__builtin_amdgcn_readlane((int)my_gate, t) >> k0) & 0xffu;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (ring_gate(min(at0 + e, held - 1))) ok |= 1u << e;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (age_of(at0 + e) > place) ok |= 1u << e;
                ok &= bits_upto8(held - at0);
            }
            if (!valid) ok = 0u;
            seen |= ok << (8 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[8 * g + e] = ((ok >> e) & 1u) ? s[8 * g + e] : SPKV_NEG_INF;
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) seen |= __shfl_xor(seen, o);
        return seen;
    };
    // weights against the column's reference as it stands; true (wave-uniform) if one is too low or not set
    bf16x8 pb[2];
    float psum, neg_ref = valid ? 0.f : -m, limit = valid ? -1.f : kSumLimit;
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
    // values of keys that no column sees to zero: a weight of zero would turn an infinity among them into a NaN
    auto clear_v = [&](int g, unsigned seen) {
        unsigned keep[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned two = seen >> (8 * g + 2 * i);
            keep[i] = (two & 1u ? 0xffffu : 0u) | (two & 2u ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int db = 0; db < NB; ++db) {
            uint4 u = __builtin_bit_cast(uint4, va[g][db]);
            u.x &= keep[0];
            u.y &= keep[1];
            u.z &= keep[2];
            u.w &= keep[3];
            va[g][db] = __builtin_bit_cast(bf16x8, u);
        }
    };
    // One half-page: its scores are in sc and its first V operands in va[0]; the scores of the next one (hp1)
    // go to sn from kf, which then holds the K operands of hp2.
    const int full = L >> 5;                                 // half-pages that need no mask
    auto process = [&](f32x16& sc, f32x16& sn, int x, const uint16_t* hp, const uint16_t* hp1, const uint16_t* hp2,
                       auto&& more) {
        const bool edge = x >= full;
        unsigned seen = 0xffffu;
        if (edge) seen = mask(sc, x);
        __builtin_amdgcn_sched_barrier(0);
        scores(sn);
        const bool low = weights(sc);
        __builtin_amdgcn_sched_barrier(0);
        if (__builtin_expect(low, 0)) rescale(sc);
        load_v(hp, 1);
        load_k(hp2);
        __builtin_amdgcn_sched_barrier(0);
        if (edge) {
            clear_v(0, seen);
            clear_v(1, seen);
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
    __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0): queries, page ids, gates
    asm volatile("" : : "s"(scale_log2e));
    // steps 0 .. kAhead - 1 are on their way before the loop; step s + kAhead is sent off in step s
    constexpr int kAhead = NW == 8 ? 3 : 4;
#pragma unroll
    for (int s = 0; s < kAhead; ++s) stage_step(s * kHps, s * kHps);
    wait_loads_but<kRowsPerWave>();
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
    if (!valid) return;
    float* pa = cut.part + pc * D + half * 4;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(pa + db * 32 + g * 8) =
                (f32x4){acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
    if (half == 0) part_ml[pc] = make_float2(m, l);
}

// The join: D / 4 threads own a column (row, head), four consecutive elements each; S such groups share a column,
// each with every S-th of its partial results, and meet in LDS (few columns of many ranges: 512 columns
// of 64 ranges in one group each took 14 us, a chain of eight round trips on a quarter of the chip).
// The sequence's own part is a set of partial results too (own.part), or comes as a call's bf16 output and fp32
// logarithm of its sum: half a step of bf16 more than from sums in 32 bits, on the share that the own tokens have.
template <int D, int S>
__global__ __launch_bounds__(256) void spkv_prefix_merge(SpkvShareCut cut, SpkvShareMerge rows, SpkvShareOwn own, int n_q_heads,
                                                         int n_kv_heads, const uint16_t* own_out, const float* own_lse,
                                                         uint16_t* out, float* lse) {      // (out may be own_out, lse own_lse)
    constexpr int TPC = D / 4, CPB = 256 / TPC, kFold = 8;
    __shared__ f32x4 s_num[S > 1 ? CPB : 1][S > 1 ? TPC : 1];
    __shared__ float2 s_ml[S > 1 ? CPB : 1];
    const int slice = (int)threadIdx.x / TPC, share = slice % S, d = ((int)threadIdx.x % TPC) * 4;
    const int64_t id = (int64_t)blockIdx.x * (CPB / S) + slice / S;      // row * Hq + head
    const bool exists = id < cut.n_out;
    const int G = n_q_heads / n_kv_heads;
    const int row = exists ? (int)(id / n_q_heads) : 0, head = exists ? (int)(id - (int64_t)row * n_q_heads) : 0;
    const int h = head / G, g = head - h * G;
    int act = -1, at = 0;
    if (rows.by_row != nullptr) {
        const int2 e = rows.by_row[row];
        act = e.x;
        at = e.y;
    } else {
        act = rows.active[row];
        at = rows.place[row];
    }
    float M = SPKV_NEG_INF, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    const int ranges = act < 0 ? 0 : cut.uniform > 0 ? cut.uniform : rows.ranges[act * n_kv_heads + h];
    int own_parts = 0;
    size_t own0 = 0;
    if (own.part != nullptr) {
        const SpkvSplit sp = own.split;
        const int pair = row * n_kv_heads + h;
        own_parts = own_ranges(own, pair);
        own0 = (size_t)pair * sp.slots * G + g;
    } else if (share == 0 && exists) {
        const uint2 ob = *reinterpret_cast<const uint2*>(own_out + id * D + d);
        const float z = own_lse[id];
        if (ranges == 0) {                                   // no prompt: the own part as it is
            *reinterpret_cast<uint2*>(out + id * D + d) = ob;
            if (lse != nullptr && d == 0) lse[id] = z;
        }
        if (z > SPKV_NEG_INF) {
            M = z * 1.4426950408889634f;
            den = 1.f;
            num = (f32x4){__builtin_bit_cast(float, ob.x << 16), __builtin_bit_cast(float, ob.x & 0xffff0000u),
                          __builtin_bit_cast(float, ob.y << 16), __builtin_bit_cast(float, ob.y & 0xffff0000u)};
        }
    }
    // partial results kFold at a time, their loads in flight together; only the rescaling is chained
    const size_t prompt0 = (size_t)h * cut.slots * cut.n_cols + (size_t)at * G + g;
    const float2* ml = reinterpret_cast<const float2*>(cut.part + (size_t)n_kv_heads * cut.slots * cut.n_cols * D);
    const float2* own_ml = reinterpret_cast<const float2*>(own.part + own.n_floats);
    const int parts = exists ? ranges + own_parts : 0;
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
            if (r0 + u * S < parts && x[u].x > SPKV_NEG_INF) {       // (a range without keys has written no sums)
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
    const float inv = den > 0.f ? 1.0f / den : 0.f;          // (a row that sees no key at all: zeros)
    uint2 packed;
    packed.x = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[0] * inv)) |
               ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[1] * inv)) << 16);
    packed.y = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[2] * inv)) |
               ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)(num[3] * inv)) << 16);
    *reinterpret_cast<uint2*>(out + id * D + d) = packed;
    if (lse != nullptr && d == 0) lse[id] = den > 0.f ? (M + log2f(den)) * 0.6931471805599453f : SPKV_NEG_INF;
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

int spkv_prefix_waves(int n_cols) { return n_cols <= 32 ? 1 : n_cols <= 64 ? 2 : n_cols <= 128 ? 4 : 8; }

template <int D>
static hipError_t launch_prefix(const SpkvView& v, const uint16_t* q, float sl, int waves, const SpkvShareCut& cut,
                                const SpkvShareTable& table, const SpkvShareRows& rows, const SpkvShareMerge& merge,
                                const SpkvShareOwn& own, const uint16_t* own_out, const float* own_lse, uint16_t* out,
                                float* lse, hipStream_t s) {
    const int items = own.part != nullptr ? own.n_pairs * own.split.slots : 0;
    const dim3 grid((unsigned)(cut.n_units + (items + waves - 1) / waves));
    if (grid.x > 0) {
        if (waves == 8) spkv_prefix_split<D, 8><<<grid, dim3(512), 0, s>>>(v, q, sl, cut, table, rows, own);
        else if (waves == 4) spkv_prefix_split<D, 4><<<grid, dim3(256), 0, s>>>(v, q, sl, cut, table, rows, own);
        else if (waves == 2) spkv_prefix_split<D, 2><<<grid, dim3(128), 0, s>>>(v, q, sl, cut, table, rows, own);
        else spkv_prefix_split<D, 1><<<grid, dim3(64), 0, s>>>(v, q, sl, cut, table, rows, own);
    }
    // groups to a column: about eight workgroups per compute unit, no more groups than there are ranges
    constexpr int CPB = 256 / (D / 4);
    int share = 8;
    while (share > 1 && (cut.n_out * share / CPB > 4096 || share > cut.slots)) share >>= 1;
    const int per_block = CPB / share;
    const dim3 merge_grid((unsigned)((cut.n_out + per_block - 1) / per_block));
    if (share == 8) spkv_prefix_merge<D, 8><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    else if (share == 4) spkv_prefix_merge<D, 4><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    else if (share == 2) spkv_prefix_merge<D, 2><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    else spkv_prefix_merge<D, 1><<<merge_grid, dim3(256), 0, s>>>(cut, merge, own, v.Hq, v.Hkv, own_out, own_lse, out, lse);
    return hipGetLastError();
}

hipError_t spkv_launch_prefix(const SpkvView& v, const uint16_t* q, float sm_scale, int waves, const SpkvShareCut& cut,
                              const SpkvShareTable& table, const SpkvShareRows& rows, const SpkvShareMerge& merge,
                              const SpkvShareOwn& own, const uint16_t* own_out, const float* own_lse, uint16_t* out,
                              float* lse, hipStream_t s) {
    const float sl = sm_scale * 1.4426950408889634f;
    return v.D == 128 ? launch_prefix<128>(v, q, sl, waves, cut, table, rows, merge, own, own_out, own_lse, out, lse, s)
                      : launch_prefix<64>(v, q, sl, waves, cut, table, rows, merge, own, own_out, own_lse, out, lse, s);
}

hipError_t spkv_launch_prefix_rows(const SpkvCu& cu, const SpkvShareActive& a, const int32_t* t_own, int n_seq,
                                   int n_kv_heads, bool appended, int n_active, int32_t* table, int32_t* by_row,
                                   int32_t* first_row, hipStream_t s) {
    spkv_prefix_rows<<<dim3((unsigned)n_seq), dim3(256), 0, s>>>(cu, a, t_own, n_seq, n_kv_heads, appended ? 1 : 0,
                                                                 n_active, reinterpret_cast<int2*>(table),
                                                                 reinterpret_cast<int2*>(by_row), first_row);
    return hipGetLastError();
}
