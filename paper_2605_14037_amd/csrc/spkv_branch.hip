// Sequences that branch, on gfx950: copies, moves and releases of whole sequences, what sequences hold as
// dense rows, and the append of rows that lie here and there.
#include "spkv_device.h"

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

// ---------------------------------------------------------------- sequences become others
// All sequences of a call change at once: sequence b becomes what source[b] was.  What a sequence holds is its
// window ring, its counters and, per head, a row of the page table.  The first sequence that takes over one whose own
// place is taken has its row of page ids, without a copy; further ones get copies of the pages in the next launch
// (spkv_fork_pages), from wherever they are by then, into the pages that they have themselves already, unless somebody
// takes those, and further ones from the pool.  Pages that are left over go back onto the stack, in this launch alone, and
// pages are handed out in the next alone.  (Copies into the pages at hand: every handing out is an atomic on one address, and
// 2600 of them -- eight copies of 32k tokens, four pages each -- were most of 148 us.)
//
// Order.  Sequences that hang together (one is the source of another and is itself replaced) are a component; the
// host has put its moves into an order in which every sequence is read before it is replaced, a cycle being opened by
// saving its first one (the flag kForkSave).  Every thread carries its own units -- 16 bytes of a ring, an entry of a
// page table row, a logit -- through all moves of the component before it takes the next, so the order of one
// thread's loads and stores is all that is needed, and what is saved is one register.
// Counters are read before any of them is written.
constexpr int kForkThreads = 256, kForkUnits = 4;             // 16 KB of a ring to a workgroup
__device__ __forceinline__ int fork_ring_units(const SpkvView& v) { return v.n_ring_pages * (spkv_page_elems(v.D) / 8); }

__global__ __launch_bounds__(kForkThreads) void spkv_fork_move(SpkvView v, SpkvForkSource from, SpkvForkMoves mv) {
    const int tid = threadIdx.x, h = blockIdx.y;
    const int m0 = mv.start[blockIdx.x], m1 = mv.start[blockIdx.x + 1];
    if (blockIdx.z > 0) {                                     // rings
        const int units = fork_ring_units(v), step = kForkThreads * kForkUnits;
        uint4* to = reinterpret_cast<uint4*>(v.ring);
        const uint4* src = reinterpret_cast<const uint4*>(from.ring);
        for (int u0 = ((int)blockIdx.z - 1) * step; u0 < units; u0 += ((int)gridDim.z - 1) * step) {
            uint4 saved[kForkUnits];
            for (int m = m0; m < m1; ++m) {
                const int d = mv.dst[m], s = mv.src[m];
                uint4* at = to + ((size_t)(d & kForkIndex) * v.Hkv + h) * units;
                const uint4* of = src + ((size_t)(s & kForkIndex) * v.Hkv + h) * units;
                uint4 x[kForkUnits];
#pragma unroll
                for (int i = 0; i < kForkUnits; ++i) {
                    const int u = u0 + i * kForkThreads + tid;
                    x[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (u < units && (s & (kForkSaved | kForkNothing)) == 0) x[i] = of[u];
                }
                if ((s & kForkSaved) != 0) {
#pragma unroll
                    for (int i = 0; i < kForkUnits; ++i) x[i] = saved[i];
                }
                if ((d & kForkSave) != 0) {
#pragma unroll
                    for (int i = 0; i < kForkUnits; ++i) {
                        const int u = u0 + i * kForkThreads + tid;
                        if (u < units) saved[i] = at[u];
                    }
                }
#pragma unroll
                for (int i = 0; i < kForkUnits; ++i) {
                    const int u = u0 + i * kForkThreads + tid;
                    if (u < units) at[u] = x[i];
                }
            }
        }
        return;
    }
    __shared__ int s_len[SPKV_MAX_BATCH], s_tokens[SPKV_MAX_BATCH], s_on[SPKV_MAX_BATCH];   // what move m brings
    __shared__ int s_own[SPKV_MAX_BATCH], s_stay[SPKV_MAX_BATCH], s_at[SPKV_MAX_BATCH];     // pages of its own, those that stay, place of the others on the stack
    __shared__ int s_most;
    if (tid == 0) s_most = 0;
    __syncthreads();
    for (int m = m0 + tid; m < m1; m += kForkThreads) {
        const int d = mv.dst[m], s = mv.src[m], i = m - m0;
        const int to = (d & kForkIndex) * v.Hkv + h, of = (s & kForkIndex) * v.Hkv + h;
        const bool nothing = (s & kForkNothing) != 0;
        s_len[i] = nothing ? 0 : from.kept_len[of];
        s_tokens[i] = nothing ? 0 : from.t_pair[of];
        s_on[i] = nothing ? 0 : from.gate_on[of];
        // its own pages: those that the copy needs stay, the others go back
        const int own = (d & kForkFree) != 0 ? (v.kept_len[to] + kPageTokens - 1) / kPageTokens : 0;
        const int pages = (s_len[i] + kPageTokens - 1) / kPageTokens, stay = (s & kForkCopy) != 0 ? min(own, pages) : 0;
        s_own[i] = own;
        s_stay[i] = stay;
        s_at[i] = own > stay ? atomicAdd(v.free_top, own - stay) : 0;
        if ((s & kForkCopy) != 0) v.pair_items[to] = stay;    // (scratch of the decoding steps)
        atomicMax(&s_most, max(own, pages));
    }
    __syncthreads();
    const int most = s_most;
    for (int i = tid; i < most; i += kForkThreads) {          // page table rows
        int saved = 0;
        for (int m = m0; m < m1; ++m) {
            const int d = mv.dst[m], s = mv.src[m];
            int32_t* at = v.page_table + ((size_t)(d & kForkIndex) * v.Hkv + h) * v.pt_cap;
            const int n = (s & kForkCopy) != 0 ? 0 : (s_len[m - m0] + kPageTokens - 1) / kPageTokens;
            const int old = i < v.pt_cap ? at[i] : 0;
            int x = saved;
            if ((s & (kForkSaved | kForkNothing)) == 0 && i < n)
                x = from.page_table[((size_t)(s & kForkIndex) * v.Hkv + h) * from.pt_cap + i];
            if (i >= s_stay[m - m0] && i < s_own[m - m0]) v.free_pages[s_at[m - m0] + i - s_stay[m - m0]] = old;
            if ((d & kForkSave) != 0) saved = old;
            if (i < min(n, v.pt_cap)) at[i] = x;
        }
    }
    for (int i = tid; i < v.w; i += kForkThreads) {           // logits of the rings
        float saved = 0.f;
        for (int m = m0; m < m1; ++m) {
            const int d = mv.dst[m], s = mv.src[m];
            float* at = v.ring_logit + ((size_t)(d & kForkIndex) * v.Hkv + h) * v.w;
            float x = 0.f;
            if ((s & kForkSaved) != 0) x = saved;
            else if ((s & kForkNothing) == 0) x = from.ring_logit[((size_t)(s & kForkIndex) * v.Hkv + h) * v.w + i];
            if ((d & kForkSave) != 0) saved = at[i];
            at[i] = x;
        }
    }
    for (int m = m0 + tid; m < m1; m += kForkThreads) {       // (all counters were read before the barrier)
        const int to = (mv.dst[m] & kForkIndex) * v.Hkv + h;
        v.kept_len[to] = s_len[m - m0];
        v.t_pair[to] = s_tokens[m - m0];
        v.gate_on[to] = s_on[m - m0];
    }
}

// Many pages to hand out: every copied pair is given the ids that it lacks, off the stack and then out of the pool, by its place among the
// pairs -- no atomic, of which all go to one address and are served one after the other.  Every workgroup, a pair's, adds up what
// the pairs before it lack.  The counters stand still meanwhile: the copies' launch moves them on, by the sum in pos_scratch[0].
__global__ __launch_bounds__(256) void spkv_fork_assign(SpkvView v, SpkvForkCopies copies) {
    __shared__ int s_sum[4];
    auto lacks = [&](int p) -> int { return max(0, min((v.kept_len[p] + kPageTokens - 1) / kPageTokens, v.pt_cap) - v.pair_items[p]); };
    const int tid = threadIdx.x, here = blockIdx.x, p = copies.dst[here / v.Hkv] * v.Hkv + here % v.Hkv;
    const int top = *v.free_top, next = *v.pool_next, mine = lacks(p);
    int32_t* row = v.page_table + (size_t)p * v.pt_cap + v.pair_items[p];
    int before = 0;
    for (int i = tid; i < here; i += 256) before += lacks(copies.dst[i / v.Hkv] * v.Hkv + i % v.Hkv);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) before += __shfl_xor(before, o);
    if ((tid & 63) == 0) s_sum[tid >> 6] = before;
    __syncthreads();
    const int id0 = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    for (int e = tid; e < mine; e += 256) {
        const int id = id0 + e, page = id < top ? v.free_pages[top - 1 - id] : next + id - max(top, 0);
        row[e] = page < v.n_pages ? page : -1;
    }
    if (tid == 0 && here == (int)gridDim.x - 1) v.pos_scratch[0] = id0 + mine;
}

// The copies: `chunk` pages of a pair to a workgroup and turn.  Pages that the pair does not have yet have been assigned, or are
// handed out by one atomic for the chunk.  A page's 32 KB (D = 128) are in flight at once, the next page's loads before this one's
// stores.  Stores without retention: never slower, whether the copies are read next or not, and 68 -> 53 us for eight copies of 30
// MB (4.6 TB/s written), 128 -> 107 for sixteen.
constexpr int kForkChunk = 16;
// Pages p0 .. of a pair, p_step apart, chunk at a time; row: its page ids, `stay` of which it has, of: those it copies.
template <int D>
__device__ __forceinline__ void copy_pages(const SpkvView& v, const SpkvForkSource& from, int32_t* row, const int32_t* of, int n, int stay,
                                           int p0, int p_step, int chunk) {
    const int tid = threadIdx.x;
    __shared__ int s_from[kForkChunk], s_to[kForkChunk];
    constexpr int kUnits = 2 * kPageTokens * D / 8 / kForkThreads;
    for (; p0 < n; p0 += p_step) {
        const int here = min(chunk, n - p0), fresh = max(0, p0 + here - max(stay, p0));
        if (tid < 64) {                                       // (chunk <= 64)
            PageBatch pb = {0, 0, 0};
            if (tid == 0) pb = alloc_page_batch(v, fresh);
            pb.stack_lo = __shfl(pb.stack_lo, 0);
            pb.from_stack = __shfl(pb.from_stack, 0);
            pb.pool_base = __shfl(pb.pool_base, 0);
            if (tid < here) {
                const int i = p0 + tid, to = i < stay ? row[i] : batch_page(v, pb, i - max(stay, p0));
                s_from[tid] = min(max(of[i], 0), from.n_pages - 1);
                s_to[tid] = to;
                if (i >= stay || to < 0) row[i] = max(to, 0);
                if (to < 0) *v.err_flag = 1;
            }
        }
        __syncthreads();
        const u32x4* pool = reinterpret_cast<const u32x4*>(from.pool);
        constexpr size_t kPageUnits = (size_t)2 * kPageTokens * D / 8;
        u32x4 x[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) x[u] = pool[s_from[0] * kPageUnits + u * kForkThreads + tid];
        for (int i = 0; i < here; ++i) {
            const int a = s_from[i], b = s_to[i];
            u32x4 y[kUnits];
#pragma unroll
            for (int u = 0; u < kUnits; ++u) y[u] = x[u];
            if (i + 1 < here) {
#pragma unroll
                for (int u = 0; u < kUnits; ++u) x[u] = pool[s_from[i + 1] * kPageUnits + u * kForkThreads + tid];
            }
            if (b < 0) continue;                              // (the pool is exhausted, and flagged)
            u32x4* to = reinterpret_cast<u32x4*>(pool_page(v, b));
#pragma unroll
            for (int u = 0; u < kUnits; ++u) __builtin_nontemporal_store(y[u], to + u * kForkThreads + tid);
            if (tid < kPageTokens) v.pos_pool[(size_t)b * kPageTokens + tid] = from.pos_pool[(size_t)a * kPageTokens + tid];
            else if (tid < 2 * kPageTokens)
                v.logit_pool[(size_t)b * kPageTokens + tid - kPageTokens] = from.logit_pool[(size_t)a * kPageTokens + tid - kPageTokens];
        }
        __syncthreads();
    }
}
template <int D>
__global__ __launch_bounds__(kForkThreads) void spkv_fork_pages(SpkvView v, SpkvForkSource from, SpkvForkCopies copies, int chunk, int assigned) {
    const int pair = copies.dst[blockIdx.z] * v.Hkv + blockIdx.y;
    const int n = min((v.kept_len[pair] + kPageTokens - 1) / kPageTokens, v.pt_cap), stay = assigned != 0 ? n : v.pair_items[pair];
    if (assigned != 0 && threadIdx.x == 0 && blockIdx.x + blockIdx.y + blockIdx.z == 0) {
        const int all = v.pos_scratch[0], top = *v.free_top, off_stack = min(max(top, 0), all);
        *v.free_top = top - off_stack;
        *v.pool_next += all - off_stack;
    }
    copy_pages<D>(v, from, v.page_table + (size_t)pair * v.pt_cap, from.page_table + ((size_t)copies.of[blockIdx.z] * v.Hkv + blockIdx.y) * from.pt_cap,
                  n, stay, blockIdx.x * chunk, gridDim.x * chunk, chunk);
}

// A few short sequences, none of which is a source itself: all in one launch.  Nothing that a workgroup reads is written but by the
// last one to be done, which writes the counters and gives back the pages left over (no page is handed out any more by then: the
// pool has to hold what goes beside what comes, which spkv_cache_fork sees to).
// One sequence of 500 tokens, D = 64, two KV heads: 5.4 us, both launches 3.4 and 3.2, and 2.4 us less of the host; seven of up to 2000, three
// heads, 63 workgroups: 9.1, 4.3 and 4.1 before.
template <int D>
__global__ __launch_bounds__(kForkThreads) void spkv_fork_few(SpkvView v, SpkvForkSource from, SpkvForkMoves mv, int chunk) {
    const int tid = threadIdx.x;
    struct Move {
        int to, of, len, pages, own;
    };
    auto move = [&](int m, int h) -> Move {
        const int s = mv.src[m];
        Move x;
        x.to = (mv.dst[m] & kForkIndex) * v.Hkv + h;
        x.of = (s & kForkNothing) != 0 ? -1 : (s & kForkIndex) * v.Hkv + h;
        x.len = x.of < 0 ? 0 : from.kept_len[x.of];
        x.pages = min((x.len + kPageTokens - 1) / kPageTokens, v.pt_cap);
        x.own = (v.kept_len[x.to] + kPageTokens - 1) / kPageTokens;
        return x;
    };
    const Move x = move(blockIdx.z, blockIdx.y);
    const int units = fork_ring_units(v), step = gridDim.x * kForkThreads;
    u32x4* ring = reinterpret_cast<u32x4*>(v.ring) + (size_t)x.to * units;
    const u32x4* src = reinterpret_cast<const u32x4*>(from.ring) + (size_t)max(x.of, 0) * units;
    for (int u0 = blockIdx.x * kForkThreads + tid; u0 < units; u0 += step * kForkUnits) {
        u32x4 r[kForkUnits];
#pragma unroll
        for (int i = 0; i < kForkUnits; ++i) {
            const int u = u0 + i * step;
            r[i] = x.of < 0 || u >= units ? (u32x4){0u, 0u, 0u, 0u} : src[u];
        }
#pragma unroll
        for (int i = 0; i < kForkUnits; ++i)
            if (u0 + i * step < units) ring[u0 + i * step] = r[i];
    }
    if (blockIdx.x == 0)
        for (int i = tid; i < v.w; i += kForkThreads)
            v.ring_logit[(size_t)x.to * v.w + i] = x.of < 0 ? 0.f : from.ring_logit[(size_t)x.of * v.w + i];
    copy_pages<D>(v, from, v.page_table + (size_t)x.to * v.pt_cap, from.page_table + (size_t)max(x.of, 0) * from.pt_cap, x.pages, min(x.own, x.pages),
                  blockIdx.x * chunk, gridDim.x * chunk, chunk);
    __shared__ int s_last;
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        s_last = atomicAdd(v.pair_ticket, 1) == (int)(gridDim.x * gridDim.y * gridDim.z) - 1;
    }
    __syncthreads();
    if (s_last == 0) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    const int n = (int)(gridDim.z * gridDim.y);
    for (int i = tid; i < n; i += kForkThreads) {
        const int m = i / v.Hkv;
        const Move y = move(m, i - m * v.Hkv);
        if (y.own > y.pages) {
            const int32_t* row = v.page_table + (size_t)y.to * v.pt_cap;
            const int at = atomicAdd(v.free_top, y.own - y.pages);
            for (int p = y.pages; p < y.own; ++p) v.free_pages[at + p - y.pages] = row[p];
        }
        const int tokens = y.of < 0 ? 0 : from.t_pair[y.of], on = y.of < 0 ? 0 : from.gate_on[y.of];
        v.kept_len[y.to] = y.len;
        v.t_pair[y.to] = tokens;
        v.gate_on[y.to] = on;
    }
    if (tid == 0) *v.pair_ticket = 0;                         // for the next launch
}

hipError_t spkv_launch_fork_move(const SpkvView& v, const SpkvForkSource& from, const SpkvForkMoves& mv, hipStream_t s) {
    const int units = v.n_ring_pages * (spkv_page_elems(v.D) / 8), step = kForkThreads * kForkUnits;
    spkv_fork_move<<<dim3(mv.n, v.Hkv, 1 + std::min((units + step - 1) / step, 1024)), dim3(kForkThreads), 0, s>>>(v, from, mv);
    return hipGetLastError();
}

// Eight workgroups to a compute unit at chunks of all / 2048 pages; where a few pages have to be handed out, a quarter of them, each with
// an atomic on the same address (15 of 32 beams of 5 MB, 2048 / 1024 / 512 / 256 workgroups 74 / 47 / 39 / 46 us, assigned 29).
constexpr int64_t kForkAssign = 256;
hipError_t spkv_launch_fork_pages(const SpkvView& v, const SpkvForkSource& from, const SpkvForkCopies& copies, int n, int64_t most_pages,
                                  int64_t all_pages, int64_t fresh_pages, hipStream_t s) {
    const int assigned = fresh_pages >= kForkAssign;
    if (assigned) spkv_fork_assign<<<dim3(n * v.Hkv), dim3(256), 0, s>>>(v, copies);
    const int64_t wanted = !assigned && fresh_pages * 8 > all_pages ? 512 : 2048;
    const int chunk = (int)std::max<int64_t>(1, std::min<int64_t>(kForkChunk, all_pages / wanted));
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((most_pages + chunk - 1) / chunk, 65535)), v.Hkv, n);
    if (v.D == 128) spkv_fork_pages<128><<<grid, dim3(kForkThreads), 0, s>>>(v, from, copies, chunk, assigned);
    else spkv_fork_pages<64><<<grid, dim3(kForkThreads), 0, s>>>(v, from, copies, chunk, assigned);
    return hipGetLastError();
}

// Up to 64 workgroups -- they take a ticket each, one after the other -- of up to 128 KB to copy, and few pages to give back, with one thread
// a head: one sequence of P pages a head emptied and one of five copied, one launch / two, us of a call that is waited for: two
// heads of 64, P = 5 19.3 / 19.4, 8 19.5 / 19.4, 16 20.6 / 19.3, 64 26 / 19, 917 120 / 21; eight heads of 128, P = 5 20.4 / 20.2, 8 20.8 / 20.4,
// 16 21.9 / 20.5, 64 29 / 21, 917 155 / 23.  False: it takes the other way.
constexpr int64_t kForkFewBack = 8;
bool spkv_launch_fork_few(const SpkvView& v, const SpkvForkSource& from, const SpkvForkMoves& mv, int64_t most_pages, int64_t most_back,
                          hipStream_t s, hipError_t* e) {
    if (most_back > kForkFewBack) return false;
    const int64_t pairs = (int64_t)mv.n * v.Hkv, bytes = (most_pages + v.n_ring_pages) * spkv_page_elems(v.D) * 2;
    if (pairs > kForkFewPairs) return false;
    const int64_t wide = std::min<int64_t>(kForkFewPairs / pairs, std::max<int64_t>(most_pages, (bytes + 16383) / 16384));
    if (bytes > wide * (128 << 10)) return false;
    const dim3 grid((unsigned)wide, v.Hkv, mv.n);
    const int chunk = (int)std::max<int64_t>(1, std::min<int64_t>(kForkChunk, (most_pages + wide - 1) / wide));
    if (v.D == 128) spkv_fork_few<128><<<grid, dim3(kForkThreads), 0, s>>>(v, from, mv, chunk);
    else spkv_fork_few<64><<<grid, dim3(kForkThreads), 0, s>>>(v, from, mv, chunk);
    *e = hipGetLastError();
    return true;
}

// -------------------------------------------------------------- what sequences hold, as rows
// A workgroup takes a half-page (32 pairs) at a time.  Rows of keys: four consecutive keys lie in 64 bytes of every
// chunk of eight elements, so a wave that takes four keys reads whole pieces of 64 bytes and writes whole rows.
// Values come as units of eight keys of one element and are turned in LDS.  Stores without retention: 242 MB out of a
// cache and into rows 105 -> 72 us, 6.7 TB/s of both; 32 MB 22.8 -> 10.7.
template <int D>
__global__ __launch_bounds__(256) void spkv_gather_pairs(SpkvView v, SpkvSequences of, SpkvPairRows out) {
    constexpr int kChunks = D / 8;
    __shared__ __attribute__((aligned(16))) uint16_t s_v[kHalfTokens][D + 8];
    const int tid = threadIdx.x, i = blockIdx.y / v.Hkv, h = blockIdx.y - i * v.Hkv, pair = of.seq[i] * v.Hkv + h;
    const int T = v.t_pair[pair], L = v.kept_len[pair], held = min(T, v.w), first = T % v.w;
    const int nA = (L + kHalfTokens - 1) >> 5, n_hp = nA + ((held + kHalfTokens - 1) >> 5);
    const int32_t* row = v.page_table + (size_t)pair * v.pt_cap;
    const size_t row0 = (size_t)blockIdx.y * out.rows;
    if (blockIdx.x == 0 && tid == 0 && out.counts != nullptr) out.counts[blockIdx.y] = L + held;
    // a ring slot's place among the window's pairs, oldest first
    auto age = [&](int slot) -> int { return T < v.w ? slot : slot - first + (slot < first ? v.w : 0); };
    for (int x = blockIdx.x; x < n_hp; x += gridDim.x) {
        const bool ring = x >= nA;
        const int k0 = (ring ? x - nA : x) * kHalfTokens, n = min((ring ? held : L) - k0, kHalfTokens);
        const int page = ring ? 0 : min(max(row[x >> 1], 0), v.n_pages - 1);
        const uint16_t* base = ring ? ring_page(v, pair, k0 >> 6) : pool_page(v, page);
        const int in0 = k0 & 63;
        auto place = [&](int r) -> int { return ring ? L + age(k0 + r) : k0 + r; };
        // all of the half-page's loads before anything is waited for
        constexpr int kMine = kHalfTokens * kChunks / 256;    // 16-byte units of keys, and of values, a thread
        uint4 kk[kMine], vl[kMine];
        const size_t e = (size_t)page * kPageTokens + in0 + (tid & 31);
        float logit = 0.f;
        int position = 0;
        if (out.k != nullptr) {
#pragma unroll
            for (int i2 = 0; i2 < kMine; ++i2) {
                const int u = i2 * 256 + tid;
                kk[i2] = *reinterpret_cast<const uint4*>(base + spkv_k_off(D, in0 + u / kChunks, u % kChunks * 8));
            }
        }
        if (out.v != nullptr) {
#pragma unroll
            for (int i2 = 0; i2 < kMine; ++i2) {
                const int u = i2 * 256 + tid;
                vl[i2] = *reinterpret_cast<const uint4*>(base + spkv_v_off(D, in0 + u / D * 8, u % D));
            }
        }
        if (tid < n) {
            logit = ring ? v.ring_logit[(size_t)pair * v.w + k0 + tid] : v.logit_pool[e];
            position = ring ? T - held + age(k0 + tid) : v.pos_pool[e];
        }
        if (out.k != nullptr) {
#pragma unroll
            for (int i2 = 0; i2 < kMine; ++i2) {
                const int u = i2 * 256 + tid, r = u / kChunks;
                if (r < n && place(r) < out.rows) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, kk[i2]), reinterpret_cast<u32x4*>(out.k + (row0 + place(r)) * D + u % kChunks * 8));
            }
        }
        if (out.v != nullptr) {
#pragma unroll
            for (int i2 = 0; i2 < kMine; ++i2) {
                const int u = i2 * 256 + tid, kc = u / D, d = u % D;
                const unsigned w[4] = {vl[i2].x, vl[i2].y, vl[i2].z, vl[i2].w};
#pragma unroll
                for (int j = 0; j < 8; ++j) s_v[8 * kc + j][d] = (uint16_t)(w[j >> 1] >> ((j & 1) * 16));
            }
            __syncthreads();
#pragma unroll
            for (int i2 = 0; i2 < kMine; ++i2) {
                const int u = i2 * 256 + tid, r = u / kChunks;
                if (r < n && place(r) < out.rows)
                    __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(&s_v[r][u % kChunks * 8]),
                                                reinterpret_cast<u32x4*>(out.v + (row0 + place(r)) * D + u % kChunks * 8));
            }
            __syncthreads();
        }
        if (tid < n && place(tid) < out.rows) {
            if (out.logits != nullptr) out.logits[row0 + place(tid)] = logit;
            if (out.positions != nullptr) out.positions[row0 + place(tid)] = position;
        }
    }
}

hipError_t spkv_launch_gather_pairs(const SpkvView& v, const SpkvSequences& of, int n, int most_half_pages, const SpkvPairRows& out,
                                    hipStream_t s) {
    const dim3 grid((unsigned)std::max(1, std::min(most_half_pages, 65535)), n * v.Hkv);
    if (v.D == 128) spkv_gather_pairs<128><<<grid, dim3(256), 0, s>>>(v, of, out);
    else spkv_gather_pairs<64><<<grid, dim3(256), 0, s>>>(v, of, out);
    return hipGetLastError();
}

// ------------------------------------------------------------------ append of chosen rows
// Token i of a sequence is row rows[cu[b] + i]; a row that is not there is flagged.  Up to kFewTokens tokens, and no more than the window
// holds: append_few_rows.  More, up to 64: the same in four passes of 16 rows whose loads are all in flight; lane j of a wave
// judges the j-th pair that leaves the window, out of the ring or, where the window is shorter than the call, one of the rows
// themselves, and only the last w rows reach the ring.  37 rows through a window of 16, 21 lists: 9.7
// us in rounds of 16, each behind the last, 7.4 so.
template <int D>
__device__ __forceinline__ void append_many_rows(const SpkvView& v, int pair, int h, int n, const uint16_t* __restrict__ k,
                                                 const uint16_t* __restrict__ vv, const float* __restrict__ f,
                                                 const int32_t* __restrict__ rows, int n_rows) {
    constexpr int kPasses = SPKV_MAX_TREE_NODES / 16;
    __shared__ int s_page;
    const int tid = threadIdx.x, lane = tid & 63, c = tid & 15;
    const bool mover = c < D / 8;
    int id = 0;                                               // lane j: row of token j
    if (lane < n) {
        const int r = rows[lane];
        if (r < 0 || r >= n_rows) *v.err_flag = 1;
        id = min(max(r, 0), n_rows - 1);
    }
    const int T = v.t_pair[pair], L = v.kept_len[pair];
    const float f_new = lane < n ? f[(size_t)id * v.Hkv + h] : 0.f;
    const int r0 = max(0, T - v.w), nr = max(0, max(0, T + n - v.w) - r0);         // pairs that leave, from position r0 on
    const float f_in = __shfl(f_new, min(max(r0 + lane - T, 0), 63));
    float f_old = 0.f;
    if (lane < nr) f_old = r0 + lane < T ? v.ring_logit[(size_t)pair * v.w + (r0 + lane) % v.w] : f_in;
    const int lp = L >> 6;
    int page = (L & 63) != 0 && lp < v.pt_cap ? v.page_table[(size_t)pair * v.pt_cap + lp] : -1;
    u32x4 k_new[kPasses], v_new[kPasses], k_old[kPasses], v_old[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int r = 16 * p + (tid >> 4), new_id = __shfl(id, r), old_id = __shfl(id, min(max(r0 + r - T, 0), 63));
        k_new[p] = v_new[p] = k_old[p] = v_old[p] = (u32x4){0u, 0u, 0u, 0u};
        if (mover && r < n && r >= n - v.w) {
            const size_t src = ((size_t)new_id * v.Hkv + h) * D + c * 8;
            k_new[p] = *reinterpret_cast<const u32x4*>(k + src);
            v_new[p] = *reinterpret_cast<const u32x4*>(vv + src);
        }
        if (mover && r < nr && r0 + r >= T) {
            const size_t src = ((size_t)old_id * v.Hkv + h) * D + c * 8;
            k_old[p] = *reinterpret_cast<const u32x4*>(k + src);
            v_old[p] = *reinterpret_cast<const u32x4*>(vv + src);
        } else if (mover && r < nr) {
            const int slot = (r0 + r) % v.w, sk = slot & 63;
            const uint16_t* sp = ring_page(v, pair, slot >> 6);
            const uint16_t* vs = sp + spkv_v_off(D, sk, c * 8);
            k_old[p] = *reinterpret_cast<const u32x4*>(sp + spkv_k_off(D, sk, c * 8));
            v_old[p] = (u32x4){vs[0] | ((unsigned)vs[8] << 16), vs[16] | ((unsigned)vs[24] << 16), vs[32] | ((unsigned)vs[40] << 16),
                               vs[48] | ((unsigned)vs[56] << 16)};
        }
    }
    const unsigned long long mask = __ballot(lane < nr && gate_passes(v, f_old, r0 + lane));
    const int kept = __popcll(mask), on = __popcll(__ballot(lane < n && gate_passes(v, f_new, T + lane)));
    const int first = (L + kPageTokens - 1) / kPageTokens, last = (L + kept + kPageTokens - 1) / kPageTokens;
    if (last > first && tid == 0) {                           // at most one page (kept <= 64)
        const int np = first < v.pt_cap ? alloc_page(v) : -1;
        if (np >= 0) v.page_table[(size_t)pair * v.pt_cap + first] = np;
        else *v.err_flag = 1;
        s_page = np;
    }
    __syncthreads();                                          // the leaving rows have been read
    const int new_page = last > first ? s_page : 0;
    if (tid == 0) {
        if (new_page >= 0) v.kept_len[pair] = L + kept;
        v.t_pair[pair] = T + n;
        v.gate_on[pair] += on;
    }
    if (new_page < 0) return;
    if (ends_in_new_half_page(L, L + kept))
        clear_list_end<D>(pool_page(v, (L + kept) >> 6 >= first ? new_page : page), L + kept, tid, 256);
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int r = 16 * p + (tid >> 4);
        const float lg_old = __shfl(f_old, r), lg_new = __shfl(f_new, r);
        if (r < nr && ((mask >> r) & 1ull)) {
            const int gi = L + __popcll(mask & ((1ull << r) - 1)), dk = gi & 63, to = (gi >> 6) >= first ? new_page : page;
            if (mover) store_row_chunk<D>(pool_page(v, to), dk, c, __builtin_bit_cast(uint4, k_old[p]), __builtin_bit_cast(uint4, v_old[p]));
            if (c == 0) {
                v.pos_pool[(size_t)to * kPageTokens + dk] = r0 + r;
                v.logit_pool[(size_t)to * kPageTokens + dk] = lg_old;
            }
        }
        if (r < n && r >= n - v.w) {
            const int slot = (T + r) % v.w;
            if (mover) store_row_chunk<D>(ring_page(v, pair, slot >> 6), slot & 63, c, __builtin_bit_cast(uint4, k_new[p]), __builtin_bit_cast(uint4, v_new[p]));
            if (c == 0) v.ring_logit[(size_t)pair * v.w + slot] = lg_new;
        }
    }
}
template <int D>
__global__ __launch_bounds__(256) void spkv_append_rows(SpkvView v, const uint16_t* __restrict__ k,
                                                        const uint16_t* __restrict__ vv, const float* __restrict__ f,
                                                        const int32_t* __restrict__ rows, int n_rows, SpkvCu cu) {
    const int pair = blockIdx.x, b = pair / v.Hkv, h = pair - b * v.Hkv;
    const int row0 = cu.v[b], n = cu.v[b + 1] - row0;
    if (n == 0) return;
    if (n > min(kFewTokens, v.w)) return append_many_rows<D>(v, pair, h, n, k, vv, f, rows + row0, n_rows);
    append_few_rows<D>(v, pair, h, n, v.t_pair[pair], v.kept_len[pair], k, vv, f, [&](int i) -> int {
        const int r = rows[row0 + i];
        if (r < 0 || r >= n_rows) *v.err_flag = 1;
        return min(max(r, 0), n_rows - 1);
    });
}

hipError_t spkv_launch_append_rows(const SpkvView& v, const uint16_t* k, const uint16_t* vv, const float* f,
                                   const int32_t* rows, int n_rows, const SpkvCu& cu, hipStream_t s) {
    if (v.D == 128) spkv_append_rows<128><<<dim3(v.n_pairs), dim3(256), 0, s>>>(v, k, vv, f, rows, n_rows, cu);
    else spkv_append_rows<64><<<dim3(v.n_pairs), dim3(256), 0, s>>>(v, k, vv, f, rows, n_rows, cu);
    return hipGetLastError();
}
