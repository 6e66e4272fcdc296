// Queries, keys and values of a layer out of one projection's rows: RMS norm of every head,
// rotation by positions on one or more axes, and the layout that the cache's calls take, in one
// pass; and the gradients of that.
#include <cmath>

#include "spkv_device.h"

// The mathematics, for a head x of D elements with weight w, pair i = (a, b) of elements and
// angle phi_i = position[axis_i] * inv_freq_i:
//   n = x w r,  r = 1 / sqrt(mean(x^2) + eps);   a' = a cos phi - b sin phi,  b' = a sin phi + b cos phi
// backward, from the gradient y of the rotated head:
//   g = y rotated by -phi;   dx = r (g w - x r^2 mean(g w x));   dw = sum over tokens and heads of g x r
//
// Bound by memory: forward reads and writes every element once, backward reads two and writes one.  Forward of 32k tokens
// (48 heads of 128, bf16: 805 MB) 153 us, 5.3 TB/s, the rate of a copy; gradients of 16k (570 MB) 118 us, 4.8 TB/s.
// A row (head of a token) lies in D / 16 lanes, sixteen elements a lane as two chunks of eight chosen
// so that both elements of every pair are in one lane: the rotation then crosses no lanes, and
// the norm's sum takes log2(D / 16) exchanges.  A workgroup takes a tile of consecutive rows, all heads of
// a token after each other, so that the angles of its few tokens are worked out once, by all
// threads, and shared through LDS while the first rows are on their way.
//
// Angles.  A position times a frequency loses the angle where it is far: 2^20 * 1.0 rad in 32 bits is off by
// 0.03.  Here a frequency is a fraction of a turn in 64 bits (fixed point), so that position *
// fraction modulo 2^64 IS the angle modulo a turn, exactly; its upper 32 bits give sine and cosine by
// octant and Taylor polynomial, to 1e-7.
struct RopeTable {
    uint64_t turn[SPKV_MAX_ROPE_PAIRS];
    uint8_t axis[SPKV_MAX_ROPE_PAIRS];
};

__device__ __forceinline__ float2 cos_sin_of_turn(unsigned turn) {
    const unsigned quadrant = (turn + 0x20000000u) >> 30;
    const float a = (float)(int)(turn - (quadrant << 30)) * 1.4629180792671596e-9f;     // 2 pi / 2^32
    const float z = a * a;
    const float s = a + a * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
    const float c = 1.f - z * (0.5f - z * (1.f / 24 - z * (1.f / 720 - z * (1.f / 40320 - z * (1.f / 3628800)))));
    const float x = (quadrant & 1u) ? s : c, y = (quadrant & 1u) ? c : s;
    return make_float2((quadrant + 1u) & 2u ? -x : x, quadrant & 2u ? -y : y);
}

// Sixteen elements of a row in one lane: chunks (of eight) c0 and c1.
struct RowChunks {
    int c0, c1;
    bool turned0, turned1;      // chunk c0 / c1 holds rotated elements (neighbouring pairs: some)
};
template <int D, bool ADJ>
__device__ __forceinline__ RowChunks row_chunks(int c, int rot_dim) {
    RowChunks r;
    if (ADJ) {
        r.c0 = c;
        r.c1 = c + D / 16;
        r.turned0 = r.c0 * 8 < rot_dim;
        r.turned1 = r.c1 * 8 < rot_dim;
    } else {                    // element i with i + rot_dim / 2 (a multiple of eight)
        const int m = rot_dim >> 4;
        r.turned0 = r.turned1 = c < m;
        r.c0 = c < m ? c : 2 * c;
        r.c1 = c < m ? c + m : 2 * c + 1;
    }
    return r;
}

template <typename T> struct Raw8;
template <> struct Raw8<uint16_t> { uint4 u; };
template <> struct Raw8<float> { uint4 u, w; };

// STREAM (see Streaming below; bf16): 1: loads, 2: stores too ask the caches for no retention.
template <int STREAM>
__device__ __forceinline__ uint4 load_unit(const void* p) {
    if (STREAM > 0) return __builtin_bit_cast(uint4, load_stream_b128(static_cast<const uint16_t*>(p)));
    return *static_cast<const uint4*>(p);
}
template <int STREAM>
__device__ __forceinline__ void store_unit(uint4 u, void* p) {
    typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
    if (STREAM > 1) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, u), static_cast<u32x4*>(p));
    else *static_cast<uint4*>(p) = u;
}
template <int STREAM>
__device__ __forceinline__ void load8(Raw8<uint16_t>& r, const uint16_t* p) { r.u = load_unit<STREAM>(p); }
template <int STREAM>
__device__ __forceinline__ void load8(Raw8<float>& r, const float* p) {
    r.u = *reinterpret_cast<const uint4*>(p);
    r.w = *reinterpret_cast<const uint4*>(p + 4);
}
template <int STREAM>
__device__ __forceinline__ void store8(const Raw8<uint16_t>& r, uint16_t* p) { store_unit<STREAM>(r.u, p); }
template <int STREAM>
__device__ __forceinline__ void store8(const Raw8<float>& r, float* p) {
    *reinterpret_cast<uint4*>(p) = r.u;
    *reinterpret_cast<uint4*>(p + 4) = r.w;
}
__device__ __forceinline__ void widen8(const Raw8<uint16_t>& r, float (&x)[8]) {
    const unsigned w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        x[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&x)[8]) {
    const unsigned w[8] = {r.u.x, r.u.y, r.u.z, r.u.w, r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(float, w[e]);
}
__device__ __forceinline__ void round8(Raw8<uint16_t>& r, const float (&x)[8]) {       // one rounding, at the end
    unsigned w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __bf16 lo = (__bf16)x[2 * e], hi = (__bf16)x[2 * e + 1];
        w[e] = (unsigned)__builtin_bit_cast(uint16_t, lo) | ((unsigned)__builtin_bit_cast(uint16_t, hi) << 16);
    }
    r.u = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void round8(Raw8<float>& r, const float (&x)[8]) {
    unsigned w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __builtin_bit_cast(unsigned, x[e]);
    r.u = make_uint4(w[0], w[1], w[2], w[3]);
    r.w = make_uint4(w[4], w[5], w[6], w[7]);
}

// Angles of tokens first .. first + n - 1 into s_cs[token][pair] (cos, sin).
__device__ __forceinline__ void fill_angles(const SpkvRope& a, const RopeTable& table, int first, int n, float2* s_cs) {
    const int pairs = a.rot_dim >> 1;
    if (pairs == 0) return;
    for (int i = threadIdx.x; i < n * pairs; i += kRopeThreads) {
        const int t = i / pairs, p = i - t * pairs;
        const int pos = a.positions[(int64_t)table.axis[p] * a.n_tokens + min(first + t, a.n_tokens - 1)];
        const uint64_t turn = (uint64_t)(int64_t)pos * table.turn[p];
        s_cs[i] = cos_sin_of_turn((unsigned)(turn >> 32));
    }
}

// The rotation of a lane's pairs by their angles (BACK: the other way).
template <int D, bool ADJ, bool BACK>
__device__ __forceinline__ void rotate16(const RowChunks& rc, int rot_dim, const float2* cs, float (&x)[8], float (&y)[8]) {
    if (ADJ) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float (&z)[8] = half ? y : x;
            const int p0 = (half ? rc.c1 : rc.c0) * 4;
            if (!(half ? rc.turned1 : rc.turned0)) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (2 * (p0 + i) < rot_dim) {
                    const float2 t = cs[p0 + i];
                    const float s = BACK ? -t.y : t.y, a = z[2 * i], b = z[2 * i + 1];
                    z[2 * i] = a * t.x - b * s;
                    z[2 * i + 1] = a * s + b * t.x;
                }
            }
        }
    } else if (rc.turned0) {
        const float4* c4 = reinterpret_cast<const float4*>(cs + rc.c0 * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 t = c4[i];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float c = u ? t.z : t.x, s0 = u ? t.w : t.y, s = BACK ? -s0 : s0;
                const float a = x[2 * i + u], b = y[2 * i + u];
                x[2 * i + u] = a * c - b * s;
                y[2 * i + u] = a * s + b * c;
            }
        }
    }
}

template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) x += __shfl_xor(x, o);
    return x;
}

// A row's place: kind 0 = query, 1 = key, 2 = value; head within the kind.
struct RowPlace {
    int token, kind, head;
};
__device__ __forceinline__ RowPlace place_of(const SpkvRope& a, int token, int hh) {
    RowPlace r;
    r.token = token;
    r.kind = hh < a.n_q ? 0 : hh < a.n_q + a.n_kv ? 1 : 2;
    r.head = hh - (r.kind == 0 ? 0 : r.kind == 1 ? a.n_q : a.n_q + a.n_kv);
    return r;
}
template <typename T>
__device__ __forceinline__ T* row_of(const SpkvRowSet (&s)[3], const RowPlace& r) {
    const SpkvRowSet& k = s[0];
    T* p = static_cast<T*>(k.p);
    int64_t ts = k.token_stride, hs = k.head_stride;
    if (r.kind == 1) {
        p = static_cast<T*>(s[1].p);
        ts = s[1].token_stride;
        hs = s[1].head_stride;
    } else if (r.kind == 2) {
        p = static_cast<T*>(s[2].p);
        ts = s[2].token_stride;
        hs = s[2].head_stride;
    }
    return p + r.token * ts + r.head * hs;
}

// One tile of rows: tile_rows consecutive rows of the order (token, head).
template <typename T, int D, bool ADJ, bool NORM, int STREAM>
__global__ __launch_bounds__(kRopeThreads) void spkv_rope_forward(SpkvRope a, RopeTable table) {
    constexpr int LPR = D / 16, RPP = kRopeThreads / LPR;      // lanes per row, rows per pass
    extern __shared__ __attribute__((aligned(16))) float s_rope[];
    float* s_w = s_rope;                                       // [2][D] weights (NORM)
    float2* s_cs = reinterpret_cast<float2*>(s_rope + (NORM ? 2 * D : 0));
    const int tid = threadIdx.x, c = tid & (LPR - 1), lane_row = tid / LPR;
    const int row0 = (int)blockIdx.x * a.tile_rows, n_rows = min(a.tile_rows, a.n_rows - row0);
    const int first = row0 / a.n_heads, last = (row0 + n_rows - 1) / a.n_heads;
    const RowChunks rc = row_chunks<D, ADJ>(c, a.rot_dim);

    int r = lane_row;
    int token = (row0 + r) / a.n_heads, hh = row0 + r - token * a.n_heads;
    Raw8<T> x0, x1;
    RowPlace at = {0, 0, 0};
    if (r < n_rows) {
        at = place_of(a, token, hh);
        const T* p = row_of<const T>(a.in, at);
        load8<STREAM>(x0, p + rc.c0 * 8);
        load8<STREAM>(x1, p + rc.c1 * 8);
    }
    if (NORM)
        for (int i = tid; i < 2 * D; i += kRopeThreads) {
            const float* w = i < D ? a.q_weight : a.k_weight;
            s_w[i] = w != nullptr ? w[i & (D - 1)] : 1.f;
        }
    fill_angles(a, table, first, last - first + 1, s_cs);
    __syncthreads();
    for (; r < n_rows; r += RPP) {
        const RowPlace here = at;
        T* o = row_of<T>(a.out, here);
        float f0[8], f1[8];
        if (here.kind < 2) {
            widen8(x0, f0);
            widen8(x1, f1);
        } else {                                               // values: as they are
            store8<STREAM>(x0, o + rc.c0 * 8);
            store8<STREAM>(x1, o + rc.c1 * 8);
        }
        if (r + RPP < n_rows) {                                // the next row travels meanwhile
            hh += RPP;
            while (hh >= a.n_heads) {
                hh -= a.n_heads;
                ++token;
            }
            at = place_of(a, token, hh);
            const T* p = row_of<const T>(a.in, at);
            load8<STREAM>(x0, p + rc.c0 * 8);
            load8<STREAM>(x1, p + rc.c1 * 8);
        }
        if (here.kind == 2) continue;                          // (a row's lanes go the same way)
        if (NORM) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += f0[e] * f0[e] + f1[e] * f1[e];
            const float r_norm = rsqrtf(row_sum<LPR>(sum) * (1.f / D) + a.eps);
            const float* w = s_w + here.kind * D;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f0[e] *= r_norm * w[rc.c0 * 8 + e];
                f1[e] *= r_norm * w[rc.c1 * 8 + e];
            }
        }
        rotate16<D, ADJ, false>(rc, a.rot_dim, s_cs + (here.token - first) * (a.rot_dim >> 1), f0, f1);
        Raw8<T> y;
        round8(y, f0);
        store8<STREAM>(y, o + rc.c0 * 8);
        round8(y, f1);
        store8<STREAM>(y, o + rc.c1 * 8);
    }
}

// Gradients.  in: those of the rotated heads (and values), x: the forward's inputs (NORM), out: the
// gradients of those.  A workgroup walks every gridDim-th tile and keeps its share of the weights'
// gradients, sixteen columns a lane: those of queries in registers, those of the fewer keys in LDS (both in
// registers left room for three waves on a SIMD instead of four).  They meet in LDS at
// the end and leave as one partial row of 2 D floats, which spkv_rope_weight_sum adds up in a
// fixed order (no atomics: equal calls give equal bits).
template <typename T, int D, bool ADJ, bool NORM, int STREAM>
__global__ __launch_bounds__(kRopeThreads, sizeof(T) == 2 ? 4 : 3) void spkv_rope_backward(SpkvRope a, RopeTable table) {
    constexpr int LPR = D / 16, RPP = kRopeThreads / LPR;
    extern __shared__ __attribute__((aligned(16))) float s_rope[];
    float* s_w = s_rope;
    f32x4* s_dwk = reinterpret_cast<f32x4*>(s_rope + 2 * D) + threadIdx.x;       // this lane's four units, kRopeThreads apart
    float2* s_cs = reinterpret_cast<float2*>(s_rope + (NORM ? 2 * D + 16 * kRopeThreads : 0));
    const int tid = threadIdx.x, c = tid & (LPR - 1), lane_row = tid / LPR;
    const RowChunks rc = row_chunks<D, ADJ>(c, a.rot_dim);
    if (NORM) {
        for (int i = tid; i < 2 * D; i += kRopeThreads) {
            const float* w = i < D ? a.q_weight : a.k_weight;
            s_w[i] = w != nullptr ? w[i & (D - 1)] : 1.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s_dwk[i * kRopeThreads] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    float dwq[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) dwq[e] = 0.f;

    for (int tile = blockIdx.x; tile < a.n_tiles; tile += gridDim.x) {
        const int row0 = tile * a.tile_rows, n_rows = min(a.tile_rows, a.n_rows - row0);
        const int first = row0 / a.n_heads, last = (row0 + n_rows - 1) / a.n_heads;
        int r = lane_row;
        int token = (row0 + r) / a.n_heads, hh = row0 + r - token * a.n_heads;
        Raw8<T> g0, g1, x0, x1;
        RowPlace at = {0, 0, 0};
        auto load_row = [&]() {
            at = place_of(a, token, hh);
            const T* p = row_of<const T>(a.in, at);
            load8<STREAM>(g0, p + rc.c0 * 8);
            load8<STREAM>(g1, p + rc.c1 * 8);
            if (NORM && at.kind < 2) {
                const T* q = row_of<const T>(a.x, at);
                load8<STREAM>(x0, q + rc.c0 * 8);
                load8<STREAM>(x1, q + rc.c1 * 8);
            }
        };
        if (r < n_rows) load_row();
        __syncthreads();                                       // the angles of the tile before are no longer read
        fill_angles(a, table, first, last - first + 1, s_cs);
        __syncthreads();
        for (; r < n_rows; r += RPP) {
            const RowPlace here = at;
            T* o = row_of<T>(a.out, here);
            float f0[8], f1[8], v0[8], v1[8];
            if (here.kind < 2) {
                widen8(g0, f0);
                widen8(g1, f1);
                if (NORM) {
                    widen8(x0, v0);
                    widen8(x1, v1);
                }
            } else {                                           // values: as they are
                store8<STREAM>(g0, o + rc.c0 * 8);
                store8<STREAM>(g1, o + rc.c1 * 8);
            }
            if (r + RPP < n_rows) {
                hh += RPP;
                while (hh >= a.n_heads) {
                    hh -= a.n_heads;
                    ++token;
                }
                load_row();
            }
            if (here.kind < 2) {                               // a row's lanes go the same way
                rotate16<D, ADJ, true>(rc, a.rot_dim, s_cs + (here.token - first) * (a.rot_dim >> 1), f0, f1);
                if (NORM) {
                    float square = 0.f, dot = 0.f;
                    const float* w = s_w + here.kind * D;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float w0 = w[rc.c0 * 8 + e], w1 = w[rc.c1 * 8 + e];
                        square += v0[e] * v0[e] + v1[e] * v1[e];
                        dot += f0[e] * w0 * v0[e] + f1[e] * w1 * v1[e];
                    }
                    square = row_sum<LPR>(square);
                    dot = row_sum<LPR>(dot);
                    const float rn = rsqrtf(square * (1.f / D) + a.eps);
                    const float back = rn * rn * dot * (1.f / D);
                    if (here.kind == 0) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            dwq[e] += f0[e] * (v0[e] * rn);
                            dwq[8 + e] += f1[e] * (v1[e] * rn);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            f32x4 p0 = s_dwk[i * kRopeThreads], p1 = s_dwk[(2 + i) * kRopeThreads];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                p0[e] += f0[4 * i + e] * (v0[4 * i + e] * rn);
                                p1[e] += f1[4 * i + e] * (v1[4 * i + e] * rn);
                            }
                            s_dwk[i * kRopeThreads] = p0;
                            s_dwk[(2 + i) * kRopeThreads] = p1;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f0[e] = rn * (f0[e] * w[rc.c0 * 8 + e] - v0[e] * back);
                        f1[e] = rn * (f1[e] * w[rc.c1 * 8 + e] - v1[e] * back);
                    }
                }
                Raw8<T> y;
                round8(y, f0);
                store8<STREAM>(y, o + rc.c0 * 8);
                round8(y, f1);
                store8<STREAM>(y, o + rc.c1 * 8);
            }
        }
    }
    if (!NORM || a.partial == nullptr) return;
    // rows of a wave meet by exchanges, waves in LDS
    float dwk[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) dwk[e] = s_dwk[(e >> 2) * kRopeThreads][e & 3];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
            dwq[e] += __shfl_xor(dwq[e], o);
            dwk[e] += __shfl_xor(dwk[e], o);
        }
    }
    __syncthreads();                                           // weights and angles are no longer read
    const int lane = tid & 63, wave = tid >> 6;
    float* s_sum = s_rope;                                     // [waves][2][D]
    if (lane < LPR) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int d = (e < 8 ? rc.c0 : rc.c1) * 8 + (e & 7);
            s_sum[(wave * 2) * D + d] = dwq[e];
            s_sum[(wave * 2 + 1) * D + d] = dwk[e];
        }
    }
    __syncthreads();
    for (int i = tid; i < 2 * D; i += kRopeThreads) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kRopeThreads / 64; ++w) sum += s_sum[w * 2 * D + i];
        a.partial[(size_t)blockIdx.x * 2 * D + i] = sum;
    }
}

// Column sums of the partial rows: a workgroup takes sixteen columns, four a thread, its threads every 64th row.
template <int D>
__global__ __launch_bounds__(256) void spkv_rope_weight_sum(const float* __restrict__ partial, int n,
                                                            float* __restrict__ dq, float* __restrict__ dk) {
    __shared__ f32x4 s[4][4];
    const int unit = threadIdx.x & 3, lane = threadIdx.x & 63, col = ((int)blockIdx.x * 4 + unit) * 4;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 16
    for (int r = threadIdx.x >> 2; r < n; r += 64) sum += *reinterpret_cast<const f32x4*>(partial + (size_t)r * 2 * D + col);
#pragma unroll
    for (int o = 4; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], o);
    if (lane < 4) s[threadIdx.x >> 6][lane] = sum;
    __syncthreads();
    if (threadIdx.x < 4) {
        sum = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
        float* out = col < D ? dq : dk;
        if (out != nullptr) *reinterpret_cast<f32x4*>(out + (col & (D - 1))) = sum;
    }
}

// Rows of a tile: as few as one pass while the chip still has room for more workgroups, and more from
// there on, so that fewer tokens are cut by tiles and their angles worked out twice.  Few heads bring many
// tokens to a tile: no more passes than the angles of 32 KB serve.
static int tile_tokens(int rows, int n_heads) { return (rows + n_heads - 2) / n_heads + 1; }
static int tile_rows(int64_t n_rows, int n_heads, int head_dim, int wanted) {
    const int pass = kRopeThreads / (head_dim / 16);
    int rows = pass;
    while (rows < 8 * pass && n_rows / (rows * 2) >= wanted &&
           (size_t)tile_tokens(rows * 2, n_heads) * (head_dim / 2) * sizeof(float2) <= 32768)
        rows *= 2;
    return rows;
}

int spkv_rope_backward_blocks(int64_t n_rows, int n_heads, int head_dim) {
    const int rows = tile_rows(n_rows, n_heads, head_dim, kRopeGradBlocks);
    return (int)std::min<int64_t>((n_rows + rows - 1) / rows, kRopeGradBlocks);
}

// Streaming.  Once a bf16 call moves more than the 256 MB of the last cache, what it reads is not there and need not stay: loads
// without retention leave the cache to what is written, for whoever reads that next -- unless that alone is more than it
// holds.  D = 128, 40 normed heads of 48, us plain / such loads / stores too, into buffers that are not in the cache: gradients of
// 6800 tokens (251 MB) 57.6 / 53.9 / 55.4, 16384 (604 MB, 201 of them written) 121 / 118 / 112, 32768 (1208, 403 written)
// 229 / 226 / 216; forward of 14000 (344) 70.8 / 70.6 / 68.1, 32768 (805, 403 written) 156 / 157 / 151.  Into the last call's
// buffers, where loads alone leave what is written for the next kernel: 6800 tokens 47.7 / 51.4 / 53.4, 16384 120 / 102 / 111, 32768
// 229 / 227 / 214; forward of 14000 67.9 / 58.1 / 67.8, 32768 156 / 157 / 150.
// fp32 calls, two loads and stores a chunk, do without: forward of 16384 tokens (805 MB) 158 / 164 / 168, gradients of 8192 (604 MB)
// 122 / 129 / 133, with D = 64 of 20000 (461 MB) 98 / 103 / 105; into the last call's buffers 158 / 163 / 168, 122 / 121 / 133, 97 / 98 / 104.
constexpr int64_t kStreamBytes = (int64_t)320 << 20, kStreamWritten = (int64_t)256 << 20;

template <typename T, int D, bool ADJ, bool NORM, int STREAM>
static hipError_t launch_rope(SpkvRope a, const RopeTable& table, bool backward, hipStream_t s) {
    a.tile_rows = tile_rows(a.n_rows, a.n_heads, D, backward ? kRopeGradBlocks : kRopeBlocks);
    a.n_tiles = (a.n_rows - 1) / a.tile_rows + 1;
    const int tokens = std::min(tile_tokens(a.tile_rows, a.n_heads), a.n_tokens);       // of a tile, at most
    size_t lds = (NORM ? 2 * D * sizeof(float) : 0) + (size_t)tokens * (a.rot_dim / 2) * sizeof(float2);
    if (!backward) {
        spkv_rope_forward<T, D, ADJ, NORM, STREAM><<<dim3(a.n_tiles), dim3(kRopeThreads), lds, s>>>(a, table);
        return hipGetLastError();
    }
    const int blocks = spkv_rope_backward_blocks(a.n_rows, a.n_heads, D);
    if (NORM) lds += (size_t)kRopeThreads * 16 * sizeof(float);      // (also room for what the waves meet in)
    spkv_rope_backward<T, D, ADJ, NORM, STREAM><<<dim3(blocks), dim3(kRopeThreads), lds, s>>>(a, table);
    if (NORM && a.partial != nullptr)
        spkv_rope_weight_sum<D><<<dim3(2 * D / 16), dim3(256), 0, s>>>(a.partial, blocks, a.dq_weight, a.dk_weight);
    return hipGetLastError();
}

template <typename T, int D, bool ADJ, bool NORM>
static hipError_t launch_rope(const SpkvRope& a, const RopeTable& table, bool backward, hipStream_t s) {
    const int64_t written = (int64_t)a.n_rows * D * sizeof(T);
    const int64_t moved = 2 * written + (backward && NORM ? (int64_t)a.n_tokens * (a.n_q + a.n_kv) * D * sizeof(T) : 0);
    if constexpr (sizeof(T) == 2) {
        if (moved > kStreamBytes)
            return written <= kStreamWritten ? launch_rope<T, D, ADJ, NORM, 1>(a, table, backward, s)
                                             : launch_rope<T, D, ADJ, NORM, 2>(a, table, backward, s);
    }
    return launch_rope<T, D, ADJ, NORM, 0>(a, table, backward, s);
}

template <typename T, int D>
static hipError_t launch_rope(const SpkvRope& a, const RopeTable& table, bool adjacent, bool norm, bool backward,
                              hipStream_t s) {
    if (norm)
        return adjacent ? launch_rope<T, D, true, true>(a, table, backward, s)
                        : launch_rope<T, D, false, true>(a, table, backward, s);
    return adjacent ? launch_rope<T, D, true, false>(a, table, backward, s)
                    : launch_rope<T, D, false, false>(a, table, backward, s);
}

hipError_t spkv_launch_rope(const SpkvRope& a, const double* inv_freq, const uint8_t* axis, int head_dim, bool fp32,
                            bool adjacent, bool norm, bool backward, hipStream_t s) {
    RopeTable table = {};
    for (int i = 0; i < a.rot_dim / 2; ++i) {
        // frequency in turns per position, its whole part dropped: positions are whole numbers
        long double part = (long double)inv_freq[i] * 0.159154943091895335768883763372514362L;
        if (!(part >= 0.0L && part < 1.0L)) part -= floorl(part);
        table.turn[i] = part >= 1.0L ? 0u : (uint64_t)(part * 18446744073709551616.0L);
        table.axis[i] = axis != nullptr ? axis[i] : 0;
    }
    if (fp32)
        return head_dim == 128 ? launch_rope<float, 128>(a, table, adjacent, norm, backward, s)
                               : launch_rope<float, 64>(a, table, adjacent, norm, backward, s);
    return head_dim == 128 ? launch_rope<uint16_t, 128>(a, table, adjacent, norm, backward, s)
                           : launch_rope<uint16_t, 64>(a, table, adjacent, norm, backward, s);
}
