// RMS norm of every query and key head with the position rotation in the same pass (moc_norm_rope), and its backward pass.
//
//   r = 1 / sqrt(mean_c x_c^2 + eps),  u_c = x_c r w_c,  and of every rotated pair of channels (a, b), with the angle t:
//   y_a = u_a cos t - u_b sin t,  y_b = u_b cos t + u_a sin t.
//   Backward:  g = the rotation by -t of dy,  xh = x r,  dw = sum over heads and tokens of g xh,
//   dx = r (w g - xh mean_c(w g xh)).
//
// Both are bound by HBM where instructions do not get in the way: each value is read once and written once, and what a row needs
// beside its own values is shared by all heads of a token.  So a warp takes a token and walks its heads - or, of few heads, each of its lane
// groups takes a token: the angles - formed in turns, in 64 bits, reduced to a part of a turn and only then rounded to 32, so that far
// positions lose nothing - are made once for all of them.
// A lane group is 16 lanes, at d = 64 eight.  A lane holds four pairs of channels of a row, the first channels of two pairs in one packed register and
// the second ones in another, whichever channels the pairs are of: the norm, the rotation and their gradients are packed multiply-adds, and the
// rotation needs no other lane.
// 33k tokens, 24 + 24 heads of 128, bf16: forward 131 us, 6.2 TB/s (94 % of what a copy reaches); backward 219 us, 5.5 TB/s: there the
// instructions of a row (some 110) keep the loads from being closer together.
// Where there are too few tokens to fill the GPU, a token's heads are dealt to several warps.
#include <algorithm>
#include <math.h>
#include <new>
#include <type_traits>

#include "moc_common.cuh"
#include "moc_tc.cuh"

namespace moc {

constexpr int kMaxPairs = 64, kMaxAxes = 4;

// by value to the kernels: turns of a pair for one step of its axis, and the axis
struct RopeTable {
    double turns[kMaxPairs];
    uint8_t axis[kMaxPairs];
};

}  // namespace moc

struct moc_rope {
    int d, n_pairs, n_axes;
    unsigned flags;
    float eps;
    moc::RopeTable tab;
};

namespace moc {

constexpr int kRopeWarps = 8;         // warps per block, each with tokens of its own

// one of the two tensors of a call
struct RopeSide {
    const void *x;                    // forward: x; backward: x (unused without a norm)
    const __nv_bfloat16 *dy;          // backward
    void *out;                        // forward: y (bf16); backward: dx (the type of x)
    const float *w;                   // null: no norm
    int64_t x_head, x_tok, dy_head, dy_tok, out_head, out_tok;
    int heads;
};

struct RopeParams {
    RopeSide side[2];                 // queries, keys
    const int32_t *pos;
    float *part;                      // backward: [blocks][2][d] sums for dw
    int n_tokens, n_axes, n_pairs;
    int units[2];                     // batches that a token's heads make
    int per_warp, n_split;            // batches a warp takes, warps that share a token
    float eps, inv_d;
};

using tc::add2;
using tc::fma2;
using tc::mul2;
using tc::pack2;
using tc::unpack2;

// A lane's four pairs: a[k] the first channels of pairs 2 k and 2 k + 1, b[k] the second ones.
struct Pairs {
    uint64_t a[2], b[2];
};
__device__ __forceinline__ uint64_t both(float v) { return pack2(v, v); }

// The channels of a lane's pairs.  Neighbours: eight consecutive ones.  Halves: lanes up to n_pairs / 4 have four channels and the four that
// are n_pairs behind them, the others eight that are not turned.  `lo`, `hi`: where its two blocks of four begin.
struct Channels {
    int lo, hi;
    __device__ __forceinline__ Channels(bool halves, int chunk, int n_pairs) {
        const int turned = n_pairs >> 2;
        lo = !halves ? chunk * 8 : chunk < turned ? chunk * 4 : 2 * n_pairs + (chunk - turned) * 8;
        hi = halves && chunk < turned ? n_pairs + chunk * 4 : lo + 4;
    }
    // channel of place i (0..3) among the first (second = 0) or second channels
    __device__ __forceinline__ int of(bool halves, int i, int second) const {
        if (halves) return (second ? hi : lo) + i;
        return lo + 2 * i + second;
    }
};

// a lane's part of a row, as it is loaded: its two blocks of four channels
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
    uint4 u;
    template <bool HALVES>
    __device__ __forceinline__ void load(const __nv_bfloat16 *row, const Channels &c) {
        if (HALVES) {
            const uint2 x = *reinterpret_cast<const uint2 *>(row + c.lo), y = *reinterpret_cast<const uint2 *>(row + c.hi);
            u = make_uint4(x.x, x.y, y.x, y.y);
        } else {
            u = *reinterpret_cast<const uint4 *>(row + c.lo);
        }
    }
    template <bool HALVES>
    __device__ __forceinline__ Pairs get() const {
        auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
        auto hi = [](uint32_t x) { return __uint_as_float(x & 0xffff0000u); };
        if (HALVES) return Pairs{{pack2(lo(u.x), hi(u.x)), pack2(lo(u.y), hi(u.y))}, {pack2(lo(u.z), hi(u.z)), pack2(lo(u.w), hi(u.w))}};
        return Pairs{{pack2(lo(u.x), lo(u.y)), pack2(lo(u.z), lo(u.w))}, {pack2(hi(u.x), hi(u.y)), pack2(hi(u.z), hi(u.w))}};
    }
};
template <> struct Raw<float> {
    float4 u, v;
    template <bool HALVES>
    __device__ __forceinline__ void load(const float *row, const Channels &c) {
        u = *reinterpret_cast<const float4 *>(row + c.lo);
        v = *reinterpret_cast<const float4 *>(row + c.hi);
    }
    template <bool HALVES>
    __device__ __forceinline__ Pairs get() const {
        if (HALVES) return Pairs{{pack2(u.x, u.y), pack2(u.z, u.w)}, {pack2(v.x, v.y), pack2(v.z, v.w)}};
        return Pairs{{pack2(u.x, u.z), pack2(v.x, v.z)}, {pack2(u.y, u.w), pack2(v.y, v.w)}};
    }
};
// to a row's channels lo.. and hi..: the result's one rounding
template <bool HALVES>
__device__ __forceinline__ void put_pairs(__nv_bfloat16 *row, const Channels &c, const Pairs &v) {
    float a[4], b[4];
    unpack2(v.a[0], a[0], a[1]); unpack2(v.a[1], a[2], a[3]);
    unpack2(v.b[0], b[0], b[1]); unpack2(v.b[1], b[2], b[3]);
    if (HALVES) {
        *reinterpret_cast<uint2 *>(row + c.lo) = make_uint2(tc::bf16x2(a[0], a[1]), tc::bf16x2(a[2], a[3]));
        *reinterpret_cast<uint2 *>(row + c.hi) = make_uint2(tc::bf16x2(b[0], b[1]), tc::bf16x2(b[2], b[3]));
    } else {
        *reinterpret_cast<uint4 *>(row + c.lo) = make_uint4(tc::bf16x2(a[0], b[0]), tc::bf16x2(a[1], b[1]), tc::bf16x2(a[2], b[2]), tc::bf16x2(a[3], b[3]));
    }
}
template <bool HALVES>
__device__ __forceinline__ void put_pairs(float *row, const Channels &c, const Pairs &v) {
    float a[4], b[4];
    unpack2(v.a[0], a[0], a[1]); unpack2(v.a[1], a[2], a[3]);
    unpack2(v.b[0], b[0], b[1]); unpack2(v.b[1], b[2], b[3]);
    *reinterpret_cast<float4 *>(row + c.lo) = HALVES ? make_float4(a[0], a[1], a[2], a[3]) : make_float4(a[0], b[0], a[1], b[1]);
    *reinterpret_cast<float4 *>(row + c.hi) = HALVES ? make_float4(b[0], b[1], b[2], b[3]) : make_float4(a[2], b[2], a[3], b[3]);
}

// the angles of a lane's four pairs at one token
struct Angles {
    uint64_t cs[2], sn[2], neg[2];
    __device__ __forceinline__ void make(const double *s_turns, const uint8_t *s_axis, const int32_t *pos, int chunk, int n_pairs) {
        float c[4], s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = chunk * 4 + i;
            c[i] = 1.f;
            s[i] = 0.f;
            if (pair < n_pairs) {
                const double t = (double)pos[s_axis[pair]] * s_turns[pair];
                sincospif(2.f * (float)(t - rint(t)), &s[i], &c[i]);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            cs[k] = pack2(c[2 * k], c[2 * k + 1]);
            sn[k] = pack2(s[2 * k], s[2 * k + 1]);
            neg[k] = pack2(-s[2 * k], -s[2 * k + 1]);
        }
    }
    // the rotation of v (BACK: by the negative angle); `turned`: which of the lane's pairs are, one bit each (FULL: all of every lane).  A
    // channel that is not turned passes as it is: times a sine of zero, its neighbour's infinity would not be zero.
    template <bool BACK, bool FULL>
    __device__ __forceinline__ Pairs turn(const Pairs &v, int turned) const {
        Pairs y;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint64_t up = BACK ? neg[k] : sn[k], down = BACK ? sn[k] : neg[k];
            y.a[k] = fma2(v.b[k], down, mul2(v.a[k], cs[k]));
            y.b[k] = fma2(v.a[k], up, mul2(v.b[k], cs[k]));
        }
        if (!FULL) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float x0, x1, y0, y1;
                const bool t0 = (turned >> (2 * k)) & 1, t1 = (turned >> (2 * k + 1)) & 1;
                unpack2(v.a[k], x0, x1); unpack2(y.a[k], y0, y1);
                y.a[k] = pack2(t0 ? y0 : x0, t1 ? y1 : x1);
                unpack2(v.b[k], x0, x1); unpack2(y.b[k], y0, y1);
                y.b[k] = pack2(t0 ? y0 : x0, t1 ? y1 : x1);
            }
        }
        return y;
    }
};
__device__ __forceinline__ float sum2(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Rows of a lane under way, and blocks per SM: what the registers hold.  (33k tokens of 24 + 24 heads, bf16: forward, six rows and three
// blocks 131 us, four and three 136, eight and two 152, four and four 136; backward, six and two 218, three and three 231,
// four and three 240, five and two 240, eight and two 235.  An fp32 projection, 12.8k tokens of 24 + 8 heads, forward: four and three
// 50, six and two 56, eight and two 58; backward, four and two 85, three 91, six 102.)
template <typename X, bool BWD>
struct RopeBatch {
    static constexpr int U = sizeof(X) == 4 ? 4 : 6;
    static constexpr int BLOCKS = BWD ? 2 : 3;
};

// FULL: every channel is turned.  BY_TOKEN: the lane groups of a warp have a token each; otherwise heads of one token in turn.
template <int D, bool HALVES, bool FULL, bool BY_TOKEN, typename X, bool BWD>
__global__ void __launch_bounds__(kRopeWarps * 32, RopeBatch<X, BWD>::BLOCKS) norm_rope_kernel(const __grid_constant__ RopeTable tab, const RopeParams p) {
    using RB = RopeBatch<X, BWD>;
    using Y = typename std::conditional<BWD, X, __nv_bfloat16>::type;
    constexpr int LPR = D / 8, RPW = 32 / LPR, U = RB::U;      // lanes a row, rows a warp
    __shared__ double s_turns[kMaxPairs];
    __shared__ uint8_t s_axis[kMaxPairs];
    __shared__ __align__(16) float s_w[2][D];                  // in the order of the lanes' pairs
    __shared__ float s_dw[BWD ? kRopeWarps : 1][2][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, chunk = lane % LPR, sub = lane / LPR;
    if (BWD) next_may_start();
    if (threadIdx.x < kMaxPairs) {
        s_turns[threadIdx.x] = tab.turns[threadIdx.x];
        s_axis[threadIdx.x] = tab.axis[threadIdx.x];
    }
    for (int i = threadIdx.x; i < 2 * D; i += kRopeWarps * 32) {
        const float *w = p.side[i / D].w;
        s_w[i / D][i % D] = w ? w[Channels(HALVES, i % D / 8, p.n_pairs).of(HALVES, i & 3, (i >> 2) & 1)] : 1.f;
    }
    __syncthreads();
    const Channels ch(HALVES, chunk, p.n_pairs);
    const int turned = p.n_pairs - chunk * 4 >= 4 ? 15 : p.n_pairs > chunk * 4 ? (1 << (p.n_pairs - chunk * 4)) - 1 : 0;
    Angles ang;
    Pairs acc[BWD ? 2 : 1] = {};
    constexpr int N_TOK = BY_TOKEN ? RPW : 1, STEP = BY_TOKEN ? 1 : RPW;      // of a warp: tokens, and heads of a token at a time
    const int64_t n_items = ((int64_t)p.n_tokens + N_TOK - 1) / N_TOK * p.n_split;
    for (int64_t item = (int64_t)blockIdx.x * kRopeWarps + warp; item < n_items; item += (int64_t)gridDim.x * kRopeWarps) {
        // (tokens' heads are split only where there are few tokens: 32 bits will do)
        const unsigned group = p.n_split == 1 ? (unsigned)item : (unsigned)item / (unsigned)p.n_split;
        const int share = (int)((unsigned)item - group * (unsigned)p.n_split);
        const int64_t mine = (int64_t)group * N_TOK + (BY_TOKEN ? sub : 0);
        const bool there = !BY_TOKEN || mine < p.n_tokens;     // the last tokens may be fewer
        const int64_t tok = there ? mine : p.n_tokens - 1;
        const int u_first = share * p.per_warp, u_end = min(p.units[0] + p.units[1], u_first + p.per_warp);
        bool made = false;
#pragma unroll
        for (int z = 0; z < 2; ++z) {                          // queries, keys
            const int u0 = z ? p.units[0] : 0, first = max(u_first, u0) - u0, last = min(u_end - u0, p.units[z]);
            if (first >= last) continue;
            const RopeSide &sd = p.side[z];
            const bool norm = sd.w != nullptr;
            int h = first * U * STEP + (BY_TOKEN ? 0 : sub); // this lane's first head of the batch
            const X *x = static_cast<const X *>(sd.x) + tok * sd.x_tok + (int64_t)h * sd.x_head;
            const __nv_bfloat16 *dy = BWD ? sd.dy + tok * sd.dy_tok + (int64_t)h * sd.dy_head : nullptr;
            Y *out = static_cast<Y *>(sd.out) + tok * sd.out_tok + (int64_t)h * sd.out_head;
            const ulonglong2 wa = *reinterpret_cast<const ulonglong2 *>(&s_w[z][chunk * 8]), wb = *reinterpret_cast<const ulonglong2 *>(&s_w[z][chunk * 8 + 4]);
#pragma unroll 1
            for (int u = first; u < last; ++u, h += U * STEP) {
                Raw<X> rx[U];
                Raw<__nv_bfloat16> rg[BWD ? U : 1];
                const int left = there ? sd.heads - h : 0, most = sd.heads - u * U * STEP;     // of this lane, of any
#pragma unroll
                for (int y = 0; y < U; ++y) {
                    rx[y] = {};
                    if (y * STEP < left && (!BWD || norm)) rx[y].template load<HALVES>(x, ch);
                    x += STEP * sd.x_head;
                    if constexpr (BWD) {
                        rg[y] = {};
                        if (y * STEP < left) rg[y].template load<HALVES>(dy, ch);
                        dy += STEP * sd.dy_head;
                    }
                }
                if (!made) {                                   // while the first rows are on their way
                    ang.make(s_turns, s_axis, p.pos + tok * p.n_axes, chunk, p.n_pairs);
                    made = true;
                }
#pragma unroll
                for (int y = 0; y < U; ++y) {
                    if (y > 0 && y * STEP >= most) break;           // (no lane has such a row)
                    Pairs v = rx[y].template get<HALVES>();
                    uint64_t r2 = 0;
                    if (norm) {
                        const uint64_t ss = fma2(v.b[1], v.b[1], fma2(v.b[0], v.b[0], fma2(v.a[1], v.a[1], mul2(v.a[0], v.a[0]))));
                        const float mean = row_sum<LPR>(sum2(ss)) * p.inv_d + p.eps;
                        // (of a row that is not there, and without an eps, 0 * inf would not be 0 in the sum for dw)
                        r2 = both(!BWD || y * STEP < left ? rsqrtf(mean) : 0.f);
#pragma unroll
                        for (int k = 0; k < 2; ++k) { v.a[k] = mul2(v.a[k], r2); v.b[k] = mul2(v.b[k], r2); }
                    }
                    if constexpr (!BWD) {
                        if (norm) {
                            v.a[0] = mul2(v.a[0], wa.x); v.a[1] = mul2(v.a[1], wa.y);
                            v.b[0] = mul2(v.b[0], wb.x); v.b[1] = mul2(v.b[1], wb.y);
                        }
                        const Pairs t = ang.template turn<false, FULL>(v, turned);
                        if (y * STEP < left) put_pairs<HALVES>(out, ch, t);
                    } else {
                        Pairs g = ang.template turn<true, FULL>(rg[y].template get<HALVES>(), turned);
                        if (norm) {
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                acc[z].a[k] = fma2(g.a[k], v.a[k], acc[z].a[k]);
                                acc[z].b[k] = fma2(g.b[k], v.b[k], acc[z].b[k]);
                            }
                            g.a[0] = mul2(g.a[0], wa.x); g.a[1] = mul2(g.a[1], wa.y);
                            g.b[0] = mul2(g.b[0], wb.x); g.b[1] = mul2(g.b[1], wb.y);
                            const uint64_t m2 = fma2(g.b[1], v.b[1], fma2(g.b[0], v.b[0], fma2(g.a[1], v.a[1], mul2(g.a[0], v.a[0]))));
                            const uint64_t nm = both(row_sum<LPR>(sum2(m2)) * -p.inv_d);
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                g.a[k] = mul2(fma2(v.a[k], nm, g.a[k]), r2);
                                g.b[k] = mul2(fma2(v.b[k], nm, g.b[k]), r2);
                            }
                        }
                        if (y * STEP < left) put_pairs<HALVES>(out, ch, g);
                    }
                    out += STEP * sd.out_head;
                }
            }
        }
    }
    if constexpr (BWD) {
        // the block's sums: the rows of a warp, then its warps, always in the same order
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            float f[8];
            unpack2(acc[z].a[0], f[0], f[1]); unpack2(acc[z].a[1], f[2], f[3]);
            unpack2(acc[z].b[0], f[4], f[5]); unpack2(acc[z].b[1], f[6], f[7]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = f[i];
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if (sub == 0) s_dw[warp][z][ch.of(HALVES, i & 3, i >> 2)] = v;
            }
        }
        __syncthreads();
        if (threadIdx.x < 2 * D) {
            const int z = threadIdx.x / D, c = threadIdx.x % D;
            float v = 0.f;
#pragma unroll
            for (int y = 0; y < kRopeWarps; ++y) v += s_dw[y][z][c];
            p.part[((size_t)blockIdx.x * 2 + z) * D + c] = v;
        }
    }
}

// dw of 32 channels: 32 threads a channel take the blocks' sums in turn, then one adds up the 32.  The order never changes.
__global__ void __launch_bounds__(1024) norm_rope_dw_kernel(const float *part, int n_blocks, int d, float *dw_q, float *dw_k) {
    __shared__ float s[32][33];
    const int groups = d / 32, z = blockIdx.x / groups, c = (blockIdx.x % groups) * 32 + (threadIdx.x & 31), y = threadIdx.x >> 5;
    float *dw = z ? dw_k : dw_q;
    previous_done();                                            // launched early: the blocks' sums are there from here on
    if (!dw) return;
    float v = 0.f;
    for (int b = y; b < n_blocks; b += 256) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = b + 32 * i < n_blocks ? part[((size_t)(b + 32 * i) * 2 + z) * d + c] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += x[i];
    }
    s[y][threadIdx.x & 31] = v;
    __syncthreads();
    if (y == 0) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) v += s[i][threadIdx.x];
        dw[c] = v;
    }
}

// the most blocks that a backward launch has: what the workspace holds sums of
constexpr int kRopeMaxBlocks = 2048;

// How a launch deals out a stream's heads: batches that a token's heads make, batches a warp takes and warps that share a token (groups of
// tokens: those of a warp), and blocks.
struct RopeSplit {
    bool by_token;
    int units[2], per_warp, n_split;
    int64_t items;
    unsigned grid;
};
// The lane groups of a warp have heads of one token in turn, next to one another in a projection; or a token each, where that has room for fewer
// rows.  Room is counted in whole batches, although rows that no lane has cost nothing: 16 + 16 and 40 + 40 heads of 128 go by token too, where in
// turn no lane would be without a row either (33k tokens 94 / 153 and 231 / 351 us, 1.12 to 1.24 times the copy's; in turn not timed).  (33k tokens, bf16, forward and backward, heads of one token and a token each: 12 + 12 heads of 128 70 / 122 and
// 73 / 120 us; 66k tokens, 6 + 2 heads of 64, 71 / 118 and 34 / 54; 264k tokens, 1 + 1 head of 128, 248 / 396 and 132 / 210.  An fp32
// projection, 6.4k tokens, 24 + 24 heads of 128, 40 / 70 and 43 / 80.  With the step from head to head as an argument of one kernel
// instead, the same cases were 77 / 138, 37 / 57 and 153 / 255.)
static RopeSplit split_norm_rope(bool fp32, bool bwd, int d, int64_t n_tokens, const int (&heads)[2], int n_sm) {
    const int U = fp32 ? RopeBatch<float, false>::U : RopeBatch<__nv_bfloat16, false>::U, rpw = 32 / (d / 8);
    const int per_sm = bwd ? RopeBatch<float, true>::BLOCKS : RopeBatch<float, false>::BLOCKS;
    int in_turn = 0, a_token = 0;                               // rows that a lane group has room for, at a token
    for (int h : heads) {
        in_turn += (h + U * rpw - 1) / (U * rpw) * rpw;
        a_token += (h + U - 1) / U;
    }
    RopeSplit p;
    p.by_token = a_token < in_turn;
    const int batch = U * (p.by_token ? 1 : rpw);               // heads of a batch
    for (int z = 0; z < 2; ++z) p.units[z] = (heads[z] + batch - 1) / batch;
    const int units = p.units[0] + p.units[1];
    // A warp takes all of its tokens' heads, unless that leaves warps without work: then as many batches of heads as give every warp
    // one (each forms the angles of its tokens again).  The longest warp is not looked at: 1,601 groups of three batches for 2,368 warps
    // (6.4k tokens, 12 + 4 heads of 64, backward) are cut in two, and some warps have four batches.
    const int64_t warps = (int64_t)n_sm * per_sm * kRopeWarps, groups = p.by_token ? (n_tokens + rpw - 1) / rpw : n_tokens;
    const int split = (int)std::min<int64_t>(units, (warps + groups - 1) / groups);
    p.per_warp = (units + split - 1) / split;
    p.n_split = (units + p.per_warp - 1) / p.per_warp;
    p.items = groups * p.n_split;
    p.grid = (unsigned)std::min<int64_t>({(p.items + kRopeWarps - 1) / kRopeWarps, (int64_t)n_sm * per_sm, (int64_t)kRopeMaxBlocks});
    return p;
}

template <int D, bool HALVES, bool FULL, bool BY_TOKEN, typename X, bool BWD>
static int launch_norm_rope_u(const moc_rope *r, const RopeParams &a, unsigned grid, float *dw_q, float *dw_k, cudaStream_t s) {
    norm_rope_kernel<D, HALVES, FULL, BY_TOKEN, X, BWD><<<grid, kRopeWarps * 32, 0, s>>>(r->tab, a);
    MOC_LAUNCH_CHECK();
    if (BWD && (dw_q || dw_k)) {
        MOC_CUDA_TRY(launch_early(true, norm_rope_dw_kernel, 2 * D / 32, 1024, 0, s, (const float *)a.part, (int)grid, D, dw_q, dw_k));
        MOC_LAUNCH_CHECK();
    }
    return MOC_OK;
}

template <int D, bool HALVES, bool FULL, typename X, bool BWD>
static int launch_norm_rope_t(const moc_rope *r, RopeParams &a, float *dw_q, float *dw_k, int n_sm, cudaStream_t s) {
    const RopeSplit p = split_norm_rope(sizeof(X) == 4, BWD, D, a.n_tokens, {a.side[0].heads, a.side[1].heads}, n_sm);
    for (int z = 0; z < 2; ++z) a.units[z] = p.units[z];
    a.per_warp = p.per_warp;
    a.n_split = p.n_split;
    return p.by_token ? launch_norm_rope_u<D, HALVES, FULL, true, X, BWD>(r, a, p.grid, dw_q, dw_k, s)
                      : launch_norm_rope_u<D, HALVES, FULL, false, X, BWD>(r, a, p.grid, dw_q, dw_k, s);
}

template <bool BWD>
static int launch_norm_rope(const moc_rope *r, RopeParams &a, int x_type, float *dw_q, float *dw_k, cudaStream_t s) {
    int dev = -1, cc = 0, n_sm = 0;
    MOC_CUDA_TRY(cudaGetDevice(&dev));
    MOC_CUDA_TRY(cudaDeviceGetAttribute(&cc, cudaDevAttrComputeCapabilityMajor, dev));
    MOC_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
    if (cc != 10) return MOC_ERR_ARCH;
    if (a.n_tokens == 0) {                                      // nothing to do but a sum of nothing
        if (dw_q) MOC_CUDA_TRY(cudaMemsetAsync(dw_q, 0, sizeof(float) * r->d, s));
        if (dw_k) MOC_CUDA_TRY(cudaMemsetAsync(dw_k, 0, sizeof(float) * r->d, s));
        return MOC_OK;
    }
    a.n_axes = r->n_axes; a.n_pairs = r->n_pairs; a.eps = r->eps; a.inv_d = 1.f / r->d;
    const bool halves = (r->flags & MOC_ROPE_HALVES) && r->n_pairs > 0, full = 2 * r->n_pairs == r->d;
    // (all of them run the same code, with their sizes known to the compiler)
    auto go = [&](auto d, auto halves_, auto full_, auto x) {
        return launch_norm_rope_t<decltype(d)::value, decltype(halves_)::value, decltype(full_)::value, decltype(x), BWD>(r, a, dw_q, dw_k, n_sm, s);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    auto by_pairs = [&](auto d, auto x) {
        if (halves) return full ? go(d, Yes{}, Yes{}, x) : go(d, Yes{}, No{}, x);
        return full ? go(d, No{}, Yes{}, x) : go(d, No{}, No{}, x);
    };
    auto by_type = [&](auto d) { return x_type == MOC_FP32 ? by_pairs(d, 0.f) : by_pairs(d, __nv_bfloat16()); };
    return r->d == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace moc

using namespace moc;

extern "C" int moc_rope_create(const moc_rope_problem *pr, moc_rope **out) {
    if (!pr || !out) return MOC_ERR_NULL;
    if (pr->head_dim != 64 && pr->head_dim != 128) return MOC_ERR_SHAPE;
    if (pr->n_pairs < 0 || 2 * (int64_t)pr->n_pairs > pr->head_dim) return MOC_ERR_SHAPE;
    if (pr->flags & ~MOC_ROPE_HALVES) return MOC_ERR_SHAPE;
    if ((pr->flags & MOC_ROPE_HALVES) && pr->n_pairs % 8 != 0) return MOC_ERR_SHAPE;
    if (!(pr->eps >= 0.f) || !isfinite(pr->eps)) return MOC_ERR_SHAPE;
    if (pr->n_pairs > 0) {
        if (!pr->pair_axis || !pr->pair_freq) return MOC_ERR_NULL;
        if (pr->n_axes < 1 || pr->n_axes > kMaxAxes) return MOC_ERR_SHAPE;
        for (int j = 0; j < pr->n_pairs; ++j)
            if (pr->pair_axis[j] < 0 || pr->pair_axis[j] >= pr->n_axes || !(fabs(pr->pair_freq[j]) <= 1e6)) return MOC_ERR_SHAPE;
    }
    moc_rope *r = new (std::nothrow) moc_rope();
    if (!r) return MOC_ERR_CUDA;
    r->d = pr->head_dim; r->n_pairs = pr->n_pairs; r->n_axes = pr->n_pairs > 0 ? pr->n_axes : 0; r->flags = pr->flags; r->eps = pr->eps;
    for (int j = 0; j < pr->n_pairs; ++j) {
        r->tab.turns[j] = pr->pair_freq[j] / 6.283185307179586476925286766559;
        r->tab.axis[j] = (uint8_t)pr->pair_axis[j];
    }
    *out = r;
    return MOC_OK;
}

extern "C" int moc_rope_destroy(moc_rope *r) {
    if (!r) return MOC_ERR_NULL;
    delete r;
    return MOC_OK;
}

extern "C" int moc_rope_workspace_bytes(const moc_rope *r, size_t *bytes) {
    if (!r || !bytes) return MOC_ERR_NULL;
    *bytes = sizeof(float) * 2 * (size_t)r->d * kRopeMaxBlocks;
    return MOC_OK;
}

// what the two calls check alike
static int check_rope_call(const moc_rope *r, int x_type, int n_tokens, int n_q, int n_k, const int32_t *pos) {
    if (!r) return MOC_ERR_NULL;
    if (x_type != MOC_BF16 && x_type != MOC_FP32) return MOC_ERR_SHAPE;
    if (n_tokens < 0 || n_q < 1 || n_q > 65535 || n_k < 0 || n_k > 65535) return MOC_ERR_SHAPE;
    if (r->n_pairs > 0 && n_tokens > 0) {
        if (!pos) return MOC_ERR_NULL;
        if (!aligned(pos, 4)) return MOC_ERR_ALIGN;
    }
    return MOC_OK;
}

extern "C" int moc_norm_rope(const moc_rope *r, int x_type, int32_t n_tokens, int32_t n_q_heads, int32_t n_k_heads, const int32_t *pos,
                             const moc_rows *q, const float *w_q, const moc_rows *q_out, const moc_rows *k, const float *w_k,
                             const moc_rows *k_out, void *stream) {
    moc::NvtxRange nvtx_range("moc_norm_rope");
    if (int e = check_rope_call(r, x_type, n_tokens, n_q_heads, n_k_heads, pos)) return e;
    const int xs = x_type == MOC_FP32 ? 4 : 2;
    RopeParams a = {};
    a.n_tokens = n_tokens;
    a.pos = pos;
    const moc_rows *in[2] = {q, k}, *out[2] = {q_out, k_out};
    const float *w[2] = {w_q, w_k};
    const int heads[2] = {n_q_heads, n_k_heads};
    for (int z = 0; z < 2; ++z) {
        RopeSide &s = a.side[z];
        s.heads = heads[z];
        if (heads[z] == 0) continue;
        if (int e = check_rows(in[z], heads[z], n_tokens, r->d, xs)) return e;
        if (int e = check_rows(out[z], heads[z], n_tokens, r->d, 2)) return e;
        if (w[z] && !aligned(w[z], 4)) return MOC_ERR_ALIGN;
        s.x = in[z]->data; s.x_head = in[z]->head_stride; s.x_tok = in[z]->token_stride;
        s.out = out[z]->data; s.out_head = out[z]->head_stride; s.out_tok = out[z]->token_stride;
        s.w = w[z];
    }
    return launch_norm_rope<false>(r, a, x_type, nullptr, nullptr, (cudaStream_t)stream);
}

extern "C" int moc_norm_rope_bwd(const moc_rope *r, int x_type, int32_t n_tokens, int32_t n_q_heads, int32_t n_k_heads, const int32_t *pos,
                                 const moc_rows *q, const float *w_q, const moc_rows *dq_out, const moc_rows *dq, float *dw_q, const moc_rows *k,
                                 const float *w_k, const moc_rows *dk_out, const moc_rows *dk, float *dw_k, void *ws, void *stream) {
    moc::NvtxRange nvtx_range("moc_norm_rope_bwd");
    if (int e = check_rope_call(r, x_type, n_tokens, n_q_heads, n_k_heads, pos)) return e;
    const int xs = x_type == MOC_FP32 ? 4 : 2;
    RopeParams a = {};
    a.n_tokens = n_tokens;
    a.pos = pos;
    const moc_rows *in[2] = {q, k}, *grad[2] = {dq_out, dk_out}, *out[2] = {dq, dk};
    const float *w[2] = {w_q, w_k};
    float *dw[2] = {dw_q, dw_k};
    const int heads[2] = {n_q_heads, n_k_heads};
    for (int z = 0; z < 2; ++z) {
        RopeSide &s = a.side[z];
        s.heads = heads[z];
        if (heads[z] == 0) { dw[z] = nullptr; continue; }
        if (int e = check_rows(grad[z], heads[z], n_tokens, r->d, 2)) return e;
        if (int e = check_rows(out[z], heads[z], n_tokens, r->d, xs)) return e;
        if (w[z]) {                                             // without a norm the gradient does not depend on x
            if (int e = check_rows(in[z], heads[z], n_tokens, r->d, xs)) return e;
            if (!dw[z]) return MOC_ERR_NULL;
            if (!aligned(w[z], 4) || !aligned(dw[z], 4)) return MOC_ERR_ALIGN;
            s.x = in[z]->data; s.x_head = in[z]->head_stride; s.x_tok = in[z]->token_stride;
        } else if (dw[z]) return MOC_ERR_SHAPE;                 // there is no such gradient
        s.dy = (const __nv_bfloat16 *)grad[z]->data; s.dy_head = grad[z]->head_stride; s.dy_tok = grad[z]->token_stride;
        s.out = out[z]->data; s.out_head = out[z]->head_stride; s.out_tok = out[z]->token_stride;
        s.w = w[z];
    }
    if (!ws) return MOC_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return MOC_ERR_ALIGN;
    a.part = static_cast<float *>(ws);
    return launch_norm_rope<true>(r, a, x_type, dw[0], dw[1], (cudaStream_t)stream);
}

// Test hook, host only: how the launch of a call on n_sm SMs deals out its work.  out: a token for each lane group, batches of queries and
// of keys, batches a warp takes, warps that share a token, items, warps
extern "C" int moc_debug_rope_split(int x_type, int bwd, int d, int64_t n_tokens, int n_q, int n_k, int n_sm, int64_t *out) {
    if (!out) return MOC_ERR_NULL;
    if ((x_type != MOC_BF16 && x_type != MOC_FP32) || (d != 64 && d != 128) || n_tokens < 1 || n_q < 1 || n_k < 0 || n_sm < 1) return MOC_ERR_SHAPE;
    const RopeSplit p = split_norm_rope(x_type == MOC_FP32, bwd != 0, d, n_tokens, {n_q, n_k}, n_sm);
    const int64_t v[7] = {p.by_token, p.units[0], p.units[1], p.per_warp, p.n_split, p.items, (int64_t)p.grid * kRopeWarps};
    std::copy(v, v + 7, out);
    return MOC_OK;
}
