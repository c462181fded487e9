// RMS norm of every query and key head with the position rotation in the same pass (moc_norm_rope), and its backward pass.
//
//   r = 1 / sqrt(mean_c x_c^2 + eps),  u_c = x_c r w_c,  and of every rotated pair of channels (a, b), with the angle t:
//   y_a = u_a cos t - u_b sin t,  y_b = u_b cos t + u_a sin t.
//   Backward:  g = the rotation by -t of dy,  xh = x r,  dw = sum over heads and tokens of g xh,
//   dx = r (w g - xh mean_c(w g xh)).
//
// Both are bound by HBM: each value is read once and written once, and what a row needs beside its own values is shared by all
// heads of a token.  So a warp takes a token and walks its heads: the angles - formed in turns, in 64 bits, reduced to a part of a
// turn and only then rounded to 32, so that far positions lose nothing - are made once for all of them.  A lane holds eight consecutive channels
// (16 bytes of bf16), 16 lanes a row at d = 128 and 8 at d = 64; four rows a lane are under way at a time.
// Where there are too few tokens to fill the GPU, a token's heads are dealt to several warps.
#include <algorithm>
#include <math.h>
#include <new>

#include "moc_common.cuh"

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

constexpr int kRopeWarps = 8;         // warps per block, each with a token of its own
constexpr int kRopeBlocksPerSm = 3;

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
    int units[2];                     // batches of rows that a token's heads make
    int per_warp, n_split;            // batches a warp takes, warps a token has
    float eps, inv_d;
};

// eight consecutive values as fp32
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { a = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const float4 *>(p)[0];
        b = reinterpret_cast<const float4 *>(p)[1];
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);       // the result's one rounding
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&v)[8]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// The angles of a lane's eight channels at one token: neighbours share an angle (interleaved pairs), or each channel has its own, whose
// partner is n_pairs channels away (halves; sn then carries the sign of the partner's term).
template <bool HALVES>
struct Angles {
    static constexpr int N = HALVES ? 8 : 4;
    float cs[N], sn[N];
    __device__ __forceinline__ void make(const double *s_turns, const uint8_t *s_axis, const int32_t *pos, int chunk, int n_pairs) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int ch = HALVES ? chunk * 8 + i : chunk * 4 + i;                 // channel, or pair
            const int pair = HALVES && ch >= n_pairs ? ch - n_pairs : ch;
            cs[i] = 1.f;
            sn[i] = 0.f;
            if (pair < n_pairs) {
                const double t = (double)pos[s_axis[pair]] * s_turns[pair];
                float s, c;
                sincospif(2.f * (float)(t - rint(t)), &s, &c);
                cs[i] = c;
                sn[i] = HALVES && ch < n_pairs ? -s : s;
            }
        }
    }
    // v <- the rotation of v (BACK: by the negative angle); partner: the lane that holds the other halves
    template <bool BACK>
    __device__ __forceinline__ void turn(float (&v)[8], int partner) const {
        if constexpr (HALVES) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float other = __shfl_sync(0xffffffffu, v[i], partner);
                // (a channel that is not turned has sn = 0; its partner, itself, may hold an infinity)
                const float t = sn[i] == 0.f ? 0.f : other * sn[i];
                v[i] = v[i] * cs[i] + (BACK ? -t : t);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = v[2 * i], b = v[2 * i + 1], s = BACK ? -sn[i] : sn[i];
                const float sb = sn[i] == 0.f ? 0.f : b * s, sa = sn[i] == 0.f ? 0.f : a * s;
                v[2 * i] = a * cs[i] - sb;
                v[2 * i + 1] = b * cs[i] + sa;
            }
        }
    }
};

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <int D, bool HALVES, typename X, bool BWD>
__global__ void __launch_bounds__(kRopeWarps * 32, BWD ? 2 : kRopeBlocksPerSm) norm_rope_kernel(const __grid_constant__ RopeTable tab, const RopeParams p) {
    constexpr int LPR = D / 8, RPW = 32 / LPR;                 // lanes a row, rows a warp
    constexpr int U = 4;                                       // rows of a lane under way
    __shared__ double s_turns[kMaxPairs];
    __shared__ uint8_t s_axis[kMaxPairs];
    __shared__ float s_dw[BWD ? kRopeWarps : 1][2][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, chunk = lane % LPR, sub = lane / LPR;
    if (threadIdx.x < kMaxPairs) {
        s_turns[threadIdx.x] = tab.turns[threadIdx.x];
        s_axis[threadIdx.x] = tab.axis[threadIdx.x];
    }
    __syncthreads();
    // the lane of the other half of this lane's channels (whole chunks: n_pairs is a multiple of eight)
    const int half = p.n_pairs >> 3;
    const int partner = HALVES ? sub * LPR + (chunk < half ? chunk + half : chunk < 2 * half ? chunk - half : chunk) : lane;
    float acc[2][8] = {};
    const int64_t n_items = (int64_t)p.n_tokens * p.n_split;
    for (int64_t item = (int64_t)blockIdx.x * kRopeWarps + warp; item < n_items; item += (int64_t)gridDim.x * kRopeWarps) {
        const int tok = (int)(item / p.n_split), part = (int)(item - (int64_t)tok * p.n_split);
        const int u_end = min(p.units[0] + p.units[1], (part + 1) * p.per_warp);
        Angles<HALVES> ang;
        bool made = false;
#pragma unroll
        for (int z = 0; z < 2; ++z) {                          // queries, keys
            const RopeSide &sd = p.side[z];
            const int u0 = z ? p.units[0] : 0, first = max(part * p.per_warp, u0), last = min(u_end, u0 + p.units[z]);
            if (first >= last) continue;
            const bool norm = sd.w != nullptr;
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = norm ? sd.w[chunk * 8 + i] : 1.f;
            const X *x = static_cast<const X *>(sd.x) + (int64_t)tok * sd.x_tok + chunk * 8;
            const __nv_bfloat16 *dy = BWD ? sd.dy + (int64_t)tok * sd.dy_tok + chunk * 8 : nullptr;
#pragma unroll 1
            for (int u = first; u < last; ++u) {
                const int h0 = (u - u0) * (U * RPW) + sub;
                Raw8<X> rx[U];
                Raw8<__nv_bfloat16> rg[BWD ? U : 1];
#pragma unroll
                for (int y = 0; y < U; ++y) {
                    const int h = h0 + y * RPW;
                    rx[y].zero();
                    if (h < sd.heads && (!BWD || norm)) rx[y].load(x + (int64_t)h * sd.x_head);
                    if constexpr (BWD) {
                        rg[y].zero();
                        if (h < sd.heads) rg[y].load(dy + (int64_t)h * sd.dy_head);
                    }
                }
                if (!made) {                                   // while the first rows are on their way
                    ang.make(s_turns, s_axis, p.pos + (int64_t)tok * p.n_axes, chunk, p.n_pairs);
                    made = true;
                }
#pragma unroll
                for (int y = 0; y < U; ++y) {
                    const int h = h0 + y * RPW;
                    float v[8], r = 1.f;
                    rx[y].get(v);
                    if (norm) {
                        float ss = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
                        r = rsqrtf(row_sum<LPR>(ss) * p.inv_d + p.eps);
                    }
                    if constexpr (!BWD) {
                        if (norm) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = v[i] * r * w[i];
                        }
                        ang.template turn<false>(v, partner);
                        if (h < sd.heads) store8(static_cast<__nv_bfloat16 *>(sd.out) + (int64_t)h * sd.out_head + (int64_t)tok * sd.out_tok + chunk * 8, v);
                    } else {
                        float g[8];
                        rg[y].get(g);
                        ang.template turn<true>(g, partner);
                        if (norm) {
                            float m = 0.f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                v[i] *= r;
                                acc[z][i] = fmaf(g[i], v[i], acc[z][i]);
                                g[i] *= w[i];
                                m = fmaf(g[i], v[i], m);
                            }
                            m = row_sum<LPR>(m) * p.inv_d;
#pragma unroll
                            for (int i = 0; i < 8; ++i) g[i] = r * (g[i] - v[i] * m);
                        }
                        if (h < sd.heads) store8(static_cast<X *>(sd.out) + (int64_t)h * sd.out_head + (int64_t)tok * sd.out_tok + chunk * 8, g);
                    }
                }
            }
        }
    }
    if constexpr (BWD) {
        // the block's sums: the rows of a warp, then its warps, always in the same order
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = acc[z][i];
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if (sub == 0) s_dw[warp][z][chunk * 8 + i] = v;
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
    if (!dw) return;
    float v = 0.f;
    for (int b = y; b < n_blocks; b += 32) v += part[((size_t)b * 2 + z) * d + c];
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

template <int D, bool HALVES, typename X, bool BWD>
static int launch_norm_rope_t(const moc_rope *r, RopeParams &a, float *dw_q, float *dw_k, int n_sm, cudaStream_t s) {
    constexpr int rows = 4 * 32 / (D / 8);
    const int per_sm = BWD ? 2 : kRopeBlocksPerSm;
    for (int z = 0; z < 2; ++z) a.units[z] = (a.side[z].heads + rows - 1) / rows;
    const int units = a.units[0] + a.units[1];
    // A warp takes all of a token's heads, unless that leaves warps without work: then as many batches of rows as give every warp
    // one (the angles are made once for each, some 200 instructions beside 350 a batch).
    const int64_t warps = (int64_t)n_sm * per_sm * kRopeWarps;
    int split = (int)std::min<int64_t>(units, (warps + a.n_tokens - 1) / a.n_tokens);
    a.per_warp = (units + split - 1) / split;
    a.n_split = (units + a.per_warp - 1) / a.per_warp;
    const int64_t items = (int64_t)a.n_tokens * a.n_split;
    const unsigned grid = (unsigned)std::min<int64_t>({(items + kRopeWarps - 1) / kRopeWarps, (int64_t)n_sm * per_sm, (int64_t)kRopeMaxBlocks});
    norm_rope_kernel<D, HALVES, X, BWD><<<grid, kRopeWarps * 32, 0, s>>>(r->tab, a);
    MOC_LAUNCH_CHECK();
    if (BWD && (dw_q || dw_k)) {
        norm_rope_dw_kernel<<<2 * D / 32, 1024, 0, s>>>(a.part, (int)grid, D, dw_q, dw_k);
        MOC_LAUNCH_CHECK();
    }
    return MOC_OK;
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
    const bool halves = (r->flags & MOC_ROPE_HALVES) && r->n_pairs > 0, f32 = x_type == MOC_FP32;
    using B = __nv_bfloat16;
    if (r->d == 128) {
        if (halves) return f32 ? launch_norm_rope_t<128, true, float, BWD>(r, a, dw_q, dw_k, n_sm, s) : launch_norm_rope_t<128, true, B, BWD>(r, a, dw_q, dw_k, n_sm, s);
        return f32 ? launch_norm_rope_t<128, false, float, BWD>(r, a, dw_q, dw_k, n_sm, s) : launch_norm_rope_t<128, false, B, BWD>(r, a, dw_q, dw_k, n_sm, s);
    }
    if (halves) return f32 ? launch_norm_rope_t<64, true, float, BWD>(r, a, dw_q, dw_k, n_sm, s) : launch_norm_rope_t<64, true, B, BWD>(r, a, dw_q, dw_k, n_sm, s);
    return f32 ? launch_norm_rope_t<64, false, float, BWD>(r, a, dw_q, dw_k, n_sm, s) : launch_norm_rope_t<64, false, B, BWD>(r, a, dw_q, dw_k, n_sm, s);
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
