// Cross attention of segments with few queries (a step of token-by-token generation): up to eight rows - queries of all the query heads that
// share a key head - against their states, on the CUDA cores.
//
// What bounds it is reading K and V, once for all the rows that share them.  On the tensor cores a query head would fill one row of a
// 128-row tile, read the states for itself and take 4300 cycles for 128 of them, where HBM needs 2800 for all heads of the group.
//
// A block has a share of a segment's states, of one key head, and up to four rows.  K and V come by asynchronous copies, 32 states a
// stage.  Eight lanes have a state, 16 channels each (8 at d = 64): four states a warp at a time; a score is a sum over the lane's
// channels and three exchanges for each row.  Each group of eight lanes keeps the running maximum, sum and output of the states that it has
// seen; they meet at the end, first in the warp, then in the block, and shares meet in cross_merge_kernel.  Everything is fp32.
// 64 sequences of some 1150 states, 24 heads on 8: 56 us, 5.4 TB/s.
#include <algorithm>

#include "moc_cross.cuh"
#include "moc_tc.cuh"

namespace moc {

using namespace tc;

struct CrossFewParams {
    const CrossFew *items;
    int Hkv, g, Lq, prows;
    CrossRows Q, K, V, O;
    float *lse, *part_o, *part_lse;
    int *status;
    float scale_log2;
};

// Four stages and three blocks an SM.  (64 sequences, 24 heads on 8, three rows a block: 56.2 us; three stages and four blocks 61,
// three stages and three blocks 63.)
constexpr int kFewKeys = 32, kFewStages = 4, kFewThreads = 128;

template <int D, int R>
__global__ void __launch_bounds__(kFewThreads, 3) cross_few_kernel(const CrossFewParams p) {
    constexpr int NC = D / 64, CH = D / 8;                 // 16-byte pieces of a lane, of a row
    constexpr int TILE = kFewKeys * D * 2;                 // bytes of K, and of V, in a stage
    extern __shared__ __align__(16) uint8_t ring[];        // [stage][K, V][state][d]
    __shared__ float s_m[4][R], s_l[4][R], s_o[4][R][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l8 = lane & 7, grp = lane >> 3;
    next_may_start();
    if (blockIdx.x == 0 && threadIdx.x == 0) p.status[ST_STATUS] = p.status[ST_DETAIL] = 0;
    const int rank = blockIdx.x / p.Hkv, hk = blockIdx.x - rank * p.Hkv;
    const CrossFew it = p.items[rank];
    const int n_stages = (it.n_keys + kFewKeys - 1) / kFewKeys;

    auto ask = [&](int s) {
        if (s < n_stages) {
            const uint32_t dst = smem_u32(ring) + (s % kFewStages) * 2 * TILE;
#pragma unroll
            for (int x = 0; x < kFewKeys * CH / kFewThreads; ++x) {
                const int i = x * kFewThreads + threadIdx.x, r = i / CH, c = i % CH, key = s * kFewKeys + r;
                const uint32_t n = key < it.n_keys ? 16u : 0u;        // (a state that is not there: zeros, at an address that is)
                const int t = it.k0 + min(key, it.n_keys - 1);
                cp_async16(dst + i * 16, p.K.row(hk, t) + c * 8, n);
                cp_async16(dst + TILE + i * 16, p.V.row(hk, t) + c * 8, n);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < kFewStages - 1; ++s) ask(s);

    auto widen = [](const uint4 &u, uint64_t (&f)[4]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    };
    // the rows, times the softmax scale and log2(e): scores come out as exponents of two
    uint64_t q[R][NC * 4], acc[R][NC * 4];
    float m[R], l[R];
    const uint64_t c2 = pack2(p.scale_log2, p.scale_log2);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = kLowest;
        l[r] = 0.f;
        const int at = it.r0 + min(r, it.nr - 1), h = hk * p.g + at / it.q_len, t = it.q0 + at % it.q_len;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            uint64_t f[4];
            widen(*reinterpret_cast<const uint4 *>(p.Q.row(h, t) + (c * 8 + l8) * 8), f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                q[r][c * 4 + i] = mul2(f[i], c2);
                acc[r][c * 4 + i] = 0ull;
            }
        }
    }
    for (int s = 0; s < n_stages; ++s) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
        __syncthreads();                                       // everybody's copies; and the stage asked for next has been read
        ask(s + kFewStages - 1);
        const uint8_t *tile = ring + (s % kFewStages) * 2 * TILE;
#pragma unroll
        for (int x = 0; x < kFewKeys / 16; ++x) {
            const int key = x * 16 + warp * 4 + grp;
            const bool there = s * kFewKeys + key < it.n_keys;
            float sc[R];
            {
                uint64_t k[NC * 4];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    uint64_t f[4];
                    widen(*reinterpret_cast<const uint4 *>(tile + (key * CH + c * 8 + l8) * 16), f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) k[c * 4 + i] = f[i];
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    uint64_t a = mul2(q[r][0], k[0]);
#pragma unroll
                    for (int i = 1; i < NC * 4; ++i) a = fma2(q[r][i], k[i], a);
                    float lo, hi;
                    unpack2(a, lo, hi);
                    sc[r] = lo + hi;
                }
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1)
#pragma unroll
                for (int r = 0; r < R; ++r) sc[r] += __shfl_xor_sync(0xffffffffu, sc[r], o);
            // the maximum moves only when a score is above it by more than 2^8 (sums stay far within fp32)
            bool moves = false;
#pragma unroll
            for (int r = 0; r < R; ++r) moves |= there && sc[r] > m[r] + 8.f;
            if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (there && sc[r] > m[r] + 8.f) {
                        const float w = ex2(m[r] - sc[r]);     // (nothing yet: 0)
                        m[r] = sc[r];
                        l[r] *= w;
                        const uint64_t w2 = pack2(w, w);
#pragma unroll
                        for (int i = 0; i < NC * 4; ++i) acc[r][i] = mul2(acc[r][i], w2);
                    }
                }
            }
            uint64_t v[NC * 4];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                uint64_t f[4];
                widen(*reinterpret_cast<const uint4 *>(tile + TILE + (key * CH + c * 8 + l8) * 16), f);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[c * 4 + i] = f[i];
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float w = there ? ex2(sc[r] - m[r]) : 0.f;
                l[r] += w;
                const uint64_t w2 = pack2(w, w);
#pragma unroll
                for (int i = 0; i < NC * 4; ++i) acc[r][i] = fma2(w2, v[i], acc[r][i]);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // the warp's four groups
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float big = fmaxf(fmaxf(m[r], __shfl_xor_sync(0xffffffffu, m[r], 8)), fmaxf(__shfl_xor_sync(0xffffffffu, m[r], 16), __shfl_xor_sync(0xffffffffu, m[r], 24)));
        const float w = l[r] == 0.f ? 0.f : ex2(m[r] - big);   // (a group without a state, or without one that weighs)
        float sum = l[r] * w;
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (lane == 0) { s_m[warp][r] = big; s_l[warp][r] = sum; }
#pragma unroll
        for (int i = 0; i < NC * 4; ++i) {
            float a, b;
            unpack2(acc[r][i], a, b);
            a *= w; b *= w;
            a += __shfl_xor_sync(0xffffffffu, a, 8); b += __shfl_xor_sync(0xffffffffu, b, 8);
            a += __shfl_xor_sync(0xffffffffu, a, 16); b += __shfl_xor_sync(0xffffffffu, b, 16);
            if (grp == 0) *reinterpret_cast<float2 *>(&s_o[warp][r][((i >> 2) * 8 + l8) * 8 + 2 * (i & 3)]) = make_float2(a, b);
        }
    }
    __syncthreads();
    // the block's four warps: two channels a thread
    for (int i = threadIdx.x; i < it.nr * (D / 2); i += kFewThreads) {
        const int r = i / (D / 2), c = i % (D / 2) * 2;
        float big = s_m[0][r], sum = 0.f, a = 0.f, b = 0.f;
#pragma unroll
        for (int y = 1; y < 4; ++y) big = fmaxf(big, s_m[y][r]);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const float w = s_l[y][r] == 0.f ? 0.f : ex2(s_m[y][r] - big);
            sum += w * s_l[y][r];
            a += w * s_o[y][r][c];
            b += w * s_o[y][r][c + 1];
        }
        // (a share whose states all weigh nothing: its row is a sum of zeros, which has no weight in the sum of shares)
        const float inv = it.slot >= 0 && sum == 0.f ? 1.f : 1.f / sum, lse = (big + log2f(sum)) * 0.6931471805599453f;
        const int at = it.r0 + r, h = hk * p.g + at / it.q_len, t = at % it.q_len;
        if (it.slot < 0) {
            *reinterpret_cast<uint32_t *>(p.O.row(h, it.q0 + t) + c) = bf16x2(a * inv, b * inv);
            if (c == 0) p.lse[(size_t)h * p.Lq + it.q0 + t] = lse;
        } else {
            const size_t row = (size_t)h * p.prows + it.slot + t;
            *reinterpret_cast<float2 *>(p.part_o + row * D + c) = make_float2(a * inv, b * inv);
            if (c == 0) p.part_lse[row] = lse;
        }
    }
}

static constexpr size_t few_smem(int d) { return (size_t)kFewStages * 2 * kFewKeys * d * 2; }

int prepare_cross_few(moc_cross *c) {
    const int r = std::min(std::max(c->few_rows, 1), 4) - 1;
    const void *const k64[4] = {(const void *)cross_few_kernel<64, 1>, (const void *)cross_few_kernel<64, 2>, (const void *)cross_few_kernel<64, 3>,
                                (const void *)cross_few_kernel<64, 4>},
               *const k128[4] = {(const void *)cross_few_kernel<128, 1>, (const void *)cross_few_kernel<128, 2>, (const void *)cross_few_kernel<128, 3>,
                                 (const void *)cross_few_kernel<128, 4>};
    MOC_CUDA_TRY(cudaFuncSetAttribute(c->d == 128 ? k128[r] : k64[r], cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_smem(c->d)));
    return MOC_OK;
}

template <int D, int R>
static int cross_few_t(const moc_cross *c, const CrossFewParams &a, cudaStream_t s) {
    cross_few_kernel<D, R><<<(unsigned)(c->few.size() * c->Hkv), kFewThreads, few_smem(D), s>>>(a);
    MOC_LAUNCH_CHECK();
    return MOC_OK;
}

template <int D>
static int cross_few_d(const moc_cross *c, const CrossFewParams &a, cudaStream_t s) {
    switch (c->few_rows) {
        case 1: return cross_few_t<D, 1>(c, a, s);
        case 2: return cross_few_t<D, 2>(c, a, s);
        case 3: return cross_few_t<D, 3>(c, a, s);
        default: return cross_few_t<D, 4>(c, a, s);
    }
}

int launch_cross_few(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws,
                     cudaStream_t s) {
    CrossFewParams a;
    a.items = c->d_few; a.Hkv = c->Hkv; a.g = c->g; a.Lq = c->Lq; a.prows = c->prows;
    a.Q = CrossRows(Q); a.K = CrossRows(K); a.V = CrossRows(V); a.O = CrossRows(O);
    a.lse = lse; a.part_o = ws_ptr<float>(ws, c->ws.part_o); a.part_lse = ws_ptr<float>(ws, c->ws.part_lse);
    a.status = ws_ptr<int>(ws, c->ws.status);
    a.scale_log2 = c->scale * 1.4426950408889634f;
    return c->d == 128 ? cross_few_d<128>(c, a, s) : cross_few_d<64>(c, a, s);
}

}  // namespace moc
