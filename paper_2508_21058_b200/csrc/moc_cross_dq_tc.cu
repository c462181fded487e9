// dQ of the cross attention: a persistent CTA per SM walks items of up to 128 query rows of a head against their segment's keys, or a
// share of them.
//
//     P = exp(scale q.k - lse),  dP = dO V^T,  dS = P (dP - delta),  dQ = scale dS K
//     T1 = Q K^T,  T2 = dO V^T   (both operands from shared memory, into TMEM; T2 has two buffers)
//     threads (two per TMEM lane) turn T1 into P, then (P, T2) into dS, written back as bf16 over the columns of T2 they have read
//     ACC += dS K                (A from TMEM, the K tile as an MN-major operand)
//
// A row's lse and delta belong to its lane, so dS costs one packed multiply and add a pair of values.  16 warps:
//   warps 0-7   lanes, two threads each: of the four 32-column chunks of a tile, thread `half` takes chunks half and 2 + half, and
//               keeps its 64 P values between T1 and T2;
//   warp 8      K and V tiles (three and two stages, running across items).  A segment's last tile comes in boxes of 16 rows, and the one
//               its end lies in row by row with zeros behind it: K is summed over, and of V's rows dP must be a number;
//   warp 9      the next item's Q and dO tiles and its lse;
//   warps 10, 11, 14, 15  its delta, 32 rows each;
//   warps 12,13 MMA issuers: warp 12 T1, warp 13 T2 and ACC.  T1(j + 1) is issued once the lanes have read T1(j), T2(j + 2)
//               after ACC(j), which reads the dS over T2(j).
// 33k queries, 512 states, 24 heads of 128: 300 to 335 us, up to 1040 TFLOP/s (by the clock that the power cap leaves).
// A pair of tiles takes 2700 cycles in a row and 400 more shared out from between items: the chain T1 -> P -> dS -> ACC of a tile bounds it (without the loads of K, V, Q and dO 14 % less).
#include <algorithm>

#include "moc_cross.cuh"
#include "moc_tc.cuh"

namespace moc {

using namespace tc;

struct CrossDqParams {
    const CrossItem *items;
    int n_work, n_all, H, g, Lq, prows;      // items of all heads: with keys, all
    CrossRows K, V, O, dO, dQ;
    const float *lse;
    float *delta;                 // [H][Lq], written here for dK and dV
    float *part;                  // [H][prows][D] shares of dQ
    int *status;
    float scale, scale_log2;
    WaitBound wait;
};

enum CrossDqWait { CQ_XFULL = 96, CQ_XEMPTY, CQ_YFULL, CQ_YEMPTY, CQ_T1FULL, CQ_T2FULL, CQ_READ, CQ_DSDONE, CQ_ACCFULL, CQ_ACCFREE, CQ_SMEM };

constexpr int kDeltaWarps = 4;    // each forms delta of 32 rows of an item
constexpr int kCrossDqThreads = 512, kCrossKStages = 3, kCrossVStages = 2;

template <int D>
__global__ void __launch_bounds__(kCrossDqThreads, 1) cross_dq_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                         const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                         const __grid_constant__ CUtensorMap tmK16, const __grid_constant__ CUtensorMap tmV16,
                                                                         const CrossDqParams p) {
    constexpr int TILE_BYTES = 128 * D * 2;
    constexpr int SUB = D / 64;
    constexpr int SUB_BYTES = 128 * 128;
    enum { X_FULL = 0, X_EMPTY, K_FULL, K_EMPTY = K_FULL + kCrossKStages, V_FULL = K_EMPTY + kCrossKStages, V_EMPTY = V_FULL + kCrossVStages,
           T1_FULL = V_EMPTY + kCrossVStages, T1_READ, T2_FULL, DS_DONE = T2_FULL + 2, ACC_FULL = DS_DONE + 2, ACC_FREE, N_BARS };
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ __align__(16) float s_ld[2][2][128];      // per item parity: -lse * log2(e) and -delta of the item's rows
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;

    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // shared tiles: Q dO | K stages | V stages
    const uint32_t sX = sbase, sK = sbase + 2 * TILE_BYTES, sV = sbase + (2 + kCrossKStages) * TILE_BYTES;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    uint32_t dyn_bytes;
    asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(dyn_bytes));
    if ((sbase - smem_u32(smem_raw)) + (uint32_t)(2 + kCrossKStages + kCrossVStages) * TILE_BYTES > dyn_bytes) {
        // the launch gave less shared memory than the tiles need: report, touch nothing
        if (threadIdx.x == 0) report_abort(p.status, CQ_SMEM);
        return;
    }
    next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        // (a wait runs out a second after the launch at the earliest)
        if (blockIdx.x == 0) p.status[ST_STATUS] = p.status[ST_DETAIL] = 0;
        mbar_init(bar(X_FULL), 2 + kDeltaWarps);            // the tiles' bytes; lse; delta
        mbar_init(bar(X_EMPTY), 2 + 8);                     // both issuers, and each lane warp when it has the item's data
        for (int t = 0; t < kCrossKStages; ++t) { mbar_init(bar(K_FULL + t), 2); mbar_init(bar(K_EMPTY + t), 1); }
        for (int t = 0; t < kCrossVStages; ++t) { mbar_init(bar(V_FULL + t), 2); mbar_init(bar(V_EMPTY + t), 1); }
        mbar_init(bar(T1_FULL), 1);
        mbar_init(bar(T1_READ), 256);
        for (int t = 0; t < 2; ++t) { mbar_init(bar(T2_FULL + t), 1); mbar_init(bar(DS_DONE + t), 256); }
        mbar_init(bar(ACC_FULL), 1);
        mbar_init(bar(ACC_FREE), 256);
        fence_barrier_init();
    }
    __syncthreads();
    if (warp == 8) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // TMEM columns: T1 [0,128)  T2 of the even tiles [128,256)  ACC [256,384)  T2 of the odd tiles [384,512)
    const uint32_t tmem = tmem_slot;
    volatile int *abort_flag = &s_abort;

    // delta_i = sum_x dO_ix O_ix of rows 32 dw .. 32 dw + 31 of every item, formed while the item before it is in work (the rows are asked
    // for an item ahead of that): a pass over dO and O less than by a launch of its own, and O is read under the products.  (33k queries
    // to 512 states, whole kernel 312 us; without delta 285; with delta formed of the tile of dO in shared memory, which comes an item
    // later, 400; with barriers of their own for Q and dO 326; with both asked for by L2 prefetches an item ahead 328.)
    auto form_delta = [&](int dw) __attribute__((always_inline)) {
        constexpr int CH = D / 8, RP = 32 / CH, B = 4;         // lanes a row, rows an instruction, instructions under way
        const int sub = lane / CH, c16 = lane % CH;
        bool ok = true;
        const int n_items = cross_items(p.n_work);
        for (int n = 0; ok && n < n_items; ++n) {
            const int id = cross_item(n), rank = id / p.H, h = id - rank * p.H;
            const CrossItem it = p.items[rank];
            if (n + 1 < n_items) {
                const int next = cross_item(n + 1), nr = next / p.H, nh = next - nr * p.H, q = p.items[nr].q0 + dw * 32 + lane;
                if (dw * 32 + lane < p.items[nr].rows)
#pragma unroll
                    for (int x = 0; x < D / 64; ++x) {
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(p.O.row(nh, q) + x * 64));
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(p.dO.row(nh, q) + x * 64));
                    }
            }
            float mine = 0.f;
#pragma unroll 1
            for (int r0 = 0; r0 < 32; r0 += B * RP) {
                uint4 a[B], b[B];
#pragma unroll
                for (int y = 0; y < B; ++y) {
                    const int r = dw * 32 + r0 + y * RP + sub;
                    a[y] = b[y] = make_uint4(0, 0, 0, 0);
                    if (r < it.rows) {
                        a[y] = __ldcg(reinterpret_cast<const uint4 *>(p.O.row(h, it.q0 + r) + c16 * 8));      // (not through L1, where the items' descriptions are)
                        b[y] = __ldcg(reinterpret_cast<const uint4 *>(p.dO.row(h, it.q0 + r) + c16 * 8));
                    }
                }
#pragma unroll
                for (int y = 0; y < B; ++y) {
                    const uint32_t u[4] = {a[y].x, a[y].y, a[y].z, a[y].w}, w[4] = {b[y].x, b[y].y, b[y].z, b[y].w};
                    float v = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v = fmaf(__uint_as_float(u[i] << 16), __uint_as_float(w[i] << 16), v);
                        v = fmaf(__uint_as_float(u[i] & 0xffff0000u), __uint_as_float(w[i] & 0xffff0000u), v);
                    }
#pragma unroll
                    for (int o = CH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                    // lane l keeps row l of the 32
                    v = __shfl_sync(0xffffffffu, v, (lane % RP) * CH);
                    if (lane / RP == r0 / RP + y) mine = v;
                }
            }
            if (dw * 32 + lane < it.rows) p.delta[(size_t)h * p.Lq + it.q0 + dw * 32 + lane] = mine;
            if (n > 0) {
                ok = __all_sync(0xffffffffu, mbar_wait(bar(X_EMPTY), (n - 1) & 1, abort_flag, p.wait, CQ_XEMPTY));
                if (!ok) break;
            }
            s_ld[n & 1][1][dw * 32 + lane] = -mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(X_FULL));
        }
        // items without keys: dQ = 0
        for (int id = p.n_work + blockIdx.x; id < p.n_all; id += gridDim.x) {
            const int rank = id / p.H, h = id - rank * p.H, q0 = p.items[rank].q0, rows = p.items[rank].rows;
            for (int x = dw * 32 + lane; x < rows * CH; x += 32 * kDeltaWarps)
                *reinterpret_cast<uint4 *>(p.dQ.row(h, q0 + x / CH) + x % CH * 8) = make_uint4(0, 0, 0, 0);
        }
    };

    if (warp < 8) {
        // ------------------------------------------------------------ lane threads
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");      // 2 x 176 + 2 x 80 = 4 x 128, what the launch gave
        const int r = threadIdx.x & 127, half = warp >> 2;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint64_t c2 = pack2(p.scale_log2, p.scale_log2);
        int gt = 0;                                       // tiles processed
        bool ok = true, t1_early = false;
        // An item's results are read and stored behind the first tile of the next one: by then its last product has long landed.
        int o_h = 0, o_q0 = 0, o_rows = 0, o_slot = 0;
        const int n_items = cross_items(p.n_work);
        for (int n = 0; ok && n_items > 0; ++n) {
            const bool have = n < n_items;
            int n_keys = 0, h = 0, q0 = 0, rows = 0, slot = 0;
            uint64_t nlse2 = 0, ndlt2 = 0;
            if (have) {
                const int id = cross_item(n), rank = id / p.H;
                const CrossItem it = p.items[rank];
                h = id - rank * p.H; n_keys = it.n_keys; q0 = it.q0; rows = it.rows; slot = it.slot;
                if (n + 1 < n_items && lane == 0) prefetch_item(p.items + cross_item(n + 1) / p.H);
                ok = mbar_wait(bar(X_FULL), n & 1, abort_flag, p.wait, CQ_XFULL);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const float nlse = s_ld[n & 1][0][r], ndlt = s_ld[n & 1][1][r];
                nlse2 = pack2(nlse, nlse);
                ndlt2 = pack2(ndlt, ndlt);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(X_EMPTY));
            }
            int k = 0;
            do {
                if (have) {
                    float pv[64];
                    const int valid = min(128, n_keys - k), st = gt & 1;
                    const uint32_t t2 = tmem + lane_off + (st ? 384u : 128u);
                    ok = t1_early || mbar_wait_spin(bar(T1_FULL), gt & 1, abort_flag, p.wait, CQ_T1FULL);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t sv[2][32];
                    tmem_ld32(tmem + lane_off + half * 32, sv[0]);
                    tmem_ld32(tmem + lane_off + (2 + half) * 32, sv[1]);
                    tmem_wait_ld();
                    tc_fence_before();
                    mbar_arrive(bar(T1_READ));                   // T1 may be overwritten
                    // (a barrier is looked at ahead of its wait, which costs some hundred cycles even if it has completed)
                    const bool t2_early = mbar_test_wait(bar(T2_FULL + st), (gt >> 1) & 1);
#pragma unroll
                    for (int rd = 0; rd < 2; ++rd) {
                        if (rd == 1 && valid <= 64) break;       // (ACC takes no step over these)
#pragma unroll
                        for (int x = 0; x < 32; x += 2) {
                            float p0, p1;
                            unpack2(fma2(pack2(__uint_as_float(sv[rd][x]), __uint_as_float(sv[rd][x + 1])), c2, nlse2), p0, p1);
                            pv[rd * 32 + x] = ex2(p0);
                            pv[rd * 32 + x + 1] = ex2(p1);
                        }
                    }
                    if (valid < 128) {
#pragma unroll
                        for (int x = 0; x < 64; ++x)
                            if (((x >> 5) * 2 + half) * 32 + (x & 31) >= valid) pv[x] = 0.f;
                    }
                    ok = t2_early || mbar_wait_spin(bar(T2_FULL + st), (gt >> 1) & 1, abort_flag, p.wait, CQ_T2FULL);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t dp[2][32];
                    tmem_ld32(t2 + half * 32, dp[0]);
                    tmem_ld32(t2 + (2 + half) * 32, dp[1]);
                    t1_early = mbar_test_wait(bar(T1_FULL), (gt + 1) & 1);
                    tmem_wait_ld();
#pragma unroll
                    for (int rd = 0; rd < 2; ++rd) {
                        if (rd == 1 && valid <= 64) break;
                        uint32_t uds[16];
#pragma unroll
                        for (int x = 0; x < 32; x += 2) {
                            float a0, a1;
                            const auto t = add2(pack2(__uint_as_float(dp[rd][x]), __uint_as_float(dp[rd][x + 1])), ndlt2);
                            unpack2(mul2(pack2(pv[rd * 32 + x], pv[rd * 32 + x + 1]), t), a0, a1);
                            uds[x >> 1] = bf16x2(a0, a1);
                        }
                        tmem_st16(t2 + (rd * 2 + half) * 32, uds);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(DS_DONE + st));
                    ++gt;
                }
                if (k == 0 && n > 0) {
                    // ---- the results of the item before: of the two warps that share the TMEM lanes, each takes 64 columns of all rows
                    // (d = 128) or 16 rows (d = 64)
                    ok = mbar_wait(bar(ACC_FULL), (n - 1) & 1, abort_flag, p.wait, CQ_ACCFULL);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    constexpr int NJ = D / 32;                       // groups of eight rows that this warp has
                    const int l4 = lane >> 2, l2 = lane & 3, cb = D == 128 ? half : 0, j0 = D == 128 ? 0 : 2 * half;
                    uint32_t v[NJ / 2][32];
#pragma unroll
                    for (int x = 0; x < NJ / 2; ++x) tmem_ld_16x256b(tmem + lane_off + 256 + ((uint32_t)(x + (j0 >> 1)) << 20) + cb * 64, v[x]);
                    tmem_wait_ld();
                    tc_fence_before();
                    mbar_arrive(bar(ACC_FREE));                      // this item's dQ may be accumulated
#pragma unroll
                    for (int y = 0; y < NJ; ++y) {
                        const int row = (warp & 3) * 32 + (j0 + y) * 8 + l4;
                        float f[16];
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            f[2 * x] = __uint_as_float(v[y >> 1][4 * x + 2 * (y & 1)]) * p.scale;
                            f[2 * x + 1] = __uint_as_float(v[y >> 1][4 * x + 2 * (y & 1) + 1]) * p.scale;
                        }
                        if (o_slot < 0) {
                            uint32_t u[8];
#pragma unroll
                            for (int x = 0; x < 8; ++x) u[x] = bf16x2(f[2 * x], f[2 * x + 1]);
                            quad_transpose(u, l2);
                            if (row < o_rows) store_quad(p.dQ.row(o_h, o_q0 + row) + cb * 64, l2, u);
                        } else if (row < o_rows) {
                            float *dst = p.part + ((size_t)o_h * p.prows + o_slot + row) * D + cb * 64 + 2 * l2;
#pragma unroll
                            for (int x = 0; x < 8; ++x) *reinterpret_cast<float2 *>(dst + 8 * x) = make_float2(f[2 * x], f[2 * x + 1]);
                        }
                    }
                }
                k += 128;
            } while (k < n_keys);
            if (!have) break;
            o_h = h; o_q0 = q0; o_rows = rows; o_slot = slot;
        }
    } else if (warp == 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        // ------------------------------------------------------------ K and V tiles
        if (lane == 0) { prefetch_tensormap(&tmK); prefetch_tensormap(&tmV); }
        int n_k = 0, n_v = 0, s3 = 0, ph3 = 0;               // K and V tiles issued; K stage and its phase
        bool ok = true;
        // a tile's rows into `dst`: whole, or in boxes of 16 with the last one row by row
        auto load = [&](uint32_t dst, const CUtensorMap *tm, const CUtensorMap *tm16, const CrossRows &src, int hk, int t0, int valid, uint32_t full) {
            const int whole = valid >> 4;
            if (lane == 0) {
                mbar_expect_tx(full, whole * 16 * D * 2);
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub) {
                    if (valid == 128) tma_load_3d(dst + sub * SUB_BYTES, tm, sub * 64, t0, hk, full);
                    else for (int b = 0; b < whole; ++b) tma_load_3d(dst + sub * SUB_BYTES + b * 2048, tm16, sub * 64, t0 + b * 16, hk, full);
                }
            }
            if (valid & 15) {
                constexpr int CH = D / 8;
#pragma unroll
                for (int x = 0; x < 16 * CH / 32; ++x) {
                    const int i = x * 32 + lane, r = whole * 16 + i / CH, c16 = i % CH;
                    cp_async16(dst + (c16 >> 3) * SUB_BYTES + sw128_offset(r, c16 & 7), src.row(hk, t0 + min(r, valid - 1)) + c16 * 8, r < valid ? 16u : 0u);
                }
                cp_async_wait_all();
                fence_proxy_async_smem();
                __syncwarp();
            }
            if (lane == 0) mbar_arrive(full);
        };
        const int n_items = cross_items(p.n_work);
        for (int n = 0; ok && n < n_items; ++n) {
            const int id = cross_item(n), rank = id / p.H, hk = (id - rank * p.H) / p.g;
            const CrossItem it = p.items[rank];
            for (int k = 0; k < it.n_keys; k += 128) {
                const int valid = min(128, it.n_keys - k), s2 = n_v & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(K_EMPTY + s3), ph3 ^ 1, abort_flag, p.wait, CQ_YEMPTY));
                if (!ok) break;
                load(sK + s3 * TILE_BYTES, &tmK, &tmK16, p.K, hk, it.k0 + k, valid, bar(K_FULL + s3));
                ++n_k;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(V_EMPTY + s2), ((n_v >> 1) & 1) ^ 1, abort_flag, p.wait, CQ_YEMPTY));
                if (!ok) break;
                load(sV + s2 * TILE_BYTES, &tmV, &tmV16, p.V, hk, it.k0 + k, valid, bar(V_FULL + s2));
                ++n_v;
                if (++s3 == kCrossKStages) { s3 = 0; ph3 ^= 1; }
            }
        }
        if (*abort_flag) {      // copies already issued must land before the shared memory is released
            int dummy_flag = 0;
            for (int b = 1; b <= kCrossKStages; ++b)
                if (n_k - b >= 0) mbar_wait(bar(K_FULL + (n_k - b) % kCrossKStages), ((n_k - b) / kCrossKStages) & 1, &dummy_flag, p.wait, CQ_YFULL);
            for (int b = 1; b <= kCrossVStages; ++b)
                if (n_v - b >= 0) mbar_wait(bar(V_FULL + ((n_v - b) & 1)), ((n_v - b) >> 1) & 1, &dummy_flag, p.wait, CQ_YFULL);
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        // ------------------------------------------------------------ the items' Q and dO and lse (looked up before the buffers are free)
        if (warp > 9) {
            form_delta(warp - 10);
        } else {
            if (lane == 0) { prefetch_tensormap(&tmQ); prefetch_tensormap(&tmdO); }
            bool ok = true;
            int n = 0;
            for (const int n_items = cross_items(p.n_work); ok && n < n_items; ++n) {
                const int id = cross_item(n), rank = id / p.H, h = id - rank * p.H;
                const CrossItem it = p.items[rank];
                float l[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = x * 32 + lane;
                    l[x] = r < it.rows ? p.lse[(size_t)h * p.Lq + it.q0 + r] : INFINITY;       // rows that are not there: P = 0
                }
                if (n > 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait(bar(X_EMPTY), (n - 1) & 1, abort_flag, p.wait, CQ_XEMPTY));
                    if (!ok) break;
                }
                if (lane == 0) {
                    mbar_expect_tx(bar(X_FULL), 2 * TILE_BYTES);
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) {
                        tma_load_3d(sX + sub * SUB_BYTES, &tmQ, sub * 64, it.q0, h, bar(X_FULL));
                        tma_load_3d(sX + TILE_BYTES + sub * SUB_BYTES, &tmdO, sub * 64, it.q0, h, bar(X_FULL));
                    }
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) s_ld[n & 1][0][x * 32 + lane] = l[x] * -1.4426950408889634f;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(X_FULL));
            }
            if (*abort_flag && n > 0) {      // the last copies issued must land before the shared memory is released
                int dummy_flag = 0;
                mbar_wait(bar(X_FULL), (n - 1) & 1, &dummy_flag, p.wait, CQ_XFULL);
            }
        }
    } else {
        // ------------------------------------------------------------ MMA issuers (a warp stays together, one lane of it issues)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp > 13) {
            form_delta(warp - 12);
        } else {
            constexpr uint32_t IDESC_ACC = idesc_bf16_f32(128, D, 0, 1);      // ACC += dS K, K MN-major
            constexpr uint32_t STAGE = TILE_BYTES >> 4;
            auto lo = [](uint64_t d) { return (uint32_t)d; };
            auto hi = [](uint64_t d) { return (uint32_t)(d >> 32); };
            bool ok = true;
            auto wait = [&](int b, int parity, int code) { ok = ok && __all_sync(0xffffffffu, mbar_wait_spin(bar(b), parity, abort_flag, p.wait, code)); };
            auto n_of = [](int valid) { return (uint32_t)(valid + 15) & ~15u; };
            int gt = 0, s3 = 0, ph3 = 0;                       // tile, its K stage and phase
            const bool side1 = uniform(warp) == 12;
            const uint64_t x1 = smem_desc_sw128(sX, 16, 1024), kk = smem_desc_sw128(sK, 16, 1024);
            const uint64_t x2 = smem_desc_sw128(sX + TILE_BYTES, 16, 1024), vv = smem_desc_sw128(sV, 16, 1024);
            const uint64_t km = smem_desc_sw128(sK, SUB_BYTES, 1024);
            // T2(t) = dO V(t)^T for tile t of the launch; `last`: it is the item's last
            auto t2 = [&](int t, int valid, bool last) {
                const int s2 = t & 1;
                wait(V_FULL + s2, (t >> 1) & 1, CQ_YFULL);
                if (!ok) return;
                tc_fence_after();
                const uint32_t d = tmem + (s2 ? 384u : 128u), idesc = idesc_bf16_f32(128, n_of(valid), 0, 0);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t o = ((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4;
                    mma_ss_elect(d, lo(x2) + o, hi(x2), lo(vv) + s2 * STAGE + o, hi(vv), idesc, ks > 0);
                }
                tc_commit_elect(bar(T2_FULL + s2));
                tc_commit_elect(bar(V_EMPTY + s2));
                if (last) tc_commit_elect(bar(X_EMPTY));
            };
            for (int n = 0; ok && n < cross_items(p.n_work); ++n) {
                const int n_keys = uniform(p.items[cross_item(n) / p.H].n_keys), n_tiles = (n_keys + 127) >> 7;
                auto valid_of = [&](int j) { return min(128, n_keys - j * 128); };
                wait(X_FULL, n & 1, CQ_XFULL);
                if (!ok) break;
                if (side1) {
                    for (int j = 0; ok && j < n_tiles; ++j, ++gt) {
                        wait(K_FULL + s3, ph3, CQ_YFULL);
                        if (gt > 0) wait(T1_READ, (gt - 1) & 1, CQ_READ);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t idesc = idesc_bf16_f32(128, n_of(valid_of(j)), 0, 0);
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            const uint32_t o = ((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4;
                            mma_ss_elect(tmem, lo(x1) + o, hi(x1), lo(kk) + s3 * STAGE + o, hi(kk), idesc, ks > 0);
                        }
                        tc_commit_elect(bar(T1_FULL));
                        if (j + 1 == n_tiles) tc_commit_elect(bar(X_EMPTY));
                        if (++s3 == kCrossKStages) { s3 = 0; ph3 ^= 1; }
                    }
                } else {
                    t2(gt, valid_of(0), n_tiles == 1);
                    if (n_tiles > 1) t2(gt + 1, valid_of(1), n_tiles == 2);
                    for (int j = 0; ok && j < n_tiles; ++j, ++gt) {
                        const int steps = (valid_of(j) + 15) >> 4;
                        wait(DS_DONE + (gt & 1), (gt >> 1) & 1, CQ_DSDONE);
                        if (j == 0 && n > 0) wait(ACC_FREE, (n - 1) & 1, CQ_ACCFREE);      // the previous item's dQ has been read
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t ds = tmem + ((gt & 1) ? 384u : 128u);
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            if (ks < steps)                  // dS of 32 keys lies over the first half of their T2 columns
                                mma_ts_elect(tmem + 256, ds + (ks >> 1) * 32 + (ks & 1) * 8, lo(km) + s3 * STAGE + ks * (2048 >> 4), hi(km), IDESC_ACC, j > 0 || ks > 0);
                        tc_commit_elect(bar(K_EMPTY + s3));
                        if (++s3 == kCrossKStages) s3 = 0;
                        if (j + 2 < n_tiles) t2(gt + 2, valid_of(j + 2), j + 3 == n_tiles);
                    }
                    if (ok) tc_commit_elect(bar(ACC_FULL));
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
    if (threadIdx.x == 0) report_abort(p.status, s_abort);
}

int prepare_cross_dq(moc_cross *c) {
    const void *kernel = c->d == 128 ? (const void *)cross_dq_tc_kernel<128> : (const void *)cross_dq_tc_kernel<64>;
    // seven tiles, always the d = 128 footprint, so that CTAs, which each take all of the tensor memory, never share an SM
    const size_t tiles = (size_t)(2 + kCrossKStages + kCrossVStages) * 128 * 128 * 2;
    int optin = 0;
    cudaFuncAttributes fa;
    MOC_CUDA_TRY(cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, c->device));
    MOC_CUDA_TRY(cudaFuncGetAttributes(&fa, kernel));
    c->dq_smem = std::min(tiles + 1024, (size_t)optin - fa.sharedSizeBytes);
    if (c->dq_smem < tiles) return MOC_ERR_SHAPE;
    MOC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)c->dq_smem));
    return MOC_OK;
}

template <int D>
static int cross_dq_d(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, const float *lse, const moc_rows *dO,
                      const moc_rows *dQ, void *ws, cudaStream_t s) {
    CUtensorMap tmQ, tmdO, tmK, tmV, tmK16, tmV16;
    if (int r = make_tmap_rows_bf16(&tmQ, Q, c->H, c->Lq, D, 128)) return r;
    if (int r = make_tmap_rows_bf16(&tmdO, dO, c->H, c->Lq, D, 128)) return r;
    tmK = tmV = tmK16 = tmV16 = tmQ;                     // (without any states no key tile is loaded, but the maps are asked for ahead)
    if (c->Lk > 0) {
        if (int r = make_tmap_rows_bf16(&tmK, K, c->Hkv, c->Lk, D, 128)) return r;
        if (int r = make_tmap_rows_bf16(&tmV, V, c->Hkv, c->Lk, D, 128)) return r;
        if (int r = make_tmap_rows_bf16(&tmK16, K, c->Hkv, c->Lk, D, 16)) return r;
        if (int r = make_tmap_rows_bf16(&tmV16, V, c->Hkv, c->Lk, D, 16)) return r;
    }
    CrossDqParams a;
    a.items = c->d_dq_items; a.n_work = c->n_dq_work * c->H; a.n_all = (int)c->dq_items.size() * c->H;
    a.H = c->H; a.g = c->g; a.Lq = c->Lq; a.prows = c->dq_prows;
    a.K = CrossRows(K); a.V = CrossRows(V); a.O = CrossRows(O); a.dO = CrossRows(dO); a.dQ = CrossRows(dQ);
    a.lse = lse; a.delta = ws_ptr<float>(ws, c->ws.delta);
    a.part = ws_ptr<float>(ws, c->ws.part_dq);
    a.status = ws_ptr<int>(ws, c->ws.status);
    a.scale = c->scale; a.scale_log2 = c->scale * 1.4426950408889634f;
    a.wait = WaitBound::of(0);
    cross_dq_tc_kernel<D><<<cross_grid(c, c->dq_items.size()), kCrossDqThreads, c->dq_smem, s>>>(tmQ, tmdO, tmK, tmV, tmK16, tmV16, a);
    MOC_LAUNCH_CHECK();
    return MOC_OK;
}

int launch_cross_dq(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, const float *lse, const moc_rows *dO,
                    const moc_rows *dQ, void *ws, cudaStream_t s) {
    return c->d == 128 ? cross_dq_d<128>(c, Q, K, V, O, lse, dO, dQ, ws, s) : cross_dq_d<64>(c, Q, K, V, O, lse, dO, dQ, ws, s);
}

}  // namespace moc
