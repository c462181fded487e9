// dK and dV of the cross attention, key stationary.
//
//     P = exp(scale q.k - lse),  dP = dO V^T,  dS = P (dP - delta);  dV = P^T dO,  dK = scale dS^T Q
//     T1 = K Q^T,  T2 = V dO^T   (both operands from shared memory, into TMEM)
//     threads (two per TMEM lane) turn T1 into P, then (P, T2) into dS, written back to TMEM as bf16
//     ACC1 += dS Q,  ACC2 += P dO   (A from TMEM, the streamed tile as an MN-major operand)
//
// There are few key tiles (a prompt has some 500 states) and many query tiles, whose products are all alike: the plan cuts the query tiles of
// a key head and segment into parts of about the same length, and a piece is one key tile against one part.  The pieces of a part follow one another in
// the list that is dealt out to the CTAs, so that neighbours stream the same queries, out of L2.  Where a key tile has several parts, each
// leaves its fp32 sums in a slot and another launch adds them up in their order.  A shared key head's query heads are just more
// query tiles of the same key tile.
// A CTA holds the piece's 128 keys (K, V) and streams (Q, dO), 128 rows at a time, through rings of three and two stages that run
// across pieces.  Issue order: ACC2(j), T1(j+1), ACC1(j), T2(j+1): while the lanes form P(j+1) the pipe runs ACC1(j) and T2(j+1).
// 16 warps: 0-7 the lane threads, 8-11 the producers (two for each ring), 12 and 13 the MMA issuers, 14 the key tiles, 15 idle.
// 33k queries, 512 states, 24 heads of 128: 312 to 345 us, up to 1330 TFLOP/s (by the clock that the power cap leaves).
// A pair of tiles takes 3100 cycles, of which its products are 2048: the lanes' way from T1 and T2 to dS bounds it.
#include <algorithm>

#include "moc_cross.cuh"
#include "moc_tc.cuh"

namespace moc {

using namespace tc;

struct CrossKvParams {
    const CrossPiece *pieces;
    const int32_t *piece_off;
    int g, Lq;
    CrossRows Q, dO, dK, dV;
    const float *lse, *delta;
    float *part;                  // [slots][2][128][D]: dK, dV
    int *status;
    float scale, scale_log2;
    WaitBound wait;
};

enum CrossKvWait { CB_XFULL = 64, CB_YFULL, CB_YEMPTY, CB_T1FULL, CB_T2FULL, CB_PDONE, CB_DSDONE, CB_ACCFULL, CB_SMEM };

constexpr int kCrossY1 = 3, kCrossY2 = 2;      // stages of the streamed tiles Q (read twice per tile) and dO
constexpr int kCrossKvThreads = 512;

template <int D>
__global__ void __launch_bounds__(kCrossKvThreads, 1) cross_dkv_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                          const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                          const CrossKvParams p) {
    constexpr int TILE_BYTES = 128 * D * 2;
    constexpr int SUB = D / 64;
    constexpr int SUB_BYTES = 128 * 128;
    constexpr int CH = D / 8;               // 16-byte pieces per row
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    enum { X_FULL = 0, Y1_FULL = 1, Y1_EMPTY = 4, Y2_FULL = 7, Y2_EMPTY = 9, T1_FULL = 11, T2_FULL = 13, P_HALF = 15, P_DONE = 16, DS_DONE = 17,
           ACC_FULL = 19, T1_ISSUED = 20, N_BARS = 22 };
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ __align__(16) float s_ld[2][2][128];      // per streamed query, (-lse * log2(e), -delta), for tiles j and j + 1

    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // shared tiles: K V | Q stages | dO stages
    const uint32_t sX = sbase, sY1 = sbase + 2 * TILE_BYTES, sY2 = sbase + (2 + kCrossY1) * TILE_BYTES;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    uint32_t dyn_bytes;
    asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(dyn_bytes));
    if ((sbase - smem_u32(smem_raw)) + (uint32_t)(2 + kCrossY1 + kCrossY2) * TILE_BYTES > dyn_bytes) {
        // the launch gave less shared memory than the tiles need: report, touch nothing
        previous_done();
        if (threadIdx.x == 0) report_abort(p.status, CB_SMEM);
        return;
    }
    next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int b = 0; b < N_BARS; ++b)
            mbar_init(bar(b), (b >= Y1_FULL && b < Y1_EMPTY) || (b >= Y2_FULL && b < T1_FULL) || b == ACC_FULL ? 2      // two warps, or both issuers
                              : b >= P_HALF && b < ACC_FULL ? 256 : 1);
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
    // TMEM columns: T1 [0,128)  T2 [128,256)  ACC1 [256,384)  ACC2 [384,512)
    const uint32_t tmem = tmem_slot;
    volatile int *abort_flag = &s_abort;
    previous_done();
    const int piece0 = p.piece_off[blockIdx.x], piece1 = p.piece_off[blockIdx.x + 1];

    if (warp < 8) {
        // ------------------------------------------------------------ lane threads: of the four 32-column chunks of a tile, thread
        // `half` takes chunks half and 2 + half, so that the first half of P is finished first; P and dS lie over columns that
        // the thread alone has read
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");      // 2 x 168 + 80 + 88 <= 4 x 128, what the launch gave
        const int half = warp >> 2;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint64_t c2 = pack2(p.scale_log2, p.scale_log2);
        bool ok = true;
        int s3 = 0, ph3 = 0, jt = 0;                  // Y1 stage of tile jt and its phase; tiles of all pieces
        bool t1_early = false, y1_early = false;      // barriers looked at ahead of their waits
        for (int pi = piece0; ok && pi < piece1; ++pi) {
            for (const int end = jt + p.pieces[pi].u1 - p.pieces[pi].u0; jt < end; ++jt) {
                const int st = jt & 1;
                ok = t1_early || mbar_wait_spin(bar(T1_FULL + st), (jt >> 1) & 1, abort_flag, p.wait, CB_T1FULL);
                ok = ok && (y1_early || mbar_wait(bar(Y1_FULL + s3), ph3, abort_flag, p.wait, CB_YFULL));
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                constexpr uint32_t t2c = 128u;                // T2, then dS
                float pv[64];
                uint32_t sv[2][32];
                tmem_ld32(tmem + lane_off + half * 32, sv[0]);
                tmem_ld32(tmem + lane_off + (2 + half) * 32, sv[1]);
                tmem_wait_ld();
                bool t2_early = false;
#pragma unroll
                for (int rd = 0; rd < 2; ++rd) {
                    const int ch = rd * 2 + half;
                    const uint32_t (&s)[32] = sv[rd];
                    if (rd == 1) t2_early = mbar_test_wait(bar(T2_FULL + st), (jt >> 1) & 1);
#pragma unroll
                    for (int x = 0; x < 32; x += 4) {
                        const ulonglong2 l = *reinterpret_cast<const ulonglong2 *>(&s_ld[st][0][ch * 32 + x]);
                        const uint64_t nl[2] = {l.x, l.y};
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float p0, p1;
                            unpack2(fma2(pack2(__uint_as_float(s[x + 2 * y]), __uint_as_float(s[x + 2 * y + 1])), c2, nl[y]), p0, p1);
                            pv[rd * 32 + x + 2 * y] = ex2(p0);
                            pv[rd * 32 + x + 2 * y + 1] = ex2(p1);
                        }
                    }
                    uint32_t ups[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) ups[x] = bf16x2(pv[rd * 32 + 2 * x], pv[rd * 32 + 2 * x + 1]);
                    tmem_st16(tmem + lane_off + ch * 32, ups);
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(rd == 0 ? P_HALF : P_DONE));      // the first, then the second 64 columns of P
                }
                ok = t2_early || mbar_wait_spin(bar(T2_FULL + st), (jt >> 1) & 1, abort_flag, p.wait, CB_T2FULL);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                uint32_t dpv[2][32];
                tmem_ld32(tmem + lane_off + t2c + half * 32, dpv[0]);
                tmem_ld32(tmem + lane_off + t2c + (2 + half) * 32, dpv[1]);
                tmem_wait_ld();
#pragma unroll
                for (int rd = 0; rd < 2; ++rd) {
                    const int ch = rd * 2 + half;
                    const uint32_t (&dp)[32] = dpv[rd];
                    uint32_t uds[16];
#pragma unroll
                    for (int x = 0; x < 32; x += 4) {
                        const ulonglong2 d = *reinterpret_cast<const ulonglong2 *>(&s_ld[st][1][ch * 32 + x]);
                        const uint64_t nd[2] = {d.x, d.y};
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float a0, a1;
                            unpack2(mul2(pack2(pv[rd * 32 + x + 2 * y], pv[rd * 32 + x + 2 * y + 1]),
                                         add2(pack2(__uint_as_float(dp[x + 2 * y]), __uint_as_float(dp[x + 2 * y + 1])), nd[y])), a0, a1);
                            uds[(x >> 1) + y] = bf16x2(a0, a1);
                        }
                    }
                    tmem_st16(tmem + lane_off + t2c + ch * 32, uds);
                }
                if (++s3 == kCrossY1) { s3 = 0; ph3 ^= 1; }
                t1_early = mbar_test_wait(bar(T1_FULL + (st ^ 1)), ((jt + 1) >> 1) & 1);
                y1_early = mbar_test_wait(bar(Y1_FULL + s3), ph3);
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar(DS_DONE + st));
            }
            // ---- results: dK = scale ACC1, dV = ACC2.  Of the two warps that share the TMEM lanes, each takes 64 columns of all rows
            // (d = 128) or 16 rows (d = 64); four lanes write 128 contiguous bytes of a row
            if (ok) ok = mbar_wait(bar(ACC_FULL), (pi - piece0) & 1, abort_flag, p.wait, CB_ACCFULL);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const CrossPiece pc = p.pieces[pi];              // (read here: kept from before the loop, it would take the loop's registers)
            constexpr int NJ = D / 32;                       // groups of eight rows that this warp has
            const int l4 = lane >> 2, l2 = lane & 3, cb = D == 128 ? half : 0, j0 = D == 128 ? 0 : 2 * half;
#pragma unroll 1
            for (int side = 0; side < 2; ++side) {
                uint32_t v[NJ / 2][32];
                __syncwarp();
#pragma unroll
                for (int x = 0; x < NJ / 2; ++x)
                    tmem_ld_16x256b(tmem + lane_off + 256 + side * 128 + ((uint32_t)(x + (j0 >> 1)) << 20) + cb * 64, v[x]);
                tmem_wait_ld();
                tc_fence_before();                           // (before this thread's next P, which the next piece's sums wait for)
                const float w = side ? 1.f : p.scale;
                const CrossRows &out = side ? p.dV : p.dK;
#pragma unroll
                for (int y = 0; y < NJ; ++y) {
                    const int row = (warp & 3) * 32 + (j0 + y) * 8 + l4;
                    float f[16];
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        f[2 * x] = __uint_as_float(v[y >> 1][4 * x + 2 * (y & 1)]) * w;
                        f[2 * x + 1] = __uint_as_float(v[y >> 1][4 * x + 2 * (y & 1) + 1]) * w;
                    }
                    if (pc.slot < 0) {
                        uint32_t u[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) u[x] = bf16x2(f[2 * x], f[2 * x + 1]);
                        quad_transpose(u, l2);
                        if (row < pc.keys) store_quad(out.row(pc.h, pc.k0 + row) + cb * 64, l2, u);
                    } else if (row < pc.keys) {
                        float *dst = p.part + (((size_t)pc.slot * 2 + side) * 128 + row) * D + cb * 64 + 2 * l2;
#pragma unroll
                        for (int x = 0; x < 8; ++x) *reinterpret_cast<float2 *>(dst + 8 * x) = make_float2(f[2 * x], f[2 * x + 1]);
                    }
                }
            }
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------ producers: Q rows by the first two warps, dO rows by the other two, each
        // warp 64 rows of every tile.  Full tiles come by TMA, a segment's last by 16-byte copies: the tiles are summed over, and what stands
        // behind the segment's end times P = 0 need not be 0.  Behind its end dO has zeros, but Q its last row again: a row of zeros times a
        // key of minus infinity, which has no weight, would not be a number, where that row's product is one if any is.  (Both directions of 64
        // segments of one query and 1500 states, 24 heads on 8: 600 us, with rows of zeros 595; with dO's repeated too 602.)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        const int pw = warp - 8, wsub = pw & 1;
        const bool y1 = pw < 2;
        int st = 0, ph = 0, jt = 0;                        // stage of tile jt in this warp's ring, and its phase
        const int n_st = y1 ? kCrossY1 : kCrossY2, b_full = y1 ? Y1_FULL : Y2_FULL, b_empty = y1 ? Y1_EMPTY : Y2_EMPTY;
        const uint32_t ring = y1 ? sY1 : sY2;
        const CUtensorMap *tile_map = y1 ? &tmQ : &tmdO;
        const CrossRows src = y1 ? p.Q : p.dO;
        if (lane == 0) prefetch_tensormap(tile_map);
        bool ok = true;
        for (int pi = piece0; ok && pi < piece1; ++pi) {
            const CrossPiece pc = p.pieces[pi];
            const int tiles = (pc.q1 - pc.q0 + 127) >> 7;
            // lse and delta of this lane's two rows of a tile, one tile ahead; a row that is not there gets lse = +inf: its P is zero
            float q_lse[2], q_del[2];
            int h = 0, t0 = 0;
            auto look_up = [&](int u) {
                const int gh = u / tiles;
                h = pc.h * p.g + gh;
                t0 = pc.q0 + (u - gh * tiles) * 128;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int q = t0 + wsub * 64 + x * 32 + lane;
                    q_lse[x] = INFINITY;
                    q_del[x] = 0.f;
                    if (y1 && q < pc.q1) {
                        q_lse[x] = p.lse[(size_t)h * p.Lq + q];
                        q_del[x] = p.delta[(size_t)h * p.Lq + q];
                    }
                }
            };
            look_up(pc.u0);
            for (int u = pc.u0; u < pc.u1; ++u, ++jt) {
                const int c_h = h, c_t0 = t0;
                const float c_lse[2] = {q_lse[0], q_lse[1]}, c_del[2] = {q_del[0], q_del[1]};
                if (u + 1 < pc.u1) look_up(u + 1);
                ok = mbar_wait(bar(b_empty + st), ph ^ 1, abort_flag, p.wait, CB_YEMPTY);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t dst = ring + st * TILE_BYTES;
                const bool whole = c_t0 + 128 <= pc.q1;
                if (whole) {
                    if (lane == 0) {
#pragma unroll
                        for (int sub = 0; sub < SUB; ++sub)
                            tma_load_3d(dst + sub * SUB_BYTES + wsub * 64 * 128, tile_map, sub * 64, c_t0 + wsub * 64, c_h, bar(b_full + st));
                    }
                } else {
                    constexpr int RP = 32 / CH;            // rows per instruction
                    const int c16 = lane % CH;
#pragma unroll 1
                    for (int r8 = 0; r8 < 64; r8 += 8)     // (eight rows at a time, in which the swizzle repeats)
#pragma unroll
                        for (int rb = 0; rb < 8; rb += RP) {
                            const int rl = rb + lane / CH, q = c_t0 + wsub * 64 + r8 + rl;
                            cp_async16(dst + (c16 >> 3) * SUB_BYTES + (wsub * 64 + r8) * 128 + sw128_offset(rl, c16 & 7),
                                       src.row(c_h, min(q, pc.q1 - 1)) + c16 * 8, y1 || q < pc.q1 ? 16u : 0u);
                        }
                }
                if (y1) {
                    // the lanes have finished with the lse / delta of tile jt - 2
                    if (jt >= 2) ok = mbar_wait(bar(DS_DONE + (jt & 1)), ((jt - 2) >> 1) & 1, abort_flag, p.wait, CB_DSDONE);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        s_ld[jt & 1][0][wsub * 64 + x * 32 + lane] = c_lse[x] * -1.4426950408889634f;
                        s_ld[jt & 1][1][wsub * 64 + x * 32 + lane] = -c_del[x];
                    }
                }
                if (!whole) {
                    cp_async_wait_all();
                    fence_proxy_async_smem();
                }
                __syncwarp();
                // one of the ring's two warps (the announcement of a whole tile's bytes is its arrival, behind lse and delta)
                if (lane == 0) {
                    if (whole) mbar_expect_tx(bar(b_full + st), TILE_BYTES / 2);
                    else mbar_arrive(bar(b_full + st));
                }
                if (++st == n_st) { st = 0; ph ^= 1; }
            }
        }
        if (*abort_flag) {      // copies already issued must land before the shared memory is released
            cp_async_wait_all();
            int dummy_flag = 0;
            for (int b = 0; b <= n_st; ++b)                // (tile jt may be under way without its arrival: that wait runs out, by when it has landed)
                if (jt - b >= 0) mbar_wait(bar(b_full + (jt - b) % n_st), ((jt - b) / n_st) & 1, &dummy_flag, p.wait, CB_YFULL);
        }
    } else {
        // ------------------------------------------------------------ MMA issuers: warp 12 owns the T1 / P side (T1, ACC2), warp 13 the
        // T2 / dS side (T2, ACC1)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 14 && lane == 0) {
            // the pieces' key tiles, each when the products of the one before it are done
            int n_x = 0;
            bool ok = true;
            for (int pi = piece0; ok && pi < piece1; ++pi) {
                const CrossPiece pc = p.pieces[pi];
                if (n_x > 0) ok = mbar_wait(bar(ACC_FULL), (n_x - 1) & 1, abort_flag, p.wait, CB_ACCFULL);
                if (!ok) break;
                mbar_expect_tx(bar(X_FULL), 2 * TILE_BYTES);
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub) {      // (rows behind the piece's keys are another's: nobody looks at their sums)
                    tma_load_3d(sX + sub * SUB_BYTES, &tmK, sub * 64, pc.k0, pc.h, bar(X_FULL));
                    tma_load_3d(sX + TILE_BYTES + sub * SUB_BYTES, &tmV, sub * 64, pc.k0, pc.h, bar(X_FULL));
                }
                ++n_x;
            }
            if (*abort_flag && n_x > 0) {
                int dummy_flag = 0;
                mbar_wait(bar(X_FULL), (n_x - 1) & 1, &dummy_flag, p.wait, CB_XFULL);
            }
        } else if (warp <= 13) {                // the warp stays together, one lane of it issues
            const bool side1 = uniform(warp) == 12;
            constexpr uint32_t IDESC_T = idesc_bf16_f32(128, 128, 0, 0);      // T = X Y^T, both K-major
            constexpr uint32_t IDESC_ACC = idesc_bf16_f32(128, D, 0, 1);      // ACC += (TMEM) Y, Y MN-major
            constexpr uint32_t STAGE = TILE_BYTES >> 4;
            const uint64_t x1 = smem_desc_sw128(sX, 16, 1024), x2 = smem_desc_sw128(sX + TILE_BYTES, 16, 1024);
            const uint64_t y1k = smem_desc_sw128(sY1, 16, 1024), y2k = smem_desc_sw128(sY2, 16, 1024);
            const uint64_t y1m = smem_desc_sw128(sY1, SUB_BYTES, 1024), y2m = smem_desc_sw128(sY2, SUB_BYTES, 1024);
            auto lo = [](uint64_t d) { return (uint32_t)d; };
            auto hi = [](uint64_t d) { return (uint32_t)(d >> 32); };
            bool ok = true;
            auto wait = [&](int b, int parity, int code) { ok = ok && __all_sync(0xffffffffu, mbar_wait_spin(bar(b), parity, abort_flag, p.wait, code)); };
            auto t1 = [&](int s3) {         // T1 = K Q^T, Q in stage s3
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t o = ((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4;
                    mma_ss_elect(tmem, lo(x1) + o, hi(x1), lo(y1k) + s3 * STAGE + o, hi(y1k), IDESC_T, ks > 0);
                }
            };
            auto t2 = [&](int s2) {         // T2 = V dO^T
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t o = ((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4;
                    mma_ss_elect(tmem + 128, lo(x2) + o, hi(x2), lo(y2k) + s2 * STAGE + o, hi(y2k), IDESC_T, ks > 0);
                }
            };
            auto acc1 = [&](int s3, bool add) {   // ACC1 (+)= dS Q
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    mma_ts_elect(tmem + 256, tmem + 128 + (ks >> 1) * 32 + (ks & 1) * 8, lo(y1m) + s3 * STAGE + ks * (2048 >> 4), hi(y1m), IDESC_ACC, add || ks > 0);
            };
            auto acc2 = [&](int s2, int half, bool add) {   // ACC2 (+)= P dO, the K steps of one half of P
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    mma_ts_elect(tmem + 384, tmem + (half * 2 + (ks >> 1)) * 32 + (ks & 1) * 8, lo(y2m) + s2 * STAGE + (half * 4 + ks) * (2048 >> 4), hi(y2m),
                                 IDESC_ACC, add || half > 0 || ks > 0);
            };
            int j = 0, s3 = 0, ph3 = 0, n_turn = 0;               // tile of all pieces; its Y1 stage and phase; T1_ISSUED so far
            for (int pi = piece0; ok && pi < piece1; ++pi) {
                const int n_tiles = uniform(p.pieces[pi].u1 - p.pieces[pi].u0);
                const int pn = pi - piece0, j0 = j;
                wait(X_FULL, pn & 1, CB_XFULL);
                if (side1) {
                    // ACC2(j) starts on the first half of P(j); T1(j+1) follows ACC2(j), which reads the P written over T1(j)
                    wait(Y1_FULL + s3, ph3, CB_YFULL);
                    if (!ok) break;
                    tc_fence_after();
                    t1(s3);
                    tc_commit_elect(bar(T1_FULL + (j & 1)));
                    if (++s3 == kCrossY1) { s3 = 0; ph3 ^= 1; }   // from here on the stage of tile j + 1
                    for (; ok && j < j0 + n_tiles; ++j) {
                        const bool more = j + 1 < j0 + n_tiles;
                        wait(Y2_FULL + (j & 1), (j >> 1) & 1, CB_YFULL);
                        wait(P_HALF, j & 1, CB_PDONE);
                        if (!ok) break;
                        tc_fence_after();
                        acc2(j & 1, 0, j > j0);
                        if (more) wait(Y1_FULL + s3, ph3, CB_YFULL);
                        wait(P_DONE, j & 1, CB_PDONE);
                        if (!ok) break;
                        tc_fence_after();
                        acc2(j & 1, 1, true);
                        if (more) {
                            t1(s3);
                            tc_commit_elect(bar(T1_FULL + ((j + 1) & 1)));
                            if (++s3 == kCrossY1) { s3 = 0; ph3 ^= 1; }
                        }
                        tc_commit_elect(bar(Y2_EMPTY + (j & 1)));             // one of two arrivals
                        // the other side may use the pipe again (two barriers: this side may be one tile ahead, never two)
                        if (more) {
                            if (lane == 0) mbar_arrive(bar(T1_ISSUED + (n_turn & 1)));
                            ++n_turn;
                        }
                    }
                } else {
                    // The lanes wait for T1(j+1) as soon as dS(j) is done, so this side keeps out of the pipe while the other issues
                    // it: ACC1(j) waits for that issue, and T2(j+1) follows ACC1(j), which reads the dS written over T2(j).
                    wait(Y2_FULL + (j & 1), (j >> 1) & 1, CB_YFULL);
                    if (!ok) break;
                    tc_fence_after();
                    t2(j & 1);
                    tc_commit_elect(bar(T2_FULL + (j & 1)));
                    tc_commit_elect(bar(Y2_EMPTY + (j & 1)));
                    for (; ok && j < j0 + n_tiles; ++j) {
                        const int jn = j + 1;
                        const bool more = jn < j0 + n_tiles;
                        if (more) {
                            wait(T1_ISSUED + (n_turn & 1), (n_turn >> 1) & 1, CB_T1FULL);
                            ++n_turn;
                        }
                        wait(Y1_FULL + s3, ph3, CB_YFULL);                     // (long there: dS(j) follows T1(j))
                        wait(DS_DONE + (j & 1), (j >> 1) & 1, CB_DSDONE);
                        if (!ok) break;
                        tc_fence_after();
                        acc1(s3, j > j0);
                        tc_commit_elect(bar(Y1_EMPTY + s3));
                        if (++s3 == kCrossY1) { s3 = 0; ph3 ^= 1; }
                        if (more) {
                            wait(Y2_FULL + (jn & 1), (jn >> 1) & 1, CB_YFULL);
                            if (!ok) break;
                            t2(jn & 1);
                            tc_commit_elect(bar(T2_FULL + (jn & 1)));
                            tc_commit_elect(bar(Y2_EMPTY + (jn & 1)));
                        }
                    }
                }
                if (ok) tc_commit_elect(bar(ACC_FULL));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
    if (threadIdx.x == 0) report_abort(p.status, s_abort);
}

int prepare_cross_dkv(moc_cross *c) {
    const void *kernel = c->d == 128 ? (const void *)cross_dkv_tc_kernel<128> : (const void *)cross_dkv_tc_kernel<64>;
    // seven tiles, always the d = 128 footprint, so that CTAs, which each take all of the tensor memory, never share an SM
    const size_t tiles = (size_t)(2 + kCrossY1 + kCrossY2) * 128 * 128 * 2;
    int optin = 0;
    cudaFuncAttributes fa;
    MOC_CUDA_TRY(cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, c->device));
    MOC_CUDA_TRY(cudaFuncGetAttributes(&fa, kernel));
    c->dkv_smem = std::min(tiles + 1024, (size_t)optin - fa.sharedSizeBytes);
    if (c->dkv_smem < tiles) return MOC_ERR_SHAPE;
    MOC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)c->dkv_smem));
    return MOC_OK;
}

template <int D>
static int cross_dkv_d(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const float *lse, const moc_rows *dO,
                       const moc_rows *dK, const moc_rows *dV, void *ws, cudaStream_t s) {
    CUtensorMap tmK, tmV, tmQ, tmdO;       // Q and dO: tiles of 64 rows
    if (int r = make_tmap_rows_bf16(&tmK, K, c->Hkv, c->Lk, D, 128)) return r;
    if (int r = make_tmap_rows_bf16(&tmV, V, c->Hkv, c->Lk, D, 128)) return r;
    if (int r = make_tmap_rows_bf16(&tmQ, Q, c->H, c->Lq, D, 64)) return r;
    if (int r = make_tmap_rows_bf16(&tmdO, dO, c->H, c->Lq, D, 64)) return r;
    CrossKvParams a;
    a.pieces = c->d_pieces; a.piece_off = c->d_piece_off; a.g = c->g; a.Lq = c->Lq;
    a.Q = CrossRows(Q); a.dO = CrossRows(dO); a.dK = CrossRows(dK); a.dV = CrossRows(dV);
    a.lse = lse; a.delta = ws_ptr<float>(ws, c->ws.delta);
    a.part = ws_ptr<float>(ws, c->ws.part_kv);
    a.status = ws_ptr<int>(ws, c->ws.status);
    a.scale = c->scale; a.scale_log2 = c->scale * 1.4426950408889634f;
    a.wait = WaitBound::of(0);
    // A short launch begins while dQ's, or the one that adds up its shares, ends: of these it needs delta (82 queries, 755 states, 6 heads, both
    // directions in a graph: 34.2 us, 35.1 one after the other).  A long one does not: its CTAs would lie where SMs come free, not with
    // neighbours that stream the same queries side by side (33k queries, 512 states, 24 heads: 845 us, 836 one after the other).
    const bool early = c->pieces.size() <= (size_t)c->n_sm;
    MOC_CUDA_TRY(launch_early(early, cross_dkv_tc_kernel<D>, (unsigned)(c->piece_off.size() - 1), kCrossKvThreads, c->dkv_smem, s, tmK, tmV, tmQ, tmdO, a));
    MOC_LAUNCH_CHECK();
    return MOC_OK;
}

int launch_cross_dkv(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const float *lse, const moc_rows *dO,
                     const moc_rows *dK, const moc_rows *dV, void *ws, cudaStream_t s) {
    return c->d == 128 ? cross_dkv_d<128>(c, Q, K, V, lse, dO, dK, dV, ws, s) : cross_dkv_d<64>(c, Q, K, V, lse, dO, dK, dV, ws, s);
}

}  // namespace moc
