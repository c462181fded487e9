// Tensor-core forward of the cross attention (tcgen05 MMA, TMEM accumulators, TMA-fed tiles): one persistent CTA per SM walks items
// of up to 256 query rows of a head - two 128-row tiles that share every key tile - against their segment's keys, or a share of them.
//
// Online softmax, a query row per thread:  m' = max(m, scale s),  P = exp2(scale log2(e) s - m'),  l = l alpha + sum P,
// O = O alpha + P V, with O rescaled only when the maximum grows by more than 2^8 (P stays below that, l in fp32).  P is rounded to
// bf16 for its contraction, as in the stream's own attention: V is bf16, and both operands of a product have one type; two products of
// a P in two parts would take half as much again of the tensor pipe.  The sum takes it unrounded.  (O against 64 bits, normal inputs, in the
// 2-norm: 2.3e-3 of its size, of which 1.7e-3 are its own rounding to bf16.)
//
// 12 warps:
//   warps 0-3 / 4-7  softmax of query tile 0 / 1 (TMEM lane = row): S from TMEM, P back over it as packed bf16 (the first 64 keys
//              are handed over before the other 64 are formed), the item's results.  The exponentials of the two tiles take turns;
//   warp 8     K and V tiles of 128 keys, two stages each, running across items.  A segment's last tile comes in boxes of 16 rows, and of V
//              the box that its end lies in row by row with zeros behind it: P is zero there, but what stands behind a segment's keys - padding,
//              or another's - may be infinite, and 0 * inf is not 0;
//   warps 9, 10  MMA issuers, one per query tile:  S(0), then  O += P V(j),  S(j + 1)  per key tile;
//   warp 11    query tiles into a ring of three: the next item's are on their way while this one is in work.
// Items are sorted by length and dealt out in turn; the next item's S(0) runs while this one's results are stored.
// 33k queries, 512 states, 24 heads of 128: 195 to 212 us, up to 1060 TFLOP/s (by the clock that the power cap leaves).
// A key tile of both query tiles takes 3450 cycles, of which its products are 2048: the two softmax groups and their exponentials bound it, and the start and end of an item (2800 cycles to four key tiles).
// Every wait is bounded; one that runs out flags the workspace's status word, and the CTA drains its copies and leaves.
#include <algorithm>

#include "moc_cross.cuh"
#include "moc_tc.cuh"

namespace moc {

using namespace tc;

struct CrossFwdParams {
    const CrossItem *items;
    int n_all, H, g, Lq, prows;        // n_all: items of all heads
    CrossRows V, O;
    float *lse, *part_o, *part_lse;
    int *status;
    int first;                         // the call's first launch clears the status
    float scale_log2;
    WaitBound wait;
};

enum CrossWait { CW_QFULL = 1, CW_KFULL, CW_VFULL, CW_SFULL, CW_PFULL, CW_OFULL, CW_KEMPTY, CW_VEMPTY, CW_TURN, CW_PHALF, CW_QEMPTY, CW_OFREE };

constexpr int kCrossThreads = 384;

template <int D>
__global__ void __launch_bounds__(kCrossThreads, 1) cross_fwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                                        const __grid_constant__ CUtensorMap tmK,
                                                                        const __grid_constant__ CUtensorMap tmV,
                                                                        const __grid_constant__ CUtensorMap tmK16,
                                                                        const __grid_constant__ CUtensorMap tmV16, const CrossFwdParams p) {
    constexpr int TILE_BYTES = 128 * D * 2;
    constexpr int SUB = D / 64;            // 64-column (128-byte) sub-tiles per row
    constexpr int SUB_BYTES = 128 * 128;
    enum { Q_FULL = 0, Q_EMPTY = 6, K_FULL = 9, K_EMPTY = 11, V_FULL = 13, V_EMPTY = 15, S_FULL = 17, P_HALF = 19, P_FULL = 21, O_FULL = 23,
           O_FREE = 25, TURN = 27, N_BARS = 29 };
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;

    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // shared tiles: Q ring of three | K stages | V stages
    const uint32_t sQ = sbase, sK = sbase + 3 * TILE_BYTES, sV = sbase + 5 * TILE_BYTES;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };

    next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        // (a wait runs out a second after the launch at the earliest)
        if (p.first && blockIdx.x == 0) p.status[ST_STATUS] = p.status[ST_DETAIL] = 0;
        for (int t = 0; t < 3; ++t) {
            mbar_init(bar(Q_FULL + t), 1);             // [query tile][buffer]: each issuer sees every phase of its own
            mbar_init(bar(Q_FULL + 3 + t), 1);
            mbar_init(bar(Q_EMPTY + t), 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(bar(K_FULL + t), 1);
            mbar_init(bar(K_EMPTY + t), 2);            // one arrival per MMA issuer
            mbar_init(bar(V_FULL + t), 2);             // the boxes', and the rows' that come one by one
            mbar_init(bar(V_EMPTY + t), 2);
            mbar_init(bar(S_FULL + t), 1);
            mbar_init(bar(P_HALF + t), 128);
            mbar_init(bar(P_FULL + t), 128);
            mbar_init(bar(O_FULL + t), 1);
            mbar_init(bar(O_FREE + t), 128);
            mbar_init(bar(TURN + t), 128);
        }
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
    // TMEM columns: S0/P0 [0,128) S1/P1 [128,256) O0 [256,384) O1 [384,512)
    const uint32_t tmem = tmem_slot;
    volatile int *abort_flag = &s_abort;

    if (warp < 8) {
        // ------------------------------------------------------------ softmax and results
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");      // 2 x 224 + 56 = 3 x 168, what the launch gave
        const int g = warp >> 2;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + g * 128 + lane_off, tO = tmem + 256 + g * 128 + lane_off;
        const float c = p.scale_log2;
        enum : uint32_t { S_ODD = 1, TURN_ODD = 2, TURNED = 4, MINE_ODD = 8 };   // key tiles; in two-tile items; any of these; items
        uint32_t bits = 0;
        bool ok = true;
        for (int n = 0;; ++n) {
            const int id = cross_item(n);
            if (n * (int)gridDim.x >= p.n_all) break;
            if (id >= p.n_all) continue;
            const int rank = id / p.H, h = id - rank * p.H;
            const CrossItem it = p.items[rank];
            const bool two = it.rows > 128;
            if (g == 1 && !two) continue;
            const int tile_rows = min(128, it.rows - g * 128);
            if (it.n_keys == 0) {
                // no states: O = 0, lse = -inf
                const int r = threadIdx.x & 127;
                for (int x = r; x < tile_rows * (D / 8); x += 128)
                    *reinterpret_cast<uint4 *>(p.O.row(h, it.q0 + g * 128 + x / (D / 8)) + x % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
                if (r < tile_rows) p.lse[(size_t)h * p.Lq + it.q0 + g * 128 + r] = -INFINITY;
                continue;
            }
            float m_run = kLowest, l_run = 0.f;
            for (int k = 0; k < it.n_keys; k += 128) {
                const int valid = min(128, it.n_keys - k);
                ok = mbar_wait(bar(S_FULL + g), bits & S_ODD, abort_flag, p.wait, CW_SFULL);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                uint32_t v[4][32];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) tmem_ld32(tS + ch * 32, v[ch]);
                tmem_wait_ld();
                if (valid < 128) {
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch)
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (ch * 32 + x >= valid) v[ch][x] = 0xff800000u;   // -inf
                }
                float m4[4];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    m4[ch] = -INFINITY;
#pragma unroll
                    for (int x = 0; x < 32; x += 2) m4[ch] = max3(m4[ch], __uint_as_float(v[ch][x]), __uint_as_float(v[ch][x + 1]));
                }
                // (looked at ahead of its wait, which costs some hundred cycles even if the turn has come)
                const bool my_turn = !two || (g == 0 && !(bits & TURNED)) || mbar_test_wait(bar(TURN + (g ^ 1)), ((bits & TURN_ODD) ? 1 : 0) ^ (g == 1 ? 0 : 1));
                const float m_new = fmaxf(m_run, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * c);
                float alpha = 1.f;
                if (k == 0) {
                    m_run = m_new;
                } else if (m_new - m_run > 8.f) {
                    alpha = exp2f(m_run - m_new);
                    m_run = m_new;
                }
                // The exponentials of the two tiles take turns, so that each has the arithmetic pipes to itself while the other's MMAs run.
                if (!__all_sync(0xffffffffu, my_turn)) {
                    ok = mbar_wait(bar(TURN + (g ^ 1)), ((bits & TURN_ODD) ? 1 : 0) ^ (g == 1 ? 0 : 1), abort_flag, p.wait, CW_TURN);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                }
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    // this tile's P V of the keys before has completed (its commit precedes this S)
#pragma unroll 1
                    for (int ch = 0; ch < D / 32; ++ch) {
                        uint32_t o[32];
                        tmem_ld32(tO + ch * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                        tmem_st32(tO + ch * 32, o);
                    }
                }
                const uint64_t c2 = pack2(c, c), nm2 = pack2(-m_run, -m_run);
                uint64_t sum_a = 0ull, sum_b = 0ull;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    uint32_t u[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        float a0, a1;
                        unpack2(fma2(pack2(__uint_as_float(v[ch][2 * x]), __uint_as_float(v[ch][2 * x + 1])), c2, nm2), a0, a1);
                        a0 = ex2(a0);
                        a1 = ex2(a1);
                        if (x & 1) sum_b = add2(sum_b, pack2(a0, a1));
                        else sum_a = add2(sum_a, pack2(a0, a1));
                        u[x] = bf16x2(a0, a1);
                        if (ch == 3 && x == 11) {
                            // the turn is handed over before the last few: that takes about as long as they do
                            asm volatile("" ::"r"(u[x]), "r"(u[x - 1]), "r"(u[x - 2]) : "memory");
                            if (two) mbar_arrive(bar(TURN + g));
#pragma unroll
                            for (int y = x + 1; y < 16; ++y) asm volatile("" : "+r"(v[3][2 * y]), "+r"(v[3][2 * y + 1]));
                        }
                    }
                    tmem_st16(tS + ch * 16, u);
                    if (ch == 1) {
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive(bar(P_HALF + g));
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar(P_FULL + g));
                float s0, s1;
                unpack2(add2(sum_a, sum_b), s0, s1);
                l_run = l_run * alpha + (s0 + s1);
                bits ^= S_ODD;
                if (two) bits = (bits ^ TURN_ODD) | TURNED;
            }
            if (!ok) break;
            // ---- results, in the 16 x 256-bit shape of the tensor memory: four lanes write 128 contiguous bytes of a row
            constexpr int CB = D / 64;
            const int l4 = lane >> 2, l2 = lane & 3, row = (warp & 3) * 32 + lane;
            // (a share whose states all weigh nothing: its row is a sum of zeros, which has no weight in the sum of shares)
            const float inv_l = it.slot >= 0 && l_run == 0.f ? 1.f : 1.f / l_run, lse = (m_run + log2f(l_run)) * 0.6931471805599453f;
            if (row < tile_rows) {
                if (it.slot < 0) p.lse[(size_t)h * p.Lq + it.q0 + g * 128 + row] = lse;
                else p.part_lse[(size_t)h * p.prows + it.slot + g * 128 + row] = lse;
            }
            ok = mbar_wait(bar(O_FULL + g), (bits & MINE_ODD) ? 1 : 0, abort_flag, p.wait, CW_OFULL);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            bits ^= MINE_ODD;
            tc_fence_after();
            uint32_t o[2 * CB][32];
#pragma unroll
            for (int x = 0; x < 2 * CB; ++x) tmem_ld_16x256b(tO + ((x / CB) << 20) + (x % CB) * 64, o[x]);
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(bar(O_FREE + g));                // the issuer may start the next item's P V, which overwrites O
#pragma unroll
            for (int j = 0; j < 4; ++j) {                // rows 8 j + l4 of the warp's 32
                const float w = __shfl_sync(0xffffffffu, inv_l, j * 8 + l4);
                const int r = (warp & 3) * 32 + j * 8 + l4;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const uint32_t (&a)[32] = o[(j >> 1) * CB + cb];
                    float f[16];
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        f[2 * x] = __uint_as_float(a[4 * x + 2 * (j & 1)]) * w;
                        f[2 * x + 1] = __uint_as_float(a[4 * x + 2 * (j & 1) + 1]) * w;
                    }
                    if (it.slot < 0) {
                        uint32_t u[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) u[x] = bf16x2(f[2 * x], f[2 * x + 1]);
                        quad_transpose(u, l2);
                        if (r < tile_rows) store_quad(p.O.row(h, it.q0 + g * 128 + r) + cb * 64, l2, u);
                    } else if (r < tile_rows) {
                        float *dst = p.part_o + ((size_t)h * p.prows + it.slot + g * 128 + r) * D + cb * 64 + 2 * l2;
#pragma unroll
                        for (int x = 0; x < 8; ++x) *reinterpret_cast<float2 *>(dst + 8 * x) = make_float2(f[2 * x], f[2 * x + 1]);
                    }
                }
            }
        }
    } else if (warp == 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ K and V tiles
        if (lane == 0) { prefetch_tensormap(&tmK); prefetch_tensormap(&tmV); }
        int n_kv = 0, k_last = -1, v_last = -1;
        bool ok = true;
        for (int n = 0; ok; ++n) {
            const int id = cross_item(n);
            if (n * (int)gridDim.x >= p.n_all) break;
            if (id >= p.n_all) continue;
            const int rank = id / p.H, hk = (id - rank * p.H) / p.g;
            const CrossItem it = p.items[rank];
            for (int k = 0; k < it.n_keys; k += 128) {
                const int valid = min(128, it.n_keys - k), st = n_kv & 1, t0 = it.k0 + k;
                const uint32_t ph = (n_kv >> 1) & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(K_EMPTY + st), ph ^ 1, abort_flag, p.wait, CW_KEMPTY));
                if (!ok) break;
                const int boxes = (valid + 15) >> 4, whole = valid >> 4;
                if (lane == 0) {
                    mbar_expect_tx(bar(K_FULL + st), boxes * 16 * D * 2);
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) {
                        const uint32_t dst = sK + st * TILE_BYTES + sub * SUB_BYTES;
                        if (valid == 128) tma_load_3d(dst, &tmK, sub * 64, t0, hk, bar(K_FULL + st));
                        else for (int b = 0; b < boxes; ++b) tma_load_3d(dst + b * 2048, &tmK16, sub * 64, t0 + b * 16, hk, bar(K_FULL + st));
                    }
                }
                k_last = n_kv;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(V_EMPTY + st), ph ^ 1, abort_flag, p.wait, CW_VEMPTY));
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(bar(V_FULL + st), whole * 16 * D * 2);
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) {
                        const uint32_t dst = sV + st * TILE_BYTES + sub * SUB_BYTES;
                        if (valid == 128) tma_load_3d(dst, &tmV, sub * 64, t0, hk, bar(V_FULL + st));
                        else for (int b = 0; b < whole; ++b) tma_load_3d(dst + b * 2048, &tmV16, sub * 64, t0 + b * 16, hk, bar(V_FULL + st));
                    }
                }
                if (boxes > whole) {                     // the box that the segment's end lies in: its rows, and zeros
                    constexpr int CH = D / 8;
#pragma unroll
                    for (int x = 0; x < 16 * CH / 32; ++x) {
                        const int i = x * 32 + lane, r = whole * 16 + i / CH, c16 = i % CH;
                        cp_async16(sV + st * TILE_BYTES + (c16 >> 3) * SUB_BYTES + sw128_offset(r, c16 & 7),
                                   p.V.row(hk, t0 + min(r, valid - 1)) + c16 * 8, r < valid ? 16u : 0u);
                    }
                    cp_async_wait_all();
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (lane == 0) mbar_arrive(bar(V_FULL + st));
                v_last = n_kv;
                ++n_kv;
            }
        }
        if (*abort_flag) {      // copies already issued must land before the shared memory is released
            int dummy_flag = 0;
            for (int b = 0; b < 2; ++b) {
                const int kj = k_last - b, vj = v_last - b;
                if (kj >= 0) mbar_wait(bar(K_FULL + (kj & 1)), (kj >> 1) & 1, &dummy_flag, p.wait, CW_KFULL);
                if (vj >= 0) mbar_wait(bar(V_FULL + (vj & 1)), (vj >> 1) & 1, &dummy_flag, p.wait, CW_VFULL);
            }
        }
    } else if (warp < 11) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ MMA issuers (the warp stays together, one lane issues)
        const int g = uniform(warp - 9);
        constexpr uint32_t IDESC_PV = idesc_bf16_f32(128, D, 0, 1);
        const uint64_t q_desc0 = smem_desc_sw128(sQ, 16, 1024), k_desc0 = smem_desc_sw128(sK, 16, 1024);
        const uint64_t v_desc0 = smem_desc_sw128(sV, SUB_BYTES, 1024);
        constexpr uint64_t STAGE = TILE_BYTES >> 4;      // next tile, in address-field units
        int qb = 0;
        auto issue_qk = [&](int st, int valid) {
            const uint32_t idesc_qk = idesc_bf16_f32(128, (valid + 15) & ~15, 0, 0);
            const uint64_t qd = q_desc0 + qb * STAGE, kd = k_desc0 + (st ? STAGE : 0);
            const uint32_t q_lo = (uint32_t)qd, q_hi = (uint32_t)(qd >> 32), k_lo = (uint32_t)kd, k_hi = (uint32_t)(kd >> 32);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t o = ((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4;
                mma_ss_elect(tmem + g * 128, q_lo + o, q_hi, k_lo + o, k_hi, idesc_qk, ks > 0);
            }
        };
        auto issue_pv = [&](int st, int ks0, int ks1, bool accumulate) {       // 16 keys a step
            const uint64_t vd = v_desc0 + (st ? STAGE : 0);
            const uint32_t v_lo = (uint32_t)vd, v_hi = (uint32_t)(vd >> 32);
            const uint32_t d_o = tmem + 256 + g * 128, a_p = tmem + g * 128;
            if (ks1 - ks0 == 4) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) mma_ts_elect(d_o, a_p + (ks0 + ks) * 8, v_lo + (ks0 + ks) * (2048 >> 4), v_hi, IDESC_PV, accumulate || ks > 0);
            } else {
                for (int ks = ks0; ks < ks1; ++ks) mma_ts_elect(d_o, a_p + ks * 8, v_lo + ks * (2048 >> 4), v_hi, IDESC_PV, accumulate || ks > ks0);
            }
        };
        int n_mine = 0, n_kv = 0, n_p = 0, n_qtile = 0;  // items with this tile, K/V tiles, P tiles, query tiles before this item
        uint32_t q_phase = 0;                            // bit b: parity of the next load of this tile into buffer b
        bool ok = true;
        auto wait = [&](int b, uint32_t parity, int code) {
            return __all_sync(0xffffffffu, mbar_wait_spin(bar(b), parity, abort_flag, p.wait, code)) != 0;
        };
        for (int n = 0; ok; ++n) {
            const int id = cross_item(n);
            if (n * (int)gridDim.x >= p.n_all) break;
            if (id >= p.n_all) continue;
            const CrossItem it = p.items[id / p.H];
            const int rows = uniform(it.rows), n_keys = uniform(it.n_keys), n_tiles = (n_keys + 127) >> 7;
            if (n_tiles == 0) continue;
            const int q_seq = n_qtile + g;
            n_qtile += rows > 128 ? 2 : 1;
            if (g == 1 && rows <= 128) {
                // no second tile: this issuer only keeps the ring's accounting (a stage is released by two arrivals)
                for (int jt = 0; ok && jt < n_tiles; ++jt) {
                    const int st = n_kv & 1;
                    const uint32_t ph = (n_kv >> 1) & 1;
                    ok = wait(K_FULL + st, ph, CW_KFULL) && wait(V_FULL + st, ph, CW_VFULL);
                    if (!ok) break;
                    if (lane == 0) {
                        mbar_arrive(bar(K_EMPTY + st));
                        mbar_arrive(bar(V_EMPTY + st));
                    }
                    ++n_kv;
                }
                continue;
            }
            qb = q_seq % 3;
            ok = ok && wait(Q_FULL + 3 * g + qb, (q_phase >> qb) & 1, CW_QFULL);
            q_phase ^= 1u << qb;
            ok = ok && wait(K_FULL + (n_kv & 1), (n_kv >> 1) & 1, CW_KFULL);
            if (!ok) break;
            tc_fence_after();
            issue_qk(n_kv & 1, min(128, n_keys));
            tc_commit_elect(bar(S_FULL + g));
            tc_commit_elect(bar(K_EMPTY + (n_kv & 1)));
            if (n_tiles == 1) tc_commit_elect(bar(Q_EMPTY + qb));
            for (int jt = 0; ok && jt < n_tiles; ++jt) {
                const int st = n_kv & 1, sn = (n_kv + 1) & 1, valid = min(128, n_keys - jt * 128);
                const uint32_t ph = (n_kv >> 1) & 1, phn = ((n_kv + 1) >> 1) & 1;
                const bool more = jt + 1 < n_tiles;
                if (!wait(V_FULL + st, ph, CW_VFULL)) { ok = false; break; }
                if (more && !wait(K_FULL + sn, phn, CW_KFULL)) { ok = false; break; }
                const int steps = (valid + 15) >> 4, half = min(steps, 4);
                if (!wait(P_HALF + g, n_p & 1, CW_PHALF)) { ok = false; break; }
                // the first P V of an item overwrites O: the previous item's has been read
                if (jt == 0 && n_mine > 0 && !wait(O_FREE + g, (n_mine - 1) & 1, CW_OFREE)) { ok = false; break; }
                tc_fence_after();
                issue_pv(st, 0, half, jt > 0);
                if (!wait(P_FULL + g, n_p & 1, CW_PFULL)) { ok = false; break; }
                tc_fence_after();
                if (steps > half) issue_pv(st, half, steps, true);
                // a commit between two groups of MMAs leaves the pipe idle: the next S goes out first, then all commits
                if (more) {
                    issue_qk(sn, min(128, n_keys - (jt + 1) * 128));
                    tc_commit_elect(bar(S_FULL + g));
                    tc_commit_elect(bar(V_EMPTY + st));
                    tc_commit_elect(bar(K_EMPTY + sn));
                    if (jt + 2 == n_tiles) tc_commit_elect(bar(Q_EMPTY + qb));      // the item's last S
                } else {
                    tc_commit_elect(bar(V_EMPTY + st));
                    tc_commit_elect(bar(O_FULL + g));
                }
                ++n_kv;
                ++n_p;
            }
            ++n_mine;
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ query tiles
        if (lane == 0) {
            prefetch_tensormap(&tmQ);
            int n_qtile = 0;
            uint32_t q_phase = 0;                        // bit 3 g + buffer: parity of the next phase of that Q_FULL
            bool ok = true;
            for (int n = 0; ok; ++n) {
                const int id = cross_item(n);
                if (n * (int)gridDim.x >= p.n_all) break;
                if (id >= p.n_all) continue;
                const int rank = id / p.H, h = id - rank * p.H;
                const CrossItem it = p.items[rank];
                if (it.n_keys == 0) continue;
                for (int g = 0; g < (it.rows > 128 ? 2 : 1); ++g) {
                    const int qb = n_qtile % 3, qf = 3 * g + qb;
                    ok = mbar_wait(bar(Q_EMPTY + qb), ((n_qtile / 3) & 1) ^ 1, abort_flag, p.wait, CW_QEMPTY);
                    if (!ok) break;
                    mbar_expect_tx(bar(Q_FULL + qf), TILE_BYTES);
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub)      // (rows behind the item's end are another's, or zeros: nobody looks at their S)
                        tma_load_3d(sQ + qb * TILE_BYTES + sub * SUB_BYTES, &tmQ, sub * 64, it.q0 + g * 128, h, bar(Q_FULL + qf));
                    q_phase ^= 1u << qf;
                    ++n_qtile;
                }
            }
            if (*abort_flag) {
                int dummy_flag = 0;
                for (int b = 0; b < 6; ++b) mbar_wait(bar(Q_FULL + b), ((q_phase >> b) & 1) ^ 1, &dummy_flag, p.wait, CW_QFULL);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
    if (threadIdx.x == 0) report_abort(p.status, s_abort);
}

// always the d = 128 footprint: more than half an SM's shared memory, so that CTAs, which each take all of the tensor memory, never share one
constexpr size_t kSmem = 7 * (size_t)128 * 128 * 2 + 1024;

int prepare_cross_fwd(moc_cross *c) {
    const void *kernel = c->d == 128 ? (const void *)cross_fwd_tc_kernel<128> : (const void *)cross_fwd_tc_kernel<64>;
    MOC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));
    return MOC_OK;
}

template <int D>
static int cross_fwd_d(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws,
                       bool first, cudaStream_t s) {
    CUtensorMap tmQ, tmK, tmV, tmK16, tmV16;
    if (int r = make_tmap_rows_bf16(&tmQ, Q, c->H, c->Lq, D, 128)) return r;
    tmK = tmV = tmK16 = tmV16 = tmQ;                     // (without any states no key tile is loaded, but the maps are asked for ahead)
    if (c->Lk > 0) {
        if (int r = make_tmap_rows_bf16(&tmK, K, c->Hkv, c->Lk, D, 128)) return r;
        if (int r = make_tmap_rows_bf16(&tmV, V, c->Hkv, c->Lk, D, 128)) return r;
        if (int r = make_tmap_rows_bf16(&tmK16, K, c->Hkv, c->Lk, D, 16)) return r;
        if (int r = make_tmap_rows_bf16(&tmV16, V, c->Hkv, c->Lk, D, 16)) return r;
    }
    CrossFwdParams a;
    a.items = c->d_items; a.n_all = (int)c->items.size() * c->H;
    a.H = c->H; a.g = c->g; a.Lq = c->Lq; a.prows = c->prows;
    a.V = CrossRows(V); a.O = CrossRows(O); a.lse = lse;
    a.part_o = ws_ptr<float>(ws, c->ws.part_o); a.part_lse = ws_ptr<float>(ws, c->ws.part_lse);
    a.status = ws_ptr<int>(ws, c->ws.status); a.first = first;
    a.scale_log2 = c->scale * 1.4426950408889634f;
    a.wait = WaitBound::of(0);
    cross_fwd_tc_kernel<D><<<cross_grid(c, c->items.size()), kCrossThreads, kSmem, s>>>(tmQ, tmK, tmV, tmK16, tmV16, a);
    MOC_LAUNCH_CHECK();
    return MOC_OK;
}

int launch_cross_fwd(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws,
                     bool first, cudaStream_t s) {
    return c->d == 128 ? cross_fwd_d<128>(c, Q, K, V, O, lse, ws, first, s) : cross_fwd_d<64>(c, Q, K, V, O, lse, ws, first, s);
}

}  // namespace moc
