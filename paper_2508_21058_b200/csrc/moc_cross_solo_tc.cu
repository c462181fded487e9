// Tensor-core forward of the cross attention for items of one 128-row query tile (segments of up to 128 queries, last tiles).
//
// With one query tile the chain of a key tile, S -> softmax -> P V -> S, has nothing to run beside it: 4200 cycles in the kernel of
// two-tile items, as much as two tiles take there together.  Here the two softmax groups work on the same query rows and take every other
// key tile, each with its own S and O in tensor memory, its own running maximum and sum and its own K and V stage; at an item's end
// the first group reads both O, which lie in the same tensor memory lanes, and puts them together:
//     m = max(m0, m1),  O = (2^(m0 - m) O0 + 2^(m1 - m) O1) / (2^(m0 - m) l0 + 2^(m1 - m) l1).
// Arithmetic, masking and the zeros behind a segment's last value row: as in moc_cross_fwd_tc.cu.
//
// 257 queries (three tiles) against 32,760 states, 24 heads of 128, in shares of 128 key tiles: 162 us, 2150 cycles a key tile.
//
// 12 warps: 0-3 / 4-7 the softmax groups, 8 the query tiles (a ring of three) and K, 9 and 10 an MMA issuer for each group, 11 V.
#include <algorithm>

#include "moc_cross.cuh"
#include "moc_tc.cuh"

namespace moc {

using namespace tc;

struct CrossSoloParams {
    const CrossItem *items;
    int n_all, H, g, Lq, prows;       // n_all: items of all heads, each with keys
    CrossRows V, O;
    float *lse, *part_o, *part_lse;
    int *status;
    int first;                         // the call's first launch clears the status
    float scale_log2;
    WaitBound wait;
};

enum CrossSoloWait { CS_QFULL = 32, CS_KFULL, CS_VFULL, CS_SFULL, CS_PFULL, CS_OFULL, CS_KEMPTY, CS_VEMPTY, CS_ML, CS_PHALF, CS_QEMPTY, CS_OFREE };

constexpr int kCrossSoloThreads = 384;

template <int D>
__global__ void __launch_bounds__(kCrossSoloThreads, 1) cross_solo_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                                             const __grid_constant__ CUtensorMap tmK,
                                                                             const __grid_constant__ CUtensorMap tmV,
                                                                             const __grid_constant__ CUtensorMap tmK16,
                                                                             const __grid_constant__ CUtensorMap tmV16, const CrossSoloParams p) {
    constexpr int TILE_BYTES = 128 * D * 2;
    constexpr int SUB = D / 64;
    constexpr int SUB_BYTES = 128 * 128;
    // pairs: per group
    enum { Q_FULL = 0, Q_EMPTY = 3, K_FULL = 6, K_EMPTY = 8, V_FULL = 10, V_EMPTY = 12, S_FULL = 14, P_HALF = 16, P_FULL = 18, O_FULL = 20,
           O_FREE = 22, ML = 24, N_BARS = 25 };
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ float s_ml[2][128];                 // the second group's maximum and sum
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;

    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // shared tiles: Q ring of three | K of either group | V of either group
    const uint32_t sQ = sbase, sK = sbase + 3 * TILE_BYTES, sV = sbase + 5 * TILE_BYTES;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };

    next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        // (a wait runs out a second after the launch at the earliest)
        if (p.first && blockIdx.x == 0) p.status[ST_STATUS] = p.status[ST_DETAIL] = 0;
        for (int t = 0; t < 3; ++t) {
            mbar_init(bar(Q_FULL + t), 1);
            mbar_init(bar(Q_EMPTY + t), 2);            // both issuers: each sees every phase of Q_FULL
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(bar(K_FULL + t), 1);
            mbar_init(bar(K_EMPTY + t), 1);
            mbar_init(bar(V_FULL + t), 2);             // the boxes', and the rows' that come one by one
            mbar_init(bar(V_EMPTY + t), 1);
            mbar_init(bar(S_FULL + t), 1);
            mbar_init(bar(P_HALF + t), 128);
            mbar_init(bar(P_FULL + t), 128);
            mbar_init(bar(O_FULL + t), 1);
            mbar_init(bar(O_FREE + t), 128);           // the first group's threads
        }
        mbar_init(bar(ML), 128);
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
    const int n_items = cross_items(p.n_all);

    if (warp < 8) {
        // ------------------------------------------------------------ softmax and results
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");      // 2 x 224 + 56 = 3 x 168, what the launch gave
        const int g = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + g * 128 + lane_off;
        const float c = p.scale_log2;
        int n_tile = 0, n_own = 0, n_ml = 0;               // key tiles and items of this group; items with two groups
        bool ok = true;
        for (int n = 0; ok && n < n_items; ++n) {
            const int id = cross_item(n), rank = id / p.H, h = id - rank * p.H;
            const CrossItem it = p.items[rank];
            if (n + 1 < n_items && lane == 0) prefetch_item(p.items + cross_item(n + 1) / p.H);
            float m_run = kLowest, l_run = 0.f;
            for (int k = g * 128; k < it.n_keys; k += 256) {
                const int valid = min(128, it.n_keys - k);
                ok = mbar_wait_spin(bar(S_FULL + g), n_tile & 1, abort_flag, p.wait, CS_SFULL);
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
                const float m_new = fmaxf(m_run, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * c);
                float alpha = 1.f;
                if (k == g * 128) {
                    m_run = m_new;
                } else if (m_new - m_run > 8.f) {
                    alpha = exp2f(m_run - m_new);
                    m_run = m_new;
                }
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    // this group's P V of the keys before has completed (its commit precedes this S)
                    const uint32_t tO = tmem + 256 + g * 128 + lane_off;
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
                ++n_tile;
            }
            if (!ok) break;
            const bool both = it.n_keys > 128;
            if (g == 1) {
                if (both) {
                    // the last item's have been read, and its O1
                    if (n_ml > 0) {
                        ok = mbar_wait(bar(O_FREE + 1), (n_ml - 1) & 1, abort_flag, p.wait, CS_OFREE);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                    }
                    s_ml[0][row] = m_run;
                    s_ml[1][row] = l_run;
                    mbar_arrive(bar(ML));
                    ++n_ml;
                }
                continue;
            }
            // ---- results of both groups
            float m1 = kLowest, l1 = 0.f;
            if (both) {
                ok = mbar_wait(bar(ML), n_ml & 1, abort_flag, p.wait, CS_ML);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                m1 = s_ml[0][row];
                l1 = s_ml[1][row];
            }
            const float big = fmaxf(m_run, m1), e0 = ex2(m_run - big), e1 = both ? ex2(m1 - big) : 0.f;
            // (a share whose states all weigh nothing: its row is a sum of zeros, which has no weight in the sum of shares)
            const float sum = e0 * l_run + e1 * l1, inv = it.slot >= 0 && sum == 0.f ? 1.f : 1.f / sum, w0 = e0 * inv, w1 = e1 * inv;
            if (row < it.rows) {
                const float lse = (big + log2f(sum)) * 0.6931471805599453f;
                if (it.slot < 0) p.lse[(size_t)h * p.Lq + it.q0 + row] = lse;
                else p.part_lse[(size_t)h * p.prows + it.slot + row] = lse;
            }
            ok = mbar_wait(bar(O_FULL), n_own & 1, abort_flag, p.wait, CS_OFULL);
            if (both) ok = ok && mbar_wait(bar(O_FULL + 1), n_ml & 1, abort_flag, p.wait, CS_OFULL);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ++n_own;
            n_ml += both;
            tc_fence_after();
            // in the 16 x 256-bit shape of the tensor memory: four lanes write 128 contiguous bytes of a row
            constexpr int CB = D / 64;
            const int l4 = lane >> 2, l2 = lane & 3;
            const uint32_t tO = tmem + 256 + lane_off;
#pragma unroll
            for (int x = 0; x < 2 * CB; ++x) {
                const int cb = x % CB;
                const uint32_t at = ((x / CB) << 20) + cb * 64;
                uint32_t a[32], b[32];
                __syncwarp();
                tmem_ld_16x256b(tO + at, a);
                if (both) tmem_ld_16x256b(tO + 128 + at, b);
                tmem_wait_ld();
                if (x == 2 * CB - 1) {                       // the next item's P V may overwrite both
                    tc_fence_before();
                    mbar_arrive(bar(O_FREE));
                    if (both) mbar_arrive(bar(O_FREE + 1));
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {                // rows 8 j + l4 of the warp's 32
                    const int j = (x / CB) * 2 + y, r = (warp & 3) * 32 + j * 8 + l4;
                    const float u0 = __shfl_sync(0xffffffffu, w0, j * 8 + l4), u1 = __shfl_sync(0xffffffffu, w1, j * 8 + l4);
                    float f[16];
#pragma unroll
                    for (int z = 0; z < 16; ++z) {
                        const int i = 4 * (z >> 1) + 2 * y + (z & 1);
                        f[z] = __uint_as_float(a[i]) * u0;
                        if (both) f[z] = fmaf(__uint_as_float(b[i]), u1, f[z]);
                    }
                    if (it.slot < 0) {
                        uint32_t u[8];
#pragma unroll
                        for (int z = 0; z < 8; ++z) u[z] = bf16x2(f[2 * z], f[2 * z + 1]);
                        quad_transpose(u, l2);
                        if (r < it.rows) store_quad(p.O.row(h, it.q0 + r) + cb * 64, l2, u);
                    } else if (r < it.rows) {
                        float *dst = p.part_o + ((size_t)h * p.prows + it.slot + r) * D + cb * 64 + 2 * l2;
#pragma unroll
                        for (int z = 0; z < 8; ++z) *reinterpret_cast<float2 *>(dst + 8 * z) = make_float2(f[2 * z], f[2 * z + 1]);
                    }
                }
            }
        }
    } else if (warp == 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ query tiles and K
        if (lane == 0) {
            prefetch_tensormap(&tmQ);
            prefetch_tensormap(&tmK);
            int n_k = 0, used[2] = {0, 0}, n = 0;            // key tiles of the item's groups so far
            bool ok = true;
            for (; ok && n < n_items; ++n) {
                const int id = cross_item(n), rank = id / p.H, h = id - rank * p.H, hk = h / p.g, qb = n % 3;
                const CrossItem it = p.items[rank];
                ok = mbar_wait(bar(Q_EMPTY + qb), ((n / 3) & 1) ^ 1, abort_flag, p.wait, CS_QEMPTY);
                if (!ok) break;
                mbar_expect_tx(bar(Q_FULL + qb), TILE_BYTES);
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub)          // (rows behind the item's end are another's, or zeros: nobody looks at their S)
                    tma_load_3d(sQ + qb * TILE_BYTES + sub * SUB_BYTES, &tmQ, sub * 64, it.q0, h, bar(Q_FULL + qb));
                for (int k = 0; k < it.n_keys; k += 128, ++n_k) {
                    const int g = (k >> 7) & 1, valid = min(128, it.n_keys - k), t0 = it.k0 + k, boxes = (valid + 15) >> 4;
                    ok = mbar_wait(bar(K_EMPTY + g), (used[g] & 1) ^ 1, abort_flag, p.wait, CS_KEMPTY);
                    if (!ok) break;
                    ++used[g];
                    mbar_expect_tx(bar(K_FULL + g), boxes * 16 * D * 2);
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) {
                        const uint32_t dst = sK + g * TILE_BYTES + sub * SUB_BYTES;
                        if (valid == 128) tma_load_3d(dst, &tmK, sub * 64, t0, hk, bar(K_FULL + g));
                        else for (int b = 0; b < boxes; ++b) tma_load_3d(dst + b * 2048, &tmK16, sub * 64, t0 + b * 16, hk, bar(K_FULL + g));
                    }
                }
                if (!ok) { ++n; break; }
            }
            if (*abort_flag) {      // copies already issued must land before the shared memory is released
                int dummy_flag = 0;
                for (int g = 0; g < 2; ++g)
                    if (used[g] > 0) mbar_wait(bar(K_FULL + g), (used[g] - 1) & 1, &dummy_flag, p.wait, CS_KFULL);
                for (int b = 1; b <= 3; ++b)
                    if (n - b >= 0) mbar_wait(bar(Q_FULL + (n - b) % 3), ((n - b) / 3) & 1, &dummy_flag, p.wait, CS_QFULL);
            }
        }
    } else if (warp == 11) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ V
        if (lane == 0) prefetch_tensormap(&tmV);
        int used0 = 0, used1 = 0;                            // tiles of either group
        bool ok = true;
        for (int n = 0; ok && n < n_items; ++n) {
            const int id = cross_item(n), rank = id / p.H, hk = (id - rank * p.H) / p.g;
            const CrossItem it = p.items[rank];
            for (int k = 0; k < it.n_keys; k += 128) {
                const int g = (k >> 7) & 1, valid = min(128, it.n_keys - k), t0 = it.k0 + k, whole = valid >> 4;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(V_EMPTY + g), ((g ? used1 : used0) & 1) ^ 1, abort_flag, p.wait, CS_VEMPTY));
                if (!ok) break;
                if (g) ++used1;
                else ++used0;
                const uint32_t tile = sV + g * TILE_BYTES;
                if (lane == 0) {
                    mbar_expect_tx(bar(V_FULL + g), whole * 16 * D * 2);
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) {
                        if (valid == 128) tma_load_3d(tile + sub * SUB_BYTES, &tmV, sub * 64, t0, hk, bar(V_FULL + g));
                        else for (int b = 0; b < whole; ++b) tma_load_3d(tile + sub * SUB_BYTES + b * 2048, &tmV16, sub * 64, t0 + b * 16, hk, bar(V_FULL + g));
                    }
                }
                if (valid & 15) {                            // the box that the segment's end lies in: its rows, and zeros
                    constexpr int CH = D / 8;
#pragma unroll
                    for (int x = 0; x < 16 * CH / 32; ++x) {
                        const int i = x * 32 + lane, r = whole * 16 + i / CH, c16 = i % CH;
                        cp_async16(tile + (c16 >> 3) * SUB_BYTES + sw128_offset(r, c16 & 7), p.V.row(hk, t0 + min(r, valid - 1)) + c16 * 8, r < valid ? 16u : 0u);
                    }
                    cp_async_wait_all();
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (lane == 0) mbar_arrive(bar(V_FULL + g));
            }
        }
        if (*abort_flag) {
            int dummy_flag = 0;
            if (used0 > 0) mbar_wait(bar(V_FULL), (used0 - 1) & 1, &dummy_flag, p.wait, CS_VFULL);
            if (used1 > 0) mbar_wait(bar(V_FULL + 1), (used1 - 1) & 1, &dummy_flag, p.wait, CS_VFULL);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ MMA issuers (the warp stays together, one lane issues): group g's tiles
        const int g = uniform(warp - 9);
        constexpr uint32_t IDESC_PV = idesc_bf16_f32(128, D, 0, 1);
        const uint64_t q_desc0 = smem_desc_sw128(sQ, 16, 1024);
        const uint64_t k_desc = smem_desc_sw128(sK + g * TILE_BYTES, 16, 1024), v_desc = smem_desc_sw128(sV + g * TILE_BYTES, SUB_BYTES, 1024);
        constexpr uint64_t STAGE = TILE_BYTES >> 4;          // next tile, in address-field units
        int qb = 0, n_own = 0, n_tile = 0;                   // Q buffer; items and key tiles of this group
        auto issue_qk = [&](int valid) {
            const uint32_t idesc_qk = idesc_bf16_f32(128, (valid + 15) & ~15, 0, 0);
            const uint64_t qd = q_desc0 + qb * STAGE;
            const uint32_t q_lo = (uint32_t)qd, q_hi = (uint32_t)(qd >> 32), k_lo = (uint32_t)k_desc, k_hi = (uint32_t)(k_desc >> 32);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t o = ((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4;
                mma_ss_elect(tmem + g * 128, q_lo + o, q_hi, k_lo + o, k_hi, idesc_qk, ks > 0);
            }
        };
        auto issue_pv = [&](int ks0, int ks1, bool accumulate) {       // 16 keys a step
            const uint32_t v_lo = (uint32_t)v_desc, v_hi = (uint32_t)(v_desc >> 32), d_o = tmem + 256 + g * 128, a_p = tmem + g * 128;
            for (int ks = ks0; ks < ks1; ++ks) mma_ts_elect(d_o, a_p + ks * 8, v_lo + ks * (2048 >> 4), v_hi, IDESC_PV, accumulate || ks > ks0);
        };
        bool ok = true;
        auto wait = [&](int b, uint32_t parity, int code) {
            return __all_sync(0xffffffffu, mbar_wait_spin(bar(b), parity, abort_flag, p.wait, code)) != 0;
        };
        for (int n = 0; ok && n < n_items; ++n) {
            const int n_keys = uniform(p.items[cross_item(n) / p.H].n_keys);
            qb = n % 3;
            ok = wait(Q_FULL + qb, (n / 3) & 1, CS_QFULL);
            if (!ok) break;
            if (g * 128 >= n_keys) {                         // the other group's tile alone
                if (lane == 0) mbar_arrive(bar(Q_EMPTY + qb));
                continue;
            }
            ok = wait(K_FULL + g, n_tile & 1, CS_KFULL);
            if (!ok) break;
            tc_fence_after();
            issue_qk(min(128, n_keys - g * 128));
            tc_commit_elect(bar(S_FULL + g));
            tc_commit_elect(bar(K_EMPTY + g));
            if (g * 128 + 256 >= n_keys) tc_commit_elect(bar(Q_EMPTY + qb));      // the item's last S of this group
            for (int k = g * 128; ok && k < n_keys; k += 256, ++n_tile) {
                const int valid = min(128, n_keys - k), steps = (valid + 15) >> 4, half = min(steps, 4);
                const bool more = k + 256 < n_keys;
                if (!wait(V_FULL + g, n_tile & 1, CS_VFULL)) { ok = false; break; }
                if (!wait(P_HALF + g, n_tile & 1, CS_PHALF)) { ok = false; break; }
                // the first P V of an item overwrites O: the previous item's has been read
                if (k == g * 128 && n_own > 0 && !wait(O_FREE + g, (n_own - 1) & 1, CS_OFREE)) { ok = false; break; }
                tc_fence_after();
                issue_pv(0, half, k > g * 128);
                if (more && !wait(K_FULL + g, (n_tile + 1) & 1, CS_KFULL)) { ok = false; break; }
                if (!wait(P_FULL + g, n_tile & 1, CS_PFULL)) { ok = false; break; }
                tc_fence_after();
                if (steps > half) issue_pv(half, steps, true);
                if (more) {
                    issue_qk(min(128, n_keys - k - 256));
                    tc_commit_elect(bar(S_FULL + g));
                    tc_commit_elect(bar(V_EMPTY + g));
                    tc_commit_elect(bar(K_EMPTY + g));
                    if (k + 512 >= n_keys) tc_commit_elect(bar(Q_EMPTY + qb));
                } else {
                    tc_commit_elect(bar(V_EMPTY + g));
                    tc_commit_elect(bar(O_FULL + g));
                }
            }
            ++n_own;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
    if (threadIdx.x == 0) report_abort(p.status, s_abort);
}

// always the d = 128 footprint: more than half an SM's shared memory, so that CTAs, which each take all of the tensor memory, never share one
constexpr size_t kSmem = 7 * (size_t)128 * 128 * 2 + 1024;

int prepare_cross_solo(moc_cross *c) {
    const void *kernel = c->d == 128 ? (const void *)cross_solo_tc_kernel<128> : (const void *)cross_solo_tc_kernel<64>;
    MOC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));
    return MOC_OK;
}

template <int D>
static int cross_solo_d(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws,
                        bool first, cudaStream_t s) {
    CUtensorMap tmQ, tmK, tmV, tmK16, tmV16;
    if (int r = make_tmap_rows_bf16(&tmQ, Q, c->H, c->Lq, D, 128)) return r;
    if (int r = make_tmap_rows_bf16(&tmK, K, c->Hkv, c->Lk, D, 128)) return r;
    if (int r = make_tmap_rows_bf16(&tmV, V, c->Hkv, c->Lk, D, 128)) return r;
    if (int r = make_tmap_rows_bf16(&tmK16, K, c->Hkv, c->Lk, D, 16)) return r;
    if (int r = make_tmap_rows_bf16(&tmV16, V, c->Hkv, c->Lk, D, 16)) return r;
    CrossSoloParams a;
    a.items = c->d_solo; a.n_all = (int)c->solo.size() * c->H;
    a.H = c->H; a.g = c->g; a.Lq = c->Lq; a.prows = c->prows;
    a.V = CrossRows(V); a.O = CrossRows(O); a.lse = lse;
    a.part_o = ws_ptr<float>(ws, c->ws.part_o); a.part_lse = ws_ptr<float>(ws, c->ws.part_lse);
    a.status = ws_ptr<int>(ws, c->ws.status); a.first = first;
    a.scale_log2 = c->scale * 1.4426950408889634f;
    a.wait = WaitBound::of(0);
    cross_solo_tc_kernel<D><<<cross_grid(c, c->solo.size()), kCrossSoloThreads, kSmem, s>>>(tmQ, tmK, tmV, tmK16, tmV16, a);
    MOC_LAUNCH_CHECK();
    return MOC_OK;
}

int launch_cross_solo(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws,
                      bool first, cudaStream_t s) {
    return c->d == 128 ? cross_solo_d<128>(c, Q, K, V, O, lse, ws, first, s) : cross_solo_d<64>(c, Q, K, V, O, lse, ws, first, s);
}

}  // namespace moc
