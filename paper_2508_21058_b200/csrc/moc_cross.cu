// Cross attention to encoder states of another length (moc_cross_attend, moc_cross_attend_bwd): the plan, the entry points and the small
// kernels that put shares together.  The attention itself: moc_cross_fwd_tc.cu, moc_cross_solo_tc.cu (one query tile), moc_cross_few.cu (few queries), moc_cross_dq_tc.cu, moc_cross_dkv_tc.cu.
#include <string.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "moc_cross.cuh"
#include "moc_tc.cuh"

namespace moc {

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Rows, items of all heads, rows of partial results and pieces are counted in 32 bits, some to spare for a tile's last row and a round of items.
constexpr int64_t kMostCount = (1ll << 31) - 1024;

static int check_cross(const moc_cross_problem *pr) {
    if (pr->n_heads < 1 || pr->n_heads > 65535 || pr->n_kv_heads < 1 || pr->n_heads % pr->n_kv_heads != 0) return MOC_ERR_SHAPE;
    if (pr->head_dim != 64 && pr->head_dim != 128) return MOC_ERR_SHAPE;
    if (pr->n_segments < 0 || !std::isfinite(pr->softmax_scale) || pr->softmax_scale < 0.f) return MOC_ERR_SHAPE;
    if (!pr->q_off || !pr->k_off) return MOC_ERR_NULL;
    if (pr->q_off[0] != 0 || pr->k_off[0] != 0) return MOC_ERR_CHUNK_TABLE;
    for (int s = 0; s < pr->n_segments; ++s) {
        if (pr->q_off[s + 1] < pr->q_off[s] || pr->k_off[s + 1] < pr->k_off[s]) return MOC_ERR_CHUNK_TABLE;
        if (pr->k_len && (pr->k_len[s] < 0 || pr->k_len[s] > pr->k_off[s + 1] - pr->k_off[s])) return MOC_ERR_CHUNK_TABLE;
    }
    const int64_t Lq = pr->q_off[pr->n_segments], Lk = pr->k_off[pr->n_segments];
    if (Lq * pr->n_heads >= kMostCount || Lk * pr->n_kv_heads >= kMostCount) return MOC_ERR_SHAPE;
    return MOC_OK;
}

// Shares of the keys.  With many items of like lengths the longest-first walk balances the CTAs by itself; with few, or with some far longer
// than the others, an item is cut into shares of `c` key tiles, whose results another launch puts together.  c is the one with the
// least estimated time `t`, in key tiles of two-tile items (3450 cycles): the slowest CTA's walk, where an item costs 0.8 beside its
// tiles (2800: its first loads and its results) and a key tile of a single query tile `single`, plus `join` for the second launch.
// (61 segments of 200 queries, 24 heads of 128, one of them with 32,760 states, the others with 77: forward 151 us and backward 544; with
// that one's items whole, 24 CTAs on them and the others done, 476 and 710.  All of 512 states, 33k queries: 202 and 650, uncut by either rule.)
// The costs were measured at d = 128 and are taken for d = 64 too: (12 heads of 64, 40 segments of 700 queries, 38 with 100 states and two
// with 30,000 and 20,000: forward 377 -> 215 us, backward 672 -> 683.)
// (No share has more than 16384 key tiles, some 50 ms: a bounded wait lasts a second.)
constexpr int kMostTiles = 16384;
struct Shares { int c; double t; };
static Shares share_tiles(const std::vector<CrossItem> &items, int H, int n_sm, double single, double join) {
    int longest = 1;
    double total = 0;
    for (const CrossItem &i : items) {
        const int nt = (i.n_keys + 127) / 128;
        longest = std::max(longest, nt);
        if (nt > 0) total += 0.8 + (i.rows > 128 ? 1.0 : single) * nt;
    }
    const double mean = total * H / n_sm;
    std::vector<double> cost;
    const bool many = items.size() * (size_t)H >= 4 * (size_t)n_sm;
    // the slowest walk with shares of c tiles, as they are dealt out (cross_item)
    auto walk = [&](int c) {
        cost.clear();
        for (const CrossItem &i : items) {
            const int nt = (i.n_keys + 127) / 128, n = std::max(1, (nt + c - 1) / c);
            for (int x = 0; x < n && nt > 0; ++x) cost.push_back(0.8 + (i.rows > 128 ? 1.0 : single) * ((int)((int64_t)nt * (x + 1) / n) - (int)((int64_t)nt * x / n)));
        }
        std::sort(cost.begin(), cost.end(), [](double a, double b) { return a > b; });
        const int64_t n_all = (int64_t)cost.size() * H;
        double t = 0;
        for (int b = 0; b < n_sm; ++b) {
            double mine = 0;
            for (int64_t at = 0, odd = 0; at < n_all; at += n_sm, odd ^= 1) {
                const int64_t id = at + (odd ? n_sm - 1 - b : b);
                if (id < n_all) mine += cost[id / H];
            }
            t = std::max(t, mine);
        }
        return t;
    };
    if (many && walk(longest) <= 1.2 * mean + join) return Shares{std::min(longest, kMostTiles), mean};
    Shares best{longest, 1e300};
    // (an item alone may be the whole mean of n_sm CTAs; of many items, each p takes a while)
    for (int p = 1; p <= std::min(longest, 2 * n_sm); p += many ? 1 + p / 4 : 1) {
        const int c = (longest + p - 1) / p;
        const double t = walk(c) + (c < longest ? join : 0.0);
        if (t < best.t) best = Shares{c, t};
        // shorter shares only cost more, unless it is a few long items that they are cut from
        if (cost.size() * (size_t)H > 4 * (size_t)n_sm && cost[0] <= 0.5 * mean) break;
    }
    best.c = std::min(best.c, kMostTiles);
    return best;
}

// cuts the items into shares of at most c key tiles; the longest items first.  false: there are more than can be counted
static bool cut_items(std::vector<CrossItem> &items, std::vector<CrossMerge> &merges, int &prows, int c, int H) {
    int64_t shares = 0, rows = prows;
    for (const CrossItem &i : items) {
        const int nt = (i.n_keys + 127) / 128, n = std::max(1, (nt + c - 1) / c);
        shares += n;
        if (n > 1) rows += (int64_t)n * i.rows;
    }
    if (shares * H >= kMostCount || rows >= kMostCount) return false;
    std::vector<CrossItem> out;
    for (const CrossItem &i : items) {
        const int nt = (i.n_keys + 127) / 128, n = std::max(1, (nt + c - 1) / c);
        if (n == 1) { out.push_back(i); continue; }
        merges.push_back(CrossMerge{i.q0, i.rows, prows, n});
        for (int x = 0; x < n; ++x) {
            const int t0 = (int)((int64_t)nt * x / n), t1 = (int)((int64_t)nt * (x + 1) / n);
            CrossItem p = i;
            p.k0 = i.k0 + t0 * 128;
            p.n_keys = std::min(i.n_keys, t1 * 128) - t0 * 128;
            p.slot = prows;
            prows += i.rows;
            out.push_back(p);
        }
    }
    std::stable_sort(out.begin(), out.end(), [](const CrossItem &a, const CrossItem &b) { return (a.n_keys + 127) / 128 > (b.n_keys + 127) / 128; });
    items.swap(out);
    return true;
}

static int derive_cross(moc_cross *c, const moc_cross_problem *pr) {
    const int S = pr->n_segments;
    c->H = pr->n_heads; c->Hkv = pr->n_kv_heads; c->g = pr->n_heads / pr->n_kv_heads; c->d = pr->head_dim;
    c->Lq = pr->q_off[S]; c->Lk = pr->k_off[S];
    c->scale = pr->softmax_scale != 0.f ? pr->softmax_scale : 1.f / std::sqrt((float)c->d);
    auto keys = [&](int s) { return pr->k_len ? pr->k_len[s] : pr->k_off[s + 1] - pr->k_off[s]; };
    auto is_few = [&](int s) {
        const int n = pr->q_off[s + 1] - pr->q_off[s];
        return n > 0 && (int64_t)n * c->g <= kFewRows && keys(s) > 0;
    };
    // Few queries: shares of the states, of 128 at least.  Three blocks are resident on an SM.  Either no more shares than that, all under
    // way at once, the launch as long as the longest; or four for every SM, the longest first, the launch about the mean and one
    // more share long.  (1 head, 1M states: 108 us and 136; 64 sequences of 375 to 1500, 24 heads on 8, which no single wave
    // takes in equal parts: 65 and 56; six and eight for every SM 58 and 63.)
    int64_t few_work = 0, few_longest = 0;
    auto few_blocks = [&](int s) { return ((pr->q_off[s + 1] - pr->q_off[s]) * c->g + 3) / 4; };
    for (int s = 0; s < S; ++s)
        if (is_few(s)) {
            few_work += (int64_t)keys(s) * c->Hkv * few_blocks(s);
            few_longest = std::max<int64_t>(few_longest, keys(s));
        }
    const int64_t slots = 3 * (int64_t)c->n_sm, mean = few_work / slots;
    auto round_share = [](int64_t n) { return std::max<int64_t>(128, (n + 31) / 32 * 32); };
    int64_t few_share = round_share(few_work / (4 * (int64_t)c->n_sm));
    for (int64_t one = round_share(mean); few_work > 0 && one < 2 * few_longest + 128 && one <= mean + few_share; one = round_share(one + one / 16 + 1)) {
        int64_t n = 0;
        for (int s = 0; s < S; ++s)
            if (is_few(s)) n += (keys(s) + one - 1) / one * c->Hkv * few_blocks(s);
        if (n <= slots) { few_share = one; break; }
    }
    for (int s = 0; s < S; ++s) {
        if (!is_few(s)) continue;
        const int q_len = pr->q_off[s + 1] - pr->q_off[s], rows = q_len * c->g, blocks = (rows + 3) / 4, nk = keys(s);
        const int n = (int)((nk + few_share - 1) / few_share);
        if (((int64_t)c->few.size() + (int64_t)n * blocks) * c->Hkv >= kMostCount || c->prows + (int64_t)n * q_len >= kMostCount) return MOC_ERR_SHAPE;
        for (int x = 0; x < n; ++x) {
            const int k0 = (int)((int64_t)nk * x / n), k1 = (int)((int64_t)nk * (x + 1) / n);
            for (int b = 0; b < blocks; ++b) {
                const int r0 = rows * b / blocks, r1 = rows * (b + 1) / blocks;
                c->few.push_back(CrossFew{pr->q_off[s], q_len, pr->k_off[s] + k0, k1 - k0, n > 1 ? c->prows + x * q_len : -1, r0, r1 - r0, 0});
                c->few_rows = std::max(c->few_rows, r1 - r0);
            }
        }
        if (n > 1) {
            c->merges.push_back(CrossMerge{pr->q_off[s], q_len, c->prows, n});
            c->prows += n * q_len;
        }
    }
    std::stable_sort(c->few.begin(), c->few.end(), [](const CrossFew &a, const CrossFew &b) { return a.n_keys > b.n_keys; });
    // The forward's items: 256 rows, or a segment's last ones.  A key tile takes 3450 cycles for two query tiles; for a single one 4200 in
    // the same kernel, 2100 in the one that has both softmax groups on one tile, which is a launch of its own.  So: all in the first
    // kernel, or the single tiles in the second, or everything in tiles of 128 in the second, whichever is estimated shortest.
    // (257 queries, 32k states, 24 heads: 188, 178 and 169 us; 576 queries, 77 states, 4 heads: 8.5 the first, 8.5 the last.)
    std::vector<CrossItem> two, one, half, none;
    for (int s = 0; s < S; ++s) {
        for (int q = pr->q_off[s]; !is_few(s) && q < pr->q_off[s + 1]; q += kCrossRows) {
            const CrossItem i{q, std::min(kCrossRows, pr->q_off[s + 1] - q), pr->k_off[s], keys(s), -1, {}};
            (i.n_keys == 0 ? none : i.rows <= 128 ? one : two).push_back(i);
        }
        for (int q = pr->q_off[s]; q < pr->q_off[s + 1]; q += 128) {
            const CrossItem i{q, std::min(128, pr->q_off[s + 1] - q), pr->k_off[s], keys(s), -1, {}};
            c->dq_items.push_back(i);
            if (i.n_keys > 0 && !is_few(s)) half.push_back(i);
        }
    }
    std::vector<CrossItem> both = two;
    both.insert(both.end(), one.begin(), one.end());
    const double alone = 4200.0 / 3450.0, solo = 2100.0 / 3450.0, join = 3.5, launch = 1.5;
    const Shares together = share_tiles(both, c->H, c->n_sm, alone, join), halves = share_tiles(half, c->H, c->n_sm, solo, join),
                 pairs = share_tiles(two, c->H, c->n_sm, alone, join), singles = share_tiles(one, c->H, c->n_sm, solo, 0.5);
    // (two launches, and K and V do not stay in L2 between them: 168 us and a merge of 10, where one launch of all tiles takes 162 and 7)
    int64_t states = 0;
    for (int s = 0; s < S; ++s) states += keys(s);
    const bool in_l2 = states * c->Hkv * c->d * 4 <= (96ll << 20);
    const double apart = two.empty() || one.empty() || !in_l2 ? 1e300 : pairs.t + singles.t + launch;
    Shares cut = together;
    if (halves.t < std::min(together.t, apart)) {
        c->solo.swap(half);
        if (!cut_items(c->solo, c->merges, c->prows, halves.c, c->H)) return MOC_ERR_SHAPE;
    } else if (apart < together.t) {
        c->items.swap(two);
        c->solo.swap(one);
        if (!cut_items(c->solo, c->merges, c->prows, singles.c, c->H)) return MOC_ERR_SHAPE;
        cut = pairs;
    } else {
        c->items.swap(both);
    }
    c->items.insert(c->items.end(), none.begin(), none.end());
    if (!cut_items(c->items, c->merges, c->prows, cut.c, c->H)) return MOC_ERR_SHAPE;
    // The second tile's warps wait through a CTA's items of one tile for the next of two, and no longer than two seconds.  Where there are more
    // than some 0.6 of that (4200 cycles a key tile, at 1.3 GHz), the items of two come first.
    int64_t ones = 0;
    for (const CrossItem &i : c->items) ones += i.rows <= 128 ? (i.n_keys + 127) / 128 : 0;
    if (ones * c->H / c->n_sm > 200000) std::stable_partition(c->items.begin(), c->items.end(), [](const CrossItem &i) { return i.rows > 128; });
    if (!cut_items(c->dq_items, c->dq_merges, c->dq_prows, share_tiles(c->dq_items, c->H, c->n_sm, 1.0, 3.0).c, c->H)) return MOC_ERR_SHAPE;
    for (const CrossMerge &m : c->merges) {
        c->most_merge_rows = std::max(c->most_merge_rows, m.rows);
        c->most_merge_n = std::max(c->most_merge_n, m.n);
    }
    for (const CrossItem &i : c->dq_items) c->n_dq_work += i.n_keys > 0;

    // Key-stationary pass.  The query tiles of a (key head, segment) are cut into parts of about the same length, and every key tile of
    // the segment against one part is a piece; a key tile with several parts is a sum of slots.  Pieces of the same part follow one another, so
    // that CTAs that run side by side stream the same queries, out of L2 (stretches of all pairs in a row, each CTA at another place
    // of the stream: 33k queries, 512 states, 24 heads 340 us and 1.6 GB from DRAM; so 331 us and 0.42 GB).
    struct Group { int h, s; int64_t units; int n; };                // pairs of a key tile; pieces of a part
    std::vector<Group> groups;
    int64_t longest = 0;
    for (int h = 0; h < c->Hkv; ++h)
        for (int s = 0; s < S; ++s) {
            const int64_t units = (int64_t)c->g * ((pr->q_off[s + 1] - pr->q_off[s] + 127) / 128);
            const int nk = units == 0 ? 0 : keys(s);                 // states that somebody reads
            if (nk > 0) groups.push_back(Group{h, s, units, (nk + 127) / 128});
            if (nk > 0) longest = std::max(longest, units);
            for (int k = pr->k_off[s] + nk; k < pr->k_off[s + 1]; k += 128)
                c->sums.push_back(CrossSum{h, k, std::min(128, pr->k_off[s + 1] - k), 0, 0, {}});
        }
    std::stable_sort(groups.begin(), groups.end(), [](const Group &a, const Group &b) { return a.units > b.units; });
    // The length of a part with the least estimated time: rounds of n_sm pieces, each as long as its first, where a piece costs two pairs
    // beside its own (its key tile, its results, the launch that adds them up).
    int64_t part = std::max<int64_t>(longest, 1);
    double best = 1e300;
    for (int64_t n = 1; n <= std::min<int64_t>(longest, 256); ++n) {
        const int64_t len = (longest + n - 1) / n;
        double t = 0;
        int64_t at = 0;                                              // pieces so far
        for (const Group &g : groups) {
            const int64_t parts = (g.units + len - 1) / len, end = at + parts * g.n;
            // rounds that begin in this group
            t += (double)((end + c->n_sm - 1) / c->n_sm - (at + c->n_sm - 1) / c->n_sm) * (2.0 + (double)g.units / parts);
            at = end;
        }
        if (t < best) { best = t; part = len; }
        if (at > 64ll * c->n_sm) break;                              // (shorter parts only cost more)
    }
    part = std::min<int64_t>(part, 1 << 16);                         // (a bounded wait lasts a second, as long as 500000 pairs)
    int64_t n_pieces = 0;
    for (const Group &g : groups) n_pieces += (g.units + part - 1) / part * g.n;
    if (n_pieces >= kMostCount) return MOC_ERR_SHAPE;
    std::vector<CrossPiece> all;
    for (const Group &g : groups) {
        const int64_t parts = (g.units + part - 1) / part;
        const int s = g.s, slot0 = c->kv_slots;
        for (int64_t x = 0; x < parts; ++x)
            for (int kt = 0; kt < g.n; ++kt) {
                const int k0 = pr->k_off[s] + kt * 128, rows = std::min(128, keys(s) - kt * 128);
                all.push_back(CrossPiece{g.h, k0, rows, pr->q_off[s], pr->q_off[s + 1], (int)(g.units * x / parts), (int)(g.units * (x + 1) / parts),
                                         parts > 1 ? slot0 + (int)(kt * parts + x) : -1});
                if (x == 0 && parts > 1) c->sums.push_back(CrossSum{g.h, k0, rows, slot0 + (int)(kt * parts), (int)parts, {}});
            }
        if (parts > 1) c->kv_slots += (int)(parts * g.n);
    }
    // dealt to the CTAs in turn, every other round in reverse
    const int64_t n_cta = std::min<int64_t>(c->n_sm, (int64_t)all.size());
    c->piece_off.push_back(0);
    for (int64_t b = 0; b < n_cta; ++b) {
        for (int64_t r = 0; r * n_cta < (int64_t)all.size(); ++r) {
            const int64_t i = r * n_cta + ((r & 1) ? n_cta - 1 - b : b);
            if (i < (int64_t)all.size()) c->pieces.push_back(all[i]);
        }
        c->piece_off.push_back((int)c->pieces.size());
    }
    CrossLayout &w = c->ws;
    const size_t H = c->H, d = c->d;
    w.status = 0;
    w.part_o = 256;
    w.part_lse = up256(w.part_o + 4 * H * c->prows * d);
    w.fwd_end = up256(w.part_lse + 4 * H * c->prows);
    w.delta = w.fwd_end;
    w.part_dq = up256(w.delta + 4 * H * c->Lq);
    w.part_kv = up256(w.part_dq + 4 * H * c->dq_prows * d);
    w.bwd_end = up256(w.part_kv + 4 * 2 * (size_t)c->kv_slots * 128 * d);
    return MOC_OK;
}

// The launches that put shares together begin while the one before them still runs, and wait for its results.
template <typename... P, typename... A>
static cudaError_t launch_after(void (*kernel)(P...), dim3 grid, cudaStream_t s, A &&...args) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = grid; c.blockDim = dim3(256); c.stream = s;
    c.attrs = &at; c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, std::forward<A>(args)...);
}

// ---- shares of the forward: O = sum_i w_i O_i / sum_i w_i, w_i = exp(lse_i - max lse), four shares' loads under way.  A warp has a row, or,
// WIDE, the eight warps of a block have one and every eighth share each.
template <int D, bool WIDE>
__global__ void __launch_bounds__(256) cross_merge_kernel(const CrossMerge *merges, const float *part_o, const float *part_lse, int prows,
                                                          CrossRows O, float *lse, int Lq) {
    constexpr int V = D / 32, W = WIDE ? 8 : 1;                // channels of a lane, warps of a row
    __shared__ float s_o[WIDE ? 8 : 1][D], s_sum[8];
    const CrossMerge m = merges[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, row = WIDE ? blockIdx.z : blockIdx.z * 8 + warp;
    previous_done();
    if (row >= m.rows) return;                                 // (WIDE: the whole block)
    const size_t at = (size_t)h * prows + m.slot + row;
    float big = kLowest;
    for (int i = lane; i < m.n; i += 32) big = fmaxf(big, part_lse[at + (size_t)i * m.rows]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    float acc[V] = {}, sum = 0.f;
    for (int i = WIDE ? warp : 0; i < m.n; i += 4 * W) {
        float2 v[4][V / 2];
        float w[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const size_t src = at + (size_t)min(i + x * W, m.n - 1) * m.rows;
            w[x] = part_lse[src];
#pragma unroll
            for (int y = 0; y < V / 2; ++y) v[x][y] = *reinterpret_cast<const float2 *>(part_o + src * D + lane * V + 2 * y);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (i + x * W >= m.n) break;
            const float e = __expf(w[x] - big);
            sum += e;
#pragma unroll
            for (int y = 0; y < V / 2; ++y) {
                acc[2 * y] = fmaf(e, v[x][y].x, acc[2 * y]);
                acc[2 * y + 1] = fmaf(e, v[x][y].y, acc[2 * y + 1]);
            }
        }
    }
    if constexpr (WIDE) {                                      // in the order of the warps
        if (lane == 0) s_sum[warp] = sum;
#pragma unroll
        for (int y = 0; y < V; ++y) s_o[warp][lane * V + y] = acc[y];
        __syncthreads();
        if (warp > 0) return;
        sum = 0.f;
#pragma unroll
        for (int y = 0; y < V; ++y) acc[y] = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            sum += s_sum[x];
#pragma unroll
            for (int y = 0; y < V; ++y) acc[y] += s_o[x][lane * V + y];
        }
    }
    const float inv = 1.f / sum;
    uint32_t *dst = reinterpret_cast<uint32_t *>(O.row(h, m.q0 + row) + lane * V);
#pragma unroll
    for (int x = 0; x < V; x += 2) dst[x / 2] = tc::bf16x2(acc[x] * inv, acc[x + 1] * inv);
    if (lane == 0) lse[(size_t)h * Lq + m.q0 + row] = big + __logf(sum);
}

// ---- shares of a gradient: out = sum of the slots, in their order; 16 bytes a lane, so a warp has one row at d = 128, two at 64
template <int D>
__device__ __forceinline__ void sum_row(const float *src, size_t stride, int n, __nv_bfloat16 *dst) {
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < n; i += 4) {
        float4 v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = i + x < n ? *reinterpret_cast<const float4 *>(src + (i + x) * stride) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < 4; ++x) { acc.x += v[x].x; acc.y += v[x].y; acc.z += v[x].z; acc.w += v[x].w; }
    }
    *reinterpret_cast<uint2 *>(dst) = make_uint2(tc::bf16x2(acc.x, acc.y), tc::bf16x2(acc.z, acc.w));
}
template <int D>
__global__ void __launch_bounds__(256) cross_sum_dq_kernel(const CrossMerge *merges, const float *part, int prows, CrossRows dQ) {
    const CrossMerge m = merges[blockIdx.x];
    const int h = blockIdx.y, at = (blockIdx.z * 256 + threadIdx.x) * 4, row = at / D, col = at % D;
    next_may_start();
    previous_done();
    if (row < m.rows)
        sum_row<D>(part + ((size_t)h * prows + m.slot + row) * D + col, (size_t)m.rows * D, m.n, dQ.row(h, m.q0 + row) + col);
}
template <int D>
__global__ void __launch_bounds__(256) cross_sum_kv_kernel(const CrossSum *sums, const float *part, CrossRows dK, CrossRows dV) {
    const CrossSum m = sums[blockIdx.x];
    const int side = blockIdx.y, at = (blockIdx.z * 256 + threadIdx.x) * 4, row = at / D, col = at % D;
    previous_done();
    if (row < m.rows)
        sum_row<D>(part + (((size_t)m.slot * 2 + side) * 128 + row) * D + col, (size_t)2 * 128 * D, m.n, (side ? dV : dK).row(m.h, m.k0 + row) + col);
}

static int enter_cross(const moc_cross *c) {
    if (!c) return MOC_ERR_NULL;
    int dev = -1;
    MOC_CUDA_TRY(cudaGetDevice(&dev));
    return dev == c->device ? MOC_OK : MOC_ERR_ARCH;
}
static int check_ws(const void *ws) { return !ws ? MOC_ERR_WORKSPACE : aligned(ws, 256) ? MOC_OK : MOC_ERR_ALIGN; }

}  // namespace moc

using namespace moc;

extern "C" int moc_cross_create(const moc_cross_problem *pr, moc_cross **out) {
    if (!pr || !out) return MOC_ERR_NULL;
    if (int r = check_cross(pr)) return r;
    int dev = -1, cc = 0, n_sm = 0;
    MOC_CUDA_TRY(cudaGetDevice(&dev));
    MOC_CUDA_TRY(cudaDeviceGetAttribute(&cc, cudaDevAttrComputeCapabilityMajor, dev));
    MOC_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
    if (cc != 10) return MOC_ERR_ARCH;
    moc_cross *c = new (std::nothrow) moc_cross();
    if (!c) return MOC_ERR_CUDA;
    c->device = dev;
    c->n_sm = n_sm;
    try {                                                       // (the tables' memory)
        if (int r = derive_cross(c, pr)) {
            delete c;
            return r;
        }
        size_t o = 0;
        auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
        const size_t a = take(sizeof(CrossItem) * c->items.size()), b = take(sizeof(CrossItem) * c->dq_items.size()),
                     m = take(sizeof(CrossMerge) * c->merges.size()), dm = take(sizeof(CrossMerge) * c->dq_merges.size()),
                     fe = take(sizeof(CrossFew) * c->few.size()), so = take(sizeof(CrossItem) * c->solo.size()),
                     p = take(sizeof(CrossPiece) * c->pieces.size()), po = take(4 * c->piece_off.size()),
                     su = take(sizeof(CrossSum) * c->sums.size());
        std::vector<char> host(o);
        auto up = [&](size_t at, const void *src, size_t bytes) { if (bytes) memcpy(host.data() + at, src, bytes); };
        up(a, c->items.data(), sizeof(CrossItem) * c->items.size());
        up(b, c->dq_items.data(), sizeof(CrossItem) * c->dq_items.size());
        up(so, c->solo.data(), sizeof(CrossItem) * c->solo.size());
        up(fe, c->few.data(), sizeof(CrossFew) * c->few.size());
        up(m, c->merges.data(), sizeof(CrossMerge) * c->merges.size());
        up(dm, c->dq_merges.data(), sizeof(CrossMerge) * c->dq_merges.size());
        up(p, c->pieces.data(), sizeof(CrossPiece) * c->pieces.size());
        up(po, c->piece_off.data(), 4 * c->piece_off.size());
        up(su, c->sums.data(), sizeof(CrossSum) * c->sums.size());
        cudaError_t e = cudaMalloc(&c->d_blob, o);
        if (e == cudaSuccess) {
            // on a stream of its own: on the legacy stream the copy would wait for what the caller has under way there
            cudaStream_t st = nullptr;
            e = table_stream(&st);
            if (e == cudaSuccess) e = cudaMemcpyAsync(c->d_blob, host.data(), o, cudaMemcpyHostToDevice, st);
            if (e == cudaSuccess) e = cudaStreamSynchronize(st);
        }
        if (e != cudaSuccess) {
            set_cuda_error(e, "cross attention tables");
            if (c->d_blob) cudaFree(c->d_blob);
            delete c;
            return MOC_ERR_CUDA;
        }
        int r = MOC_OK;
        for (auto prepare : {prepare_cross_fwd, prepare_cross_solo, prepare_cross_few, prepare_cross_dq, prepare_cross_dkv})
            if (!r) r = prepare(c);
        if (r) {
            cudaFree(c->d_blob);
            delete c;
            return r;
        }
        char *d = static_cast<char *>(c->d_blob);
        c->d_items = (CrossItem *)(d + a); c->d_dq_items = (CrossItem *)(d + b); c->d_few = (CrossFew *)(d + fe); c->d_solo = (CrossItem *)(d + so);
        c->d_merges = (CrossMerge *)(d + m); c->d_dq_merges = (CrossMerge *)(d + dm);
        c->d_pieces = (CrossPiece *)(d + p); c->d_piece_off = (int32_t *)(d + po); c->d_sums = (CrossSum *)(d + su);
    } catch (...) {
        delete c;
        return MOC_ERR_CUDA;
    }
    *out = c;
    return MOC_OK;
}

extern "C" int moc_cross_destroy(moc_cross *c) {
    if (!c) return MOC_ERR_NULL;
    if (c->d_blob) cudaFree(c->d_blob);
    delete c;
    return MOC_OK;
}

extern "C" int moc_cross_workspace_bytes(const moc_cross *c, int with_bwd, size_t *bytes) {
    if (!c || !bytes) return MOC_ERR_NULL;
    *bytes = with_bwd ? c->ws.bwd_end : c->ws.fwd_end;
    return MOC_OK;
}

extern "C" int moc_cross_attend(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse,
                                void *ws, void *stream) {
    moc::NvtxRange nvtx_range("moc_cross_attend");
    if (int r = enter_cross(c)) return r;
    for (const moc_rows *t : {Q, O}) if (int r = check_rows(t, c->H, c->Lq, c->d, 2)) return r;
    for (const moc_rows *t : {K, V}) if (int r = check_rows(t, c->Hkv, c->Lk, c->d, 2)) return r;
    if (c->Lq > 0 && !lse) return MOC_ERR_NULL;
    if (!aligned(lse, 4)) return MOC_ERR_ALIGN;
    if (int r = check_ws(ws)) return r;
    cudaStream_t s = (cudaStream_t)stream;
    if (c->Lq == 0) {
        MOC_CUDA_TRY(cudaMemsetAsync(ws_ptr<int>(ws, c->ws.status), 0, 8, s));
        return MOC_OK;
    }
    // (the first of them clears the status)
    if (!c->few.empty())
        if (int r = launch_cross_few(c, Q, K, V, O, lse, ws, s)) return r;
    if (!c->solo.empty())
        if (int r = launch_cross_solo(c, Q, K, V, O, lse, ws, c->few.empty(), s)) return r;
    if (!c->items.empty())
        if (int r = launch_cross_fwd(c, Q, K, V, O, lse, ws, c->few.empty() && c->solo.empty(), s)) return r;
    if (!c->merges.empty()) {
        const bool wide = c->most_merge_n > 16;
        const dim3 grid((unsigned)c->merges.size(), c->H, wide ? c->most_merge_rows : (c->most_merge_rows + 7) / 8);
        const float *po = ws_ptr<float>(ws, c->ws.part_o), *pl = ws_ptr<float>(ws, c->ws.part_lse);
        auto kernel = c->d == 128 ? (wide ? cross_merge_kernel<128, true> : cross_merge_kernel<128, false>)
                                  : (wide ? cross_merge_kernel<64, true> : cross_merge_kernel<64, false>);
        MOC_CUDA_TRY(launch_after(kernel, grid, s, (const CrossMerge *)c->d_merges, po, pl, c->prows, CrossRows(O), lse, c->Lq));
        MOC_LAUNCH_CHECK();
    }
    return MOC_OK;
}

extern "C" int moc_cross_attend_bwd(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O,
                                    const float *lse, const moc_rows *dO, const moc_rows *dQ, const moc_rows *dK, const moc_rows *dV, void *ws,
                                    void *stream) {
    moc::NvtxRange nvtx_range("moc_cross_attend_bwd");
    if (int r = enter_cross(c)) return r;
    for (const moc_rows *t : {Q, O, dO, dQ}) if (int r = check_rows(t, c->H, c->Lq, c->d, 2)) return r;
    for (const moc_rows *t : {K, V, dK, dV}) if (int r = check_rows(t, c->Hkv, c->Lk, c->d, 2)) return r;
    if (c->Lq > 0 && !lse) return MOC_ERR_NULL;
    if (!aligned(lse, 4)) return MOC_ERR_ALIGN;
    if (int r = check_ws(ws)) return r;
    cudaStream_t s = (cudaStream_t)stream;
    if (c->Lq > 0) {
        if (int r = launch_cross_dq(c, Q, K, V, O, lse, dO, dQ, ws, s)) return r;
        // (each of the launches that follow waits for the one before it)
        if (!c->dq_merges.empty()) {
            const dim3 g2((unsigned)c->dq_merges.size(), c->H, c->d / 8);      // 1024 values a block
            const float *part = ws_ptr<float>(ws, c->ws.part_dq);
            MOC_CUDA_TRY(launch_after(c->d == 128 ? cross_sum_dq_kernel<128> : cross_sum_dq_kernel<64>, g2, s, (const CrossMerge *)c->d_dq_merges, part,
                                      c->dq_prows, CrossRows(dQ)));
            MOC_LAUNCH_CHECK();
        }
        if (!c->pieces.empty())
            if (int r = launch_cross_dkv(c, Q, K, V, lse, dO, dK, dV, ws, s)) return r;
    } else {
        MOC_CUDA_TRY(cudaMemsetAsync(ws_ptr<int>(ws, c->ws.status), 0, 8, s));
    }
    if (!c->sums.empty()) {
        const dim3 g3((unsigned)c->sums.size(), 2, c->d / 8);
        const float *part = ws_ptr<float>(ws, c->ws.part_kv);
        MOC_CUDA_TRY(launch_after(c->d == 128 ? cross_sum_kv_kernel<128> : cross_sum_kv_kernel<64>, g3, s, (const CrossSum *)c->d_sums, part, CrossRows(dK),
                                  CrossRows(dV)));
        MOC_LAUNCH_CHECK();
    }
    return MOC_OK;
}

// The key tiles that the CTAs of a launch walk, of the sorted items of every head: the most that one has, and the mean.
static void walks(const std::vector<CrossItem> &items, int H, int n_sm, int64_t *out) {
    const int64_t n_all = (int64_t)items.size() * H, n_cta = std::min<int64_t>(n_all, n_sm);
    out[0] = out[1] = 0;
    for (int64_t b = 0; b < n_cta; ++b) {
        int64_t tiles = 0;
        for (int64_t n = 0; n * n_cta < n_all; ++n) {
            const int64_t id = n * n_cta + ((n & 1) ? n_cta - 1 - b : b);
            if (id < n_all) tiles += (items[id / H].n_keys + 127) / 128;
        }
        out[0] = std::max(out[0], tiles);
        out[1] += tiles;
    }
    out[1] = n_cta > 0 ? (out[1] + n_cta - 1) / n_cta : 0;
}

// The most key tiles that a CTA of the two-tile launch walks in items of one query tile before one of two, whose second tile's warps wait
// through them.
static int64_t longest_wait(const std::vector<CrossItem> &items, int H, int n_sm) {
    const int64_t n_all = (int64_t)items.size() * H, n_cta = std::min<int64_t>(n_all, n_sm);
    int64_t most = 0;
    for (int64_t b = 0; b < n_cta; ++b) {
        int64_t run = 0;
        for (int64_t n = 0; n * n_cta < n_all; ++n) {
            const int64_t id = n * n_cta + ((n & 1) ? n_cta - 1 - b : b);
            if (id >= n_all || items[id / H].n_keys == 0) continue;
            if (items[id / H].rows <= 128) {
                run += (items[id / H].n_keys + 127) / 128;
            } else {
                most = std::max(most, run);
                run = 0;
            }
        }
    }
    return most;
}

// Test hook, host only: the launches of a problem on a GPU of n_sm SMs.  out: items of the forward's kernels (two query tiles, one, few
// queries) that have keys, and rows to put together; items of dQ that have keys; pieces of dK/dV; slots of their sums; the longest
// walk and the mean one of the two-tile launch, the one-tile launch and dQ, in key tiles; the longest wait in the first of these
extern "C" int moc_debug_cross_plan(const moc_cross_problem *pr, int n_sm, int64_t *out) {
    if (!pr || !out) return MOC_ERR_NULL;
    if (int r = check_cross(pr)) return r;
    if (n_sm < 1) return MOC_ERR_SHAPE;
    moc_cross c = {};
    c.n_sm = n_sm;
    try {
        if (int r = derive_cross(&c, pr)) return r;
    } catch (...) {
        return MOC_ERR_CUDA;
    }
    auto with_keys = [](const std::vector<CrossItem> &items) { return std::count_if(items.begin(), items.end(), [](const CrossItem &i) { return i.n_keys > 0; }); };
    out[0] = with_keys(c.items) * c.H; out[1] = (int64_t)c.solo.size() * c.H; out[2] = (int64_t)c.few.size() * c.Hkv; out[3] = (int64_t)c.prows * c.H;
    out[4] = with_keys(c.dq_items) * c.H; out[5] = (int64_t)c.pieces.size(); out[6] = c.kv_slots;
    walks(c.items, c.H, n_sm, out + 7);
    walks(c.solo, c.H, n_sm, out + 9);
    walks(c.dq_items, c.H, n_sm, out + 11);
    out[13] = longest_wait(c.items, c.H, n_sm);
    return MOC_OK;
}

extern "C" int moc_cross_get_status(const moc_cross *c, const void *ws, void *stream, int *device_status, int *detail) {
    if (int r = enter_cross(c)) return r;
    if (!device_status) return MOC_ERR_NULL;
    if (int r = check_ws(ws)) return r;
    int32_t st[2] = {0, 0};
    MOC_CUDA_TRY(cudaMemcpyAsync(st, ws_ptr<int32_t>(ws, c->ws.status), sizeof st, cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    MOC_CUDA_TRY(cudaStreamSynchronize((cudaStream_t)stream));
    *device_status = st[0];
    if (detail) *detail = st[1];
    return MOC_OK;
}
