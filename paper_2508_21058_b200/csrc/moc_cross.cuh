// Cross attention: the plan's tables and what its files share.
#pragma once
#include <vector>

#include "moc_common.cuh"

namespace moc {

// A work item of the forward (up to 256 query rows of one segment) or of dQ (up to 128), of every head: its queries, its keys (n_keys
// may be 0), and where its share's results go if there are other shares: the first row of partial results, -1 for none.
struct __align__(16) CrossItem { int32_t q0, rows, k0, n_keys, slot, pad[3]; };
// A share of the states of a segment with few queries, of every key head: rows [r0, r0 + nr) of the q_len queries of each of the key
// head's query heads; row r is query r mod q_len of query head r / q_len.
struct __align__(16) CrossFew { int32_t q0, q_len, k0, n_keys, slot, r0, nr, pad; };
// Rows whose partial results are put together: n times `rows`, from row `slot` of a head's partial results on.
struct __align__(16) CrossMerge { int32_t q0, rows, slot, n; };
// A piece of the key-stationary pass: up to 128 keys of a key head against units [u0, u1) of query rows; unit u: query head
// h * group + u / q_tiles, rows q0 + 128 (u mod q_tiles) of the segment's [q0, q1).
struct __align__(16) CrossPiece { int32_t h, k0, keys, q0, q1, u0, u1, slot; };
// Rows of a key head's dK and dV that are sums of n slots (0: zeros).
struct __align__(16) CrossSum { int32_t h, k0, rows, slot, n, pad[3]; };

constexpr int kCrossRows = 256;
// Where a running maximum begins: below every score but not minus infinity, so that a score of minus infinity weighs 2^-inf = 0, not
// 2^(inf - inf), also where a row has seen no other yet.  A row, or a share of its states, that sees no other has a sum of 0 and a log-sum-exp
// of minus infinity.
constexpr float kLowest = -3.402823466e38f;

// Rows of a key head up to which a segment counts as one with few queries.  Not a measured crossover: 64 segments of one query and 1500
// states take 77 us with three rows a key head there (24 heads on 8), and 163 with 12 or 24 (on 2 or 1) on the tensor cores, where each
// query head has a tile of its own; neither was tried the other way.
constexpr int kFewRows = 8;

struct CrossLayout {
    size_t status;
    size_t part_o, part_lse;       // forward: [H][prows][d] and [H][prows] fp32
    size_t fwd_end;
    size_t delta;                  // [H][Lq]
    size_t part_dq;                // [H][dq_prows][d] fp32
    size_t part_kv;                // [slots][2][128][d] fp32
    size_t bwd_end;
};

}  // namespace moc

struct moc_cross {
    int H, Hkv, g, d, Lq, Lk, device, n_sm;
    float scale;
    std::vector<moc::CrossItem> items, solo, dq_items; // per head, the longest first; solo: items of one query tile with a launch of their own
    std::vector<moc::CrossMerge> merges, dq_merges;    // per head
    std::vector<moc::CrossPiece> pieces;
    std::vector<int32_t> piece_off;                    // of every CTA of the key-stationary pass
    std::vector<moc::CrossSum> sums;
    std::vector<moc::CrossFew> few;                    // per key head, the longest first
    int few_rows = 0;                                  // the most rows that one has
    int most_merge_rows = 0, most_merge_n = 0;         // of the forward's merges
    int prows = 0, dq_prows = 0, kv_slots = 0;         // rows of partial results of a head, the same of dQ; slots in all
    int n_dq_work = 0;                                 // dQ's items that have keys: the others, which come last, only need zeros
    void *d_blob = nullptr;
    moc::CrossItem *d_items, *d_solo, *d_dq_items;
    moc::CrossFew *d_few;
    moc::CrossMerge *d_merges, *d_dq_merges;
    moc::CrossPiece *d_pieces;
    int32_t *d_piece_off;
    moc::CrossSum *d_sums;
    moc::CrossLayout ws;
    size_t dq_smem = 0, dkv_smem = 0;                  // shared memory of their launches
};

namespace moc {

// a caller's rows of bf16 on the device
struct CrossRows {
    __nv_bfloat16 *p;
    int64_t head, tok;
    CrossRows() = default;
    explicit CrossRows(const moc_rows *r) : p(static_cast<__nv_bfloat16 *>(r->data)), head(r->head_stride), tok(r->token_stride) {}
#ifdef __CUDACC__
    __device__ __forceinline__ __nv_bfloat16 *row(int h, int t) const { return p + h * head + t * tok; }
#endif
};

#ifdef __CUDACC__
// A CTA's n-th item of a list that is sorted by length: every other round in reverse, so that no CTA has the longest of each.
__device__ __forceinline__ int cross_item(int n) {
    return n * (int)gridDim.x + ((n & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
}
// how many of the first `n_all` items a CTA has
__device__ __forceinline__ int cross_items(int n_all) {
    const int rounds = n_all / (int)gridDim.x, rest = n_all - rounds * (int)gridDim.x;
    return rounds + (((rounds & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x) < rest ? 1 : 0);
}
// asks for an item's description ahead of its use
__device__ __forceinline__ void prefetch_item(const CrossItem *item) { asm volatile("prefetch.global.L1 [%0];" ::"l"(item)); }
#endif

// what the kernels of a plan's launches need of the runtime, once
int prepare_cross_fwd(moc_cross *c);
int prepare_cross_solo(moc_cross *c);
int prepare_cross_few(moc_cross *c);
int prepare_cross_dq(moc_cross *c);
int prepare_cross_dkv(moc_cross *c);

int launch_cross_solo(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws, bool first, cudaStream_t s);
int launch_cross_few(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws,
                     cudaStream_t s);
int launch_cross_fwd(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, float *lse, void *ws, bool first, cudaStream_t s);
// (also writes delta)
int launch_cross_dq(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const moc_rows *O, const float *lse, const moc_rows *dO,
                    const moc_rows *dQ, void *ws, cudaStream_t s);
int launch_cross_dkv(const moc_cross *c, const moc_rows *Q, const moc_rows *K, const moc_rows *V, const float *lse, const moc_rows *dO,
                     const moc_rows *dK, const moc_rows *dV, void *ws, cudaStream_t s);
// items: rows of one head's tile list x heads, as one launch of up to `most` CTAs
static inline unsigned cross_grid(const moc_cross *c, size_t items) {
    const size_t n = items * (size_t)c->H;
    return (unsigned)(n < (size_t)c->n_sm ? n : (size_t)c->n_sm);
}

}  // namespace moc
