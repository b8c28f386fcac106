// Attention of the rows of draft trees over a cache kept in pages (include/sdv.h: sdv_tree_attention).
#pragma once
#include <cuda.h>
#include <math_constants.h>

#include "paged.cuh"
#include "tree_plan.h"

namespace sdv {

constexpr int kTreeThreads = 192;      // warps 0..3: softmax, a tile row per thread; 4: copies; 5: tensor-core issue
constexpr int kTreeBlocksPerSm = 2;
constexpr int kTreeMaxBlocks = 1024;   // of a launch: twice the SMs

template <int HD>
struct TreeShape {
    static constexpr int kAtoms = HD / 64;                        // 64-column swizzled slabs of a row
    static constexpr int kQBytes = kTreeTileRows * HD * 2;
    static constexpr int kSlotBytes = kTreeKeys * HD * 2;         // keys or values of a tile
    static constexpr int kSlots = HD == 128 ? 5 : 11;
    static constexpr int kCtlBytes = HD == 128 ? 1024 : 2048;
    static constexpr int kSmemBytes = kQBytes + kSlots * kSlotBytes + kCtlBytes;   // two blocks an SM: at most 113 KB each
    static_assert(kSmemBytes <= 113 * 1024, "two blocks per SM");
};

struct TreeParams : TreeLists {
    void* out;
    const void* v;                     // pool, for values that are not finite
    const int *block_table, *parent;
    float* part_o;                     // [2][block][part_rows / 4][HD / 8][4][8]: four rows' 32 bytes make a line, for the storing warp and for the merge
    float2* part_ml;                   // [2][block][part_rows] maximum (log2 units), sum
    int* status;
    long long out_row_stride, out_head_stride, table_stride, page_stride, head_stride, token_stride;
    int page_shift, n_pages, part_rows, blocks, q_step;
    float scale_log2e;
    int clear;                         // rows that nobody computes are filled
    int copies;                        // keys or values of tiles that a block copies at most: no limit but in tests
    unsigned long long wait_limit_ns, drain_limit_ns;   // waits that may be given up; those that keep copies and products from outliving the block
};

// Tiles of all sequences, summed up by a block: thread t has the sequences [t * per, (t + 1) * per).
template <int WARPS>
struct TreeScan {
    int warp_sum[WARPS], before[WARPS * 32];   // before: within its warp
    __device__ __forceinline__ static int per(const TreeLists& P) { return (P.n_seqs + WARPS * 32 - 1) / (WARPS * 32); }
    template <bool EARLY>
    __device__ __forceinline__ void fill(const TreeLists& P) {   // all threads; a barrier follows
        const int tid = threadIdx.x, lane = tid & 31, n = per(P), b0 = min(tid * n, P.n_seqs), b1 = min(b0 + n, P.n_seqs);
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += tree_tiles(P, tree_seq<EARLY>(P, b));
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        before[tid] = incl - sum;
        if (lane == 31) warp_sum[tid >> 5] = incl;
    }
    __device__ __forceinline__ int total() const {
        int t = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) t += warp_sum[w];
        return t;
    }
    // The sequence that has tile `tile` (below the total), and how far into it; whole warps.
    __device__ __forceinline__ int find_tile(const TreeLists& P, int& tile, TreeSeq& s) const {
        const int lane = threadIdx.x & 31;
        int w = 0;
#pragma unroll
        for (int k = 0; k < WARPS - 1; ++k)
            if (w == k && tile >= warp_sum[k]) {
                tile -= warp_sum[k];
                ++w;
            }
        const int t = w * 32 + 31 - __clz(__ballot_sync(0xffffffffu, before[w * 32 + lane] <= tile));   // the last thread that begins at or before it
        tile -= before[t];
        int b = t * per(P);
        for (;; ++b) {
            s = tree_seq(P, b);
            const int n = tree_tiles(P, s);
            if (tile < n || b + 1 >= P.n_seqs) return b;
            tile -= n;
        }
    }
};

__device__ __forceinline__ void tma_load_3d(void* smem_dst, const void* map, int x, int y, int z, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(smem_dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* smem_dst, const void* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(smem_dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
                 : "memory");
}

template <typename T> __device__ __forceinline__ uint32_t tree_idesc(uint32_t n);
template <> __device__ __forceinline__ uint32_t tree_idesc<__nv_bfloat16>(uint32_t n) { return umma_idesc_bf16(128u, n); }
template <> __device__ __forceinline__ uint32_t tree_idesc<__half>(uint32_t n) { return umma_idesc_bf16(128u, n) & ~((1u << 7) | (1u << 10)); }   // both operands fp16

// Probabilities are relative to 2^shift for a row's largest score.  fp16 has bits for 2^-24 to 2^15.99: with the largest at 2^7 to 2^15, those of 2^-31 of it still count
// (at 1 to 2^8, a flat tail of 2^-25 each vanished from the outputs but not from the sums: 2^-9 of a row's mass behind 65536 keys).  bf16 has fp32's range.
template <typename T> constexpr float kProbShift = 0.f;
template <> constexpr float kProbShift<__half> = 7.f;

// Clears what is infinite or NaN among the two 16-bit numbers of a word; whether there was any.
template <typename T> __device__ __forceinline__ bool clear_not_finite(uint32_t& w) {
    constexpr uint32_t kExp = Half16<T>::kExponent;
    const bool lo = (w & kExp) == kExp, hi = ((w >> 16) & kExp) == kExp;
    w &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
    return lo || hi;
}

// Two fp32 numbers in a 64-bit register: one instruction for both.
__device__ __forceinline__ uint64_t pack_f32x2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Bit masks of the rows on the way from every row of a tree to its root, by doubling: lane l has rows l and l + 32.
__device__ __forceinline__ void tree_masks(const TreeParams& P, const TreeSeq& s, int lane, unsigned long long& m0, unsigned long long& m1) {
    int p0 = lane, p1 = lane + 32;   // how far up the mask reaches: a row points at itself once it is at the root
    m0 = 1ull << lane;
    m1 = 1ull << (lane + 32);
    if (lane > 0 && lane < s.rows) {
        const int p = P.parent[s.first + lane];
        p0 = p < 0 || p >= lane ? 0 : p;
    }
    if (lane + 32 < s.rows) {
        const int p = P.parent[s.first + lane + 32];
        p1 = p < 0 || p >= lane + 32 ? 0 : p;
    }
    m0 |= 1ull << p0;
    m1 |= 1ull << p1;
#pragma unroll 1
    for (int step = 0; step < 6 && __any_sync(0xffffffffu, p0 > 0 && p0 != lane || p1 > 0 && p1 != lane + 32); ++step) {
        const unsigned long long a0 = __shfl_sync(0xffffffffu, m0, p0 & 31), a1 = __shfl_sync(0xffffffffu, m1, p0 & 31);
        const unsigned long long b0 = __shfl_sync(0xffffffffu, m0, p1 & 31), b1 = __shfl_sync(0xffffffffu, m1, p1 & 31);
        const int q0 = __shfl_sync(0xffffffffu, p0, p0 & 31), q1 = __shfl_sync(0xffffffffu, p1, p0 & 31);
        const int r0 = __shfl_sync(0xffffffffu, p0, p1 & 31), r1 = __shfl_sync(0xffffffffu, p1, p1 & 31);
        m0 |= p0 < 32 ? a0 : a1;
        m1 |= p1 < 32 ? b0 : b1;
        p0 = p0 < 32 ? q0 : q1;
        p1 = p1 < 32 ? r0 : r1;
    }
}

// Values of the rows `rows` of the tree that are not finite, columns c .. c + 31, added to a row's output: the product left them out.  An infinity times any
// probability is the infinity, so no weight is needed.  Rare.
template <typename T>
__device__ __forceinline__ void tree_add_not_finite(const TreeParams& P, const TreeCursor& cur, unsigned long long rows, int c, uint32_t (&o)[32]) {
#pragma unroll 1
    for (; rows; rows &= rows - 1) {
        const int key = cur.s.length + __ffsll((long long)rows) - 1;
        const int page = P.block_table[cur.b * P.table_stride + (key >> P.page_shift)];
        if (page < 0 || page >= P.n_pages) continue;
        const T* v = (const T*)P.v + page * P.page_stride + cur.h * P.head_stride + (key & (P.page_size - 1)) * P.token_stride + c;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float x = Half16<T>::up(v[i]);
            if (!isfinite(x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
        }
    }
}

// Rows that nobody computes, shared out over the blocks, by one warp: zeros in those of no sequence, NaN in those of a sequence past SDV_TREE_ROWS.
template <typename T, int HD>
__device__ __forceinline__ void tree_clear(const TreeParams& P, int lane) {
    const int words = P.g * P.n_kv * (HD / 8);   // 16 bytes each, of a row
    const auto fill = [&](int from, int until, uint32_t with) {
        for (int r = from + (int)blockIdx.x; r < until; r += P.blocks)
            for (int i = lane; i < words; i += 32)
                *reinterpret_cast<uint4*>((T*)P.out + r * P.out_row_stride + i / (HD / 8) * P.out_head_stride + i % (HD / 8) * 8) = make_uint4(with, with, with, with);
    };
    fill(0, rows_begin(P.cu_rows, 0, P.n_rows), 0u);
    fill(rows_begin(P.cu_rows, P.n_seqs, P.n_rows), P.n_rows, 0u);
    for (int b0 = 0; b0 < P.n_seqs; b0 += 32) {
        const int b = b0 + lane;
        unsigned many = __ballot_sync(0xffffffffu, b < P.n_seqs && rows_count(P.cu_rows, b, P.n_rows) > SDV_TREE_ROWS);
        for (; many; many &= many - 1) {
            const int at = b0 + __ffs(many) - 1;
            fill(rows_begin(P.cu_rows, at, P.n_rows) + SDV_TREE_ROWS, rows_begin(P.cu_rows, at + 1, P.n_rows), 0x7fff7fffu);
        }
    }
}

// out = sum_t softmax(scale q k_t) v_t with running maxima and sums.  A tile is 64 keys by up to 128 tile rows (a tile row is one query head of one row; the rows of a
// sequence and the heads that share a KV head read the keys together).  All tiles of all sequences, KV heads and tiles of rows are one list, cut into equal shares
// over two blocks an SM whatever the lengths: a block works through parts of one or of many items, and what it did not do alone is merged by tree_merge_kernel from
// un-normalised outputs, maxima and sums in the workspace.  (Short tables are dealt out in whole items instead, see the host.)
// Within a block: one warp copies keys and values, box by box of a page, into a ring of tiles (tensor maps: any strides, five tiles of 16 KB in flight a block); one issues S = Q K^T
// into one of two tensor-memory buffers and, when four warps have turned it into probabilities in place (a tile row a thread, no exchange between threads), P V, which adds up in
// tensor memory.  The output is rescaled only when a row's maximum grew by more than 2^8 (this and probabilities in tensor memory are published methods, named at
// dense_attention_kernel): probabilities stay below 2^8 (fp16: 2^15, see kProbShift) and their sums, in fp32, lose nothing.  S of the next tile is
// computed during the softmax of this one.  Probabilities are rounded to the 16-bit type for the second product, as its operand has to be; sums take them unrounded.
// Bound by memory where the cache is long: 64 sequences of one row over up to 8192 tokens (619 MB, 7 heads a KV head) take 97 us here and 104 with the merge, 5.9 TB/s; a run of
// many seconds is bound by power, 113 us.  24 trees of up to 40 rows (244 MB) take 49 us: 37 for the bytes, 4 until the first scores, the rest until the slowest block is through
// (blocks of equal shares end up to 15 percent apart).  Several tiles of rows read the keys again from L2
// each: 64 rows of 28 + 4 heads over 16000 tokens take 34.7 us (bytes 5.2, products 9.1).  They draw 3.8 TB/s from L2, less than a row a sequence draws through it from HBM: a block
// takes 2 us a tile of 64 keys, its one stream's chain of load, S, softmax and P V.
// Places behind a sequence's end hold anything: their values are cleared in shared memory (0 x NaN is not 0).  Rows of the tree
// that a row does not see take part in its product with probability 0: infinities and NaN among their values are cleared too, and added
// by those who see them at the end.
template <typename T, int HD>
__global__ void __launch_bounds__(kTreeThreads, kTreeBlocksPerSm)
tree_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_q1, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                      const __grid_constant__ TreeParams P) {
    using S = TreeShape<HD>;
    constexpr int KSTEPS = HD / 16;
    extern __shared__ __align__(1024) uint8_t tree_smem[];
    uint8_t *Qs = tree_smem, *ring = Qs + S::kQBytes;
    struct Ctl {
        uint64_t full[S::kSlots], empty[S::kSlots], s_full[2], p_ready[2], pv_done[2], q_ready, q_free, drained;
        unsigned long long bad[4];     // rows of the tree with values that are not finite, by item (modulo 4)
        uint32_t tmem_base;
        int abort_flag;
        TreeScan<kTreeThreads / 32> scan;
    };
    Ctl* ctl = reinterpret_cast<Ctl*>(ring + S::kSlots * S::kSlotBytes);
    static_assert(sizeof(Ctl) <= S::kCtlBytes, "control block");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
    if (tid == 0) {
        for (int s = 0; s < S::kSlots; ++s) {
            mbar_init(&ctl->full[s], 1);
            mbar_init(&ctl->empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&ctl->s_full[i], 1);
            mbar_init(&ctl->p_ready[i], 4);
            mbar_init(&ctl->pv_done[i], 1);
        }
        for (int i = 0; i < 4; ++i) ctl->bad[i] = 0;
        mbar_init(&ctl->drained, 1);
        mbar_init(&ctl->q_ready, 1);
        mbar_init(&ctl->q_free, 1);
        ctl->abort_flag = 0;
        mbar_fence_init();
    }
    for (int i = tid; i < S::kQBytes / 16; i += kTreeThreads) reinterpret_cast<uint4*>(Qs)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    if (warp == 5) tmem_alloc(&ctl->tmem_base, 256);   // S0 | S1, 64 columns each | O, HD columns
    if (warp == 4 && lane < 4) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &map_q : lane == 1 ? &map_q1 : lane == 2 ? &map_k : &map_v) : "memory");
    grid_dep_wait();
    ctl->scan.fill<false>(P);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem_base;
    grid_dep_launch();   // behind the wait: the merge reads the lengths at once
    TreeCursor cur;
    {
        const TreeCut cut(ctl->scan.total(), P.blocks);
        int offset = cut.begin((int)blockIdx.x);
        const int n = cut.begin((int)blockIdx.x + 1) - offset;
        cur.left = 0;
        if (n > 0) {
            TreeSeq s;
            const int b = ctl->scan.find_tile(P, offset, s);
            cur.start(P, b, s, offset, n);
        }
    }

    if (warp == 4) {
        // ---- copies: K0 V0 K1 V1 ... through the ring
        const int box_keys = min(P.page_size, kTreeKeys), boxes = kTreeKeys / box_keys;   // per slab
        const int my_box = lane % boxes, my_atom = lane / boxes;
        uint32_t s = 0, par = 0;
        int issued = 0;
        bool ok = true;
        const auto page_of = [&](const TreeCursor& c, int tile) {   // page of this lane's box of a tile
            const int key = tile * kTreeKeys + my_box * box_keys;
            return my_atom < S::kAtoms && key < c.s.keys ? P.block_table[c.b * P.table_stride + (key >> P.page_shift)] : -1;
        };
        int page = cur.left > 0 ? page_of(cur, cur.tile) : -1;
        while (cur.left > 0 && ok) {
            const int n = cur.run(P);
            TreeCursor nxt = cur;
            nxt.skip(P, n);
            for (int j = 0; j < n && ok; ++j) {
                if (issued >= P.copies) {
                    ok = false;
                    break;
                }
                const int tile = cur.tile + j, key = tile * kTreeKeys + my_box * box_keys;
                const int next_page = j + 1 < n ? page_of(cur, tile + 1) : nxt.left > 0 ? page_of(nxt, nxt.tile) : -1;
                const bool mine = my_atom < S::kAtoms && key < cur.s.keys;
                const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * (uint32_t)box_keys * 128u;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    ok = ok && mbar_wait_bounded(&ctl->empty[s], par ^ 1u, &ctl->abort_flag, P.wait_limit_ns);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(&ctl->full[s], bytes);
                    __syncwarp();
                    // (x a multiple of 64 elements; a page outside the pool reads as zeros)
                    if (mine)
                        tma_load_4d(ring + s * S::kSlotBytes + my_atom * (kTreeKeys * 128) + my_box * box_keys * 128, kv ? &map_v : &map_k, my_atom * 64, key & (P.page_size - 1),
                                    cur.h, page, &ctl->full[s]);
                    ++issued;
                    if (++s == S::kSlots) { s = 0; par ^= 1u; }
                }
                page = next_page;
            }
            cur = nxt;
        }
        // the copies still in flight are waited for (bounded): where a wait was given up, here or later, nobody else does
        for (int back = 0; back < S::kSlots && back < issued; ++back) {
            if (s == 0) { s = S::kSlots; par ^= 1u; }
            --s;
            if (!mbar_drain(&ctl->full[s], par, P.drain_limit_ns)) break;
        }
    } else if (warp == 5) {
        // ---- tensor-core issue
        const uint32_t id_s = tree_idesc<T>(kTreeKeys), id_o = tree_idesc<T>(HD) | (1u << 16);   // B of P V: features contiguous
        const uint32_t qa = smem_u32(Qs), ra = smem_u32(ring);
        bool ok = true;
        uint32_t item = 0;
        uint32_t s_k = 0, par_k = 0;                    // slot of the next keys
        uint32_t n_s = 0, n_p = 0;                      // tiles whose scores / products were issued
        const auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && mbar_wait_bounded(bar, parity, &ctl->abort_flag, P.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
        };
        // The queries of an item, all heads of the group: `q_step` rows a copy, the last ones one by one.  Other tile rows keep what they hold, zeros to begin with: products with
        // them cost power (a long run over 64 sequences of one row took 121 us a call with the neighbours' queries in them, 114 with zeros).
        const auto load_q = [&](const TreeCursor& c) {
            if (elect_one()) {
                const int rows = min(P.chunk, c.s.rows - c.c * P.chunk), row0 = c.s.first + c.c * P.chunk;
                mbar_arrive_expect_tx(&ctl->q_ready, (uint32_t)(S::kAtoms * 128 * rows * P.g));
                for (int r = 0; r < rows;) {
                    const bool many = rows - r >= P.q_step;
#pragma unroll
                    for (int a = 0; a < S::kAtoms; ++a)
                        tma_load_3d(Qs + a * (kTreeTileRows * 128) + r * P.g * 128, many ? &map_q : &map_q1, a * 64, c.h * P.g, row0 + r, &ctl->q_ready);
                    r += many ? P.q_step : 1;
                }
            }
            __syncwarp();
        };
        uint32_t q_loads = 0;
        if (cur.left > 0) {
            load_q(cur);
            ++q_loads;
        }
        const auto scores = [&](bool last) {
            // the buffer held the probabilities of the tile two back: products into different accumulators are not ordered among themselves
            // (waited for is the newest product: within an item that of the tile two back)
            if (n_p > 0) wait(&ctl->pv_done[(n_p - 1u) & 1u], ((n_p - 1u) >> 1) & 1u);
            wait(&ctl->full[s_k], par_k);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t d = tmem + (n_s & 1u) * kTreeKeys, k = ra + s_k * S::kSlotBytes;
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks)
                    umma_bf16(d, umma_desc_sw128(qa + (uint32_t)((ks >> 2) * (kTreeTileRows * 128) + (ks & 3) * 32)),
                              umma_desc_sw128(k + (uint32_t)((ks >> 2) * (kTreeKeys * 128) + (ks & 3) * 32)), id_s, (uint32_t)ks);
                umma_commit(&ctl->empty[s_k]);
                umma_commit(&ctl->s_full[n_s & 1u]);
                if (last) umma_commit(&ctl->q_free);
            }
            __syncwarp();
            ++n_s;
            s_k += 2;                                   // the values lie between
            if (s_k >= S::kSlots) { s_k -= S::kSlots; par_k ^= 1u; }
        };
        uint32_t s_v = 1, par_v = 0;
        while (cur.left > 0 && ok) {
            const int n = cur.run(P);
            TreeCursor nxt = cur;
            nxt.skip(P, n);
            wait(&ctl->q_ready, item & 1u);
            if (ok) scores(n == 1);
            for (int j = 0; j < n && ok; ++j) {
                if (j + 1 < n) scores(j + 2 == n);
                if (j + 1 == n && nxt.left > 0) {   // the item's last scores are under way: the next item's queries take the place of this one's behind them
                    wait(&ctl->q_free, item & 1u);
                    if (!ok) break;
                    load_q(nxt);
                    ++q_loads;
                }
                wait(&ctl->full[s_v], par_v);
                wait(&ctl->p_ready[n_p & 1u], (n_p >> 1) & 1u);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t p = tmem + (n_p & 1u) * kTreeKeys, v = ra + s_v * S::kSlotBytes;
#pragma unroll
                    for (int ks = 0; ks < kTreeKeys / 16; ++ks)   // 16 keys: 16 rows of 128 bytes of every slab; 8 packed columns of P
                        umma_bf16_tmem_a(tmem + 2 * kTreeKeys, p + (uint32_t)ks * 8u, umma_desc_sw128_mn(v + (uint32_t)ks * 2048u, kTreeKeys * 128), id_o,
                                         (uint32_t)(j | ks));
                    umma_commit(&ctl->empty[s_v]);
                    umma_commit(&ctl->pv_done[n_p & 1u]);
                }
                __syncwarp();
                ++n_p;
                s_v += 2;
                if (s_v >= S::kSlots) { s_v -= S::kSlots; par_v ^= 1u; }
            }
            ++item;
            cur = nxt;
        }
        if (q_loads) mbar_drain(&ctl->q_ready, (q_loads - 1u) & 1u, P.drain_limit_ns);   // where a wait was given up, nobody else waits for the last copy
        // tensor and shared memory are given back only when no product uses them any more, whoever gave up a wait: this warp, or those who wait for its last product
        if (n_s) {
            if (elect_one()) umma_commit(&ctl->drained);
            __syncwarp();
            mbar_drain(&ctl->drained, 0, P.drain_limit_ns);
        }
    } else {
        // ---- softmax: tile row t
        const int t = tid;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16, to = tmem + lanes + 2 * kTreeKeys;
        bool ok = true;
        uint32_t n_t = 0, item = 0;
        int mask_b = -1;
        unsigned long long anc0 = 0, anc1 = 0;
        uint32_t v_slot = 1, v_par = 0;
        while (cur.left > 0) {
            const int n = cur.run(P);
            const TreeSeq& sq = cur.s;
            const int jt = t / P.g, j = cur.c * P.chunk + jt, hh = t - jt * P.g;                       // row of the sequence, head of the group
            const int rows_here = min(P.chunk, sq.rows - cur.c * P.chunk) * P.g;
            const bool real = t < rows_here, some = warp * 32 < rows_here;                             // this row, any row of the warp
            unsigned long long see = j < 63 ? (2ull << j) - 1 : ~0ull;                                 // rows of the sequence this row sees
            if (P.parent) {
                if (mask_b != cur.b) {
                    tree_masks(P, sq, lane, anc0, anc1);
                    mask_b = cur.b;
                }
                const unsigned long long a0 = __shfl_sync(0xffffffffu, anc0, j & 31), a1 = __shfl_sync(0xffffffffu, anc1, j & 31);
                see = j < 32 ? a0 : a1;
            }
            float m = real ? -CUDART_INF_F : CUDART_INF_F, l = 0.f;   // (the probabilities of a tile row without a query are zeros)
            TreeCursor nxt = cur;
            nxt.skip(P, n);
            for (int k = 0; k < n; ++k, ++n_t) {
                const int key0 = (cur.tile + k) * kTreeKeys, new0 = sq.length - key0, left = sq.keys - key0;   // first new key, keys left, within the tile
                const uint32_t ts = tmem + lanes + (n_t & 1u) * kTreeKeys;
                ok = ok && mbar_wait_bounded(&ctl->s_full[n_t & 1u], (n_t >> 1) & 1u, &ctl->abort_flag, P.wait_limit_ns);
                const bool tail = new0 < kTreeKeys;    // rows of the tree, or the end, among the keys
                if (tail) {
                    ok = ok && mbar_wait_bounded(&ctl->full[v_slot], v_par, &ctl->abort_flag, P.wait_limit_ns);
                    if (ok) {
                        // two threads a key, half of its columns each
                        const int key = t >> 1;
                        uint4* vr = reinterpret_cast<uint4*>(ring + v_slot * S::kSlotBytes + key * 128);
                        bool wrong = false;
#pragma unroll
                        for (int i = (t & 1) * 4; i < (t & 1) * 4 + 4; ++i) {
#pragma unroll
                            for (int a = 0; a < S::kAtoms; ++a) {
                                uint4* w = vr + a * (kTreeKeys * 8) + i;
                                if (key >= left) *w = make_uint4(0, 0, 0, 0);
                                else if (key >= new0) {
                                    uint4 x = *w;
                                    if (clear_not_finite<T>(x.x) | clear_not_finite<T>(x.y) | clear_not_finite<T>(x.z) | clear_not_finite<T>(x.w)) {
                                        *w = x;
                                        wrong = true;
                                    }
                                }
                            }
                        }
                        if (wrong) atomicOr(&ctl->bad[item & 3u], 1ull << (key - new0));
                    }
                    fence_proxy_async_smem();
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (some) {
                    tc_fence_after();
                    uint32_t v[2][32];
                    tmem_ld32(ts, v[0]);
                    tmem_ld32(ts + 32u, v[1]);
                    tmem_ld_wait();
                    if (tail) {
                        // keys before the new ones, and the new ones on the row's path
                        const int old = max(new0, 0);
                        unsigned long long vis = old >= 64 ? ~0ull : (1ull << old) - 1;
                        if (new0 >= 0) vis |= new0 < 64 ? see << new0 : 0ull;
                        else vis |= -new0 < 64 ? see >> -new0 : 0ull;
                        if (left < 64) vis &= (1ull << left) - 1;
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (!((vis >> i) & 1ull)) v[i >> 5][i & 31] = 0xff800000u;   // -inf
                    }
                    float m4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                    for (int i = 0; i < 64; i += 2) m4[(i >> 1) & 3] = fmaxf(fmaxf(m4[(i >> 1) & 3], __uint_as_float(v[i >> 5][i & 31])), __uint_as_float(v[i >> 5][(i & 31) + 1]));
                    const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * P.scale_log2e;
                    const bool grow = real && mx > m + 8.f;   // also the first tile that shows this row a key
                    const bool rescale = grow && m != -CUDART_INF_F;
                    if (__any_sync(0xffffffffu, rescale)) {
                        // the product of the tile before has to be complete (it is the newest one, as this tile's waits for this
                        // warp, and the one two before it is complete, as these scores came after it: with two barriers the parity is unambiguous)
                        ok = mbar_wait_bounded(&ctl->pv_done[(n_t - 1u) & 1u], ((n_t - 1u) >> 1) & 1u, &ctl->abort_flag, P.wait_limit_ns);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        tc_fence_after();
                        const float f = rescale ? exp2f(m - mx) : 1.f;
                        l *= f;
#pragma unroll 1
                        for (int c = 0; c < HD; c += 16) {
                            float o[16];
                            uint32_t x[16];
                            tmem_ld16(to + (uint32_t)c, o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(o[i] * f);
                            tmem_st16(to + (uint32_t)c, x);
                        }
                    }
                    if (grow) m = mx;
                    const float ref = m == -CUDART_INF_F ? 0.f : m - kProbShift<T>;
                    const uint64_t sc2 = pack_f32x2(P.scale_log2e, P.scale_log2e), ref2 = pack_f32x2(-ref, -ref);
                    uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t pk[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float x, y;
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[c][i]), __uint_as_float(v[c][i + 1])), sc2, ref2), x, y);
                            x = ex2_ftz(x);
                            y = ex2_ftz(y);
                            sum2[(i >> 1) & 1] = add_f32x2(sum2[(i >> 1) & 1], pack_f32x2(x, y));
                            pk[i / 2] = Half16<T>::pack(x, y);
                        }
                        tmem_st16(ts + 16u * (uint32_t)c, pk);   // over scores this thread has read
                    }
                    {
                        float x, y;
                        unpack_f32x2(add_f32x2(sum2[0], sum2[1]), x, y);
                        l += x + y;
                    }
                    tmem_st_wait();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->p_ready[n_t & 1u]);
                v_slot += 2;
                if (v_slot >= S::kSlots) { v_slot -= S::kSlots; v_par ^= 1u; }
            }
            if (ok) ok = mbar_wait_bounded(&ctl->pv_done[(n_t - 1u) & 1u], ((n_t - 1u) >> 1) & 1u, &ctl->abort_flag, P.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            const bool whole = n == sq.tiles;
            if (some) {
                tc_fence_after();
                const unsigned long long bad = *(volatile unsigned long long*)&ctl->bad[item & 3u] & see;
                const int slot = (int)blockIdx.x + (item ? P.blocks : 0);   // an item that is not the block's first is its last, or whole
                float* po = P.part_o + (long long)slot * P.part_rows * HD + (t >> 2) * (4 * HD) + (t & 3) * 8;
                T* dst = (T*)P.out + (sq.first + j) * P.out_row_stride + (cur.h * P.g + hh) * P.out_head_stride;
                const float sc = whole ? 1.f / l : 1.f;
                if (!whole && real) P.part_ml[(long long)slot * P.part_rows + t] = ok ? make_float2(m, l) : make_float2(0.f, CUDART_NAN_F);
#pragma unroll 1
                for (int c = 0; c < HD; c += 32) {
                    uint32_t o[32];
                    if (ok) {
                        tmem_ld32(to + (uint32_t)c, o);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0x7fc00000u;   // NaN
                    }
                    if (real && ok && bad) tree_add_not_finite<T>(P, cur, bad, c, o);
                    if (real && whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4*>(dst + c + i) =
                                make_uint4(Half16<T>::pack(__uint_as_float(o[i]) * sc, __uint_as_float(o[i + 1]) * sc), Half16<T>::pack(__uint_as_float(o[i + 2]) * sc, __uint_as_float(o[i + 3]) * sc),
                                           Half16<T>::pack(__uint_as_float(o[i + 4]) * sc, __uint_as_float(o[i + 5]) * sc), Half16<T>::pack(__uint_as_float(o[i + 6]) * sc, __uint_as_float(o[i + 7]) * sc));
                    } else if (real) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) st_global_v8(po + (c + i) * 4, o + i);
                    }
                    __syncwarp();   // tensor memory is read by whole warps
                }
                tc_fence_before();
            }
            // nobody is at the item after the next before this thread has been through the next one, and all are done with the one two back
            if (tid == 0) ctl->bad[(item + 2u) & 3u] = 0;
            ++item;
            cur = nxt;
        }
    }
    if (P.clear && warp == 4) tree_clear<T, HD>(P, lane);   // (the copying warp is the first to be through; from within its branch, the chain over 65536 tokens took 0.5 us more)
    __syncwarp();
    __syncthreads();
    if (warp == 5) tmem_dealloc(tmem, 256);
    if (tid == 0 && ctl->abort_flag && P.status) atomicExch(P.status, 1);
}

// Output rows whose keys several blocks went through: un-normalised partial outputs weighted by 2^(maximum - largest maximum).  A unit is four tile rows of an
// item, or 16 columns of them where there are so few units that each has a block; a lane has four columns of one row.  A warp takes a unit; those with more than
// twelve parts, and the fine ones, are gone through by whole blocks (a long cache of few sequences is cut into up to 150 parts).  Neighbouring units are in different blocks, so that a long
// sequence among short ones has many blocks' help.  Where the parts are follows from the lengths alone and is worked out before the attention is waited for.
// Bound by latency: 1.2 us behind the attention's last block, then a round trip to L2 of about 1 us for every two parts and 64 columns (alone) or five parts (together), the store:
// 2.5 to 5 us in all.  (Loops are kept short: unrolled further, instruction fetches and spilled registers took more than they saved.)
constexpr int kMergeWarps = 8, kMergeThreads = kMergeWarps * 32, kMergeDeep = 5 /* parts a warp has in flight */, kMergeFew = 12;
struct TreeUnit {
    int block0, n;        // first block with a part, parts
    int row, rows, col;   // first tile row, rows, first column
    int first, h, j0;     // first row of the sequence, KV head, first (row, head of the group) of the unit within the sequence
    bool late;            // of block0 it is the second partial item
    __device__ __forceinline__ int slot(int i, int blocks) const { return block0 + i + (i == 0 && late ? blocks : 0); }
};

__device__ __forceinline__ void tree_add(float4& o, float w, const float4& x) { o.x += w * x.x; o.y += w * x.y; o.z += w * x.z; o.w += w * x.w; }
__device__ __forceinline__ void tree_scale(float4& o, float w) { o.x *= w; o.y *= w; o.z *= w; o.w *= w; }

// What a lane has of a unit: a row, four columns of every group of 32.
template <typename T, int HD>
struct TreeMergeRow {
    const float2* ml;
    const float* o;    // (at most 1024 blocks of two parts of 128 rows of 128 columns: offsets within 32 bits)
    __device__ __forceinline__ TreeMergeRow(const TreeParams& P, const TreeUnit& q, int my_row, int lane) {
        ml = P.part_ml + q.row + my_row;
        o = P.part_o + q.row * HD + (lane >> 3) * 32 + my_row * 8 + (lane & 1) * 4;
    }
    __device__ __forceinline__ void store(const TreeParams& P, const TreeUnit& q, int my_row, int lane, int c, const float4& v, float sum) const {
        const float sc = 1.f / sum;
        const int r = q.j0 + my_row, j = r / P.g, hh = r - j * P.g;
        T* dst = (T*)P.out + (q.first + j) * P.out_row_stride + (q.h * P.g + hh) * P.out_head_stride + (lane >> 3) * 8 + (lane & 1) * 4;
        if (my_row < q.rows) *reinterpret_cast<uint2*>(dst + c) = make_uint2(Half16<T>::pack(v.x * sc, v.y * sc), Half16<T>::pack(v.z * sc, v.w * sc));
    }
};

// Adds parts i0, i0 + step, ... of a unit, up to five, to (maximum, sum, output).
template <int HD>
__device__ __forceinline__ void tree_gather(const TreeParams& P, const TreeUnit& q, const float2* ml0, const float* o0, int i0, int step, float& m, float& l, float4& o) {
    float2 ml[kMergeDeep];
    float4 x[kMergeDeep];
#pragma unroll
    for (int t = 0; t < kMergeDeep; ++t) {
        const int i = i0 + t * step;
        ml[t] = make_float2(-CUDART_INF_F, 0.f);
        if (i < q.n) {
            const int at = q.slot(i, P.blocks) * P.part_rows;
            ml[t] = ml0[at];
            x[t] = *reinterpret_cast<const float4*>(o0 + at * HD);
        }
    }
    float mx = m;
#pragma unroll
    for (int t = 0; t < kMergeDeep; ++t) mx = fmaxf(mx, ml[t].x);
    const float ref = mx == -CUDART_INF_F ? 0.f : mx, keep = exp2f(m - ref);
    m = mx;
    l *= keep;
    tree_scale(o, keep);
#pragma unroll
    for (int t = 0; t < kMergeDeep; ++t)
        if (i0 + t * step < q.n) {
            const float f = exp2f(ml[t].x - ref);
            l += f * ml[t].y;
            tree_add(o, f, x[t]);
        }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kMergeThreads, 3) tree_merge_kernel(const __grid_constant__ TreeParams P, int group, int split) {
    __shared__ TreeScan<kMergeWarps> scan;
    __shared__ int unit0[kMergeThreads];   // first unit of every thread's first sequence
    __shared__ TreeUnit shared_unit[kMergeWarps];
    __shared__ float4 shared_o[kMergeWarps][32];
    __shared__ float2 shared_ml[kMergeWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, my_row = (lane >> 1) & 3;
    const bool fine = split * 16 == HD;
    const int place = fine ? lane & 15 : lane, few = fine ? 1 : kMergeFew;
    // Units are numbered by the (row, query head) pairs of a KV head in fours, every sequence and every tile of rows beginning a new one: with n rows before it, a sequence
    // begins behind ceil(n g / 4) fours, as many broken ones as there are sequences before it, and as many as whole tiles fit n.  (The host sees to it that the number of
    // units stays within 32 bits.)
    const auto first_unit = [&](int b) {
        const unsigned first = rows_begin<true>(P.cu_rows, b, P.n_rows);
        return (int)((first * P.g + 3u) / 4u + first / P.chunk) + b;
    };
    const int chunk_units = (P.chunk * P.g + 3) / 4;
    const int per = TreeScan<kMergeWarps>::per(P);
    unit0[threadIdx.x] = (int)threadIdx.x * per < P.n_seqs ? first_unit((int)threadIdx.x * per) : INT_MAX;
    scan.fill<true>(P);
    __syncthreads();
    const int total = scan.total(), cols = HD / split;
    const TreeCut cut(total, P.blocks);
    const unsigned tasks = ((unsigned)(P.n_rows * P.g + 3) / 4u + (unsigned)P.n_rows / P.chunk + P.n_seqs) * P.n_kv * split;
    bool waited = false;
    for (unsigned p0 = blockIdx.x; p0 < tasks; p0 += gridDim.x * group) {
        if (warp < group) {
            const unsigned task = p0 + warp * gridDim.x;
            TreeUnit q;
            q.n = 0;
            if (task < tasks && total > 0) {
                const unsigned u = task / split, unit_u = u / P.n_kv;
                const int unit = (int)unit_u;
                q.col = (int)(task - u * split) * cols;
                q.h = (int)(u - unit_u * P.n_kv);
                // the last sequence that begins at or before the unit, and the tiles before it
                int tile0 = 0;
                int w = 0;
                while (w < kMergeWarps - 1 && unit0[(w + 1) * 32] <= unit) tile0 += scan.warp_sum[w++];
                const int t = w * 32 + max(0, 31 - __clz(__ballot_sync(0xffffffffu, unit0[w * 32 + lane] <= unit)));
                tile0 += scan.before[t];
                int b = t * per;
                const int end = min(b + per, P.n_seqs) - 1;
                while (b < end && first_unit(b + 1) <= unit) tile0 += tree_tiles(P, tree_seq<true>(P, b++));
                const TreeSeq s = tree_seq<true>(P, b);
                const int u0 = unit - first_unit(b);
                if (u0 >= 0 && u0 < s.chunks * chunk_units && s.tiles > 0) {
                    const int c = u0 / chunk_units, rows = min(P.chunk, s.rows - c * P.chunk) * P.g;
                    q.row = (u0 - c * chunk_units) * 4;
                    if (q.row < rows) {
                        q.first = s.first;
                        q.j0 = c * P.chunk * P.g + q.row;
                        q.rows = min(4, rows - q.row);
                        tile0 += (q.h * s.chunks + c) * s.tiles;
                        q.block0 = cut.owner(tile0);
                        q.n = cut.owner(tile0 + s.tiles - 1) - q.block0 + 1;
                        q.late = cut.begin(q.block0) < tile0;
                    }
                }
            }
            if (lane == 0) shared_unit[warp] = q;
        }
        if (!waited) {
            grid_dep_wait();   // the parts are there
            grid_dep_launch();
        }
        waited = true;
        __syncwarp();
        bool many = false;
        if (warp < group) {
            const TreeUnit& q = shared_unit[warp];
            many = q.n > few;
            if (q.n > 1 && !many) {
                TreeMergeRow<T, HD> row(P, q, my_row, lane);
#pragma unroll 1
                for (int c = 0; c < HD; c += 64) {   // two groups of 32 columns
                    float m = -CUDART_INF_F, l = 0.f;
                    float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
                    for (int i = 0; i < q.n; i += 2) {   // two parts at a time
                        const int at = q.slot(i, P.blocks) * P.part_rows, next = q.slot(i + 1, P.blocks) * P.part_rows;
                        const bool two = i + 1 < q.n;
                        const float2 a = row.ml[at], b = two ? row.ml[next] : make_float2(-CUDART_INF_F, 0.f);
                        float4 x[2], y[2];
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            x[g] = *reinterpret_cast<const float4*>(row.o + at * HD + (c + g * 32) * 4);
                            if (two) y[g] = *reinterpret_cast<const float4*>(row.o + next * HD + (c + g * 32) * 4);
                        }
                        const float mx = fmaxf(m, fmaxf(a.x, b.x)), ref = mx == -CUDART_INF_F ? 0.f : mx, keep = exp2f(m - ref), fa = exp2f(a.x - ref), fb = exp2f(b.x - ref);
                        m = mx;
                        l = l * keep + fa * a.y + fb * b.y;
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            tree_scale(o[g], keep);
                            tree_add(o[g], fa, x[g]);
                            if (two) tree_add(o[g], fb, y[g]);
                        }
                    }
#pragma unroll
                    for (int g = 0; g < 2; ++g) row.store(P, q, my_row, lane, c + g * 32, o[g], l);
                }
            }
        }
        if (!__syncthreads_or(many)) continue;
        // Together, one unit after the other.  Fine units: every half warp has parts of its own.  Others: warps in turn have a group of 32 columns, and the parts are shared out among
        // those of a group.
        const int groups = fine ? 1 : cols / 32, halves = fine ? 2 : 1, step = kMergeWarps / groups * halves;
#pragma unroll 1
        for (int k = 0; k < group; ++k) {
            const TreeUnit& q = shared_unit[k];
            if (q.n <= few) continue;   // the same for the whole block
            TreeMergeRow<T, HD> row(P, q, my_row, place);
            const int c = q.col + warp % groups * 32;
            float m = -CUDART_INF_F, l = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int i0 = warp / groups * halves + (fine ? lane >> 4 : 0); i0 < q.n; i0 += kMergeDeep * step) tree_gather<HD>(P, q, row.ml, row.o + c * 4, i0, step, m, l, o);
            shared_o[warp][lane] = o;
            shared_ml[warp][lane] = make_float2(m, l);
            __syncthreads();
            if (warp < groups) {
                // fine: half a warp's lanes add up the other half's as well
                float mx = -CUDART_INF_F, sum = 0.f;
                for (int t = warp; t < kMergeWarps; t += groups) mx = fmaxf(mx, fmaxf(shared_ml[t][lane].x, shared_ml[t][lane ^ (halves - 1) * 16].x));
                const float ref = mx == -CUDART_INF_F ? 0.f : mx;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int t = 0; t < kMergeWarps / groups * halves; ++t) {
                    const int w = warp + (t / halves) * groups, at = lane ^ (t & (halves - 1)) * 16;
                    const float2 ml = shared_ml[w][at];
                    const float f = exp2f(ml.x - ref);
                    sum += f * ml.y;
                    tree_add(v, f, shared_o[w][at]);
                }
                if (place == lane) row.store(P, q, my_row, place, c, v, sum);
            }
            __syncthreads();
        }
        // a warp still looks for units to take together while another could be at the next ones
        if (p0 + gridDim.x * group < tasks) __syncthreads();
    }
}

}  // namespace sdv
