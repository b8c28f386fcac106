// Verification of drafted tokens against the target's probabilities (include/sdv.h: sdv_verify_sampled).
#pragma once
#include "paged.cuh"

namespace sdv {

constexpr int kVerifyThreads = 512, kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyTile = 512;             // vocabulary entries a warp sums up at a time: sixteen a lane
constexpr int kVerifyMaxCluster = 8;

__device__ __forceinline__ void st_cluster_f8(uint32_t addr, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory"); }

// What the drawn token's distribution is made of.
struct VerifyRest {
    const float *p, *q;      // target's row; rejected draft's row or null
    const int* out;          // tokens without a share (shared memory)
    int n_out, vocab;
    bool wide;               // rows start on 16-byte boundaries
};

// Sixteen entries of a tile: lane's four from each of four places `apart` entries apart (0 past the end), as the fp32 pairs whose differences are the shares: an entry without
// a share is 0 - 0.  The difference of two fp32 numbers and their sum over a vocabulary are near enough exact in 64 bits.
__device__ __forceinline__ void verify_load(const VerifyRest& d, int first, int apart, float (&p)[16], float (&q)[16]) {
    if (first + 3 * apart + 3 < d.vocab && d.wide) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(d.p + first + k * apart));
            p[4 * k] = v.x; p[4 * k + 1] = v.y; p[4 * k + 2] = v.z; p[4 * k + 3] = v.w;
        }
        if (d.q) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(d.q + first + k * apart));
                q[4 * k] = v.x; q[4 * k + 1] = v.y; q[4 * k + 2] = v.z; q[4 * k + 3] = v.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = first + (i >> 2) * apart + (i & 3);
            p[i] = at < d.vocab ? __ldcg(d.p + at) : 0.f;
            q[i] = d.q && at < d.vocab ? __ldcg(d.q + at) : 0.f;
        }
    }
    for (int n = 0; n < d.n_out; ++n) {
        const int at = d.out[n] - first;
        if ((unsigned)at < (unsigned)(3 * apart + 4)) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (at == (i >> 2) * apart + (i & 3)) p[i] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (!d.q) q[i] = 0.f;
        const bool has = p[i] > 0.f && p[i] > q[i];   // NaN has none
        p[i] = has ? p[i] : 0.f;
        q[i] = has ? fmaxf(q[i], 0.f) : 0.f;
    }
}

// A cluster takes one sequence.  All its blocks go through the drafts (at most 64 rows, one gather each; a row is looked at on its own, with the shares of its earlier
// siblings, and the path is walked once); each sums up its part of the distribution that remains, tile by tile in a fixed order; every block writes its sum into the others' shared memory, and the block whose
// part holds the drawn token reads that one tile again.  Sums in 64 bits: a token's share may be 10^-9 of the whole, fp32 sums would draw its neighbour.  A token's place is that of the
// exact sums up to a relative 10^-15.  Bound by the chain of round trips (lengths, rows, shares, row, exchange, tile): 7.5 us for one
// sequence; 64 at a vocabulary of 152064 with draft probabilities 17.7 us, 15.7 with the 78 MB in L2, of which reading them takes 11.9 (memory is 41 % busy, conversions 29 %, the 64-bit pipe 9 %).  Two blocks an SM (their registers), all resident at once.
__global__ void __launch_bounds__(kVerifyThreads, 2) verify_sampled_kernel(const __grid_constant__ sdv_verify_args a, int tiles_per_block) {
    extern __shared__ double tile_sum[];   // [tiles_per_block]
    __shared__ int tok[SDV_TREE_ROWS], par[SDV_TREE_ROWS], out[SDV_TREE_ROWS], path[SDV_TREE_ROWS], child[SDV_TREE_ROWS];
    __shared__ float share[SDV_TREE_ROWS];
    __shared__ unsigned char again[SDV_TREE_ROWS];
    __shared__ int n_path, n_out, rejected_row;
    __shared__ double sums[2][kVerifyMaxCluster];   // of every block's share
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int CS = (int)cluster_size(), rank = (int)cluster_rank(), b = (int)blockIdx.x / CS;
    grid_dep_wait();
    grid_dep_launch();   // behind the wait: what comes next may rely on all that came before
    const int first = rows_begin(a.cu_rows, b, a.n_rows), all = rows_count(a.cu_rows, b, a.n_rows), T = min(all, SDV_TREE_ROWS);
    if (blockIdx.x == 0) {   // rows of no sequence
        const int from = rows_begin(a.cu_rows, a.n_seqs, a.n_rows), until = rows_begin(a.cu_rows, 0, a.n_rows);
        for (int r = tid; r < a.n_rows; r += kVerifyThreads) {
            if (r >= until && r < from) continue;
            a.out_tokens[r] = a.out_rows[r] = -1;
            if (a.out_slots) a.out_slots[r] = -1;
        }
    }
    if (T == 0) {   // the whole cluster
        if (rank == 0 && tid == 0) a.accept_len[b] = -1;
        return;
    }
    cluster_arrive_relaxed();   // waited for before anything is written to another block, which has started by then
    const float draw = a.uniforms[first];
    const int i = tid;
    float u = 0.f, q = 1.f;
    if (i < SDV_TREE_ROWS) {
        int p = -1, x = -1;
        float s = 0.f;
        if (i > 0 && i < T) {
            p = a.parent ? a.parent[first + i] : i - 1;
            if (p < 0 || p >= i) p = 0;
            x = a.tokens[first + i];
            u = a.uniforms[first + i];
            if (x >= 0 && x < a.vocab) {
                s = __ldcg(a.target + (first + p) * a.target_stride + x);
                if (a.draft) {
                    q = __ldcg(a.draft + (first + i) * a.draft_stride + x);
                    if (q < 0.f) q = 0.f;
                }
            }
        }
        tok[i] = x;
        par[i] = p;
        share[i] = s > 0.f ? s : 0.f;
        child[i] = SDV_TREE_ROWS;
    }
    __syncthreads();
    // siblings: whether an earlier one carries the same token, then what the earlier ones leave
    if (i < T) {
        bool same = false;
        if (a.parent)
            for (int s = 1; s < i; ++s) same |= par[s] == par[i] && tok[s] == tok[i];
        again[i] = same;
    }
    __syncthreads();
    if (i < T) {
        bool yes = false;
        if (i > 0) {
            if (a.draft) {
                yes = (double)u * (double)q < (double)share[i];
            } else {
                double gone = 0.0;
                if (a.parent)
                    for (int s = 1; s < i; ++s)
                        if (par[s] == par[i] && !again[s]) gone += (double)share[s];
                yes = !again[i] && (double)u * (1.0 - gone) < (double)share[i];
            }
        }
        if (yes) atomicMin(&child[par[i]], i);   // the first accepted child is followed
    }
    __syncthreads();
    if (tid == 0) {
        int n = 0, at = 0;
        path[0] = 0;
        while (child[at] < SDV_TREE_ROWS) {
            at = child[at];
            path[++n] = at;
        }
        n_path = n;
        n_out = 0;
        rejected_row = -1;
    }
    __syncthreads();
    const int a_len = n_path, last = path[a_len];
    if (i > 0 && i < T && par[i] == last) {   // a rejected child: every child of the last accepted row is one
        if (a.draft) rejected_row = i;
        else out[atomicAdd(&n_out, 1)] = tok[i];   // any order: a set
    }
    if (rank == 0) {
        // rows from the sequence's first on; the entry of the drawn token is written last, by whoever finds it
        for (int r = tid; r < all; r += kVerifyThreads) {
            a.out_rows[first + r] = r <= a_len ? path[min(r, SDV_TREE_ROWS - 1)] : -1;
            if (r != a_len) a.out_tokens[first + r] = r < a_len ? tok[path[min(r + 1, SDV_TREE_ROWS - 1)]] : -1;
        }
        if (a.out_slots) {
            for (int r = tid; r < all; r += kVerifyThreads) {
                int to = -1;
                for (int k = 1; k <= a_len; ++k)
                    if (path[k] == r && k != r) to = a.slots[first + k];
                a.out_slots[first + r] = to;
            }
        }
        if (tid == 0) a.accept_len[b] = a_len;
    }
    __syncthreads();
    VerifyRest d;
    d.vocab = a.vocab;
    d.p = a.target + (first + last) * a.target_stride;
    d.q = rejected_row >= 0 ? a.draft + (first + rejected_row) * a.draft_stride : nullptr;
    d.out = out;
    d.n_out = n_out;
    d.wide = (((uintptr_t)d.p | (uintptr_t)d.q) & 15) == 0;
    const int tiles = (a.vocab + kVerifyTile - 1) / kVerifyTile, tile0 = rank * tiles_per_block, mine = max(0, min(tiles - tile0, tiles_per_block));
    for (int attempt = 0;; ++attempt) {
        for (int t = warp; t < mine; t += kVerifyWarps) {
            float p[16], q[16];
            verify_load(d, (tile0 + t) * kVerifyTile + lane * 4, 128, p, q);
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += d.q ? (double)p[i] - (double)q[i] : (double)p[i];
#pragma unroll
            for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            if (lane == 0) tile_sum[t] = sum;
        }
        __syncthreads();
        if (warp == 0) {
            double sum = 0.0;
            for (int t = lane; t < mine; t += 32) sum += tile_sum[t];
#pragma unroll
            for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            if (attempt == 0) cluster_wait();
            // to every block of the cluster; each attempt has a place of its own, so that nobody waits for the readers
            if (lane < CS) st_cluster_f8(map_shared_rank(smem_u32(&sums[attempt][rank]), lane), sum);
            __syncwarp();
        } else if (attempt == 0) {
            cluster_wait();
        }
        cluster_sync();
        double before = 0.0, whole = 0.0;
        for (int k = 0; k < CS; ++k) whole += sums[attempt][k];
        const double goal = (double)draw * whole;
        int holder = -1;   // the first block behind which the cumulative sum exceeds the goal, else the last one with a share
        {
            double cum = 0.0;
            bool done = false;
            for (int k = 0; k < CS && !done; ++k) {
                const double x = sums[attempt][k];
                if (x > 0.0) {
                    holder = k;
                    before = cum;
                    done = cum + x > goal;
                }
                cum += x;
            }
        }
        if (!(whole > 0.0)) {
            if (attempt == 0 && (d.q || d.n_out)) {   // nothing is left: the target's distribution itself
                d.q = nullptr;
                d.n_out = 0;
                __syncthreads();   // tile_sum has been read
                continue;
            }
            if (rank == 0 && tid == 0) a.out_tokens[first + a_len] = -1;
            return;
        }
        if (rank != holder || warp > 0) return;
        // tile: the same rule over this block's tiles
        double cum = before, at_before = before;
        int at = -1;
        bool done = false;
        for (int t0 = 0; t0 < mine && !done; t0 += 32) {
            const double x = t0 + lane < mine ? tile_sum[t0 + lane] : 0.0;
            double incl = x;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const double v = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl += v;
            }
            const unsigned some = __ballot_sync(0xffffffffu, x > 0.0), over = __ballot_sync(0xffffffffu, x > 0.0 && cum + incl > goal);
            if (some) {
                const int l = over ? __ffs(over) - 1 : 31 - __clz(some);
                at = t0 + l;
                at_before = cum + __shfl_sync(0xffffffffu, incl - x, l);
                done = over != 0;
            }
            cum += __shfl_sync(0xffffffffu, incl, 31);
        }
        // entry: again over the tile's, a lane sixteen in a row
        float p[16], q[16];
        const int from = (tile0 + at) * kVerifyTile + lane * 16;
        verify_load(d, from, 4, p, q);
        double part = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) part += (double)p[i] - (double)q[i];
        double incl = part;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const double v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        double sum = at_before + (incl - part);
        int hit = -1, some = -1;   // the first entry behind which the sum exceeds the goal, the last one with a share
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const double w = (double)p[i] - (double)q[i];
            sum += w;
            if (w > 0.0) {
                some = i;
                if (hit < 0 && sum > goal) hit = i;
            }
        }
        const unsigned has = __ballot_sync(0xffffffffu, some >= 0), over = __ballot_sync(0xffffffffu, hit >= 0);
        const int l = over ? __ffs(over) - 1 : has ? 31 - __clz(has) : 0;
        if (lane == l) a.out_tokens[first + a_len] = from + (over ? hit : some);
        return;
    }
}

}  // namespace sdv
