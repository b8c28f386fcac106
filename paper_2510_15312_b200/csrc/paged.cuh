// Slots and rotary append of a cache kept in pages (include/sdv.h: sdv_paged_slots, sdv_rope_append).
#pragma once
#include <cuda_fp16.h>
#include <limits.h>

#include "../../include/sdv.h"
#include "ptx.cuh"
#include "tree_plan.h"

namespace sdv {

// Largest index i in [0, n] with a[i] <= x, for ascending a[0 .. n]; -1 if there is none.
__device__ __forceinline__ int last_not_above(const int* a, int n, int x) {
    int lo = -1, hi = n + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ------------------------------------------------------------------------------------------ slots
constexpr int kSlotThreads = 512;

// Every block sums up all sequences' needs (they are few: at most 4096) and takes its share of the rows and of the new table entries, which find their
// sequence by bisection in shared memory: one launch and no block waits for another.  Bound by latency: launch, a round trip to
// memory for the lengths, one for the tables (4.4 us for 5 sequences of 20 rows, 5.4 for 1000 of up to 47 rows and 33298 pages).
// With parents each row walks up to its root, a load a step, 50 ns: made for draft trees, a prompt of 9000 rows whose parents are given as well takes 0.47 ms, and one of 262144 rows,
// the most that the host lets through with parents, 33 ms.
struct SlotShared {
    int row0[SDV_MAX_SEQUENCES + 1];   // first row of every sequence
    int need0[SDV_MAX_SEQUENCES + 1];  // pages needed by the sequences before
    int warp_sum[kSlotThreads / 32];
    int refused, head;
};

// Pages that sequence b wants; need: those it lacks, 0 where its row of the table is too short for it (fits = false).
__device__ __forceinline__ long long slots_want(const sdv_slots_args& a, int b, int rows, int& need, bool& narrow) {
    const long long tokens = (long long)max(a.kv_len[b], 0) + rows;
    const long long want = rows > 0 ? (tokens + a.page_size - 1) / a.page_size : 0;
    narrow = want > a.table_width;
    need = narrow ? 0 : max(0, (int)want - min(max(a.n_held[b], 0), a.table_width));
    return want;
}

__global__ void __launch_bounds__(kSlotThreads) paged_slots_kernel(const __grid_constant__ sdv_slots_args a) {
    __shared__ SlotShared s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = a.n_seqs;
    grid_dep_wait();
    grid_dep_launch();   // behind the wait: what comes next may rely on all that came before
    const int head = max(*a.free_state, 0);
    // needs of this thread's sequences, summed up over the block.  The sum of all needs stays below 2^31: each is at most
    // table_width, and the host refuses n_seqs * table_width beyond that.
    const int per = (B + kSlotThreads - 1) / kSlotThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    int sum = 0;
    for (int b = b0; b < b1; ++b) {
        int need;
        bool narrow;
        s.row0[b] = rows_begin(a.cu_rows, b, a.n_rows);
        slots_want(a, b, rows_count(a.cu_rows, b, a.n_rows), need, narrow);
        s.need0[b] = sum;
        sum += need;
    }
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
    }
    if (lane == 31) s.warp_sum[warp] = incl;
    if (tid == 0) {
        s.refused = 0;
        s.head = head;
        s.row0[B] = rows_begin(a.cu_rows, B, a.n_rows);
    }
    __syncthreads();
    int base = incl - sum;
    for (int w = 0; w < warp; ++w) base += s.warp_sum[w];
    for (int b = b0; b < b1; ++b) s.need0[b] += base;
    if (tid == kSlotThreads - 1) s.need0[B] = base + sum;
    __syncthreads();
    const auto taken = [&](int b) {   // whether sequence b's need is met
        const int need = s.need0[b + 1] - s.need0[b];
        return need == 0 || (long long)head + s.need0[b + 1] <= a.n_free;
    };
    if (blockIdx.x == 0) {
        int refused = 0, last = head;
        for (int b = b0; b < b1; ++b) {
            int need;
            bool narrow;
            slots_want(a, b, max(0, s.row0[b + 1] - s.row0[b]), need, narrow);
            const bool fits = !narrow && taken(b);
            a.n_held_out[b] = a.n_held[b] + (fits ? need : 0);
            if (fits && need) last = head + s.need0[b + 1];
            refused += fits ? 0 : 1;
        }
        if (last > head) atomicMax(&s.head, last);
        if (refused) atomicAdd(&s.refused, refused);
        __syncthreads();
        if (tid == 0) {
            a.free_state_out[0] = s.head;
            a.free_state_out[1] = s.refused;
        }
    }
    const int stride = (int)gridDim.x * kSlotThreads, first = (int)blockIdx.x * kSlotThreads + tid;
    // new entries of the block table: entry e of all needs is the list's e-th page behind its head
    const int entries = s.need0[B];
    for (int e = first; e < entries; e += stride) {
        const int b = last_not_above(s.need0, B, e);
        if (b < B && taken(b)) a.block_table[b * a.table_stride + max(a.n_held[b], 0) + (e - s.need0[b])] = a.free_pages[head + e];
    }
    // rows
    for (int r = first; r < a.n_rows; r += stride) {
        const int b = last_not_above(s.row0, B, r);
        int slot = -1, position = 0;
        if (b >= 0 && b < B && r < s.row0[b + 1]) {
            const int local = r - s.row0[b], length = max(a.kv_len[b], 0);
            int depth = local;
            if (a.parent) {
                depth = 0;
                for (int i = local; i > 0; ++depth) {
                    const int p = a.parent[s.row0[b] + i];
                    i = p < 0 || p >= i ? 0 : p;
                }
            }
            position = (int)min((long long)length + depth, (long long)INT_MAX);
            int need;
            bool narrow;
            slots_want(a, b, s.row0[b + 1] - s.row0[b], need, narrow);
            if (!narrow && taken(b)) {
                const long long token = (long long)length + local;
                const int page_at = (int)(token / a.page_size), offset = (int)(token % a.page_size), held = min(max(a.n_held[b], 0), a.table_width);
                // entries behind the held ones may be on their way by another block: from the list, where they come from
                const int page = page_at < held ? a.block_table[b * a.table_stride + page_at] : a.free_pages[head + s.need0[b] + (page_at - held)];
                const long long at = (long long)page * a.page_size + offset;
                slot = page < 0 || at > INT_MAX ? -1 : (int)at;
            }
        }
        a.slots[r] = slot;
        a.positions[r] = position;
    }
}

// ------------------------------------------------------------------------------------------ rotary embedding and append
constexpr int kRopeThreads = 256;

template <typename T> struct Half16;
template <> struct Half16<__nv_bfloat16> {
    static constexpr uint32_t kExponent = 0x7f80u;   // all ones: infinite or NaN
    static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
};
template <> struct Half16<__half> {
    static constexpr uint32_t kExponent = 0x7c00u;
    static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};

// W 16-bit elements moved at once.
template <int W> struct Words;
template <> struct Words<8> { typedef uint4 type; };
template <> struct Words<2> { typedef uint32_t type; };
template <> struct Words<1> { typedef uint16_t type; };
template <typename T, int W>
union Elements {
    typename Words<W>::type w;
    T e[W];
    __device__ __forceinline__ Elements() {}
};

// Cosines and sines of n rows from row t0 on, [row][pair].  An angle is worked out in 64 bits as a fraction of a turn: a position of 10^6 in fp32 is off by up to 0.03 rad.
__device__ __forceinline__ void rope_turns(const sdv_rope_args& a, int t0, int n, float2* turn) {
    const int half = a.rot_dim / 2;
    grid_dep_wait();
    grid_dep_launch();   // behind the wait: what comes next may rely on all that came before
    for (int i = threadIdx.x; i < n * half; i += kRopeThreads) {
        const int t = i / half, p = i - t * half;
        const double turns = (double)a.positions[t0 + t] * a.frequencies[p] * 0.15915494309189533577;   // 1 / (2 pi)
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[i] = make_float2(c * a.factor, s * a.factor);
    }
}

template <typename T>
__device__ __forceinline__ void rope_turn(T& lo, T& hi, float2 cs) {
    const float b = Half16<T>::up(lo), d = Half16<T>::up(hi);
    lo = Half16<T>::down(b * cs.x - d * cs.y);
    hi = Half16<T>::down(d * cs.x + b * cs.y);
}

// Where row r of a head goes in the pages; null: nowhere.
template <typename T>
__device__ __forceinline__ T* rope_place(const sdv_rope_args& a, const sdv_pages& pages, void* base, int r, int h) {
    const int slot = a.slots[r];
    if (slot < 0 || slot >= (long long)pages.n_pages * pages.page_size) return nullptr;
    const int page = slot / pages.page_size, token = slot - page * pages.page_size;
    return (T*)base + page * pages.page_stride + h * pages.head_stride + token * pages.token_stride;
}

// A block takes `tokens` rows: their cosines and sines once, then all heads of q, k and v in units of 2 W elements, W on either side of the pairs (half layout: only where
// the halves are multiples of W) or W neighbouring pairs.  A unit is read whole before it is written, so q may be turned in place.
// Bound by memory for prompts (8191 rows of 24 + 8 heads of 128: 28.9 us, 5.8 TB/s), by latency for the rows of a step.
template <typename T, bool INTERLEAVED, int W>
__global__ void __launch_bounds__(kRopeThreads, 8) rope_append_kernel(const __grid_constant__ sdv_rope_args a, const __grid_constant__ sdv_pages pages, int tokens) {
    extern __shared__ float2 turn[];   // [token][pair] cosine, sine
    const int half = a.rot_dim / 2, t0 = (int)blockIdx.x * tokens, n = min(tokens, a.n_rows - t0);
    rope_turns(a, t0, n, turn);
    __syncthreads();
    const int per_head = a.head_dim / (2 * W), q_units = a.q ? a.n_q_heads * per_head : 0, k_units = a.k ? a.n_kv_heads * per_head : 0, units = q_units + 2 * k_units;
    for (int i = threadIdx.x; i < n * units; i += kRopeThreads) {
        const int t = i / units, r = t0 + t;
        int u = i - t * units;
        const bool is_q = u < q_units, is_v = u >= q_units + k_units;
        u -= is_q ? 0 : is_v ? q_units + k_units : q_units;
        const int h = u / per_head, at = u - h * per_head;
        const T* src;
        T* dst;
        if (is_q) {
            src = (const T*)a.q + r * a.q_row_stride + h * a.q_head_stride;
            dst = (T*)a.q_out + r * a.out_row_stride + h * a.out_head_stride;
        } else {
            src = is_v ? (const T*)a.v + r * a.v_row_stride + h * a.v_head_stride : (const T*)a.k + r * a.k_row_stride + h * a.k_head_stride;
            dst = rope_place<T>(a, pages, is_v ? pages.v : pages.k, r, h);
            if (!dst) continue;
        }
        // elements e0 .. and e1 .. of the head; pairs p .. p + W - 1 where they are turned
        const int pair = at * W;
        int e0 = at * 2 * W, e1 = e0 + W;
        const bool turned = !is_v && pair < half;
        if (turned && !INTERLEAVED) {
            e0 = pair;
            e1 = pair + half;
        }
        typedef typename Words<W>::type Word;
        Elements<T, W> x, y;
        x.w = *reinterpret_cast<const Word*>(src + e0);
        y.w = *reinterpret_cast<const Word*>(src + e1);
        if (turned) {
            const float2* cs = turn + t * half + pair;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                if (INTERLEAVED && W > 1 && pair + j >= half) break;
                // the pair's members: in the half layout x[j], y[j]; interleaved, neighbours in the 2 W elements x, y
                T& lo = INTERLEAVED ? (2 * j < W ? x.e[(2 * j) % W] : y.e[(2 * j) % W]) : x.e[j];
                T& hi = INTERLEAVED ? (2 * j + 1 < W ? x.e[(2 * j + 1) % W] : y.e[(2 * j + 1) % W]) : y.e[j];
                rope_turn(lo, hi, cs[j]);
            }
        }
        *reinterpret_cast<Word*>(dst + e0) = x.w;
        *reinterpret_cast<Word*>(dst + e1) = y.w;
    }
}

// Half layout with halves that are no multiple of eight: the partners of eight aligned elements do not lie on a 16-byte boundary.  The heads of q and k go through shared memory,
// `heads` of a row at a time, and are turned there in place, two pairs a thread; global memory sees 16-byte accesses only.  A thread keeps its place within the heads and
// steps from head to head without a division.  (Two bytes at a time from global memory, 51 pairs took 123 us; so they take 46, where 56,
// which need no stage, take 32: the rows of a block follow each other, load, turn and store of each behind barriers.)
template <typename T>
__global__ void __launch_bounds__(kRopeThreads, 8) rope_staged_kernel(const __grid_constant__ sdv_rope_args a, const __grid_constant__ sdv_pages pages, int tokens, int heads) {
    extern __shared__ uint4 stage[];   // [head][16 bytes] | [token][pair] cosine, sine
    const int half = a.rot_dim / 2, t0 = (int)blockIdx.x * tokens, n = min(tokens, a.n_rows - t0), per_head = a.head_dim / 8, words = (half + 1) / 2;
    float2* turn = reinterpret_cast<float2*>(stage + heads * per_head);
    rope_turns(a, t0, n, turn);
    const int q_heads = a.q ? a.n_q_heads : 0, k_heads = a.k ? a.n_kv_heads : 0;
    const int my_head = (int)threadIdx.x / per_head, my_chunk = (int)threadIdx.x - my_head * per_head, head_step = kRopeThreads / per_head;   // 16 bytes of a head (at most 32)
    const int my_row = (int)threadIdx.x / words, my_pair = ((int)threadIdx.x - my_row * words) * 2, row_step = kRopeThreads / words;           // two pairs (at most 64)
    for (int t = 0; t < n; ++t) {
        const int r = t0 + t;
        const float2* cs = turn + t * half + my_pair;
        for (int h0 = 0; h0 < q_heads + k_heads; h0 += heads) {
            const int count = min(heads, q_heads + k_heads - h0);
            if (my_head < head_step) {
                for (int h = my_head; h < count; h += head_step) {
                    const int hd = h0 + h;
                    const T* src = hd < q_heads ? (const T*)a.q + r * a.q_row_stride + hd * a.q_head_stride : (const T*)a.k + r * a.k_row_stride + (hd - q_heads) * a.k_head_stride;
                    stage[h * per_head + my_chunk] = *reinterpret_cast<const uint4*>(src + my_chunk * 8);
                }
            }
            __syncthreads();
            if (my_row < row_step) {
                const bool two = my_pair + 1 < half;
                const float2 c0 = cs[0], c1 = two ? cs[1] : c0;
                for (int h = my_row; h < count; h += row_step) {
                    T* lo = reinterpret_cast<T*>(stage + h * per_head) + my_pair;
                    T* hi = lo + half;
                    if (two) {
                        Elements<T, 2> x, y;
                        x.w = *reinterpret_cast<const uint32_t*>(lo);
                        y.e[0] = hi[0];
                        y.e[1] = hi[1];
                        rope_turn(x.e[0], y.e[0], c0);
                        rope_turn(x.e[1], y.e[1], c1);
                        *reinterpret_cast<uint32_t*>(lo) = x.w;
                        hi[0] = y.e[0];
                        hi[1] = y.e[1];
                    } else {   // the last of an odd number of pairs
                        T x = lo[0], y = hi[0];
                        rope_turn(x, y, c0);
                        lo[0] = x;
                        hi[0] = y;
                    }
                }
            }
            __syncthreads();
            if (my_head < head_step) {
                for (int h = my_head; h < count; h += head_step) {
                    const int hd = h0 + h;
                    T* dst = hd < q_heads ? (T*)a.q_out + r * a.out_row_stride + hd * a.out_head_stride : rope_place<T>(a, pages, pages.k, r, hd - q_heads);
                    if (dst) *reinterpret_cast<uint4*>(dst + my_chunk * 8) = stage[h * per_head + my_chunk];
                }
            }
            __syncthreads();
        }
        if (my_head < head_step) {
            for (int h = my_head; h < k_heads; h += head_step) {   // values are only moved
                T* dst = rope_place<T>(a, pages, pages.v, r, h);
                if (dst) *reinterpret_cast<uint4*>(dst + my_chunk * 8) = *reinterpret_cast<const uint4*>((const T*)a.v + r * a.v_row_stride + h * a.v_head_stride + my_chunk * 8);
            }
        }
    }
}

}  // namespace sdv
