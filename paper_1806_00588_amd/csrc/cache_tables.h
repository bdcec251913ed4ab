// Block tables of a paged cache (lsh_cache_advance): rows continue their parents', as the state rows of lsh_beam_advance do, by
// their tables instead of by copies; blocks are taken for new tokens, every new token gets its slot.
//
// Nothing but the tables says which blocks are in use: a block is free if no row continues with it and no row begins a copy of
// it in this call.  So beams that die need no release, and there is no list that could disagree with the tables.  Free blocks
// are given out lowest first, to rows in order: the result is a function of the inputs.
//
// Bound by latency: three dependent passes (who continues with what; how many blocks each row needs and which are free; tables
// and slots) over a few bytes.
#pragma once
#include "device_utils.h"

namespace lshbeam {

struct TablesArgs {
    int S, B, T, n_blocks, block, width;
    const int32_t* parents;      // [R] beam of the sentence, or null: every row is its own parent
    const int32_t* n_new;        // [R] or null: T, and 0 for rows without a parent
    const int32_t* tables_in;    // [R, width]
    const int32_t* lengths_in;   // [R]
    int32_t* tables_out;
    int32_t* lengths_out;
    int32_t* slots;              // [R, T]
    int32_t* copy_from;          // [R]
    int32_t* shared;             // [S]
    int32_t* status;             // [2]
    struct RowPlan* plan;        // workspace [R]
    int32_t* base;               // workspace [R]: where the row's blocks begin in `free_ids`
    int32_t* free_ids;           // workspace [n_blocks]
    uint8_t* used;               // workspace [n_blocks rounded up to 16]
};

// What a row continues with and asks for.
struct RowPlan {
    int32_t old_len;    // tokens it continues with
    int32_t n_new;      // tokens to come
    int32_t need;       // blocks to take; -1: the row asks for more than its table or T holds
    int32_t copy;       // block that its first new block begins as a copy of, or -1
};

__device__ __forceinline__ int blocks_of(int tokens, int block) { return (int)(((int64_t)tokens + block - 1) / block); }

// The row whose table row r continues (-1: none), and how many tokens of it.
__device__ __forceinline__ int parent_row(const TablesArgs& a, int r, int* tokens) {
    const int b = a.parents ? a.parents[r] : r % a.B;
    *tokens = 0;
    if (b < 0 || b >= a.B) return -1;
    const int p = r - r % a.B + b;
    *tokens = min(max(a.lengths_in[p], 0), (int)min((int64_t)a.width * a.block, (int64_t)INT32_MAX));
    return p;
}

// Row r's plan; `or_all` is an OR over the threads that share the work (all of them call it).
template <typename F>
__device__ __forceinline__ RowPlan plan_row(const TablesArgs& a, int r, int p, int old_len, int thread, int threads, F or_all) {
    int want = a.n_new ? max(a.n_new[r], 0) : (p < 0 ? 0 : a.T);
    RowPlan plan{old_len, want, 0, -1};
    const int n_old = blocks_of(old_len, a.block);
    bool others = false;
    const bool partial = want > 0 && old_len % a.block != 0;
    const int32_t last = partial ? a.tables_in[(int64_t)p * a.width + n_old - 1] : -1;
    if (partial) {   // does another row of the sentence continue with the block that this one would write on?
        const int r0 = r - r % a.B;
        for (int o = thread; o < a.B; o += threads) {
            int tokens = 0;
            const int q = r0 + o == r ? -1 : parent_row(a, r0 + o, &tokens);
            if (q >= 0 && blocks_of(tokens, a.block) >= n_old) others |= a.tables_in[(int64_t)q * a.width + n_old - 1] == last;
        }
    }
    others = or_all(others);
    const int64_t len = (int64_t)old_len + want;
    if (want > a.T || len > (int64_t)a.width * a.block || len > INT32_MAX) { plan.need = -1; return plan; }
    plan.copy = others && last >= 0 && last < a.n_blocks ? last : -1;
    plan.need = blocks_of((int)len, a.block) - n_old + (plan.copy >= 0);
    return plan;
}

__global__ void __launch_bounds__(256) k_tables_clear(TablesArgs a) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i * 16 < a.n_blocks) reinterpret_cast<uint4*>(a.used)[i] = make_uint4(0, 0, 0, 0);
}

// grid = R workgroups: the row continues its parent's table; the blocks that it names are in use.
__global__ void __launch_bounds__(256) k_tables_rows(TablesArgs a) {
    const int r = blockIdx.x;
    int old_len;
    const int p = parent_row(a, r, &old_len);
    const RowPlan plan = plan_row(a, r, p, old_len, threadIdx.x, 256, [](bool v) { return __syncthreads_or(v) != 0; });
    if (threadIdx.x == 0) a.plan[r] = plan;
    const int n_old = blocks_of(old_len, a.block);
    for (int j = threadIdx.x; j < a.width; j += 256) {
        const int32_t id = j < n_old ? a.tables_in[(int64_t)p * a.width + j] : -1;
        a.tables_out[(int64_t)r * a.width + j] = id;
        if (id >= 0 && id < a.n_blocks) a.used[id] = 1;
    }
}

// One workgroup: where each row's blocks begin among the free ones, the free ones (as many as are wanted), the status.
__global__ void __launch_bounds__(1024) k_tables_take(TablesArgs a) {
    __shared__ uint32_t wsum[17];
    const int R = a.S * a.B;
    int64_t want = 0;
    int refused = 0;
    for (int r0 = 0; r0 < R; r0 += 1024) {
        const int r = r0 + threadIdx.x;
        const int need = r < R ? a.plan[r].need : 0;
        uint32_t total = 0;
        const uint32_t incl = block_incl_scan((uint32_t)max(need, 0), wsum, &total);
        if (r < R) a.base[r] = (int32_t)min(want + incl - max(need, 0), (int64_t)INT32_MAX);
        want += total;
        refused += __syncthreads_count(need < 0);
    }
    int64_t found = 0;
    for (int i0 = 0; i0 < a.n_blocks && found < want; i0 += 16 * 1024) {
        const int i = i0 + 16 * threadIdx.x;
        uint32_t bits = 0;
        if (i < a.n_blocks) {
            const uint4 v = *reinterpret_cast<const uint4*>(a.used + i);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 16; ++k) bits |= (uint32_t)(i + k < a.n_blocks && !(w[k >> 2] >> (8 * (k & 3)) & 1u)) << k;
        }
        uint32_t total = 0;
        const uint32_t n = __builtin_popcount(bits);
        int64_t at = found + block_incl_scan(n, wsum, &total) - n;
        for (; bits; bits &= bits - 1, ++at)
            if (at < want) a.free_ids[at] = i + __builtin_ctz(bits);
        found += total;
    }
    if (threadIdx.x == 0) {
        a.status[0] = (int32_t)min(max(want - found, (int64_t)0), (int64_t)INT32_MAX);
        a.status[1] = refused;
    }
}

// Tables, lengths and slots of row r, once it is known that all rows get what they ask for (`ok`), else without new tokens.
__device__ __forceinline__ void finish_row(const TablesArgs& a, int r, const RowPlan& plan, bool ok, const int32_t* free_ids, int thread, int threads) {
    const int n_old = blocks_of(plan.old_len, a.block), first = n_old - (plan.copy >= 0);
    const int len = ok ? plan.old_len + plan.n_new : plan.old_len, end = blocks_of(len, a.block);
    int32_t* table = a.tables_out + (int64_t)r * a.width;
    if (ok)
        for (int j = first + thread; j < end; j += threads) table[j] = free_ids[j - first];
    for (int t = thread; t < a.T; t += threads) {
        int32_t slot = -1;
        if (ok && t < plan.n_new) {
            const int pos = plan.old_len + t, j = pos / a.block;
            const int32_t id = j >= first ? free_ids[j - first] : table[j];
            if (id >= 0 && id < a.n_blocks) slot = id * a.block + pos % a.block;
        }
        a.slots[(int64_t)r * a.T + t] = slot;
    }
    if (thread == 0) {
        a.lengths_out[r] = len;
        a.copy_from[r] = ok ? plan.copy : -1;
    }
}

// Leading blocks that all rows of sentence s with tokens have in common, whole blocks only.  One row: all of its whole blocks.
// More: a block taken in this call is nobody else's, so it ends where the first row's new blocks begin at the latest.
// `lead` is shared memory; ends with a barrier.
__device__ __forceinline__ void shared_blocks(const TablesArgs& a, int s, const RowPlan* plan, bool ok, int* lead, int* rows, int* ref) {
    if (threadIdx.x == 0) { lead[0] = lead[1] = INT32_MAX; *rows = 0; *ref = INT32_MAX; }
    __syncthreads();
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const RowPlan p = plan[b];
        const int len = ok ? p.old_len + p.n_new : p.old_len;
        if (len <= 0) continue;
        atomicAdd(rows, 1);
        atomicMin(ref, b);
        atomicMin(&lead[0], len / a.block);
        atomicMin(&lead[1], blocks_of(p.old_len, a.block) - (ok && p.copy >= 0));
    }
    __syncthreads();
    const int n = *rows, first = *ref, most = n == 0 ? 0 : n == 1 ? lead[0] : min(lead[0], lead[1]);
    __syncthreads();
    if (threadIdx.x == 0) lead[0] = most;
    __syncthreads();
    if (n > 1) {
        const int32_t* t0 = a.tables_out + (int64_t)s * a.B * a.width;
        for (int b = first + 1; b < a.B; ++b) {
            const RowPlan p = plan[b];
            if ((ok ? p.old_len + p.n_new : p.old_len) <= 0) continue;
            for (int j = threadIdx.x; j < most; j += blockDim.x)
                if (t0[(int64_t)b * a.width + j] != t0[(int64_t)first * a.width + j]) { atomicMin(&lead[0], j); break; }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) a.shared[s] = lead[0];
}

// grid = R workgroups.
__global__ void __launch_bounds__(256) k_tables_finish(TablesArgs a) {
    __shared__ int lead[2], rows, ref;
    const int r = blockIdx.x;
    const bool ok = a.status[0] == 0 && a.status[1] == 0;
    if (a.shared && r % a.B == 0) shared_blocks(a, r / a.B, a.plan + r, ok, lead, &rows, &ref);
    const RowPlan plan = a.plan[r];
    finish_row(a, r, plan, ok, a.free_ids + (ok ? a.base[r] : 0), threadIdx.x, 256);
}

}  // namespace lshbeam
