// Block tables of a paged cache (lsh_cache_advance): rows continue their parents', as the state rows of lsh_beam_advance do, by
// their tables instead of by copies; blocks are taken for new tokens, every new token gets its slot.
//
// Nothing but the tables says which blocks are in use: a block is free if no row continues with it and no row begins a copy of
// it in this call.  So beams that die need no release, and there is no list that could disagree with the tables.  Free blocks
// are given out lowest first, to rows in order: the result is a function of the inputs.
//
// Bound by latency: three dependent passes (who continues with what; how many blocks each row needs and which are free; tables
// and slots) over a few bytes.  Small calls are one workgroup's (k_tables_once), which has plans and a bitmap of the pool in LDS:
// 12 rows of 20 blocks 6.5 to 7.5 us, where the four launches of the others take 15 to 16 to be made (640 rows of 256 blocks: kernels of 1.8,
// 5.1, 4.0 and 5.6).
#pragma once
#include "device_utils.h"

namespace lshbeam {

struct RowPlan;
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
    RowPlan* plan;        // workspace [R]
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

// Row r's plan, but for what other rows say: `last` is the block that it would write on, or -1 (a whole number of blocks, or nothing new).
__device__ __forceinline__ RowPlan plan_row(const TablesArgs& a, int r, int p, int old_len, int32_t* last) {
    const RowPlan plan{old_len, a.n_new ? max(a.n_new[r], 0) : (p < 0 ? 0 : a.T), 0, -1};
    *last = plan.n_new > 0 && old_len % a.block != 0 ? a.tables_in[(int64_t)p * a.width + old_len / a.block] : -1;
    return plan;
}
// Does row q (-1: none) with `tokens` tokens continue with block `last` where row r's table ends?
__device__ __forceinline__ bool continues(const TablesArgs& a, int q, int tokens, int old_len, int32_t last) {
    const int n = blocks_of(old_len, a.block);
    return q >= 0 && blocks_of(tokens, a.block) >= n && a.tables_in[(int64_t)q * a.width + n - 1] == last;
}
// `others`: another row continues with the row's last block.
__device__ __forceinline__ void finish_plan(const TablesArgs& a, RowPlan& plan, int32_t last, bool others) {
    const int64_t len = (int64_t)plan.old_len + plan.n_new;
    if (plan.n_new > a.T || len > (int64_t)a.width * a.block || len > INT32_MAX) { plan.need = -1; return; }
    plan.copy = others && last >= 0 && last < a.n_blocks ? last : -1;
    plan.need = blocks_of((int)len, a.block) - blocks_of(plan.old_len, a.block) + (plan.copy >= 0);
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
    int32_t last;
    RowPlan plan = plan_row(a, r, p, old_len, &last);
    bool others = false;
    if (last >= 0)
        for (int o = threadIdx.x; o < a.B; o += 256) {
            int tokens = 0;
            const int q = r - r % a.B + o;
            if (q != r) others |= continues(a, parent_row(a, q, &tokens), tokens, old_len, last);
        }
    finish_plan(a, plan, last, __syncthreads_or(others) != 0);
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
// More: a block taken in this call is nobody else's, so it ends where the first row's new blocks begin at the latest.  `threads`
// threads share the work; min_all makes each of four values the smallest of all of them.
template <typename F>
__device__ __forceinline__ int shared_blocks(const TablesArgs& a, int s, const RowPlan* plan, bool ok, int thread, int threads, F min_all) {
    auto length = [&](const RowPlan& p) { return ok ? p.old_len + p.n_new : p.old_len; };
    int v[4] = {INT32_MAX, INT32_MAX, INT32_MAX, INT32_MAX};   // first row, last one (negative), whole blocks, old ones
    for (int b = thread; b < a.B; b += threads) {
        const RowPlan p = plan[b];
        if (length(p) <= 0) continue;
        v[0] = min(v[0], b);
        v[1] = min(v[1], -b);
        v[2] = min(v[2], length(p) / a.block);
        v[3] = min(v[3], blocks_of(p.old_len, a.block) - (ok && p.copy >= 0));
    }
    min_all(v);
    const int first = v[0], last = -v[1], most = min(v[2], v[3]);
    if (first == INT32_MAX) return 0;
    if (first == last) return v[2];
    const int32_t* t0 = a.tables_out + (int64_t)s * a.B * a.width;
    v[0] = most;
    for (int j = thread; j < most; j += threads) {
        const int32_t id = t0[(int64_t)first * a.width + j];
        bool same = true;
        for (int b0 = first + 1; b0 <= last; b0 += 8) {   // eight rows asked for together, whether they have tokens or not
            int32_t other[8];
            bool empty[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int b = min(b0 + k, last);
                other[k] = t0[(int64_t)b * a.width + j];
                empty[k] = length(plan[b]) <= 0;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) same &= empty[k] | (other[k] == id);
        }
        if (!same) v[0] = min(v[0], j);
    }
    min_all(v);
    return v[0];
}

__device__ __forceinline__ void wave_min(int (&v)[4]) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = min(v[k], __shfl_xor(v[k], off, kWave));
}

// grid = R workgroups, after S more if blocks in common are asked for.
__global__ void __launch_bounds__(256) k_tables_finish(TablesArgs a) {
    __shared__ int least[4][4];
    const int common = a.shared ? a.S : 0, r = (int)blockIdx.x - common;
    const bool ok = (a.status[0] | a.status[1]) == 0;
    if (r < 0) {
        const int s = blockIdx.x;
        const int n = shared_blocks(a, s, a.plan + (int64_t)s * a.B, ok, threadIdx.x, 256, [&](int (&v)[4]) {
            wave_min(v);
            __syncthreads();
            if (lane_id() == 0)
#pragma unroll
                for (int k = 0; k < 4; ++k) least[wave_id()][k] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = min(min(least[0][k], least[1][k]), min(least[2][k], least[3][k]));
        });
        if (threadIdx.x == 0) a.shared[s] = n;
        return;
    }
    const RowPlan plan = a.plan[r];
    finish_row(a, r, plan, ok, a.free_ids + (ok ? a.base[r] : 0), threadIdx.x, 256);
}

// One workgroup does all of it.  LDS: the rows' plans, parents, last blocks and bases, a bit for each block of the pool (18 KB at most).
// The limits are where it is no slower than the four launches, which take 15 to 16 us a call whatever the size: 12 rows of 20 blocks
// 7.8 us a call, 64 of 64 10.7 (a pool of 4096 blocks; 13 with 131 072), 4 of 1024 8 to 15; beyond them 160 rows of 64 23, 1024 of 32 70, and
// one row of 4096 new tokens 57, 8 of 512 13 to 18.
constexpr int kOnceRows = 64, kOnceEntries = 4096, kOnceBlocks = 1 << 17, kOnceNew = 256, kOnceSlots = 2048;
inline bool tables_at_once(int64_t R, int64_t width, int64_t n_blocks, int64_t T) {
    return R <= kOnceRows && R * width <= kOnceEntries && n_blocks <= kOnceBlocks && T <= kOnceNew && R * T <= kOnceSlots;
}
inline size_t once_lds(int64_t R, int64_t n_blocks) { return (size_t)R * (sizeof(RowPlan) + 16) + (size_t)((n_blocks + 31) / 32) * 4; }
__global__ void __launch_bounds__(1024) k_tables_once(TablesArgs a) {
    extern __shared__ int32_t once[];
    __shared__ uint32_t wsum[17];
    const int R = a.S * a.B, tid = threadIdx.x, words = (a.n_blocks + 31) / 32;
    RowPlan* plan = reinterpret_cast<RowPlan*>(once);
    int32_t *parent = once + 4 * R, *last = parent + R, *others = last + R, *base = others + R;
    uint32_t* used = reinterpret_cast<uint32_t*>(base + R);
    for (int i = tid; i < words; i += 1024) used[i] = 0;
    int32_t my_last = -1;
    if (tid < R) {
        int old_len;
        const int p = parent_row(a, tid, &old_len);
        plan[tid] = plan_row(a, tid, p, old_len, &my_last);
        parent[tid] = p;
        last[tid] = my_last;
        others[tid] = 0;
    }
    __syncthreads();
    for (int e = tid; e < R * a.B; e += 1024) {          // pairs of rows of a sentence
        const int r = (int)((unsigned)e / (unsigned)a.B), q = r - r % a.B + e - r * a.B;
        if (q != r && last[r] >= 0 && continues(a, parent[q], plan[q].old_len, plan[r].old_len, last[r])) others[r] = 1;
    }
    for (int e = tid; e < R * a.width; e += 1024) {      // the parents' tables; their blocks are in use
        const int r = (int)((unsigned)e / (unsigned)a.width), j = e - r * a.width;
        const int32_t id = j < blocks_of(plan[r].old_len, a.block) ? a.tables_in[(int64_t)parent[r] * a.width + j] : -1;
        a.tables_out[e] = id;
        if (id >= 0 && id < a.n_blocks) atomicOr(&used[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    int need = 0;
    if (tid < R) {
        RowPlan mine = plan[tid];
        finish_plan(a, mine, my_last, others[tid] != 0);
        plan[tid] = mine;
        need = mine.need;
    }
    const int refused = __syncthreads_count(need < 0);
    uint32_t want = 0, found = 0;                        // (at most R * (width + 1) blocks)
    const uint32_t incl = block_incl_scan((uint32_t)max(need, 0), wsum, &want);
    if (tid < R) base[tid] = (int32_t)(incl - max(need, 0));
    const int per = (words + 1023) / 1024;               // words of a thread, one after the other
    auto free_bits = [&](int i) {
        uint32_t bits = ~used[i];
        if (i == words - 1 && (a.n_blocks & 31)) bits &= (1u << (a.n_blocks & 31)) - 1u;
        return bits;
    };
    uint32_t n = 0;
    for (int i = tid * per; i < min(words, (tid + 1) * per); ++i) n += __builtin_popcount(free_bits(i));
    uint32_t at = block_incl_scan(n, wsum, &found) - n;
    for (int i = tid * per; i < min(words, (tid + 1) * per) && at < want; ++i)
        for (uint32_t bits = free_bits(i); bits && at < want; bits &= bits - 1) a.free_ids[at++] = 32 * i + __builtin_ctz(bits);
    const bool ok = refused == 0 && want <= found;
    if (tid == 0) {
        a.status[0] = want > found ? (int32_t)(want - found) : 0;
        a.status[1] = refused;
    }
    __syncthreads();                                     // (the workgroup's writes are there for all of it)
    // 16 lanes to a row
    for (int r = tid >> 4; r < R; r += 64) finish_row(a, r, plan[r], ok, a.free_ids + (ok ? base[r] : 0), tid & 15, 16);
    if (a.shared)
        for (int s = wave_id(); s < a.S; s += 16) {
            const int lead = shared_blocks(a, s, plan + s * a.B, ok, lane_id(), kWave, [](int (&v)[4]) { wave_min(v); });
            if (lane_id() == 0) a.shared[s] = lead;
        }
}

}  // namespace lshbeam
