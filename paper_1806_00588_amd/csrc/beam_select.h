// Beam selection from dense logits (lsh_beam_select).  Per hidden row r of S * B
//   lse_r = log sum_w exp x[r, w] over the allowed words,   score[r, w] = beam_scores[r] + x[r, w] - lse_r
// and per sentence the N best (beam, word) by (score in 64 bits, lower beam, lower word).
//
// The logits are read once: k_select_tiles leaves the largest logit of every tile of 128 words (16 lanes of 8 words: one
// 16-byte load of 16-bit words, two of fp32) and per wave the pair (max, sum of exp).  k_select_words, a workgroup per sentence,
// finds from those the scores that a winner can have and opens the tiles that hold such a score.  A score grows with the logit
// within a row, so a tile's best score is that of its largest logit, in any rounding.  Where a sentence has at most 64 pieces of
// 512 words, k_select_small does all of it from registers in one launch.
//
// Sums: exp in fp32 of differences from the wave's largest (the dominant terms err by an ulp of their own), eight of them added
// in fp32, those sums in fp64; lse and scores in fp64.  Scores of different beams are compared, and an lse that is off by 1e-6 (what
// fp32 sums give at 200 000 words) would change the places of neighbours some 1e-6 apart: one in 10^4 pairs.
#pragma once
#include <hip/hip_fp16.h>

#include "device_utils.h"

namespace lshbeam {

enum { kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2 };
template <int TYPE> struct WordOf { using type = uint16_t; };
template <> struct WordOf<kTypeF32> { using type = float; };

constexpr int kSelWords = 8;                   // words of a lane in a row, one after the other
constexpr int kSelTile = 16 * kSelWords;       // words of a record
constexpr int kSelPiece = kWave * kSelWords;   // words of a wave at a time: four tiles
constexpr int kSelBatch = 4;                   // pieces whose loads a wave has under way together
constexpr int kSelThreads = 1024;              // of the workgroup of a sentence
constexpr int kSelListed = 2048;               // tiles, and words, that it can list
constexpr int kSelSmall = 64;                  // pieces of a sentence that k_select_small takes: four of a wave

struct SelPart { double sum; float max; float pad; };   // of a wave's words of a row: sum exp(x - max)

struct SelArgs {
    const void* x;            // logits [R, ld]
    int64_t ld;
    const uint8_t* allowed;   // bit w % 8 of byte w / 8 of row r: word w may follow; null: all may
    int64_t allowed_pitch;    // bytes; 0: one row for all
    const float* scores;      // [R]
    int V, B, N;
    int tiles;                // of a row
    int pieces;               // pieces of a wave of k_select_tiles
    int parts;                // its waves of a row
    float* tile_max;          // [R, tiles]
    SelPart* part;            // [R, parts]
    int32_t* out_beam;        // [S, N]
    int32_t* out_word;
    float* out_score;
    float* out_lse;           // [R] or null
};

// exp(d) for d <= 0 (or NaN): 2^(d log2 e), log2 e in two parts -- with one, every term would be off by |d| * 1.3e-8, all on the same side.
__device__ __forceinline__ float exp_diff(float d) {
    return __builtin_amdgcn_exp2f(fmaf(d, 1.44269502162933349609375f, d * 1.92596302e-8f));
}

template <int TYPE> __device__ __forceinline__ float word_f32(typename WordOf<TYPE>::type v) {
    if constexpr (TYPE == kTypeF32) return v;
    else if constexpr (TYPE == kTypeBf16) return __uint_as_float((uint32_t)v << 16);
    else return __half2float(__ushort_as_half(v));
}

// Logits of words w .. w + 7 of a row as they lie in memory, and which of them count: those inside the row that are allowed.  Rows
// may begin at any element.
template <int TYPE> struct Words {
    using T = typename WordOf<TYPE>::type;
    uint32_t w[TYPE == kTypeF32 ? 8 : 4];
    uint32_t bits;
    __device__ __forceinline__ void load(const SelArgs& a, int64_t r, int at) {
        bits = 0;
        if (at >= a.V) return;
        const T* p = static_cast<const T*>(a.x) + r * a.ld + at;
        bits = 0xffu;
        if (a.allowed) bits = a.allowed[r * a.allowed_pitch + (at >> 3)];
        if (at + kSelWords <= a.V) {
#pragma unroll
            for (int h = 0; h < (TYPE == kTypeF32 ? 2 : 1); ++h) {
                const Chunk16U<T> v = *reinterpret_cast<const Chunk16U<T>*>(p + 4 * h);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[4 * h + i] = v.w[i];
            }
        } else {
            bits &= 0xffu >> (at + kSelWords - a.V);
#pragma unroll
            for (int i = 0; i < kSelWords; ++i) {
                const uint32_t v = at + i < a.V ? (uint32_t)word_bits(p[i]) : 0u;
                if constexpr (TYPE == kTypeF32) w[i] = v;
                else w[i >> 1] = i & 1 ? w[i >> 1] | v << 16 : v;
            }
        }
    }
    static __device__ __forceinline__ uint32_t word_bits(float v) { return __float_as_uint(v); }
    static __device__ __forceinline__ uint32_t word_bits(uint16_t v) { return v; }
    // ... as fp32, -inf where they do not count
    __device__ __forceinline__ void get(float (&x)[kSelWords]) const {
#pragma unroll
        for (int i = 0; i < kSelWords; ++i) {
            if constexpr (TYPE == kTypeF32) x[i] = __uint_as_float(w[i]);
            else x[i] = word_f32<TYPE>((T)(w[i >> 1] >> (16 * (i & 1)) & 0xffffu));
        }
        if (bits != 0xffu) {
#pragma unroll
            for (int i = 0; i < kSelWords; ++i) x[i] = bits >> i & 1u ? x[i] : -INFINITY;
        }
    }
};
template <int TYPE>
__device__ __forceinline__ void load_words(const SelArgs& a, int64_t r, int at, float (&x)[kSelWords]) {
    Words<TYPE> w;
    w.load(a, r, at);
    w.get(x);
}

__device__ __forceinline__ float max_of(const float (&x)[kSelWords]) {   // (a NaN is not the largest; it shows in the sum)
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}
// sum exp(x - m); an infinite m counts as 0, so that +inf gives +inf, nothing gives 0 and a NaN gives NaN
__device__ __forceinline__ float sum_exp(const float (&x)[kSelWords], float m) {
    const float z = isinf(m) ? 0.f : m;
    float e[kSelWords];
#pragma unroll
    for (int i = 0; i < kSelWords; ++i) e[i] = exp_diff(x[i] - z);
    return ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// grid = R * ceil(parts / 4) workgroups of four waves; a wave takes `pieces` pieces of a row, one after the other.  Bound by memory: 640
// rows of 200 000 words, bf16, 256 MB in 64 us (4.0 TB/s).
template <int TYPE>
__global__ void __launch_bounds__(256) k_select_tiles(SelArgs a) {
    const int per_row = (a.parts + 3) >> 2;
    const int64_t r = blockIdx.x / per_row;
    const int part = (blockIdx.x - (int)r * per_row) * 4 + __builtin_amdgcn_readfirstlane(wave_id());
    if (part >= a.parts) return;
    const int ln = lane_id();
    const int n_pieces = (a.V + kSelPiece - 1) / kSelPiece;
    const int end = min(n_pieces, (part + 1) * a.pieces);
    float m = -INFINITY;
    double sum = 0.0;
    Words<TYPE> next[kSelBatch];
    auto ask = [&](int p) {
#pragma unroll
        for (int i = 0; i < kSelBatch; ++i)
            if (p + i < end) next[i].load(a, r, (p + i) * kSelPiece + ln * kSelWords);
    };
    ask(part * a.pieces);
    for (int p = part * a.pieces; p < end; p += kSelBatch) {
        Words<TYPE> now_[kSelBatch];
#pragma unroll
        for (int i = 0; i < kSelBatch; ++i) now_[i] = next[i];
        ask(p + kSelBatch);              // (while these are worked on)
        float now = m;
#pragma unroll
        for (int i = 0; i < kSelBatch; ++i) {
            if (p + i >= end) continue;
            float x[kSelWords];
            now_[i].get(x);
            const float top = row16_max(max_of(x));
            now = fmaxf(now, top);
            const int t = (p + i) * 4 + (ln >> 4);
            if ((ln & 15) == 0 && t < a.tiles) a.tile_max[r * a.tiles + t] = top;
        }
        now = wave_max_f32(now);
        if (now > m) {
            if (m > -INFINITY) sum *= exp((double)m - (double)now);
            m = now;
        }
#pragma unroll
        for (int i = 0; i < kSelBatch; ++i) {
            if (p + i >= end) continue;
            float x[kSelWords];
            now_[i].get(x);
            sum += (double)sum_exp(x, m);
        }
    }
    sum = wave_sum_f64(sum);
    if (ln == 0) a.part[r * a.parts + part] = SelPart{sum, m, 0.f};
}

// ---- keys ---------------------------------------------------------------------------------------

// A score's place among all scores: 64 bits, larger is better; 0 where the score is not finite in fp32.
__device__ __forceinline__ uint64_t score_key(double s) {
    const float f = (float)s;
    if (!(fabsf(f) < INFINITY)) return 0;
    const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);   // (-0 and 0 are equal)
    return (u >> 63) ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ float key_score(uint64_t k) {
    const uint64_t u = (k >> 63) ? k & 0x7fffffffffffffffull : ~k;
    return (float)__longlong_as_double((long long)u);
}
__device__ __forceinline__ uint32_t pair_of(int beam, int word) { return (uint32_t)beam << 24 | (uint32_t)word; }

struct SelShared {
    double off[256];                    // of each beam: score - log of the sum of exp(x - top), ...
    float top[256];                     // ... its largest logit
    float rough[256];                   // off in 32 bits
    uint64_t key[kSelListed];
    uint32_t pair[kSelListed];
    uint32_t tile[kSelListed];
    uint32_t hist[256];
    uint32_t wsum[kSelThreads / kWave + 1];
    float wave_best[kSelThreads / kWave];
    uint32_t n_tiles, n_words, digit, need, above;
};

// beam score + (x - lse), lse = top + log sum: the difference of two logits first, which loses nothing where both are huge (a row of
// nothing but the type's lowest value).
__device__ __forceinline__ double score_of(const SelShared& sh, int b, float x) { return sh.off[b] + ((double)x - (double)sh.top[b]); }

// A key such that at least N of the threads' keys reach it, if as many are not 0 (else 1): the N-th largest, or one not far below.
// All threads call it; it ends with a barrier.
__device__ __forceinline__ uint64_t nth_of_threads(SelShared& sh, uint64_t key, int N) {
    uint64_t prefix = 0;
    uint32_t need = (uint32_t)N;
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
        __syncthreads();
        if (key && (shift == 56 || (key >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[(uint32_t)(key >> shift) & 255u], 1u);
        __syncthreads();
        if (threadIdx.x < kWave) {   // lane l: bins 255 - 4 l down to 252 - 4 l
            const int hi = 255 - 4 * lane_id();
            const uint32_t c0 = sh.hist[hi], c1 = sh.hist[hi - 1], c2 = sh.hist[hi - 2], c3 = sh.hist[hi - 3];
            const uint32_t incl = wave_incl_scan(c0 + c1 + c2 + c3), before = incl - (c0 + c1 + c2 + c3);
            if (lane_id() == kWave - 1 && incl < need) sh.digit = 256;   // fewer than N
            if (before < need && incl >= need) {
                uint32_t b = before, d = hi;
                if (b + c0 < need) { b += c0; --d; if (b + c1 < need) { b += c1; --d; if (b + c2 < need) { b += c2; --d; } } }
                sh.digit = d;
                sh.need = need - b;
                sh.above = sh.hist[d];
            }
        }
        __syncthreads();
        const uint32_t d = sh.digit;
        if (d > 255) return 1;           // (only in the first round)
        prefix = prefix << 8 | d;
        need = sh.need;
        if (sh.above <= need + 32) return prefix << shift;   // the whole bin may come along
        __syncthreads();
    }
    return prefix;
}

// The score in 32 bits, -inf where there is none.  It errs by 2^-23 of the largest of its parts.
__device__ __forceinline__ float rough_score(const SelShared& sh, int b, float x) {
    const float f = sh.rough[b] + (x - sh.top[b]);
    return fabsf(f) < INFINITY ? f : -INFINITY;
}

// Which scores can be among the N best, given that each thread knows the rough score of a word of its own (-inf: none): at least N of
// the threads' scores are let in, and few more.  Scores are told apart by their distance from the best, in sixteenths; one sixteenth
// more than needed is let in, which is far more than rough scores err by as long as the best is below 2^15 (no row's off is above
// the best, so that what is let in has no large parts).  Where it is not, or the N-th is 16 and more away, `none` says so.
// All threads call it; it ends with a barrier.
struct SelLimit {
    float best, width;
    bool none;
    __device__ __forceinline__ bool lets(float f) const { return (best - f) * 16.f < width; }
};
__device__ __forceinline__ SelLimit limit_of_threads(SelShared& sh, float f, int N) {
    const float top = wave_max_f32(f);
    if (lane_id() == 0) sh.wave_best[wave_id()] = top;
    if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
    __syncthreads();
    SelLimit to{row16_max(sh.wave_best[lane_id() & 15]), 0.f, true};
    const float d = (to.best - f) * 16.f;
    if (d < 256.f) atomicAdd(&sh.hist[(int)d], 1u);   // (-inf - -inf is NaN: not counted)
    __syncthreads();
    // lane l of every wave: bins 4 l .. 4 l + 3
    const uint32_t* h = sh.hist + 4 * lane_id();
    const uint32_t c0 = h[0], c1 = h[1], c2 = h[2], c3 = h[3], incl = wave_incl_scan(c0 + c1 + c2 + c3), before = incl - (c0 + c1 + c2 + c3);
    const uint64_t here = __ballot(before < (uint32_t)N && incl >= (uint32_t)N);
    if (here && fabsf(to.best) < 32768.f) {
        int b = 4 * lane_id();
        if (before + c0 < (uint32_t)N) { ++b; if (before + c0 + c1 < (uint32_t)N) { ++b; if (before + c0 + c1 + c2 < (uint32_t)N) ++b; } }
        to.width = (float)((int)wave_read_lane((uint32_t)b, __builtin_ctzll(here)) + 2);
        to.none = false;
    }
    __syncthreads();
    return to;
}

// m: the row's largest logit, sum: of exp(x - m).
__device__ __forceinline__ void put_offset(const SelArgs& a, SelShared& sh, int64_t r, int b, float m, double sum, float score) {
    const double lg = log(sum);          // (of nothing: -inf)
    sh.off[b] = (double)score - lg;
    sh.top[b] = m;
    sh.rough[b] = (float)sh.off[b];
    if (a.out_lse) a.out_lse[r] = (float)(m > -INFINITY ? (double)m + lg : lg);
}
// The row's lse from its parts, by a wave; also its offset in shared memory.  first: the first 64 parts and the row's score, asked
// for while the row before was worked on.
struct RowStart {
    SelPart part;
    float score;
    __device__ __forceinline__ void ask(const SelArgs& a, int64_t r, const SelPart* of_row, int parts) {
        part = lane_id() < parts ? of_row[lane_id()] : SelPart{0.0, -INFINITY, 0.f};
        score = a.scores[r];
    }
};
__device__ __forceinline__ void row_offset(const SelArgs& a, SelShared& sh, int64_t r, int b, const SelPart* part, int parts, const RowStart& first) {
    const int ln = lane_id();
    float m = first.part.max;
    for (int i = ln + kWave; i < parts; i += kWave) m = fmaxf(m, part[i].max);
    m = wave_max_f32(m);
    double sum = 0.0;
    for (int i = ln; i < parts; i += kWave) {
        const SelPart p = i < kWave ? first.part : part[i];
        sum += isinf(m) || isinf(p.max) ? p.sum : p.sum * exp((double)p.max - (double)m);
    }
    sum = wave_sum_f64(sum);
    if (ln == 0) put_offset(a, sh, r, b, m, sum, first.score);
}

// The same for a row of at most 16 parts, by 16 lanes: lane i's part p (sum 0, max -inf: none).  8 sentences of 60 beams, 753 words,
// bf16: 20.0 us a call, 24.1 with a wave for each row.
__device__ __forceinline__ void row_offset16(const SelArgs& a, SelShared& sh, int64_t r, int b, const SelPart& p, float score) {
    const float m = row16_max(p.max);
    double sum = isinf(m) || isinf(p.max) ? p.sum : p.sum * exp((double)p.max - (double)m);
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
    if ((lane_id() & 15) == 0) put_offset(a, sh, r, b, m, sum, score);
}

// The N best of sh.key / sh.pair [n], n <= kSelListed, to the outputs of sentence s; empty places behind them.  A word's rank is how
// many are before it: lane j of every wave holds words j and j + 64, a ballot for each word that the wave ranks (a thread for each word
// and a loop over the others waited for LDS in every turn).
__device__ __forceinline__ void rank_words(const SelArgs& a, SelShared& sh, int s, int n) {
    const int ln = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    constexpr int kWaves = kSelThreads / kWave;
    uint64_t k[2];
    uint32_t p[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const bool in = ln + kWave * h < n;
        k[h] = in ? sh.key[ln + kWave * h] : 0;
        p[h] = in ? sh.pair[ln + kWave * h] : 0xffffffffu;
    }
    auto rank_one = [&](uint64_t key, uint32_t pair) {
        int rank = __popcll(__ballot(k[0] > key || (k[0] == key && p[0] < pair)));
        if (n > kWave) rank += __popcll(__ballot(k[1] > key || (k[1] == key && p[1] < pair)));
        for (int o = 2 * kWave; o < n; o += kWave) {
            const bool in = o + ln < n;
            const uint64_t ko = in ? sh.key[o + ln] : 0;
            const uint32_t po = in ? sh.pair[o + ln] : 0xffffffffu;
            rank += __popcll(__ballot(ko > key || (ko == key && po < pair)));
        }
        if (ln == 0 && rank < a.N) {
            const size_t at = (size_t)s * a.N + rank;
            a.out_beam[at] = (int32_t)(pair >> 24);
            a.out_word[at] = (int32_t)(pair & 0xffffffu);
            a.out_score[at] = key_score(key);
        }
    };
#pragma unroll
    for (int h = 0; h < 2; ++h)
        for (int e = wv; e < kWave && e + kWave * h < n; e += kWaves)
            rank_one((uint64_t)wave_read_lane((uint32_t)(k[h] >> 32), e) << 32 | wave_read_lane((uint32_t)k[h], e), wave_read_lane(p[h], e));
    for (int e = 2 * kWave + wv; e < n; e += kWaves) rank_one(sh.key[e], sh.pair[e]);
    for (int i = n + threadIdx.x; i < a.N; i += kSelThreads) {
        const size_t at = (size_t)s * a.N + i;
        a.out_beam[at] = -1;
        a.out_word[at] = -1;
        a.out_score[at] = -INFINITY;
    }
}

// The N best of ALL words of a sentence whatever their ties, several times over the logits: for lists that overflow.  The N-th
// largest key by radix, tiles without a part in it passed over; the words above it in any order, those equal to it in order of
// beam and word as far as there is room.
template <int TYPE>
__device__ __forceinline__ void select_all_words(const SelArgs& a, SelShared& sh, int s) {
    const int wv = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id();
    const int pieces = (a.V + kSelPiece - 1) / kSelPiece, units = a.B * pieces;
    uint64_t prefix = 0;
    uint32_t need = (uint32_t)a.N;
    bool all = false;                    // fewer than N words have a score
    for (int shift = 56; shift >= 0 && !all; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
        __syncthreads();
        for (int u = wv; u < units; u += kSelThreads / kWave) {
            const int b = u / pieces, w = (u - b * pieces) * kSelPiece + ln * kSelWords;
            if (w >= a.V) continue;
            float x[kSelWords];
            load_words<TYPE>(a, (int64_t)s * a.B + b, w, x);
#pragma unroll
            for (int i = 0; i < kSelWords; ++i) {
                const uint64_t k = score_key(score_of(sh, b, x[i]));
                if (k && (shift == 56 || (k >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[(uint32_t)(k >> shift) & 255u], 1u);
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int d = 255;
            while (d >= 0 && sh.hist[d] < need) need -= sh.hist[d--];
            sh.digit = d < 0 ? 256u : (uint32_t)d;
            sh.need = need;
        }
        __syncthreads();
        all = sh.digit > 255;            // (only in the first round)
        prefix = prefix << 8 | (sh.digit & 255u);
        need = sh.need;
    }
    // prefix: the N-th largest key; `need` of the words that have it belong to the N best
    if (threadIdx.x == 0) sh.n_words = 0;
    __syncthreads();
    uint32_t ties = 0;                   // of the units so far (the same in all threads)
    for (int u0 = 0; u0 < units; u0 += kSelThreads / kWave) {
        const int u = u0 + wv, b = min(u / pieces, a.B - 1), w = (u - b * pieces) * kSelPiece + ln * kSelWords;
        uint64_t k[kSelWords];
        uint32_t mine = 0;
        if (u < units && w < a.V) {
            float x[kSelWords];
            load_words<TYPE>(a, (int64_t)s * a.B + b, w, x);
#pragma unroll
            for (int i = 0; i < kSelWords; ++i) { k[i] = score_key(score_of(sh, b, x[i])); mine += !all && k[i] == prefix; }
        } else {
#pragma unroll
            for (int i = 0; i < kSelWords; ++i) k[i] = 0;
        }
        uint32_t total = 0;
        uint32_t at = ties + block_incl_scan(mine, sh.wsum, &total) - mine;
#pragma unroll
        for (int i = 0; i < kSelWords; ++i) {
            const bool tie = !all && k[i] == prefix;
            const bool in = tie ? at < need : k[i] && (all || k[i] > prefix);
            at += tie;
            if (in) {
                const uint32_t to = atomicAdd(&sh.n_words, 1u);
                if (to < kSelListed) { sh.key[to] = k[i]; sh.pair[to] = pair_of(b, w + i); }
            }
        }
        ties += total;
    }
    __syncthreads();
    rank_words(a, sh, s, (int)sh.n_words);
}

// grid = S workgroups, each a chain of loads and barriers: 10 us for 12 rows of 40 000 words, 16 for 64 times 10 of 200 000.
template <int TYPE>
__global__ void __launch_bounds__(kSelThreads) k_select_words(SelArgs a) {
    __shared__ SelShared sh;
    const int s = blockIdx.x, wv = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id();
    const int64_t r0 = (int64_t)s * a.B;
    // Up to 256 units of 64 tiles of a row: wave w has units w, w + 16, ..., its sixteen under way together and kept.  More of them:
    // the parts first, then the tiles of those that can have a winner (2 sentences of 56 beams, 193 407 words in fp32: all tiles,
    // twice, 92 us a call, parts first below 40).
    constexpr int kHeld = 16, kWaves = kSelThreads / kWave;
    const int runs = (a.tiles + kWave - 1) / kWave, units = a.B * runs;
    const float* top = a.tile_max + r0 * a.tiles;
    auto ask = [&](int u0, float (&x)[kHeld]) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int u = u0 + i * kWaves;
            x[i] = -INFINITY;
            if (u >= units) continue;
            const int b = (int)((unsigned)u / (unsigned)runs), t = (u - b * runs) * kWave + ln;
            if (t < a.tiles) x[i] = top[(int64_t)b * a.tiles + t];
        }
    };
    float held[kHeld];
    const bool by_tiles = units <= kHeld * kWaves;
    if (by_tiles) ask(wv, held);
    if (threadIdx.x == 0) sh.n_tiles = sh.n_words = 0;
    const SelPart* parts = a.part + r0 * a.parts;
    if (a.parts <= 16) {
        for (int b = threadIdx.x >> 4; b < a.B; b += kSelThreads / 16)
            row_offset16(a, sh, r0 + b, b, (ln & 15) < a.parts ? parts[b * a.parts + (ln & 15)] : SelPart{0.0, -INFINITY, 0.f}, a.scores[r0 + b]);
    } else if (wv < a.B) {
        RowStart now;
        now.ask(a, r0 + wv, parts + (int64_t)wv * a.parts, a.parts);
        for (int b = wv; b < a.B; b += kWaves) {
            RowStart next = now;
            if (b + kWaves < a.B) next.ask(a, r0 + b + kWaves, parts + (int64_t)(b + kWaves) * a.parts, a.parts);
            row_offset(a, sh, r0 + b, b, parts + (int64_t)b * a.parts, a.parts, now);
            now = next;
        }
    }
    __syncthreads();
    // the threads' best tiles, or parts: N distinct ones reach the N-th of them, and no word below can be among the N best
    float best = -INFINITY;
    const int n_parts = a.B * a.parts;
    if (by_tiles) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {   // in the place of the maxima
            const int u = wv + i * kWaves;
            if (u >= units) continue;
            held[i] = rough_score(sh, (int)((unsigned)u / (unsigned)runs), held[i]);
            best = fmaxf(best, held[i]);
        }
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < n_parts; i += kSelThreads) best = fmaxf(best, rough_score(sh, (int)((unsigned)i / (unsigned)a.parts), parts[i].max));
    }
    const SelLimit limit = limit_of_threads(sh, best, a.N);
    auto list = [&](int u) {             // (a lane of the wave's unit u)
        const int b = (int)((unsigned)u / (unsigned)runs), t = (u - b * runs) * kWave + ln;
        if (t >= a.tiles) return;
        const uint32_t to = atomicAdd(&sh.n_tiles, 1u);
        if (to < kSelListed) sh.tile[to] = (uint32_t)(b * a.tiles + t);
    };
    uint64_t least = 1;
    if (!limit.none && by_tiles) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (wv + i * kWaves < units && limit.lets(held[i])) list(wv + i * kWaves);
    } else if (!limit.none) {            // the parts that can have a winner, then their tiles
#pragma unroll 4
        for (int i = threadIdx.x; i < n_parts; i += kSelThreads) {
            if (!limit.lets(rough_score(sh, (int)((unsigned)i / (unsigned)a.parts), parts[i].max))) continue;
            const uint32_t to = atomicAdd(&sh.n_words, 1u);
            if (to < kSelListed) sh.pair[to] = (uint32_t)i;
        }
        __syncthreads();
        const int n = (int)sh.n_words;
        __syncthreads();
        if (threadIdx.x == 0) { sh.n_words = 0; if (n > kSelListed) sh.n_tiles = kSelListed + 1; }
        for (int j = threadIdx.x >> 4; j < (n > kSelListed ? 0 : n); j += kSelThreads / 16) {
            const int i = (int)sh.pair[j], b = (int)((unsigned)i / (unsigned)a.parts), t0 = (i - b * a.parts) * a.pieces * (kSelPiece / kSelTile);
            for (int t = t0 + (ln & 15); t < min(t0 + a.pieces * (kSelPiece / kSelTile), a.tiles); t += 16)
                if (limit.lets(rough_score(sh, b, top[(int64_t)b * a.tiles + t]))) {
                    const uint32_t to = atomicAdd(&sh.n_tiles, 1u);
                    if (to < kSelListed) sh.tile[to] = (uint32_t)(b * a.tiles + t);
                }
        }
    } else {                             // scores far apart, huge, or fewer than N: the same by keys
        uint64_t key = 0;
        auto key_of = [&](int u) {
            const int b = (int)((unsigned)u / (unsigned)runs), t = (u - b * runs) * kWave + ln;
            return t < a.tiles ? score_key(score_of(sh, b, top[(int64_t)b * a.tiles + t])) : 0;
        };
        for (int u = wv; u < units; u += kWaves) { const uint64_t k = key_of(u); key = k > key ? k : key; }
        least = nth_of_threads(sh, key, a.N);
        for (int u = wv; u < units; u += kWaves)
            if (key_of(u) >= least) list(u);
    }
    __syncthreads();
    const int n = (int)sh.n_tiles;
    if (n <= kSelListed) {
        for (int i = threadIdx.x >> 4; i < n; i += kSelThreads / 16) {   // 16 lanes open a tile
            const int t = (int)sh.tile[i], b = t / a.tiles, w = (t - b * a.tiles) * kSelTile + (ln & 15) * kSelWords;
            if (w >= a.V) continue;
            float x[kSelWords];
            load_words<TYPE>(a, r0 + b, w, x);
#pragma unroll
            for (int j = 0; j < kSelWords; ++j) {
                if (!limit.none && !limit.lets(rough_score(sh, b, x[j]))) continue;
                const uint64_t k = score_key(score_of(sh, b, x[j]));
                if (k >= least) {
                    const uint32_t to = atomicAdd(&sh.n_words, 1u);
                    if (to < kSelListed) { sh.key[to] = k; sh.pair[to] = pair_of(b, w + j); }
                }
            }
        }
    }
    __syncthreads();
    if (n <= kSelListed && sh.n_words <= kSelListed) rank_words(a, sh, s, (int)sh.n_words);
    else select_all_words<TYPE>(a, sh, s);
}

// grid = S workgroups; sentences of at most kSelSmall pieces (B * ceil(V / 512)): every word stays in a register of its thread.
// 4 rows of 1000 words: 6.2 us.
template <int TYPE>
__global__ void __launch_bounds__(kSelThreads) k_select_small(SelArgs a) {
    __shared__ SelShared sh;
    __shared__ SelPart part[kSelSmall];
    constexpr int kOwn = kSelSmall / (kSelThreads / kWave);   // pieces of a wave
    const int s = blockIdx.x, wv = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id();
    const int64_t r0 = (int64_t)s * a.B;
    const int pieces = (a.V + kSelPiece - 1) / kSelPiece, units = a.B * pieces;
    float x[kOwn][kSelWords];
    const int row = threadIdx.x >> 4;    // (B <= kSelSmall: every row has 16 lanes)
    const float score = row < a.B ? a.scores[r0 + row] : 0.f;
    if (threadIdx.x == 0) sh.n_words = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int u = wv + i * (kSelThreads / kWave), b = u / pieces, w = (u - b * pieces) * kSelPiece + ln * kSelWords;
        if (u < units && w < a.V) load_words<TYPE>(a, r0 + b, w, x[i]);
        else {
#pragma unroll
            for (int j = 0; j < kSelWords; ++j) x[i][j] = -INFINITY;
        }
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int u = wv + i * (kSelThreads / kWave);
        if (u < units) {
            const float m = wave_max_f32(max_of(x[i]));
            const double sum = wave_sum_f64((double)sum_exp(x[i], m));
            if (ln == 0) part[u] = SelPart{sum, m, 0.f};
        }
    }
    __syncthreads();
    if (pieces <= 16) {
        if (row < a.B) row_offset16(a, sh, r0 + row, row, (ln & 15) < pieces ? part[row * pieces + (ln & 15)] : SelPart{0.0, -INFINITY, 0.f}, score);
    } else {
        for (int b = wv; b < a.B; b += kSelThreads / kWave) {
            RowStart start;
            start.ask(a, r0 + b, part + b * pieces, pieces);
            row_offset(a, sh, r0 + b, b, part + b * pieces, pieces, start);
        }
    }
    __syncthreads();
    float lane_best[kOwn], best = -INFINITY;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int u = wv + i * (kSelThreads / kWave);
        lane_best[i] = u < units ? rough_score(sh, u / pieces, max_of(x[i])) : -INFINITY;
        best = fmaxf(best, lane_best[i]);
    }
    const SelLimit limit = limit_of_threads(sh, best, a.N);
    uint64_t least = 1;
    if (limit.none) {
        uint64_t key = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int u = wv + i * (kSelThreads / kWave);
            const uint64_t k = u < units ? score_key(score_of(sh, u / pieces, max_of(x[i]))) : 0;
            key = k > key ? k : key;
        }
        least = nth_of_threads(sh, key, a.N);
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int u = wv + i * (kSelThreads / kWave), b = min(u / pieces, a.B - 1);
        const int w = (u - b * pieces) * kSelPiece + ln * kSelWords;
        if (u >= units || (!limit.none && !limit.lets(lane_best[i]))) continue;   // (the lane's others are no better)
#pragma unroll
        for (int j = 0; j < kSelWords; ++j) {
            if (!limit.none && !limit.lets(rough_score(sh, b, x[i][j]))) continue;
            const uint64_t k = score_key(score_of(sh, b, x[i][j]));
            if (k >= least) {
                const uint32_t to = atomicAdd(&sh.n_words, 1u);
                if (to < kSelListed) { sh.key[to] = k; sh.pair[to] = pair_of(b, w + j); }
            }
        }
    }
    __syncthreads();
    if (sh.n_words <= kSelListed) rank_words(a, sh, s, (int)sh.n_words);
    else select_all_words<TYPE>(a, sh, s);
}

}  // namespace lshbeam
