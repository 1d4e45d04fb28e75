// Eviction of single tokens: the choice of the tokens to keep by their weight, and the smaller cache made of them.
#include "common.hpp"
#include "stream_kv.hpp"

#include <type_traits>

namespace ra {

// ---- choice ----------------------------------------------------------------------------------------------------------------
// Keys that order like the weights: the sign bit flipped for positive numbers, all bits for negative ones; both zeros alike.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = as_u32(w + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

struct SelectTokensArgs {
    const float* weights;    // [B][n_pos]
    const int32_t* seg_len;  // [B][R_max]
    const int32_t* n_rounds;
    int n_pos, R_max, budget, keep_first, keep_last, unit;  // unit: of kept_off, for 16 tokens
    long long stride;
    int32_t *kept_idx, *n_kept, *kept_len;
    long long* kept_off;
    float* kept_weights;
};

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kDigit = 11, kBins = 1 << kDigit;  // three digits: 11, 11 and 10 bits of the key
constexpr int kChunk = 256;                      // positions that a wave reads with one instruction: four a lane
constexpr int kChunks = 8;                       // ... that it has in flight
constexpr int kCandidates = 8192;                // keys that share the first digit with the threshold and fit into LDS
constexpr int kManyPositions = 65536;            // positions from which several workgroups take a sequence (SelectParts)

typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));

// Bins of the counts, each four times over: lanes that meet in a bin meet in a quarter of it only.
__device__ __forceinline__ void count_bin(int* hist, uint32_t bin) { atomicAdd(&hist[bin * 4 + (threadIdx.x & 3)], 1); }
__device__ __forceinline__ int lanes_below(unsigned long long mask) {
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

// Positions of a sequence: n of them; the first lo and those from hi on are kept whatever they weigh, and `need` of the others, K
// in all.
struct TokenRange {
    int n, K, lo, hi, need;
    __device__ __forceinline__ TokenRange(const SelectTokensArgs& a, int tokens) {
        n = tokens;
        K = min(a.budget, n);
        lo = min(a.keep_first, n);
        hi = n - min(a.keep_last, n - lo);
        need = K - lo - (n - hi);
    }
    __device__ __forceinline__ bool all() const { return need >= hi - lo; }  // ... of the middle are kept
    __device__ __forceinline__ bool none() const { return need <= 0; }
    __device__ __forceinline__ bool inside(int p0) const { return p0 >= lo && p0 + kChunk <= hi; }  // the whole chunk lies in the middle
};
// The keys of the middle that are kept: those above `key`, and the first `equal` of those equal to it.
struct Threshold {
    uint32_t key;
    int equal;
};

// First positions of the rounds, and of the end, cut off at n_pos, which is returned.  1024 threads, R_max <= 1024; a barrier at
// its end.
__device__ __forceinline__ int round_starts(const SelectTokensArgs& a, int b, int* start, int* wave_sum) {
    const int r = threadIdx.x, wave = r >> 6;
    static_assert(kMaxRounds <= kSelThreads, "a thread for every round");
    int len = r < a.R_max ? a.seg_len[(size_t)b * a.R_max + r] : 0;
    if (r >= a.n_rounds[b]) len = 0;
    len = min(max(len, 0), a.n_pos);  // (64 of them add up to 2^30 at most)
    const int incl = wave_inclusive_sum(len);
    if ((r & 63) == 63) wave_sum[wave] = min(incl, a.n_pos);
    __syncthreads();
    int before = 0;
    for (int i = 0; i < wave; ++i) before = min(before + wave_sum[i], a.n_pos);
    if (r < a.R_max) start[r] = min(before + incl - len, a.n_pos);
    if (r == kSelThreads - 1) start[a.R_max] = min(before + incl, a.n_pos);
    __syncthreads();
    return start[a.R_max];
}

// Up to kChunks chunks of n weights, from chunk c0 to c_hi - 1.  Past the end: zeros.
struct Chunks {
    float x[kChunks][4];
};
__device__ __forceinline__ Chunks load_chunks(const float* w, int n, int c0, int c_hi) {
    const int lane = threadIdx.x & 63;
    Chunks c;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
        const int p = (c0 + j) * kChunk + lane * 4;
        float4_any v = {0.f, 0.f, 0.f, 0.f};
        if (c0 + j < c_hi) {
            if (p + 4 <= n) {
                v = *reinterpret_cast<const float4_any*>(w + p);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (p + e < n) v[e] = w[p + e];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) c.x[j][e] = v[e];
    }
    return c;
}
// The chunks c_lo .. c_hi - 1 of n weights by a wave, the first kChunks of which it holds: f(first position of the chunk, the lane's
// four weights).
template <typename F>
__device__ __forceinline__ void each_chunk(const Chunks& held, const float* w, int n, int c_lo, int c_hi, F f) {
    if (c_lo >= c_hi) return;
    Chunks c = held;
    for (int c0 = c_lo;;) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
            if (c0 + j < c_hi) f((c0 + j) * kChunk, c.x[j]);
        c0 += kChunks;
        if (c0 >= c_hi) break;
        c = load_chunks(w, n, c0, c_hi);
    }
}

// Counts of a digit, and what is found in them.
struct DigitCounts {
    int hist[kBins * 4];
    uint32_t digit;  // at which the counts, from the largest digit down, reach what is left ...
    int left;        // ... of which so much is left then ...
    int here;        // ... of so many candidates
    int wave_sum[kSelWaves];
};
__device__ __forceinline__ void clear_counts(DigitCounts& d) {  // no barrier
    for (int i = threadIdx.x; i < kBins; i += kSelThreads) *reinterpret_cast<int4*>(&d.hist[4 * i]) = make_int4(0, 0, 0, 0);
}
__device__ __forceinline__ int count_of(const DigitCounts& d, int bin) {
    const int4 four = *reinterpret_cast<const int4*>(&d.hist[bin * 4]);
    return four.x + four.y + four.z + four.w;
}
// `count`: thread t's counts of the digits top - N t, top - N t - 1, ... (N a thread, top the largest digit).  Ends with a barrier.
template <int N>
__device__ __forceinline__ void find_digit(DigitCounts& d, const int (&count)[N], int left) {
    const int tid = threadIdx.x, wave = tid >> 6;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) mine += count[i];
    const int incl = wave_inclusive_sum(mine);
    if ((tid & 63) == 63) d.wave_sum[wave] = incl;
    __syncthreads();
    int taken = incl - mine;
    for (int i = 0; i < kSelWaves; ++i) taken += i < wave ? d.wave_sum[i] : 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (taken < left && taken + count[i] >= left) {  // one digit of one thread
            d.digit = (uint32_t)(kSelThreads * N - 1 - N * tid - i);
            d.left = left - taken;
            d.here = count[i];
        }
        taken += count[i];
    }
    __syncthreads();
}
template <int BITS>
__device__ __forceinline__ void find_digit(DigitCounts& d, int left) {
    constexpr int N = (1 << BITS) / kSelThreads;
    int count[N];
#pragma unroll
    for (int i = 0; i < N; ++i) count[i] = count_of(d, kSelThreads * N - 1 - N * (int)threadIdx.x - i);
    find_digit(d, count, left);
}
constexpr int kShift1 = 32 - kDigit, kShift2 = kShift1 - kDigit;  // of the first and the second digit; the third has kShift2 bits

// Adds the chunks' positions of the middle to the counts of their first (second, third) digit, if they share those before with
// `key`.  No barrier.
template <int LEVEL>
__device__ __forceinline__ void count_digit(DigitCounts& d, const TokenRange& range, const Chunks& held, const float* w, int c_lo, int c_hi, uint32_t key) {
    const int lane = threadIdx.x & 63;
    constexpr int kAbove = LEVEL == 1 ? 31 : LEVEL == 2 ? kShift1 : kShift2, kShift = LEVEL == 1 ? kShift1 : LEVEL == 2 ? kShift2 : 0;
    constexpr uint32_t kMask = LEVEL == 3 ? (1u << kShift2) - 1 : kBins - 1;
    int zeros = 0;  // weights of zero, which whole rounds have and which would queue at one address, are counted by the wave
    each_chunk(held, w, range.n, c_lo, c_hi, [&](int p0, const float (&x)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int p = p0 + lane * 4 + e;
            const uint32_t k = weight_key(x[e]);
            const bool counts = (range.inside(p0) || (p >= range.lo && p < range.hi)) && (LEVEL == 1 || k >> kAbove == key >> kAbove);
            zeros += __popcll(__ballot(counts && x[e] == 0.f));
            if (counts && x[e] != 0.f) count_bin(d.hist, k >> kShift & kMask);
        }
    });
    if (lane == 0 && zeros > 0) atomicAdd(&d.hist[(0x80000000u >> kShift & kMask) * 4], zeros);
}

// Writes the kept positions of the wave's chunks: kept for certain before them `sure`, with the threshold's key `ties`.
// below(round, kept positions below its start), by any lane, for the rounds that start in the chunks; keep(place, position, weight).
// 0: dropped, 1: kept, 2: kept if it is among the first `equal` of its kind
__device__ __forceinline__ int fate(const TokenRange& range, const Threshold& t, int p0, int p, float x) {
    const uint32_t key = weight_key(x);
    const int of_middle = range.all() ? 1 : range.none() ? 0 : key > t.key ? 1 : key == t.key ? 2 : 0;
    return range.inside(p0) ? of_middle : p >= range.n ? 0 : p < range.lo || p >= range.hi ? 1 : of_middle;
}
template <typename Below, typename Keep>
__device__ __forceinline__ void write_kept(const TokenRange& range, const Threshold& t, const Chunks& held, const float* w, int c_lo, int c_hi, int sure, int ties,
                                           const int* start, int R, Below below, Keep keep) {
    const int lane = threadIdx.x & 63;
    int at = sure + min(ties, t.equal);
    // the round whose start comes next: the first that starts at or behind these chunks
    int round = 0;
    for (int r0 = 0; r0 <= R; r0 += 64) round += __popcll(__ballot(r0 + lane <= R && start[min(r0 + lane, R)] < c_lo * kChunk));
    each_chunk(held, w, range.n, c_lo, c_hi, [&](int p0, const float (&x)[4]) {
        // positions in order: lane by lane, four each
        unsigned long long kept[4], maybe[4];
        int f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = fate(range, t, p0, p0 + lane * 4 + e, x[e]);
            maybe[e] = __ballot(f[e] == 2);
        }
        bool mine[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[e] = f[e] == 1;
        if (maybe[0] | maybe[1] | maybe[2] | maybe[3]) {
            int tie = ties;
#pragma unroll
            for (int e = 0; e < 4; ++e) tie += lanes_below(maybe[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mine[e] |= f[e] == 2 && tie < t.equal;
                tie += f[e] == 2;
            }
        }
        int j = at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            kept[e] = __ballot(mine[e]);
            j += lanes_below(kept[e]);
        }
        for (int starts = 64; starts == 64; round += starts) {  // a lane each (many: rounds of a few tokens, and those behind the last)
            const int in = start[min(round + lane, R)] - p0, in_lane = in >> 2, in_e = in & 3;
            const bool here = round + lane <= R && in < kChunk;
            if (here) {
                int under = at;
#pragma unroll
                for (int e = 0; e < 4; ++e) under += __popcll(kept[e] & ((1ull << in_lane) - 1)) + (e < in_e && (kept[e] >> in_lane & 1));
                below(round + lane, under);
            }
            starts = __popcll(__ballot(here));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (mine[e]) keep(j++, p0 + lane * 4 + e, x[e]);
            at += __popcll(kept[e]);
            ties += __popcll(maybe[e]);
        }
    });
}

// Lengths and places of the rounds from the kept positions below their starts (below[R_max]: K), by the first wave.
template <typename Below>
__device__ __forceinline__ void write_rounds(const SelectTokensArgs& a, int b, int K, Below below) {
    const int lane = threadIdx.x & 63;
    long long off = (long long)b * a.stride;
    for (int r0 = 0; r0 < a.R_max; r0 += 64) {
        const int r = r0 + lane, len = r < a.R_max ? below(r + 1) - below(r) : 0;
        const int blocks = (len + 15) / 16, incl = wave_inclusive_sum(blocks);
        if (r < a.R_max) {
            a.kept_len[(size_t)b * a.R_max + r] = len;
            if (a.kept_off) a.kept_off[(size_t)b * a.R_max + r] = off + (long long)(incl - blocks) * a.unit;
        }
        off += (long long)__builtin_amdgcn_readlane(incl, 63) * a.unit;
    }
    if (lane == 0) a.n_kept[b] = K;
}

// n of `value` from `p` on, by the threads `tid` of `threads`: four at a time, and what is left of them.
template <typename T>
__device__ __forceinline__ void fill(T* p, int n, T value, int tid, int threads) {
    typedef T four_t __attribute__((ext_vector_type(4), aligned(4)));
    for (int j = tid; j < n / 4; j += threads) *reinterpret_cast<four_t*>(p + 4 * j) = four_t{value, value, value, value};
    if (tid < n % 4) p[n / 4 * 4 + tid] = value;
}

// One workgroup per sequence.  The `need` largest weights of the middle (what is neither among the first nor the last tokens) are
// those above a threshold key and, of those equal to it, the first ones.  The threshold is found digit by digit from counts of
// the candidates that share the digits before: over the weights for the first digit; the candidates that share it then lie in
// LDS as a rule, and the other digits are counted there (if they are more, over the weights).
// Every wave has a contiguous sixteenth of the positions: it knows how many of them it keeps, and writes them behind what the
// waves before it keep.  Counts are whole numbers: their order does not matter.
//
// Bound by what one compute unit does in a row: 131 000 weights take it 17 microseconds to count, 26 to sort out, 22 to write.
__global__ __launch_bounds__(kSelThreads) void select_tokens_kernel(SelectTokensArgs a) {
    __shared__ __align__(16) DigitCounts d;
    __shared__ int s_start[kMaxRounds + 1], s_below[kMaxRounds + 1];
    __shared__ int s_wave[kSelWaves][2];  // positions that are kept for certain, positions with the threshold's key
    __shared__ uint2 s_cand[kCandidates];  // key, position
    __shared__ int s_count;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float* w = a.weights + (size_t)b * a.n_pos;
    if (tid == 0) s_count = 0;
    clear_counts(d);
    const TokenRange range(a, round_starts(a, b, s_start, s_wave[0]));
    if (tid < kSelWaves) s_wave[tid][0] = s_wave[tid][1] = 0;
    __syncthreads();
    const int chunks = (range.n + kChunk - 1) / kChunk, c_lo = chunks * wave / kSelWaves, c_hi = chunks * (wave + 1) / kSelWaves;
    const Chunks held = load_chunks(w, range.n, c_lo, c_hi);
    Threshold t = {0, 0};
    bool counted = false;  // s_wave is complete
    if (!range.all() && !range.none()) {
        count_digit<1>(d, range, held, w, c_lo, c_hi, 0);
        __syncthreads();
        find_digit<kDigit>(d, range.need);
        const uint32_t digit1 = d.digit;
        t.key = digit1 << kShift1;
        int left = d.left;
        const bool in_lds = d.here <= kCandidates;
        clear_counts(d);
        __syncthreads();
        if (in_lds) {
            int sure = 0;
            each_chunk(held, w, range.n, c_lo, c_hi, [&](int p0, const float (&x)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = p0 + lane * 4 + e;
                    const uint32_t key = weight_key(x[e]), digit = key >> kShift1;
                    const bool middle = range.inside(p0) || (p >= range.lo && p < range.hi);
                    sure += __popcll(__ballot(middle ? digit > digit1 : p < range.n));
                    const unsigned long long take = __ballot(middle && digit == digit1);
                    if (take) {  // into the list, in any order
                        int at = 0;
                        if (lane == 0) at = atomicAdd(&s_count, __popcll(take));
                        at = __builtin_amdgcn_readfirstlane(at) + lanes_below(take);
                        if (middle && digit == digit1) s_cand[at] = make_uint2(key, (uint32_t)p);
                    }
                }
            });
            if (lane == 0) s_wave[wave][0] = sure;
            __syncthreads();
            const int n_cand = s_count;
            for (int i = tid; i < n_cand; i += kSelThreads) count_bin(d.hist, s_cand[i].x >> kShift2 & (kBins - 1));
            __syncthreads();
            find_digit<kDigit>(d, left);
            t.key |= d.digit << kShift2;
            left = d.left;
            clear_counts(d);
            __syncthreads();
            for (int i = tid; i < n_cand; i += kSelThreads)
                if (s_cand[i].x >> kShift2 == t.key >> kShift2) count_bin(d.hist, s_cand[i].x & ((1 << kShift2) - 1));
            __syncthreads();
            find_digit<kShift2>(d, left);
            t.key |= d.digit;
            t.equal = d.left;
            for (int i = tid; i < n_cand; i += kSelThreads) {
                if (s_cand[i].x < t.key) continue;
                // the wave whose positions these are: the last one that begins at or before the chunk
                const int c = (int)s_cand[i].y / kChunk;
                int owner = (int)(((long long)c * kSelWaves) / chunks);
                while (owner + 1 < kSelWaves && chunks * (owner + 1) / kSelWaves <= c) ++owner;
                atomicAdd(&s_wave[owner][s_cand[i].x == t.key], 1);
            }
            counted = true;
        } else {
            count_digit<2>(d, range, held, w, c_lo, c_hi, t.key);
            __syncthreads();
            find_digit<kDigit>(d, left);
            t.key |= d.digit << kShift2;
            left = d.left;
            clear_counts(d);
            __syncthreads();
            count_digit<3>(d, range, held, w, c_lo, c_hi, t.key);
            __syncthreads();
            find_digit<kShift2>(d, left);
            t.key |= d.digit;
            t.equal = d.left;
        }
    }
    if (!counted) {
        int n_sure = 0, n_equal = 0;
        each_chunk(held, w, range.n, c_lo, c_hi, [&](int p0, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int f = fate(range, t, p0, p0 + lane * 4 + e, x[e]);
                n_sure += __popcll(__ballot(f == 1));
                n_equal += __popcll(__ballot(f == 2));
            }
        });
        if (lane == 0) {
            s_wave[wave][0] = n_sure;
            s_wave[wave][1] = n_equal;
        }
    }
    __syncthreads();
    int sure = 0, ties = 0;
    for (int i = 0; i < wave; ++i) {
        sure += s_wave[i][0];
        ties += s_wave[i][1];
    }
    int32_t* idx = a.kept_idx + (size_t)b * a.budget;
    float* left_over = a.kept_weights ? a.kept_weights + (size_t)b * a.n_pos : nullptr;
    write_kept(range, t, held, w, c_lo, c_hi, sure, ties, s_start, a.R_max, [&](int r, int under) { s_below[r] = under; },
               [&](int j, int p, float x) {
                   idx[j] = p;
                   if (left_over) left_over[j] = x;
               });
    fill(idx + range.K, a.budget - range.K, (int32_t)-1, tid, kSelThreads);
    if (left_over) fill(left_over + range.K, a.n_pos - range.K, 0.f, tid, kSelThreads);
    // starts behind the last chunk (and all of them, if there are no tokens): everything kept lies below
    for (int r = tid; r <= a.R_max; r += kSelThreads)
        if (s_start[r] >= chunks * kChunk) s_below[r] = range.K;
    __syncthreads();
    if (wave == 0) write_rounds(a, b, range.K, [&](int r) { return s_below[r]; });
}

// ---- the same by several workgroups per sequence ------------------------------------------------------------------------------
// Every workgroup has a part of the positions.  Three launches count the digits, each of them adding up what the one before
// counted in all parts; one writes the kept positions, every part behind what the parts before it keep; the last one writes
// the rounds and the weights.  Until then the counts lie where those weights will: kept_weights holds them (5120 numbers a part
// of 8192 positions or more).
constexpr int kPartPositions = 8192;
constexpr int kMinParts = 8, kMaxParts = 64;  // (each adds up the counts of all)
struct SelectParts {
    int n, chunks;  // parts; chunks of a part
    // No more parts than compute units, which such a workgroup fills: twice as many took 78 microseconds instead of 51 (16 dialogues of
    // 131 000 tokens).  Where that leaves a sequence fewer than eight it is one workgroup's (64 dialogues of 48 000 tokens: 47, four
    // parts 58; 100 of 131 000: 122, two parts 170), and so are short sequences: one of 48 000 tokens 44, parts of 16384 positions
    // 39.6, of 8192 34.5; of 36 000 36 and 34; of 30 000 30 and 33.
    static bool pays(int n_pos, int B, int num_cu) { return n_pos >= kManyPositions && B <= num_cu / kMinParts; }
    static SelectParts of(int n_pos, int B, int num_cu) {
        const int most = num_cu / B < kMaxParts ? num_cu / B : kMaxParts;
        SelectParts s;
        s.chunks = kPartPositions / kChunk * ((n_pos - 1) / kPartPositions / most + 1);
        s.n = (n_pos + s.chunks * kChunk - 1) / (s.chunks * kChunk);
        return s;
    }
    // A wave's share begins with this chunk, wherever the sequence ends, so that its weights are asked for before that is known.
    __device__ int first_chunk(int part, int wave) const { return part * chunks + chunks * wave / kSelWaves; }
    __device__ int used(int positions) const { return (positions + chunks * kChunk - 1) / (chunks * kChunk); }  // parts with positions
};
constexpr int kPartNumbers = 2 * kBins + (1 << kShift2) + 2;
static_assert(kPartNumbers <= kPartPositions && (kManyPositions / kPartPositions + 1) * kPartNumbers + 4 <= kManyPositions, "they fit");
struct SelectScratch {
    int *count1, *count2, *count3;  // [parts][bins]
    int* found;                     // digit and what is left, of the first and the second level
    int* above;                     // [parts][2]: positions of the part above the first (second) digit
    __device__ __forceinline__ SelectScratch(const SelectTokensArgs& a, int b, int parts) {
        count1 = reinterpret_cast<int*>(a.kept_weights + (size_t)b * a.n_pos);
        count2 = count1 + (size_t)parts * kBins;
        count3 = count2 + (size_t)parts * kBins;
        above = count3 + ((size_t)parts << kShift2);
        found = above + 2 * parts;
    }
};

// Adds up a level's counts of all parts and finds the digit.  `mine`: the counts of this part, `before`: of the parts before it, of
// the digits that find_digit gives the thread.
template <int N>
__device__ __forceinline__ int thread_digit(int i) { return kSelThreads * N - 1 - N * (int)threadIdx.x - i; }
template <int N>
__device__ __forceinline__ void add_parts(DigitCounts& d, const int* counts, int parts, int part, int left, int (&mine)[N], int (&before)[N]) {
    int sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = mine[i] = before[i] = 0;
    for (int p0 = 0; p0 < parts; p0 += 16) {
        int c[16][N];
#pragma unroll
        for (int p = 0; p < 16; ++p)
#pragma unroll
            for (int i = 0; i < N; ++i) c[p][i] = p0 + p < parts ? counts[(size_t)(p0 + p) * (kSelThreads * N) + thread_digit<N>(i)] : 0;
#pragma unroll
        for (int p = 0; p < 16; ++p)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum[i] += c[p][i];
                mine[i] += p0 + p == part ? c[p][i] : 0;
                before[i] += p0 + p < part ? c[p][i] : 0;
            }
    }
    find_digit(d, sum, left);
}
// Sum over the threads, in every thread; two barriers.
__device__ __forceinline__ int block_sum(int v, int* wave_sum) {
    v = wave_inclusive_sum(v);
    if ((threadIdx.x & 63) == 63) wave_sum[threadIdx.x >> 6] = v;
    __syncthreads();
    int sum = 0;
    for (int i = 0; i < kSelWaves; ++i) sum += wave_sum[i];
    __syncthreads();
    return sum;
}

// grid (parts, B)
template <int LEVEL>
__global__ __launch_bounds__(kSelThreads) void select_count_kernel(SelectTokensArgs a, SelectParts parts) {
    __shared__ __align__(16) DigitCounts d;
    __shared__ int s_start[kMaxRounds + 1], s_wave[kSelWaves];
    const int part = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float* w = a.weights + (size_t)b * a.n_pos;
    const int c_lo = parts.first_chunk(part, wave);
    const Chunks held = load_chunks(w, a.n_pos, c_lo, parts.first_chunk(part, wave + 1));
    clear_counts(d);
    const TokenRange range(a, round_starts(a, b, s_start, s_wave));
    const int used = parts.used(range.n), c_hi = min(parts.first_chunk(part, wave + 1), (range.n + kChunk - 1) / kChunk);
    if (part >= used) return;
    const SelectScratch at(a, b, parts.n);
    uint32_t key = 0;
    if constexpr (LEVEL > 1) {
        const uint32_t digit1 = LEVEL == 3 ? (uint32_t)at.found[0] : 0;
        const int left = LEVEL == 3 ? at.found[1] : range.need;
        int mine[2], before[2];
        add_parts(d, LEVEL == 2 ? at.count1 : at.count2, used, part, left, mine, before);
        const uint32_t digit = d.digit;
        if (part == 0 && tid == 0) {
            at.found[2 * (LEVEL - 2)] = (int)digit;
            at.found[2 * (LEVEL - 2) + 1] = d.left;
        }
        key = LEVEL == 2 ? digit << kShift1 : digit1 << kShift1 | digit << kShift2;
        const int above = block_sum(((uint32_t)thread_digit<2>(0) > digit ? mine[0] : 0) + ((uint32_t)thread_digit<2>(1) > digit ? mine[1] : 0), s_wave);
        if (tid == 0) at.above[2 * part + LEVEL - 2] = above;
    }
    count_digit<LEVEL>(d, range, held, w, c_lo, c_hi, key);
    __syncthreads();
    constexpr int kCounts = LEVEL == 3 ? 1 << kShift2 : kBins;
    int* out = (LEVEL == 1 ? at.count1 : LEVEL == 2 ? at.count2 : at.count3) + (size_t)part * kCounts;
    for (int i = tid; i < kCounts; i += kSelThreads) out[i] = count_of(d, i);
}

// grid (parts, B): the kept positions, and in kept_len how many of them lie below the rounds' starts
__global__ __launch_bounds__(kSelThreads) void select_write_kernel(SelectTokensArgs a, SelectParts parts) {
    __shared__ __align__(16) DigitCounts d;
    __shared__ int s_start[kMaxRounds + 1], s_wave[kSelWaves], s_sure[kSelWaves], s_ties[kSelWaves];
    const int part = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float* w = a.weights + (size_t)b * a.n_pos;
    const int c_lo = parts.first_chunk(part, wave);
    const Chunks held = load_chunks(w, a.n_pos, c_lo, parts.first_chunk(part, wave + 1));
    const TokenRange range(a, round_starts(a, b, s_start, s_wave));
    const SelectScratch at(a, b, parts.n);
    int32_t* idx = a.kept_idx + (size_t)b * a.budget;
    fill(idx + range.K, a.budget - range.K, (int32_t)-1, part * kSelThreads + tid, parts.n * kSelThreads);
    int32_t* below = a.kept_len + (size_t)b * a.R_max;
    if (part == 0)  // starts behind the last chunk: everything kept lies below
        for (int r = tid; r < a.R_max; r += kSelThreads)
            if (s_start[r] >= (range.n + kChunk - 1) / kChunk * kChunk) below[r] = range.K;
    const int used = parts.used(range.n);
    if (part >= used) return;
    const int c_hi = min(parts.first_chunk(part, wave + 1), (range.n + kChunk - 1) / kChunk), p0 = part * parts.chunks * kChunk;
    int mine[1], before[1];
    add_parts(d, at.count3, used, part, at.found[3], mine, before);
    const uint32_t digit3 = d.digit;
    const Threshold t = {(uint32_t)at.found[0] << kShift1 | (uint32_t)at.found[2] << kShift2 | digit3, d.left};
    // what the parts before this one keep
    const int forced = min(range.lo, p0) + max(p0 - range.hi, 0);
    int sure = block_sum(((uint32_t)thread_digit<1>(0) > digit3 ? before[0] : 0) + (tid < part ? at.above[2 * tid] + at.above[2 * tid + 1] : 0), s_wave) + forced;
    int ties = block_sum((uint32_t)thread_digit<1>(0) == digit3 ? before[0] : 0, s_wave);
    if (range.all()) sure = p0, ties = 0;
    else if (range.none()) sure = forced, ties = 0;
    int n_sure = 0, n_ties = 0;
    each_chunk(held, w, range.n, c_lo, c_hi, [&](int p, const float (&x)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int f = fate(range, t, p, p + lane * 4 + e, x[e]);
            n_sure += __popcll(__ballot(f == 1));
            n_ties += __popcll(__ballot(f == 2));
        }
    });
    if (lane == 0) {
        s_sure[wave] = n_sure;
        s_ties[wave] = n_ties;
    }
    __syncthreads();
    for (int i = 0; i < wave; ++i) {
        sure += s_sure[i];
        ties += s_ties[i];
    }
    write_kept(range, t, held, w, c_lo, c_hi, sure, ties, s_start, a.R_max, [&](int r, int under) { if (r < a.R_max) below[r] = under; },
               [&](int j, int p, float) { idx[j] = p; });
}

// grid (pieces of kFinish weights, B)
constexpr int kFinish = 4 * kSelThreads;
__global__ __launch_bounds__(kSelThreads) void select_finish_kernel(SelectTokensArgs a) {
    __shared__ int s_start[kMaxRounds + 1], s_wave[kSelWaves], s_below[kMaxRounds + 1];
    const int part = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const float* w = a.weights + (size_t)b * a.n_pos;
    const int32_t* idx = a.kept_idx + (size_t)b * a.budget;
    float* out = a.kept_weights + (size_t)b * a.n_pos;
    const int first = part * kFinish, last = min(first + kFinish, a.n_pos);
    constexpr int kEach = kFinish / kSelThreads;
    float x[kEach];  // asked for before it is known how many are kept (-1 behind the last one)
    int from[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int j = first + i * kSelThreads + tid;
        from[i] = j < a.budget ? idx[j] : 0;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = w[max(from[i], 0)];
    const TokenRange range(a, round_starts(a, b, s_start, s_wave));
    const int kept = min(max(range.K - first, 0), last - first);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (const int j = i * kSelThreads + tid; j < kept) out[first + j] = x[i];
    fill(out + first + kept, last - first - kept, 0.f, tid, kSelThreads);
    if (part != 0) return;
    for (int r = tid; r <= a.R_max; r += kSelThreads) s_below[r] = r < a.R_max ? a.kept_len[(size_t)b * a.R_max + r] : range.K;
    __syncthreads();
    if (tid < 64) write_rounds(a, b, range.K, [&](int r) { return s_below[r]; });
}

// ---- the smaller cache -------------------------------------------------------------------------------------------------------
struct CompactArgs {
    DevView src, dst;
    const int32_t *kept_idx, *n_kept;
    int max_kept;
    int piece;  // kept tokens that a workgroup moves, whole tiles of one round
};

constexpr int kCompactTokens = 64;  // ... of them at most

// Where the tokens of a round lie: key row and first element of the value tile, for head 0, and from one head to the next.
struct RoundPlace {
    const DevView& v;
    int b, len;
    long long off, off_v;
    __device__ __forceinline__ RoundPlace(const DevView& view, int b_, int round, int len_) : v(view), b(b_), len(len_) {
        off = v.seg_off[(size_t)b * v.R_max + round];
        off_v = v.seg_off_v[(size_t)b * v.R_max + round];
    }
    __device__ __forceinline__ long long block(int t) const {
        const long long at = min(max(off + t / 16, 0ll), (long long)v.max_blocks - 1);
        return (long long)max(v.block_table[(size_t)b * v.max_blocks + at], 0) * v.Hkv;
    }
    __device__ __forceinline__ long long key_row(int t) const { return v.block_size ? block(t) * 16 + t % 16 : off * v.Hkv + t; }
    __device__ __forceinline__ long long value_tile(int t, int d) const {
        return v.block_size ? block(t) * 16 * d : (off_v * v.Hkv + (t & ~15)) * d;
    }
    __device__ __forceinline__ int key_stride() const { return v.block_size ? 16 : len; }
    __device__ __forceinline__ int value_stride(int d) const { return v.block_size ? 16 * d : ((len + 15) & ~15) * d; }
};

// grid (pieces of a sequence's rounds, B, four jobs).  A wave moves the keys or the values of one head at a time.
// Keys are rows.  Values are tiles of 16 tokens, [D][16], of which a kept token is a column: a lane owns channels, has its rows of
// two source tiles in registers or on their way, writes the columns that stay side by side into LDS, and from there every new
// tile goes out once, as 32 (64) contiguous bytes a channel; every source tile is read once.  (With a load per element, 64
// channels in 64 sectors of a tile, 2 GB moved in 663 microseconds, the second-level cache read eight times over.)
template <typename T, int D>
__global__ __launch_bounds__(256) void compact_rounds_kernel(CompactArgs a) {
    constexpr int kPieces = D * sizeof(T) / 16;  // of a key row
    constexpr int kQuads = (int)sizeof(T), kChannels = D / 64;  // 16-byte pieces of a channel's 16 tokens; channels of a lane
    constexpr int kPitch = 8 * kQuads + 2;  // 32-bit words of a channel in LDS: 32 tokens
    __shared__ long long s_key[kCompactTokens], s_tile[kCompactTokens], s_new_key[kCompactTokens], s_new_tile[kCompactTokens / 16];
    __shared__ int s_from[kCompactTokens];  // source token (-1: none)
    __shared__ int s_mask[kCompactTokens], s_valid[kCompactTokens / 16];
    __shared__ __align__(16) uint32_t s_column[4][D * kPitch];
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = a.src.R_max, n_src = min(max(a.src.n_rounds[b], 0), R), n_dst = min(max(a.dst.n_rounds[b], 0), R);
    const size_t row = (size_t)b * R;
    // the piece's round: its lengths in both caches, and what lies before it (every wave for itself)
    int round = -1, t0 = 0, len = 0, first = 0, src_len = 0, src_first = 0;
    {
        int pieces_before = 0, dst_before = 0, src_before = 0;
        for (int r0 = 0; r0 < n_dst && round < 0; r0 += 64) {
            const int r = r0 + lane;
            const int d = r < n_dst ? max(a.dst.seg_len[row + r], 0) : 0, s = r < n_src ? max(a.src.seg_len[row + r], 0) : 0;
            const int pieces = (d + a.piece - 1) / a.piece;
            const int end = wave_inclusive_sum(pieces), d_end = wave_inclusive_sum(d), s_end = wave_inclusive_sum(s);
            const int target = (int)blockIdx.x - pieces_before;
            const unsigned long long in = __ballot(end > target && end - pieces <= target);
            if (in) {
                const int at = __ffsll(in) - 1;
                round = r0 + at;
                len = __builtin_amdgcn_readlane(d, at);
                src_len = __builtin_amdgcn_readlane(s, at);
                t0 = (target - (__builtin_amdgcn_readlane(end, at) - __builtin_amdgcn_readlane(pieces, at))) * a.piece;
                first = dst_before + __builtin_amdgcn_readlane(d_end, at) - len;
                src_first = src_before + __builtin_amdgcn_readlane(s_end, at) - src_len;
            }
            pieces_before += __builtin_amdgcn_readlane(end, 63);
            dst_before += __builtin_amdgcn_readlane(d_end, 63);
            src_before += __builtin_amdgcn_readlane(s_end, 63);
        }
    }
    if (round < 0) return;
    const RoundPlace src(a.src, b, round, src_len), dst(a.dst, b, round, len);
    const int here = min(a.piece, len - t0);
    if (tid < kCompactTokens) {
        const int j = first + t0 + tid;
        int from = -1;
        if (tid < here && j < min(max(a.n_kept[b], 0), a.max_kept)) {
            from = a.kept_idx[(size_t)b * a.max_kept + j] - src_first;
            if (from < 0 || from >= src_len) from = -1;
        }
        s_from[tid] = from;
        s_key[tid] = from >= 0 ? src.key_row(from) : 0;
        if (tid < here) s_new_key[tid] = dst.key_row(t0 + tid);
        if (tid % 16 == 0 && tid < here) s_new_tile[tid / 16] = dst.value_tile(t0 + tid, D);
    }
    __syncthreads();
    // the source tiles that the piece takes columns of, one after the other: where, which columns, and the new place of the first
    int n_tiles = 0;
    if (a.src.v) {
        auto tile_of = [&](int i) { return i >= 0 && i < here && s_from[i] >= 0 ? s_from[i] >> 4 : -1; };
        for (int i0 = 0; i0 < here; i0 += 64) {
            const int i = i0 + lane, tile = tile_of(i);
            const unsigned long long starts = __ballot(tile >= 0 && tile != tile_of(i - 1));
            if (wave == 0 && (starts >> lane & 1)) {
                int mask = 0;
                for (int j = i; j < here && tile_of(j) == tile; ++j) mask |= 1 << (s_from[j] & 15);
                const int k = n_tiles + __popcll(starts & ((1ull << lane) - 1));
                s_mask[k] = i << 16 | mask;
                s_tile[k] = src.value_tile(s_from[i], D);
            }
            const unsigned long long some = __ballot(tile >= 0);
            if (wave == 0 && lane < 4) s_valid[i0 / 16 + lane] = (int)(some >> 16 * lane & 0xffff);
            n_tiles += __popcll(starts);
        }
    }
    __syncthreads();
    const int Hkv = a.src.Hkv;
    const int jobs = a.src.v ? 2 * Hkv : Hkv;
    for (int job = blockIdx.z * 4 + wave; job < jobs; job += 4 * gridDim.z) {
        const int g = job >= Hkv ? job - Hkv : job;
        if (job < Hkv) {
            constexpr int kRows = 64 / kPieces, kFlight = 8;  // rows of an instruction; instructions in flight
            const uint4* from = static_cast<const uint4*>(a.src.k);
            uint4* to = static_cast<uint4*>(const_cast<void*>(a.dst.k));
            const long long head = (long long)g * src.key_stride(), new_head = (long long)g * dst.key_stride();
            for (int i0 = 0; i0 < here; i0 += kRows * kFlight) {
                const uint4* at[kFlight];
                bool some[kFlight];
                uint4 k[kFlight];
#pragma unroll
                for (int f = 0; f < kFlight; ++f) {
                    const int i = min(i0 + f * kRows + lane / kPieces, kCompactTokens - 1);
                    some[f] = s_from[i] >= 0;
                    at[f] = from + (s_key[i] + head) * kPieces + lane % kPieces;
                    k[f] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int f = 0; f < kFlight; ++f)
                    if (some[f]) k[f] = load_once(at[f]);
#pragma unroll
                for (int f = 0; f < kFlight; ++f) {
                    const int i = i0 + f * kRows + lane / kPieces;
                    if (i < here) to[(s_new_key[i] + new_head) * kPieces + lane % kPieces] = k[f];
                }
            }
            continue;
        }
        const T* from = static_cast<const T*>(a.src.v) + (size_t)g * src.value_stride(D) + lane * 16;
        T* to = static_cast<T*>(const_cast<void*>(a.dst.v)) + (size_t)g * dst.value_stride(D) + lane * 16;
        struct Tile {  // the lane's channels (lane, lane + 64) of a source tile
            uint32_t x[kChannels][4 * kQuads];
        };
        auto load = [&](int k) {
            Tile t;
            const T* tile = from + s_tile[min(k, n_tiles - 1)];
#pragma unroll
            for (int c = 0; c < kChannels; ++c)
#pragma unroll
                for (int w = 0; w < kQuads; ++w) {
                    const uint4 v = reinterpret_cast<const uint4*>(tile + c * 1024)[w];
                    t.x[c][4 * w] = v.x, t.x[c][4 * w + 1] = v.y, t.x[c][4 * w + 2] = v.z, t.x[c][4 * w + 3] = v.w;
                }
            return t;
        };
        // the lane's channels of two new tiles, in turn: token j is column j % 32
        uint32_t* mine = s_column[wave] + lane * kPitch;
        T* columns = reinterpret_cast<T*>(mine);
        constexpr int kNextChannel = 64 * kPitch;  // words to the lane's second channel
        int written = 0;  // new tiles
        auto write_out = [&](int upto) {  // the new tiles that end before token `upto`
            while (written < upto >> 4) {
                const int valid = __builtin_amdgcn_readfirstlane(s_valid[written]);
                T* tile = to + s_new_tile[written];
#pragma unroll
                for (int c = 0; c < kChannels; ++c) {
                    uint32_t x[4 * kQuads];
#pragma unroll
                    for (int w = 0; w < 2 * kQuads; ++w) {
                        const uint2 v = *reinterpret_cast<const uint2*>(mine + c * kNextChannel + (written & 1) * 4 * kQuads + 2 * w);
                        x[2 * w] = v.x, x[2 * w + 1] = v.y;
                    }
                    if (valid != 0xffff) {  // columns behind the round's end, and those that come from nowhere: zeros
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(valid >> i & 1)) x[i * (int)sizeof(T) / 4] &= sizeof(T) == 4 ? 0u : i % 2 ? 0x0000ffffu : 0xffff0000u;
                    }
#pragma unroll
                    for (int w = 0; w < kQuads; ++w)
                        reinterpret_cast<uint4*>(tile + c * 1024)[w] = make_uint4(x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]);
                }
                ++written;
            }
        };
        auto pick = [&](const Tile& t, int k) {  // the kept columns of source tile k
            const int first_mask = __builtin_amdgcn_readfirstlane(s_mask[k]), first_j = first_mask >> 16;
            write_out(first_j);
            int j = first_j;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (first_mask >> e & 1) {
#pragma unroll
                    for (int c = 0; c < kChannels; ++c) {
                        T* at = columns + c * kNextChannel * (4 / (int)sizeof(T)) + (j & 31);
                        if constexpr (sizeof(T) == 4) *at = t.x[c][e];
                        else *at = (T)(e % 2 ? t.x[c][e / 2] >> 16 : t.x[c][e / 2]);
                    }
                    ++j;
                }
        };
        if (n_tiles > 0) {  // two tiles held, the request for the next one made in any case: no wait is for more than the tile in hand
            Tile x = load(0), y;
            for (int k = 0; k < n_tiles; k += 2) {
                y = load(k + 1);
                pick(x, k);
                if (k + 1 >= n_tiles) break;
                x = load(k + 2);
                pick(y, k + 1);
            }
        }
        write_out((here + 15) & ~15);
    }
}

// Tokens of a piece, for `tokens` tokens times groups of four jobs.  A wave takes the source tiles of a piece one after the other, and
// a piece looks its round up and reads the tiles at its ends again: as long as possible, and short enough for two workgroups a
// compute unit.  (Pieces of 16, 32, 64, 128, microseconds: one dialogue of 2 048 tokens 8.2, 10.1, 12.6, 18.8; two 16.4, 13.7, 15.5,
// 20.2; four 28.3, 24.7, 25.0, 28.4; 16 of 16 000 paged ones 685, 569, 541, 543.)
static int compact_piece(int64_t tokens, int num_cu) {
    int piece = kCompactTokens;
    while (piece > 16 && tokens / piece < 2 * num_cu) piece /= 2;
    return piece;
}

}  // namespace ra

using namespace ra;

static bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    return a != nullptr && (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

extern "C" int ra_select_tokens(ra_ctx* ctx, void* stream, const float* weights, int n_pos, const int32_t* seg_len,
                                const int32_t* n_rounds, int B, int R_max, const ra_keep_params* params, int32_t* kept_idx,
                                int32_t* n_kept, int32_t* kept_len, int64_t* kept_off, float* kept_weights) {
    RA_REQUIRE(ctx != nullptr, RA_ERR_INVALID_ARG, "select_tokens: ctx is NULL");
    RA_REQUIRE(params != nullptr, RA_ERR_INVALID_ARG, "select_tokens: params is NULL");
    RA_REQUIRE(B > 0 && R_max > 0 && n_pos > 0, RA_ERR_INVALID_ARG, "select_tokens: B, R_max and n_pos must be positive");
    RA_REQUIRE(R_max <= kMaxRounds, RA_ERR_UNSUPPORTED, "select_tokens: R_max %d exceeds %d", R_max, kMaxRounds);
    RA_REQUIRE(n_pos <= 1 << 24, RA_ERR_UNSUPPORTED, "select_tokens: n_pos %d exceeds 2^24", n_pos);
    RA_REQUIRE(params->budget > 0 && params->keep_first >= 0 && params->keep_last >= 0 &&
                   (int64_t)params->keep_first + params->keep_last <= params->budget,
               RA_ERR_INVALID_ARG, "select_tokens: budget %d has no room for the first %d and the last %d tokens", params->budget,
               params->keep_first, params->keep_last);
    RA_REQUIRE(params->block_size == 0 || params->block_size == kUnitTokens, RA_ERR_UNSUPPORTED,
               "select_tokens: block_size must be 0 or %d (got %d)", kUnitTokens, params->block_size);
    RA_REQUIRE(params->stride >= 0, RA_ERR_INVALID_ARG, "select_tokens: stride is negative");
    RA_REQUIRE(weights && seg_len && n_rounds && kept_idx && n_kept && kept_len, RA_ERR_INVALID_ARG,
               "select_tokens: NULL argument");
    const size_t weight_bytes = (size_t)B * n_pos * sizeof(float), round_bytes = (size_t)B * R_max * sizeof(int32_t);
    RA_REQUIRE(!overlap(kept_weights, weight_bytes, weights, weight_bytes), RA_ERR_INVALID_ARG,
               "select_tokens: kept_weights must be another buffer than weights");
    RA_REQUIRE(!overlap(kept_len, round_bytes, seg_len, round_bytes) && n_kept != n_rounds, RA_ERR_INVALID_ARG,
               "select_tokens: kept_len and n_kept must be other buffers than seg_len and n_rounds");
    SelectTokensArgs a = {};
    a.weights = weights;
    a.seg_len = seg_len;
    a.n_rounds = n_rounds;
    a.n_pos = n_pos;
    a.R_max = R_max;
    a.budget = params->budget;
    a.keep_first = params->keep_first;
    a.keep_last = params->keep_last;
    a.unit = params->block_size ? 1 : kUnitTokens;
    a.stride = params->stride;
    a.kept_idx = kept_idx;
    a.n_kept = n_kept;
    a.kept_len = kept_len;
    a.kept_off = reinterpret_cast<long long*>(kept_off);
    a.kept_weights = kept_weights;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (kept_weights != nullptr && SelectParts::pays(n_pos, B, ctx->num_cu)) {
        const SelectParts parts = SelectParts::of(n_pos, B, ctx->num_cu);
        const dim3 grid((unsigned)parts.n, (unsigned)B), block(kSelThreads);
        hipLaunchKernelGGL((select_count_kernel<1>), grid, block, 0, st, a, parts);
        hipLaunchKernelGGL((select_count_kernel<2>), grid, block, 0, st, a, parts);
        hipLaunchKernelGGL((select_count_kernel<3>), grid, block, 0, st, a, parts);
        hipLaunchKernelGGL(select_write_kernel, grid, block, 0, st, a, parts);
        hipLaunchKernelGGL(select_finish_kernel, dim3((unsigned)((n_pos + kFinish - 1) / kFinish), (unsigned)B), block, 0, st, a);
    } else {
        hipLaunchKernelGGL(select_tokens_kernel, dim3((unsigned)B), dim3(kSelThreads), 0, st, a);
    }
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}

extern "C" int ra_compact_rounds(ra_ctx* ctx, void* stream, const ra_kv_view* src, const int32_t* kept_idx, const int32_t* n_kept,
                                 int max_kept, const ra_kv_view* dst) {
    RA_REQUIRE(ctx != nullptr, RA_ERR_INVALID_ARG, "compact_rounds: ctx is NULL");
    RA_REQUIRE(max_kept > 0, RA_ERR_INVALID_ARG, "compact_rounds: max_kept must be positive");
    RA_REQUIRE(kept_idx != nullptr && n_kept != nullptr, RA_ERR_INVALID_ARG, "compact_rounds: kept_idx or n_kept is NULL");
    if (int rc = check_view(src, false, "compact_rounds: src")) return rc;
    if (int rc = check_view(dst, false, "compact_rounds: dst")) return rc;
    RA_REQUIRE(src->R_max > 0, RA_ERR_INVALID_ARG, "compact_rounds: R_max is 0, there is nothing to keep");
    RA_REQUIRE(src->B == dst->B && src->R_max == dst->R_max && src->Hkv == dst->Hkv && src->d == dst->d && src->dtype == dst->dtype,
               RA_ERR_INVALID_ARG, "compact_rounds: src and dst differ in B, R_max, Hkv, d or dtype");
    RA_REQUIRE((src->v == nullptr) == (dst->v == nullptr), RA_ERR_INVALID_ARG,
               "compact_rounds: values must be given in both views or in neither");
    RA_REQUIRE(src->k != dst->k && (src->v == nullptr || src->v != dst->v), RA_ERR_INVALID_ARG,
               "compact_rounds: dst needs memory of its own");
    RA_REQUIRE(src->d == 64 || src->d == 128, RA_ERR_UNSUPPORTED, "compact_rounds: head_dim %d not in {64, 128}", src->d);
    RA_REQUIRE(src->B <= 65535, RA_ERR_UNSUPPORTED, "compact_rounds: batch %d exceeds 65535", src->B);
    RA_REQUIRE(src->Hkv <= 65535, RA_ERR_UNSUPPORTED, "compact_rounds: Hkv %d exceeds 65535", src->Hkv);
    RA_REQUIRE((((uintptr_t)src->k | (uintptr_t)src->v | (uintptr_t)dst->k | (uintptr_t)dst->v) & 15) == 0, RA_ERR_INVALID_ARG,
               "compact_rounds: keys and values must be 16-byte aligned");
    CompactArgs a = {};
    a.src = to_dev(src);
    a.dst = to_dev(dst);
    a.kept_idx = kept_idx;
    a.n_kept = n_kept;
    a.max_kept = max_kept;
    const int jobs = (src->Hkv * (src->v ? 2 : 1) + 3) / 4;
    a.piece = compact_piece((int64_t)max_kept * src->B * jobs, ctx->num_cu);
    const dim3 grid((unsigned)(max_kept / a.piece + src->R_max), (unsigned)src->B, (unsigned)jobs);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (src->dtype == RA_BF16 && src->d == 128) hipLaunchKernelGGL((compact_rounds_kernel<uint16_t, 128>), grid, dim3(256), 0, st, a);
    else if (src->dtype == RA_BF16) hipLaunchKernelGGL((compact_rounds_kernel<uint16_t, 64>), grid, dim3(256), 0, st, a);
    else if (src->d == 128) hipLaunchKernelGGL((compact_rounds_kernel<uint32_t, 128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((compact_rounds_kernel<uint32_t, 64>), grid, dim3(256), 0, st, a);
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
