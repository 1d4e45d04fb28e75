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

typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));

// One more of `bin` for every lane of the wave that has one: lanes that agree with the first of them are added up before (weights
// of zero, which whole rounds have, would otherwise queue at one address).
__device__ __forceinline__ void count_bin(int* hist, bool has, int bin) {
    const unsigned long long all = __ballot(has);
    if (!all) return;
    const int lane = threadIdx.x & 63, leader = __ffsll(all) - 1, common = __builtin_amdgcn_readlane(bin, leader);
    const unsigned long long same = __ballot(has && bin == common);
    if (lane == leader) atomicAdd(&hist[common], __popcll(same));
    else if (has && bin != common) atomicAdd(&hist[bin], 1);
}

// One workgroup per sequence.  The `need` largest weights of the middle (what is neither among the first nor the last tokens) are
// those above a threshold key and, of those equal to it, the first ones.  The threshold is found digit by digit from counts of
// the candidates that share the digits before: over the weights for the first digit; the candidates that share it then lie in
// LDS as a rule, and the other digits are counted there (if they are more, over the weights).
// Every wave has a contiguous sixteenth of the positions: it knows how many of them it keeps, and writes them behind what the
// waves before it keep.  Counts are whole numbers: their order does not matter.
//
// Bound by a compute unit's share of the cache bandwidth and its round trips: three passes over the weights, 2 KB a wave and
// instruction group in flight.
__global__ __launch_bounds__(kSelThreads) void select_tokens_kernel(SelectTokensArgs a) {
    __shared__ int s_hist[kBins];
    __shared__ int s_start[kMaxRounds + 1], s_below[kMaxRounds + 1];
    __shared__ int s_wave[kSelWaves][2];  // positions that are kept for certain, positions with the threshold's key
    __shared__ uint2 s_cand[kCandidates];  // key, position
    __shared__ uint32_t s_digit;
    __shared__ int s_left, s_count, s_total;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float* w = a.weights + (size_t)b * a.n_pos;
    const int n_rounds = min(max(a.n_rounds[b], 0), a.R_max);
    // first positions of the rounds
    if (wave == 0) {
        int before = 0;
        for (int r0 = 0; r0 < a.R_max; r0 += 64) {
            const int r = r0 + lane, len = r < n_rounds ? max(a.seg_len[(size_t)b * a.R_max + r], 0) : 0;
            const int incl = wave_inclusive_sum(len);
            if (r < a.R_max) s_start[r] = min(before + incl - len, a.n_pos);
            before = min(before + __builtin_amdgcn_readlane(incl, 63), a.n_pos);
        }
        if (lane == 0) s_start[a.R_max] = s_total = before;
    }
    for (int i = tid; i < kBins; i += kSelThreads) s_hist[i] = 0;
    if (tid < kSelWaves) s_wave[tid][0] = s_wave[tid][1] = 0;
    if (tid == 0) s_count = 0;
    __syncthreads();
    const int n = s_total, K = min(a.budget, n);
    const int first = min(a.keep_first, n), last = min(a.keep_last, n - first);
    const int lo = first, hi = n - last, need = K - first - last;  // of the positions lo .. hi - 1

    // The wave's positions, kChunk at a time: f(first position of the chunk, the lane's four weights).  Past the end: zeros.
    const int chunks = (n + kChunk - 1) / kChunk, c_lo = chunks * wave / kSelWaves, c_hi = chunks * (wave + 1) / kSelWaves;
    auto each_chunk = [&](auto f) {
        for (int c0 = c_lo; c0 < c_hi; c0 += kChunks) {
            float x[kChunks][4];
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
                for (int e = 0; e < 4; ++e) x[j][e] = v[e];
            }
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
                if (c0 + j < c_hi) f((c0 + j) * kChunk, x[j]);
        }
    };
    // The digit at which the counts, from the largest one down, reach `left`; what is left of it then, and the candidates there.
    auto find_digit = [&](int bits, int left) {
        if (wave == 0) {
            int taken = 0;
            for (int i0 = (1 << bits) - 64; i0 >= 0; i0 -= 64) {
                const int bin = i0 + 63 - lane, c = s_hist[bin], incl = wave_inclusive_sum(c);
                const unsigned long long reached = __ballot(taken + incl >= left);
                if (reached) {
                    if (lane == __ffsll(reached) - 1) {
                        s_digit = (uint32_t)bin;
                        s_left = left - (taken + incl - c);
                        s_total = c;
                    }
                    break;
                }
                taken += __builtin_amdgcn_readlane(incl, 63);
            }
        }
        __syncthreads();
    };
    auto clear_bins = [&] {
        for (int i = tid; i < kBins; i += kSelThreads) s_hist[i] = 0;
        __syncthreads();
    };

    uint32_t threshold = 0;  // keys above it are kept, and the first `equal` of those equal to it
    int equal = 0;
    const bool all = need >= hi - lo, none = need <= 0;
    bool counted = false;  // s_wave is complete
    if (!all && !none) {
        constexpr int kShift1 = 32 - kDigit, kShift2 = kShift1 - kDigit;
        each_chunk([&](int p0, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int p = p0 + lane * 4 + e;
                count_bin(s_hist, p >= lo && p < hi, weight_key(x[e]) >> kShift1);
            }
        });
        __syncthreads();
        find_digit(kDigit, need);
        const uint32_t digit1 = s_digit;
        threshold = digit1 << kShift1;
        int left = s_left;
        const bool in_lds = s_total <= kCandidates;
        clear_bins();
        if (in_lds) {
            int sure = 0;
            each_chunk([&](int p0, const float (&x)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = p0 + lane * 4 + e;
                    const uint32_t key = weight_key(x[e]), digit = key >> kShift1;
                    const bool middle = p >= lo && p < hi;
                    sure += __popcll(__ballot(p < n && (!middle || digit > digit1)));
                    const unsigned long long take = __ballot(middle && digit == digit1);
                    if (!take) continue;
                    int at = 0;
                    if (lane == 0) at = atomicAdd(&s_count, __popcll(take));
                    at = __builtin_amdgcn_readfirstlane(at) + __popcll(take & ((1ull << lane) - 1));
                    if (take >> lane & 1) s_cand[at] = make_uint2(key, (uint32_t)p);
                }
            });
            if (lane == 0) s_wave[wave][0] = sure;
            __syncthreads();
            const int n_cand = s_count;
            for (int i = tid; i < n_cand; i += kSelThreads) atomicAdd(&s_hist[s_cand[i].x >> kShift2 & (kBins - 1)], 1);
            __syncthreads();
            find_digit(kDigit, left);
            threshold |= s_digit << kShift2;
            left = s_left;
            clear_bins();
            for (int i = tid; i < n_cand; i += kSelThreads)
                if (s_cand[i].x >> kShift2 == threshold >> kShift2) atomicAdd(&s_hist[s_cand[i].x & ((1 << kShift2) - 1)], 1);
            __syncthreads();
            find_digit(kShift2, left);
            threshold |= s_digit;
            equal = s_left;
            for (int i = tid; i < n_cand; i += kSelThreads) {
                if (s_cand[i].x < threshold) continue;
                // the wave whose positions these are: the last one that begins at or before the chunk
                const int c = (int)s_cand[i].y / kChunk;
                int owner = (int)(((long long)c * kSelWaves) / chunks);
                while (owner + 1 < kSelWaves && chunks * (owner + 1) / kSelWaves <= c) ++owner;
                atomicAdd(&s_wave[owner][s_cand[i].x == threshold], 1);
            }
            counted = true;
        } else {
            each_chunk([&](int p0, const float (&x)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = p0 + lane * 4 + e;
                    const uint32_t key = weight_key(x[e]);
                    count_bin(s_hist, p >= lo && p < hi && key >> kShift1 == digit1, key >> kShift2 & (kBins - 1));
                }
            });
            __syncthreads();
            find_digit(kDigit, left);
            threshold |= s_digit << kShift2;
            left = s_left;
            clear_bins();
            each_chunk([&](int p0, const float (&x)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = p0 + lane * 4 + e;
                    const uint32_t key = weight_key(x[e]);
                    count_bin(s_hist, p >= lo && p < hi && key >> kShift2 == threshold >> kShift2, key & ((1 << kShift2) - 1));
                }
            });
            __syncthreads();
            find_digit(kShift2, left);
            threshold |= s_digit;
            equal = s_left;
        }
    }
    // 0: dropped, 1: kept, 2: kept if it is among the first `equal` of its kind
    auto fate = [&](int p, float x) {
        const uint32_t key = weight_key(x);
        const int of_middle = all ? 1 : none ? 0 : key > threshold ? 1 : key == threshold ? 2 : 0;
        return p >= n ? 0 : p < lo || p >= hi ? 1 : of_middle;
    };
    if (!counted) {
        int n_sure = 0, n_equal = 0;
        each_chunk([&](int p0, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int f = fate(p0 + lane * 4 + e, x[e]);
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
    int at = 0, equal_before = 0;
    for (int i = 0; i < wave; ++i) {
        at += s_wave[i][0];
        equal_before += s_wave[i][1];
    }
    at += min(equal_before, equal);
    int32_t* idx = a.kept_idx + (size_t)b * a.budget;
    float* left_over = a.kept_weights ? a.kept_weights + (size_t)b * a.n_pos : nullptr;
    // the round whose start comes next: the first that starts at or behind this wave's part (the first wave: round 0)
    int round = 0;
    for (int r0 = 0; r0 <= a.R_max; r0 += 64)
        round += __popcll(__ballot(r0 + lane <= a.R_max && s_start[min(r0 + lane, a.R_max)] < c_lo * kChunk));
    const unsigned long long below_lane = (1ull << lane) - 1;
    each_chunk([&](int p0, const float (&x)[4]) {
        // positions in order: lane by lane, four each
        unsigned long long kept[4], maybe[4];
        int f[4], eq = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = fate(p0 + lane * 4 + e, x[e]);
            maybe[e] = __ballot(f[e] == 2);
            eq += __popcll(maybe[e] & below_lane);
        }
        eq += equal_before;
        int j = at;
        bool mine[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            mine[e] = f[e] == 1 || (f[e] == 2 && eq < equal);
            eq += f[e] == 2;
            kept[e] = __ballot(mine[e]);
            j += __popcll(kept[e] & below_lane);
        }
        while (round <= a.R_max && s_start[round] < p0 + kChunk) {
            const int in = s_start[round] - p0, in_lane = in >> 2, in_e = in & 3;
            int below = at;
#pragma unroll
            for (int e = 0; e < 4; ++e) below += __popcll(kept[e] & ((1ull << in_lane) - 1)) + (e < in_e && (kept[e] >> in_lane & 1));
            if (lane == 0) s_below[round] = below;
            ++round;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (mine[e]) {
                idx[j] = p0 + lane * 4 + e;
                if (left_over) left_over[j] = x[e];
                ++j;
            }
            at += __popcll(kept[e]);
            equal_before += __popcll(maybe[e]);
        }
    });
    for (int j = K + tid; j < a.budget; j += kSelThreads) idx[j] = -1;
    if (left_over)
        for (int j = K + tid; j < a.n_pos; j += kSelThreads) left_over[j] = 0.f;
    // starts behind the last chunk (and all of them, if there are no tokens): everything kept lies below
    for (int r = tid; r <= a.R_max; r += kSelThreads)
        if (s_start[r] >= chunks * kChunk) s_below[r] = K;
    __syncthreads();
    if (wave == 0) {
        long long off = (long long)b * a.stride;
        for (int r0 = 0; r0 < a.R_max; r0 += 64) {
            const int r = r0 + lane, len = r < a.R_max ? s_below[r + 1] - s_below[r] : 0;
            const int blocks = (len + 15) / 16, incl = wave_inclusive_sum(blocks);
            if (r < a.R_max) {
                a.kept_len[(size_t)b * a.R_max + r] = len;
                if (a.kept_off) a.kept_off[(size_t)b * a.R_max + r] = off + (long long)(incl - blocks) * a.unit;
            }
            off += (long long)__builtin_amdgcn_readlane(incl, 63) * a.unit;
        }
        if (lane == 0) a.n_kept[b] = K;
    }
}

// ---- the smaller cache -------------------------------------------------------------------------------------------------------
struct CompactArgs {
    DevView src, dst;
    const int32_t *kept_idx, *n_kept;
    int max_kept;
};

constexpr int kCompactTokens = 128;  // kept tokens that a workgroup moves: eight tiles, of one round

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

// grid (pieces of kCompactTokens of a sequence's rounds, B).  A wave moves the keys or the values of one head at a time.
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
            const int pieces = (d + kCompactTokens - 1) / kCompactTokens;
            const int end = wave_inclusive_sum(pieces), d_end = wave_inclusive_sum(d), s_end = wave_inclusive_sum(s);
            const int target = (int)blockIdx.x - pieces_before;
            const unsigned long long in = __ballot(end > target && end - pieces <= target);
            if (in) {
                const int at = __ffsll(in) - 1;
                round = r0 + at;
                len = __builtin_amdgcn_readlane(d, at);
                src_len = __builtin_amdgcn_readlane(s, at);
                t0 = (target - (__builtin_amdgcn_readlane(end, at) - __builtin_amdgcn_readlane(pieces, at))) * kCompactTokens;
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
    const int here = min(kCompactTokens, len - t0);
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

}  // namespace ra

using namespace ra;

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
    RA_REQUIRE(kept_weights != weights, RA_ERR_INVALID_ARG, "select_tokens: kept_weights must be another buffer than weights");
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
    hipLaunchKernelGGL(select_tokens_kernel, dim3((unsigned)B), dim3(kSelThreads), 0, reinterpret_cast<hipStream_t>(stream), a);
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
    const dim3 grid((unsigned)(max_kept / kCompactTokens + src->R_max), (unsigned)src->B, (unsigned)((src->Hkv * (src->v ? 2 : 1) + 3) / 4));
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (src->dtype == RA_BF16 && src->d == 128) hipLaunchKernelGGL((compact_rounds_kernel<uint16_t, 128>), grid, dim3(256), 0, st, a);
    else if (src->dtype == RA_BF16) hipLaunchKernelGGL((compact_rounds_kernel<uint16_t, 64>), grid, dim3(256), 0, st, a);
    else if (src->d == 128) hipLaunchKernelGGL((compact_rounds_kernel<uint32_t, 128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((compact_rounds_kernel<uint32_t, 64>), grid, dim3(256), 0, st, a);
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
