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
constexpr int kDigit = 11, kBins = 1 << kDigit;  // three passes: 11, 11 and 10 bits of the key

// One workgroup per sequence.  The `need` largest weights of the middle (what is neither among the first nor the last tokens) are
// those above a threshold key, found digit by digit from counts of the candidates that share the digits before, and, of those
// equal to it, the first ones.  Then every wave takes a contiguous sixteenth of the positions: it counts what it keeps, and
// writes it behind what the waves before it keep.  Counts are whole numbers: their order does not matter.
__global__ __launch_bounds__(kSelThreads) void select_tokens_kernel(SelectTokensArgs a) {
    __shared__ int s_hist[kBins];
    __shared__ int s_start[kMaxRounds + 1], s_below[kMaxRounds + 1];
    __shared__ int s_wave[kSelWaves][2];
    __shared__ uint32_t s_digit;
    __shared__ int s_left, s_total;
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
    __syncthreads();
    const int n = s_total, K = min(a.budget, n);
    const int first = min(a.keep_first, n), last = min(a.keep_last, n - first);
    const int lo = first, hi = n - last, need = K - first - last;  // of the positions lo .. hi - 1

    uint32_t threshold = 0;  // keys above it are kept, and the first `equal` of those equal to it
    int equal = 0;
    if (need > 0 && need < hi - lo) {
        int left = need;
        for (int shift = 32 - kDigit; ; shift = max(shift - kDigit, 0)) {
            // (the last digit is shorter: its upper bits are part of the one before)
            const int bits = shift == 32 - kDigit ? kDigit : shift > 0 ? kDigit : 32 - 2 * kDigit;
            for (int i = tid; i < kBins; i += kSelThreads) s_hist[i] = 0;
            __syncthreads();
            const int above = shift + bits;
            for (int p = lo + tid; p < hi; p += kSelThreads) {
                const uint32_t key = weight_key(w[p]);
                if (above == 32 || key >> above == threshold >> above) atomicAdd(&s_hist[key >> shift & ((1u << bits) - 1)], 1);
            }
            __syncthreads();
            if (wave == 0) {  // from the largest digit down: the first at which the count reaches what is left
                int taken = 0;
                for (int i0 = (1 << bits) - 64; i0 >= 0; i0 -= 64) {
                    const int bin = i0 + 63 - lane, c = s_hist[bin], incl = wave_inclusive_sum(c);
                    const unsigned long long reached = __ballot(taken + incl >= left);
                    if (reached) {
                        const int at = __ffsll(reached) - 1;
                        if (lane == at) {
                            s_digit = (uint32_t)bin;
                            s_left = left - (taken + incl - c);
                        }
                        break;
                    }
                    taken += __builtin_amdgcn_readlane(incl, 63);
                }
            }
            __syncthreads();
            threshold |= s_digit << shift;
            left = s_left;
            if (shift == 0) break;
        }
        equal = left;
    }
    const bool all = need >= hi - lo, none = need <= 0;
    // 0: dropped, 1: kept, 2: kept if it is among the first `equal` of its kind
    auto fate = [&](int p, float x) {
        if (p >= n) return 0;
        if (p < lo || p >= hi || all) return 1;
        if (none) return 0;
        const uint32_t key = weight_key(x);
        return key > threshold ? 1 : key == threshold ? 2 : 0;
    };
    const int chunks = (n + 63) / 64, c_lo = chunks * wave / kSelWaves, c_hi = chunks * (wave + 1) / kSelWaves;
    int n_sure = 0, n_equal = 0;
    for (int c = c_lo; c < c_hi; ++c) {
        const int p = c * 64 + lane, f = fate(p, p < n ? w[p] : 0.f);
        n_sure += __popcll(__ballot(f == 1));
        n_equal += __popcll(__ballot(f == 2));
    }
    if (lane == 0) {
        s_wave[wave][0] = n_sure;
        s_wave[wave][1] = n_equal;
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
    if (c_lo < c_hi) {
        for (int r0 = 0; r0 <= a.R_max; r0 += 64)
            round += __popcll(__ballot(r0 + lane <= a.R_max && s_start[min(r0 + lane, a.R_max)] < c_lo * 64));
    }
    const unsigned long long below_lane = (1ull << lane) - 1;
    for (int c = c_lo; c < c_hi; ++c) {
        const int p = c * 64 + lane;
        const float x = p < n ? w[p] : 0.f;
        const int f = fate(p, x);
        const unsigned long long maybe = __ballot(f == 2);
        const unsigned long long kept = __ballot(f == 1 || (f == 2 && equal_before + __popcll(maybe & below_lane) < equal));
        while (round <= a.R_max && s_start[round] < c * 64 + 64) {
            const int in = s_start[round] - c * 64;
            if (lane == 0) s_below[round] = at + __popcll(kept & ((1ull << in) - 1));
            ++round;
        }
        if (kept >> lane & 1) {
            const int j = at + __popcll(kept & below_lane);
            idx[j] = p;
            if (left_over) left_over[j] = x;
        }
        at += __popcll(kept);
        equal_before += __popcll(maybe);
    }
    for (int j = K + tid; j < a.budget; j += kSelThreads) idx[j] = -1;
    if (left_over)
        for (int j = K + tid; j < a.n_pos; j += kSelThreads) left_over[j] = 0.f;
    __syncthreads();
    // starts behind the last whole chunk (and all of them, if there are no tokens): everything kept lies below
    for (int r = tid; r <= a.R_max; r += kSelThreads)
        if (s_start[r] >= chunks * 64) s_below[r] = K;
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

template <typename T, int D>
__device__ __forceinline__ size_t key_row(const DevView& v, int b, long long off, int len, int g, int t) {
    if (v.block_size) {
        const long long at = min(max(off + t / 16, 0ll), (long long)v.max_blocks - 1);
        return ((size_t)max(v.block_table[(size_t)b * v.max_blocks + at], 0) * v.Hkv + g) * 16 + t % 16;
    }
    return (size_t)off * v.Hkv + (size_t)g * len + t;
}
// First element of the value tile that holds token t.
template <typename T, int D>
__device__ __forceinline__ size_t value_tile(const DevView& v, int b, long long off_k, long long off_v, int len, int g, int t) {
    if (v.block_size) {
        const long long at = min(max(off_k + t / 16, 0ll), (long long)v.max_blocks - 1);
        return ((size_t)max(v.block_table[(size_t)b * v.max_blocks + at], 0) * v.Hkv + g) * D * 16;
    }
    return ((size_t)off_v * v.Hkv + (size_t)g * ((len + 15) & ~15) + (t & ~15)) * D;
}

// grid (value tiles of a sequence's smaller cache, B): a workgroup makes one tile of 16 tokens for every KV head, a wave a
// head at a time.
template <typename T, int D>
__global__ __launch_bounds__(256) void compact_rounds_kernel(CompactArgs a) {
    constexpr int kPieces = D * sizeof(T) / 16;  // of a key row
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = a.src.R_max, n_src = min(max(a.src.n_rounds[b], 0), R), n_dst = min(max(a.dst.n_rounds[b], 0), R);
    const size_t row = (size_t)b * R;
    // the tile's round: its lengths in both caches, and what lies before it
    int round = -1, tile = 0, len = 0, first = 0, src_len = 0, src_first = 0;
    {
        int tiles_before = 0, dst_before = 0, src_before = 0;
        for (int r0 = 0; r0 < n_dst && round < 0; r0 += 64) {
            const int r = r0 + lane;
            const int d = r < n_dst ? max(a.dst.seg_len[row + r], 0) : 0, s = r < n_src ? max(a.src.seg_len[row + r], 0) : 0;
            const int tiles = (d + 15) / 16;
            const int tile_end = wave_inclusive_sum(tiles), d_end = wave_inclusive_sum(d), s_end = wave_inclusive_sum(s);
            const int target = (int)blockIdx.x - tiles_before;
            const unsigned long long in = __ballot(tile_end > target && tile_end - tiles <= target);
            if (in) {
                const int at = __ffsll(in) - 1;
                round = r0 + at;
                len = __builtin_amdgcn_readlane(d, at);
                src_len = __builtin_amdgcn_readlane(s, at);
                tile = target - (__builtin_amdgcn_readlane(tile_end, at) - __builtin_amdgcn_readlane(tiles, at));
                first = dst_before + __builtin_amdgcn_readlane(d_end, at) - len;
                src_first = src_before + __builtin_amdgcn_readlane(s_end, at) - src_len;
            }
            tiles_before += __builtin_amdgcn_readlane(tile_end, 63);
            dst_before += __builtin_amdgcn_readlane(d_end, 63);
            src_before += __builtin_amdgcn_readlane(s_end, 63);
        }
    }
    if (round < 0) return;
    // lane % 16: the tile's token, and where it comes from (-1: nowhere)
    const int t = tile * 16 + (lane & 15), j = first + t;
    int from = -1;
    if (t < len && j < min(max(a.n_kept[b], 0), a.max_kept)) {
        from = a.kept_idx[(size_t)b * a.max_kept + j] - src_first;
        if (from < 0 || from >= src_len) from = -1;
    }
    const long long so = a.src.seg_off[row + round], sv = a.src.seg_off_v[row + round];
    const long long dof = a.dst.seg_off[row + round], dv = a.dst.seg_off_v[row + round];
    const int Hkv = a.src.Hkv;
    for (int g = wave; g < Hkv; g += 4) {
        for (int x = lane; x < 16 * kPieces; x += 64) {
            const int i = x / kPieces, c = x % kPieces, src_t = __shfl(from, i, 64);
            if (tile * 16 + i >= len) continue;
            uint4 k = make_uint4(0, 0, 0, 0);
            if (src_t >= 0)
                k = reinterpret_cast<const uint4*>(static_cast<const T*>(a.src.k) + key_row<T, D>(a.src, b, so, src_len, g, src_t) * D)[c];
            reinterpret_cast<uint4*>(static_cast<T*>(const_cast<void*>(a.dst.k)) + key_row<T, D>(a.dst, b, dof, len, g, tile * 16 + i) * D)[c] = k;
        }
        if (a.src.v == nullptr) continue;
        T* out = static_cast<T*>(const_cast<void*>(a.dst.v)) + value_tile<T, D>(a.dst, b, dof, dv, len, g, tile * 16);
        const size_t my_tile = from >= 0 ? value_tile<T, D>(a.src, b, so, sv, src_len, g, from) + (from & 15) : 0;
        for (int c = lane; c < D; c += 64) {
            union {
                T e[16];
                uint4 u[sizeof(T)];
            } v;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const size_t at = ((size_t)(unsigned)__shfl((int)(my_tile >> 32), i, 64) << 32) | (unsigned)__shfl((int)my_tile, i, 64);
                v.e[i] = __shfl(from, i, 64) >= 0 ? static_cast<const T*>(a.src.v)[at + c * 16] : T(0);
            }
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4*>(out + c * 16)[i] = v.u[i];
        }
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
    RA_REQUIRE((((uintptr_t)src->k | (uintptr_t)src->v | (uintptr_t)dst->k | (uintptr_t)dst->v) & 15) == 0, RA_ERR_INVALID_ARG,
               "compact_rounds: keys and values must be 16-byte aligned");
    CompactArgs a = {};
    a.src = to_dev(src);
    a.dst = to_dev(dst);
    a.kept_idx = kept_idx;
    a.n_kept = n_kept;
    a.max_kept = max_kept;
    const dim3 grid((unsigned)(max_kept / 16 + src->R_max), (unsigned)src->B);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (src->dtype == RA_BF16 && src->d == 128) hipLaunchKernelGGL((compact_rounds_kernel<uint16_t, 128>), grid, dim3(256), 0, st, a);
    else if (src->dtype == RA_BF16) hipLaunchKernelGGL((compact_rounds_kernel<uint16_t, 64>), grid, dim3(256), 0, st, a);
    else if (src->d == 128) hipLaunchKernelGGL((compact_rounds_kernel<uint32_t, 128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((compact_rounds_kernel<uint32_t, 64>), grid, dim3(256), 0, st, a);
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
