// Attention weight of every history token, summed over the query tokens and heads of a call and added to a running total:
//   weights[p] = prev[p] + sum_{i,h} exp(scale q_ih . k_p - lse_ih).
// The attention call has left the log-sum-exp of every row, so one pass over the keys gives the probabilities themselves: no
// maximum, no second pass, and nothing that a token owes to another.
//
// Roles: S [16 rows x 16 tokens] = Q . K^T by matrix instructions, token = lane % 16, rows 4 (lane / 16) + i.  A lane adds up
// the rows that it meets of its token in one register; the four lane groups are added at the very end.  A row's term is
// 2^(c s - lse log2 e): one fused multiply-add, one exponential, one addition.
#include "common.hpp"
#include "mfma_util.hpp"
#include "stream_kv.hpp"

#include <type_traits>

namespace ra {

struct WeightArgs {
    DevView view;
    const void* q;           // [B][q_len][Hq][D]
    const float* lse;        // [B][q_len][Hq]
    const int32_t* sel_idx;  // [B][R_max] or null
    const int32_t* n_sel;
    const float* prev;  // [B][n_pos] or null
    float* weights;     // [B][n_pos]
    int q_len, Hq, G, n_pos;
    float c;  // scale * log2(e)
};

constexpr int kWeightTile = 32;  // tokens of a tile, which never crosses a round
constexpr int kWeightRows = 512;  // rows whose log-sum-exps are staged at a time

// Operand fragments of 16 rows of keys or queries and their product, per type.
template <typename T, int D>
struct Rows16;
template <int D>
struct Rows16<BF16, D> {
    static constexpr int EB = 2, N = D / 32;
    uint4 x[N];
    __device__ __forceinline__ void load(const char* row, int q4) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = reinterpret_cast<const uint4*>(row)[i * 4 + q4];
    }
    __device__ static __forceinline__ floatx4_t product(const Rows16& a, const Rows16& b) {
        floatx4_t s = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < N; ++i) s = mfma16(a.x[i], b.x[i], s);
        return s;
    }
};
template <int D>
struct Rows16<F32, D> {  // product e of step j takes channels 16 j + 4 (lane / 16) + e
    static constexpr int EB = 4, N = D / 16;
    float4 x[N];
    __device__ __forceinline__ void load(const char* row, int q4) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = reinterpret_cast<const float4*>(row)[i * 4 + q4];
    }
    __device__ static __forceinline__ floatx4_t product(const Rows16& a, const Rows16& b) {
        floatx4_t s = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].x, b.x[i].x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].y, b.x[i].y, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].z, b.x[i].z, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].w, b.x[i].w, s, 0, 0, 0);
        }
        return s;
    }
};

// grid (tiles of a sequence, B).  Workgroup = one tile; its four waves take the KV heads in turn, each all rows of its heads,
// and are added up in the order of the waves.
template <typename T, int D, bool PAGED>
__global__ __launch_bounds__(256) void token_weights_kernel(WeightArgs a) {
    typedef Rows16<T, D> Rows;
    __shared__ float s_sum[4][kWeightTile];
    __shared__ float s_lse[4][kWeightRows];
    const DevView& vw = a.view;
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, n = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n_rounds = min(max(vw.n_rounds[b], 0), vw.R_max);
    const int32_t* lens = vw.seg_len + (size_t)b * vw.R_max;

    // ---- the tile's round, and the tokens before it (every wave for itself) --------------------------------------------
    int round = -1, tile = blockIdx.x, pos = 0, len = 0, total = 0;
    {
        int tiles_before = 0;
        for (int r0 = 0; r0 < n_rounds; r0 += 64) {
            const int r = r0 + lane, mine = r < n_rounds ? max(lens[r], 0) : 0;
            const int tiles = (mine + kWeightTile - 1) / kWeightTile;
            const int tile_end = wave_inclusive_sum(tiles), tok_end = wave_inclusive_sum(mine);
            const int target = (int)blockIdx.x - tiles_before;
            const unsigned long long in = __ballot(tiles > 0 && tile_end > target && tile_end - tiles <= target);
            if (round < 0 && in) {
                const int at = __ffsll(in) - 1;
                round = r0 + at;
                len = __builtin_amdgcn_readlane(mine, at);
                tile = target - (__builtin_amdgcn_readlane(tile_end, at) - __builtin_amdgcn_readlane(tiles, at));
                pos = total + __builtin_amdgcn_readlane(tok_end, at) - len;
            }
            tiles_before += __builtin_amdgcn_readlane(tile_end, 63);
            total += __builtin_amdgcn_readlane(tok_end, 63);
        }
    }
    const float* prev = a.prev ? a.prev + (size_t)b * a.n_pos : nullptr;
    float* out = a.weights + (size_t)b * a.n_pos;
    // positions behind the last token, by the first workgroup of the sequence
    if (blockIdx.x == 0)
        for (int p = total + tid; p < a.n_pos; p += 256) out[p] = prev ? prev[p] : 0.f;
    if (round < 0) return;
    int times = a.sel_idx ? 0 : 1;  // how often the list names the round
    if (a.sel_idx) {
        const int listed = min(max(a.n_sel[b], 0), vw.R_max);
        for (int i0 = 0; i0 < listed; i0 += 64)
            times += __popcll(__ballot(i0 + lane < listed && a.sel_idx[(size_t)b * vw.R_max + min(i0 + lane, listed - 1)] == round));
    }
    const int tok0 = tile * kWeightTile, ntok = min(kWeightTile, len - tok0);
    float sum[2] = {0.f, 0.f};
    if (times > 0) {
        const int rows = a.q_len * a.G;
        const char* kbase = static_cast<const char*>(vw.k);
        const long long off = vw.seg_off[(size_t)b * vw.R_max + round];
        for (int g = wave; g < vw.Hkv; g += 4) {
            Rows keys[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = min(tok0 + h * 16 + n, len - 1);
                size_t row;
                if (PAGED) {
                    const long long at = min(max(off + t / 16, 0ll), (long long)vw.max_blocks - 1);
                    row = ((size_t)max(vw.block_table[(size_t)b * vw.max_blocks + at], 0) * vw.Hkv + g) * 16 + t % 16;
                } else {
                    row = (size_t)off * vw.Hkv + (size_t)g * len + t;
                }
                keys[h].load(kbase + row * D * Rows::EB, q4);
            }
            for (int r0 = 0; r0 < rows; r0 += kWeightRows) {
                const int here = min(kWeightRows, rows - r0);
                __builtin_amdgcn_wave_barrier();
                for (int r = lane; r < ((here + 15) & ~15); r += 64) {  // rows that add nothing: 2^-infinity
                    float x = __builtin_inff();
                    if (r < here) {
                        const int i = (r0 + r) / a.G, h = r0 + r - i * a.G;
                        x = a.lse[((size_t)b * a.q_len + i) * a.Hq + (size_t)g * a.G + h] * kLog2e;
                    }
                    s_lse[wave][r] = __builtin_fabsf(x) < __builtin_inff() ? x : __builtin_inff();
                }
                __builtin_amdgcn_wave_barrier();
                for (int r = 0; r < here; r += 16) {
                    const int row = min(r0 + r + n, rows - 1), i = row / a.G, h = row - i * a.G;
                    Rows q;
                    q.load(static_cast<const char*>(a.q) + (((size_t)b * a.q_len + i) * a.Hq + (size_t)g * a.G + h) * D * Rows::EB, q4);
                    // the queries of such a row may be anything
                    if (s_lse[wave][r + n] == __builtin_inff()) q = Rows{};
                    const floatx4_t l = *reinterpret_cast<const floatx4_t*>(&s_lse[wave][r + 4 * q4]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const floatx4_t s = Rows::product(q, keys[k]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[k] += fast_exp2(__builtin_fmaf(s[e], a.c, -l[e]));
                    }
                }
            }
        }
    }
    // ---- lane groups, then waves, in a fixed order -----------------------------------------------------------------------
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        sum[h] = xrow_sum4(sum[h]);
        if (q4 == 0) s_sum[wave][h * 16 + n] = sum[h];
    }
    __syncthreads();
    if (tid < ntok && pos + tok0 + tid < a.n_pos) {
        const int p = pos + tok0 + tid;
        const float add = (s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]);
        out[p] = (prev ? prev[p] : 0.f) + add * (float)times;
    }
}

}  // namespace ra

using namespace ra;

extern "C" int ra_token_weights(ra_ctx* ctx, void* stream, const void* q, int q_len, int Hq, const ra_kv_view* layer,
                                const int32_t* sel_idx, const int32_t* n_sel, const float* lse, float scale, const float* prev,
                                float* weights, int n_pos) {
    RA_REQUIRE(ctx != nullptr, RA_ERR_INVALID_ARG, "token_weights: ctx is NULL");
    RA_REQUIRE(q_len > 0, RA_ERR_INVALID_ARG, "token_weights: q_len must be positive");
    RA_REQUIRE(n_pos > 0, RA_ERR_INVALID_ARG, "token_weights: n_pos must be positive");
    RA_REQUIRE(q != nullptr && lse != nullptr && weights != nullptr, RA_ERR_INVALID_ARG, "token_weights: q, lse or weights is NULL");
    if (int rc = check_view(layer, false, "token_weights")) return rc;
    RA_REQUIRE(layer->R_max > 0, RA_ERR_INVALID_ARG, "token_weights: R_max is 0, there is nothing to weigh");
    RA_REQUIRE(Hq > 0 && Hq % layer->Hkv == 0, RA_ERR_INVALID_ARG, "token_weights: Hq %d is not a multiple of Hkv %d", Hq, layer->Hkv);
    RA_REQUIRE((sel_idx == nullptr) == (n_sel == nullptr), RA_ERR_INVALID_ARG,
               "token_weights: sel_idx and n_sel must both be given or both be NULL");
    RA_REQUIRE(scale > 0.f && scale == scale, RA_ERR_INVALID_ARG, "token_weights: scale must be positive");
    RA_REQUIRE(layer->d == 64 || layer->d == 128, RA_ERR_UNSUPPORTED, "token_weights: head_dim %d not in {64, 128}", layer->d);
    const int G = Hq / layer->Hkv;
    RA_REQUIRE(G <= 16, RA_ERR_UNSUPPORTED, "token_weights: Hq / Hkv = %d exceeds 16", G);
    RA_REQUIRE(layer->B <= 65535, RA_ERR_UNSUPPORTED, "token_weights: batch %d exceeds 65535", layer->B);
    RA_REQUIRE((((uintptr_t)q | (uintptr_t)layer->k) & 15) == 0, RA_ERR_INVALID_ARG, "token_weights: q and keys must be 16-byte aligned");
    const int64_t tiles = layer->max_tokens / kWeightTile + layer->R_max;
    RA_REQUIRE(tiles < (int64_t)1 << 24, RA_ERR_UNSUPPORTED, "token_weights: max_tokens too large");
    WeightArgs a = {};
    a.view = to_dev(layer);
    a.q = q;
    a.lse = lse;
    a.sel_idx = sel_idx;
    a.n_sel = n_sel;
    a.prev = prev;
    a.weights = weights;
    a.q_len = q_len;
    a.Hq = Hq;
    a.G = G;
    a.n_pos = n_pos;
    a.c = scale * kLog2e;
    const dim3 grid((unsigned)tiles, (unsigned)layer->B);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    KernelTimer timer(ctx, st);
    const bool bf16 = layer->dtype == RA_BF16, wide = layer->d == 128, paged = layer->block_size != 0;
#define RA_WEIGHTS_CASE(T_, D_, P_)                                                                              \
    if (bf16 == std::is_same<T_, BF16>::value && wide == (D_ == 128) && paged == P_)                             \
        RA_LAUNCH_TIMED((token_weights_kernel<T_, D_, P_>), grid, dim3(256), 0, st, a);
    RA_WEIGHTS_CASE(BF16, 128, false) RA_WEIGHTS_CASE(BF16, 128, true) RA_WEIGHTS_CASE(BF16, 64, false) RA_WEIGHTS_CASE(BF16, 64, true)
    RA_WEIGHTS_CASE(F32, 128, false) RA_WEIGHTS_CASE(F32, 128, true) RA_WEIGHTS_CASE(F32, 64, false) RA_WEIGHTS_CASE(F32, 64, true)
#undef RA_WEIGHTS_CASE
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
