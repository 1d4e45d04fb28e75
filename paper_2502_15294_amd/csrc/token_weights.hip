// Attention weight of every history token, summed over the query tokens and heads of a call and added to a running total:
//   weights[p] = prev[p] + sum_{i,h} exp(scale q_ih . k_p - lse_ih).
// The attention call has left the log-sum-exp of every row, so one pass over the keys gives the probabilities themselves: no
// maximum, no second pass, and nothing that a token owes to another.
//
// Roles: S [16 rows x 16 tokens] = Q . K^T by matrix instructions, token = lane % 16, rows 4 (lane / 16) + i.  A lane adds up
// the rows that it meets of its token in one register; the four lane groups are added at the very end.  A row's term is
// 2^(c s - lse log2 e): one fused multiply-add, one exponential, one addition.
//
// The tokens of a sequence's selected rounds form one list, cut evenly (in 16-token tiles) over the workgroups of the sequence; a
// tile may cross from one round into the next, since every lane has the address of its own token.  A token's sum over all heads
// stays in one workgroup, so that nothing is exchanged between them and the order of the sums is fixed.
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
    int q_len, Hq, G, n_pos, n_parts;  // n_parts: workgroups of a sequence
    float c;  // scale * log2(e)
};

constexpr int kLookup = 256;    // tokens whose places are looked up at a time
constexpr int kManyRows = 64;  // query rows per KV head from which the waves share them through LDS

// Operand fragments of 16 rows of keys or queries and their product, per type.
template <typename T, int D>
struct Rows16;
template <int D>
struct Rows16<BF16, D> {
    static constexpr int EB = 2, N = D / 32;
    typedef uint4 piece_t;
    piece_t x[N];
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
    typedef float4 piece_t;
    piece_t x[N];
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

// The share of this workgroup: part i of n of sequence b.  Workgroups go to the eight dies in turn, and every die gets
// neighbouring parts: the queries of a sequence then stay in the second-level cache of the one or two dies that read them.
struct Part {
    int b, i, n;
    __device__ __forceinline__ explicit Part(int n_) : n(n_) {
        const int dies = 8, die = blockIdx.x % dies, all = gridDim.x, each = all / dies, more = all - each * dies;
        const int mine = die * each + min(die, more) + (int)blockIdx.x / dies;
        b = mine / n;
        i = mine - b * n;
    }
};

// A sequence's selected rounds, in LDS: where the rounds begin in the history and in the list of selected tokens.
struct SelectedRounds {
    int* pos;    // [R + 1] first position of round r; of the end
    int* virt;   // [R + 1] tokens of the selected rounds before round r; all of them
    int* times;  // [R] how often the selection names round r
    static size_t bytes(int R) { return (3 * (size_t)R + 2) * sizeof(int); }
    __device__ __forceinline__ SelectedRounds(int* lds, int R) : pos(lds), virt(lds + R + 1), times(lds + 2 * R + 2) {}
};
// A token of that list.
struct TokenPlace {
    long long row[kLookup];  // its key row for head 0 ...
    int stride[kLookup];     // ... and from one head to the next
    int pos[kLookup];
    float times[kLookup];
};

// All threads (256); ends with a barrier.  What is read is asked for in one go.
__device__ __forceinline__ void selected_rounds(const SelectedRounds& sr, const WeightArgs& a, int b) {
    const DevView& vw = a.view;
    const int tid = threadIdx.x, lane = tid & 63, R = vw.R_max;
    const size_t row = (size_t)b * R;
    constexpr int N = kMaxRounds / 256;
    int len[N], sel[N];
    const int32_t* listed_rounds = a.sel_idx ? a.sel_idx : vw.seg_len;
    const int known = vw.n_rounds[b], listed_known = a.sel_idx ? a.n_sel[b] : 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int r = min(tid + 256 * j, R - 1);
        len[j] = 0, sel[j] = -1;
        if (j * 256 < R) {
            len[j] = vw.seg_len[row + r];
            sel[j] = listed_rounds[row + r];
        }
    }
    const int n_rounds = min(max(known, 0), R), listed = min(max(listed_known, 0), R);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int r = tid + 256 * j;
        if (r < R) {
            sr.pos[r] = r < n_rounds ? max(len[j], 0) : 0;
            sr.times[r] = a.sel_idx ? 0 : 1;
        }
    }
    __syncthreads();
    if (a.sel_idx) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (tid + 256 * j < listed && sel[j] >= 0 && sel[j] < n_rounds) atomicAdd(&sr.times[sel[j]], 1);  // (a count: in any order)
        __syncthreads();
    }
    if (tid < 64) {
        int pos = 0, virt = 0;
        for (int r0 = 0; r0 < R; r0 += 64) {
            const int r = r0 + lane, n = r < R ? sr.pos[r] : 0, chosen = r < R && sr.times[r] > 0 ? n : 0;
            const int pos_end = wave_inclusive_sum(n), virt_end = wave_inclusive_sum(chosen);
            if (r < R) {
                sr.pos[r] = pos + pos_end - n;
                sr.virt[r] = virt + virt_end - chosen;
            }
            pos += __builtin_amdgcn_readlane(pos_end, 63);
            virt += __builtin_amdgcn_readlane(virt_end, 63);
        }
        if (lane == 0) {
            sr.pos[R] = pos;
            sr.virt[R] = virt;
        }
    }
    __syncthreads();
}

// Positions that keep `prev`: workgroup i of n takes every n-th round that is not selected, and its share of what lies behind the
// last token.
__device__ __forceinline__ void copy_rest(const SelectedRounds& sr, const WeightArgs& a, int b, int i, int n) {
    if (a.prev == a.weights) return;
    const float* prev = a.prev ? a.prev + (size_t)b * a.n_pos : nullptr;
    float* out = a.weights + (size_t)b * a.n_pos;
    const int R = a.view.R_max, tid = threadIdx.x;
    if (a.sel_idx)
        for (int r = i; r < R; r += n) {
            if (sr.times[r] > 0) continue;
            for (int p = sr.pos[r] + tid; p < min(sr.pos[r + 1], a.n_pos); p += 256) out[p] = prev ? prev[p] : 0.f;
        }
    for (int p = sr.pos[R] + i * 256 + tid; p < a.n_pos; p += n * 256) out[p] = prev ? prev[p] : 0.f;
}

// Token v of the list into place t.  No barrier.
template <bool PAGED>
__device__ __forceinline__ void look_up(TokenPlace& tp, const SelectedRounds& sr, const WeightArgs& a, int b, int t, int v) {
    const DevView& vw = a.view;
    int lo = 0, hi = vw.R_max;  // the last round with virt <= v (an empty or unselected one ends where it begins)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sr.virt[mid] <= v) lo = mid;
        else hi = mid;
    }
    const int r = lo, in = v - sr.virt[r];
    const long long off = vw.seg_off[(size_t)b * vw.R_max + r];
    if (PAGED) {
        const long long at = min(max(off + in / 16, 0ll), (long long)vw.max_blocks - 1);
        tp.row[t] = (long long)max(vw.block_table[(size_t)b * vw.max_blocks + at], 0) * vw.Hkv * 16 + in % 16;
        tp.stride[t] = 16;
    } else {
        tp.row[t] = off * vw.Hkv + in;
        tp.stride[t] = sr.virt[r + 1] - sr.virt[r];
    }
    tp.pos[t] = sr.pos[r] + in;
    tp.times[t] = (float)sr.times[r];
}

__device__ __forceinline__ void store_weight(const WeightArgs& a, const TokenPlace& tp, int b, int t, float sum) {
    const int p = tp.pos[t];
    if (p >= a.n_pos) return;
    const size_t at = (size_t)b * a.n_pos + p;
    a.weights[at] = (a.prev ? a.prev[at] : 0.f) + sum * tp.times[t];
}

// Row r of KV head g in the order of q and lse, from the sequence's first row on.
__device__ __forceinline__ int row_index(const WeightArgs& a, const RowsPerToken& per_token, int g, int r) {
    const int i = per_token.token(r);
    return i * a.Hq + g * a.G + (r - i * a.G);
}
// Its log2-sum-exp; infinity for a row that adds nothing (2^-infinity).
__device__ __forceinline__ float lse2(float lse) {
    const float x = lse * kLog2e;
    return __builtin_fabsf(x) < __builtin_inff() ? x : __builtin_inff();
}
__device__ __forceinline__ float row_lse2(const WeightArgs& a, const RowsPerToken& per_token, const float* lse, int g, int r, int rows) {
    return r < rows ? lse2(lse[row_index(a, per_token, g, r)]) : __builtin_inff();
}

// Keys of 16 tokens as whole rows: the lanes of an instruction read 64 / kPieces rows, each of them contiguous, and the operand
// layout (lane % 16 = token) is made through a piece of LDS of the wave's own.  Read in the operand layout instead, 16
// neighbouring lanes are in 16 rows, and a wave's instruction looks up 64 cache lines for its 16: 1.3 GB of keys took 274
// microseconds, bound by that.  (Non-temporal: an instruction covers whole lines, and the keys are read once.)
template <typename T, int D>
struct KeyTile {
    static constexpr int kRowBytes = D * Rows16<T, D>::EB, kPieces = kRowBytes / 16, kRows = 64 / kPieces, kLoads = 16 / kRows;
    uint4 x[kLoads];
    __device__ __forceinline__ void load(const DevView& vw, const TokenPlace& tp, int place, int g) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int t = place + j * kRows + lane / kPieces;
            const char* row = static_cast<const char*>(vw.k) + (tp.row[t] + (long long)g * tp.stride[t]) * kRowBytes;
            x[j] = load_once(reinterpret_cast<const uint4*>(row) + lane % kPieces);
        }
    }
    // lds: 16 kPieces pieces of the wave's own; piece c of row r lies at position (c + r) mod kPieces of the row: no bank conflicts
    __device__ __forceinline__ Rows16<T, D> operand(uint4* lds) const {
        const int lane = threadIdx.x & 63, n = lane & 15, q4 = lane >> 4;
        __builtin_amdgcn_wave_barrier();  // same wave: LDS operations complete in program order
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = j * kRows + lane / kPieces;
            lds[r * kPieces + ((lane % kPieces + r) & (kPieces - 1))] = x[j];
        }
        __builtin_amdgcn_wave_barrier();
        Rows16<T, D> rows;
#pragma unroll
        for (int i = 0; i < Rows16<T, D>::N; ++i)
            rows.x[i] = __builtin_bit_cast(typename Rows16<T, D>::piece_t, lds[n * kPieces + ((i * 4 + q4 + n) & (kPieces - 1))]);
        return rows;
    }
};

// Few rows per KV head: bound by the keys' bandwidth.  The four waves take the KV heads in turn and all of the workgroup's tokens,
// 256 at a time: a head's queries stay in registers for them (the first 16 rows), and its keys come TILES tiles at a time, the next
// ones always on their way while some are worked on.  The waves' sums are added in their order, once per 256 tokens.
// grid (workgroups of a sequence x B)
template <typename T>
constexpr int kWeightWaves = std::is_same<T, F32>::value ? 2 : 3;  // of a SIMD, whose registers they share
template <typename T, int D, bool PAGED>
__global__ __launch_bounds__(256, kWeightWaves<T>) void token_weights_kernel(WeightArgs a) {
    typedef Rows16<T, D> Rows;
    typedef KeyTile<T, D> Keys;
    constexpr int TILES = std::is_same<T, F32>::value && D == 128 ? 1 : 2, kStep = 16 * TILES;
    extern __shared__ __align__(16) int s_rounds[];
    __shared__ TokenPlace tp;
    __shared__ uint4 s_tile[4][16 * Keys::kPieces];
    __shared__ float s_sum[4][kLookup];
    const DevView& vw = a.view;
    const SelectedRounds sr(s_rounds, vw.R_max);
    const Part part(a.n_parts);
    const int b = part.b, tid = threadIdx.x, lane = tid & 63, n = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    selected_rounds(sr, a, b);
    const int total = sr.virt[vw.R_max], tiles = (total + 15) / 16;
    const int v_lo = (int)((long long)tiles * part.i / part.n) * 16, v_hi = min((int)((long long)tiles * (part.i + 1) / part.n) * 16, total);
    const RowsPerToken per_token(a.G);
    const char* queries = static_cast<const char*>(a.q) + (size_t)b * a.q_len * a.Hq * (D * Rows::EB);
    const float* lse = a.lse + (size_t)b * a.q_len * a.Hq;
    const int rows = a.q_len * a.G;

    struct Query {  // 16 rows of a head and their log2-sum-exps
        Rows x;
        float l[4];
    };
    auto load_query = [&](int g, int r0) {
        Query q;
        const int at = row_index(a, per_token, g, min(r0 + n, rows - 1));
        q.x.load(queries + (size_t)at * (D * Rows::EB), q4);
        if (lse2(lse[at]) == __builtin_inff()) q.x = Rows{};  // (the queries of a row that adds nothing may be anything)
#pragma unroll
        for (int e = 0; e < 4; ++e) q.l[e] = row_lse2(a, per_token, lse, g, r0 + 4 * q4 + e, rows);
        return q;
    };
    for (int v0 = v_lo; v0 < v_hi; v0 += kLookup) {
        __syncthreads();  // the places and the sums before are read
        look_up<PAGED>(tp, sr, a, b, tid, min(v0 + tid, v_hi - 1));
        s_sum[wave][lane] = s_sum[wave][lane + 64] = s_sum[wave][lane + 128] = s_sum[wave][lane + 192] = 0.f;
        __syncthreads();
        const int here = min(kLookup, v_hi - v0), last = (here - 1) / kStep * kStep;
        for (int g = wave; g < vw.Hkv; g += 4) {
            const Query q0 = load_query(g, 0);
            struct Step {
                Keys k[TILES];
            };
            auto load = [&](int t0) {  // (behind the last step that one again: a request that is made in any case is one wait less)
                Step s;
                t0 = min(t0, last);
#pragma unroll
                for (int k = 0; k < TILES; ++k) s.k[k].load(vw, tp, t0 + k * 16, g);
                return s;
            };
            auto consume = [&](const Step& s, int t0) {
#pragma unroll
                for (int k = 0; k < TILES; ++k) {
                    const Rows keys = s.k[k].operand(s_tile[wave]);
                    float sum = 0.f;
                    auto add = [&](const Query& q) {
                        const floatx4_t x = Rows::product(q.x, keys);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum += fast_exp2(__builtin_fmaf(x[e], a.c, -q.l[e]));
                    };
                    add(q0);
                    for (int r0 = 16; r0 < rows; r0 += 16) add(load_query(g, r0));
                    sum = xrow_sum4(sum);
                    if (q4 == 0) s_sum[wave][t0 + k * 16 + n] += sum;
                }
            };
            Step x = load(0), y;
            for (int t0 = 0;;) {
                y = load(t0 + kStep);
                consume(x, t0);
                if ((t0 += kStep) > last) break;
                x = load(t0 + kStep);
                consume(y, t0);
                if ((t0 += kStep) > last) break;
            }
        }
        __syncthreads();
        if (tid < here) store_weight(a, tp, b, tid, (s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]));
    }
    copy_rest(sr, a, b, part.i, part.n);
}

// Many rows per KV head (bf16): bound by the exponentials (24 cycles of a wave's vector ALU for 64 terms, 16 of the matrix core with
// 128 channels).  The waves own tokens, up to four tiles each, whose keys of one head they keep in registers while the head's
// queries pass through LDS, 32 rows at a time, read once for the workgroup; one barrier per 32 rows and two buffers.
// grid (workgroups of a sequence x B)
template <int D, bool PAGED>
__global__ __launch_bounds__(256, 3) void token_weights_rows_kernel(WeightArgs a) {
    typedef Rows16<BF16, D> Rows;
    constexpr int TILES = 4, kGroup = 32, kPieces = D / 8, kPerThread = kGroup * kPieces / 256;  // 16-byte pieces of a row; of a group, per thread
    extern __shared__ __align__(16) int s_rounds[];
    __shared__ TokenPlace tp;
    __shared__ uint4 s_q[2][kGroup * kPieces];  // piece x of row r at position (x + r) mod kPieces of the row: no bank conflicts
    __shared__ float s_lse[2][kGroup];
    const DevView& vw = a.view;
    const SelectedRounds sr(s_rounds, vw.R_max);
    const Part part(a.n_parts);
    const int b = part.b, tid = threadIdx.x, lane = tid & 63, n = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    selected_rounds(sr, a, b);
    const int total = sr.virt[vw.R_max], tiles = (total + 15) / 16;
    const int v_lo = (int)((long long)tiles * part.i / part.n) * 16, v_hi = min((int)((long long)tiles * (part.i + 1) / part.n) * 16, total);
    const RowsPerToken per_token(a.G);
    const char* queries = static_cast<const char*>(a.q) + (size_t)b * a.q_len * a.Hq * (D * Rows::EB);
    const float* lse = a.lse + (size_t)b * a.q_len * a.Hq;
    const int rows = a.q_len * a.G, groups = (rows + kGroup - 1) / kGroup;
    for (int v0 = v_lo; v0 < v_hi; v0 += kLookup) {
        __syncthreads();  // the places and the queries before are read
        look_up<PAGED>(tp, sr, a, b, tid, min(v0 + tid, v_hi - 1));
        __syncthreads();
        // this wave's tiles of the step: dealt out evenly
        const int step_tiles = (min(kLookup, v_hi - v0) + 15) / 16;
        const int my_lo = step_tiles * wave / 4, my_tiles = step_tiles * (wave + 1) / 4 - my_lo;
        float sum[TILES];
#pragma unroll
        for (int k = 0; k < TILES; ++k) sum[k] = 0.f;
        struct Stage {
            uint4 q[kPerThread];
            float lse;  // (as it is: what is made of it here would wait for it here)
            bool ok;
        };
        int next_g = 0, next_r0 = 0;
        auto fetch = [&]() -> Stage {  // the next 32 rows of the head, or the next head's first ones
            Stage s;
            const int g = next_g, r0 = next_r0;
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) {
                const int x = tid + 256 * j, r = x / kPieces;
                s.q[j] = reinterpret_cast<const uint4*>(queries + (size_t)row_index(a, per_token, g, min(r0 + r, rows - 1)) * (D * Rows::EB))[x % kPieces];
            }
            const int r = r0 + (tid & (kGroup - 1));
            s.ok = r < rows;
            s.lse = lse[row_index(a, per_token, g, min(r, rows - 1))];
            next_r0 += kGroup;
            if (next_r0 >= rows) ++next_g, next_r0 = 0;
            return s;
        };
        Rows keys[TILES];
        Stage stage = fetch();
        const int n_groups = groups * vw.Hkv;
        for (int i = 0, g = 0, left = 0; i < n_groups; ++i, --left) {
            const int buf = i & 1;
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) {
                const int x = tid + 256 * j, r = x / kPieces;
                s_q[buf][r * kPieces + ((x % kPieces + r) & (kPieces - 1))] = stage.q[j];
            }
            if (tid < kGroup) s_lse[buf][tid] = stage.ok ? lse2(stage.lse) : __builtin_inff();
            if (left == 0) {  // the next head's keys
#pragma unroll
                for (int k = 0; k < TILES; ++k)
                    if (k < my_tiles) {
                        const int t = (my_lo + k) * 16 + n;
                        keys[k].load(static_cast<const char*>(vw.k) + (tp.row[t] + (long long)g * tp.stride[t]) * (D * Rows::EB), q4);
                    }
                wait_for_loads_so_far();  // here, once per head, not behind the join (together with the next queries) per 32 rows
                ++g;
                left = groups;
            }
            lds_barrier();
            if (i + 1 < n_groups) stage = fetch();
            auto group = [&](auto n_tiles) {
                constexpr int N = decltype(n_tiles)::value;
                const bool some_off = __any(s_lse[buf][lane & (kGroup - 1)] == __builtin_inff());
#pragma unroll
                for (int h = 0; h < kGroup / 16; ++h) {
                    Rows q;
#pragma unroll
                    for (int x = 0; x < Rows::N; ++x) q.x[x] = s_q[buf][(h * 16 + n) * kPieces + ((x * 4 + q4 + h * 16 + n) & (kPieces - 1))];
                    if (some_off && s_lse[buf][h * 16 + n] == __builtin_inff()) q = Rows{};  // (such a row's queries may be anything)
                    const floatx4_t l = *reinterpret_cast<const floatx4_t*>(&s_lse[buf][h * 16 + 4 * q4]);
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const floatx4_t s = Rows::product(q, keys[k]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[k] += fast_exp2(__builtin_fmaf(s[e], a.c, -l[e]));
                    }
                }
            };
            if (my_tiles == 4) group(std::integral_constant<int, 4>());
            else if (my_tiles == 3) group(std::integral_constant<int, 3>());
            else if (my_tiles == 2) group(std::integral_constant<int, 2>());
            else if (my_tiles == 1) group(std::integral_constant<int, 1>());
        }
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            const float x = xrow_sum4(sum[k]);
            const int t = (my_lo + k) * 16 + n;
            if (k < my_tiles && q4 == 0 && v0 + t < v_hi) store_weight(a, tp, b, t, x);
        }
    }
    copy_rest(sr, a, b, part.i, part.n);
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
    RA_REQUIRE(layer->max_tokens < (int64_t)1 << 30, RA_ERR_UNSUPPORTED, "token_weights: max_tokens too large");
    RA_REQUIRE((int64_t)q_len * G < (int64_t)1 << 27 && (int64_t)q_len * Hq < (int64_t)1 << 31, RA_ERR_UNSUPPORTED,
               "token_weights: %d query tokens are too many", q_len);
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
    const bool bf16 = layer->dtype == RA_BF16, wide = layer->d == 128, paged = layer->block_size != 0;
    const bool many = bf16 && q_len * G >= kManyRows;
    // as many workgroups as run at the same time, and none for less than a tile
    const int64_t tiles = (layer->max_tokens + 15) / 16, at_once = (int64_t)ctx->num_cu * (bf16 ? 3 : 2);
    int64_t n = (at_once + layer->B - 1) / layer->B;
    if (n > tiles) n = tiles;
    a.n_parts = (int)(n < 1 ? 1 : n);
    const dim3 grid((unsigned)(a.n_parts * layer->B));
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    KernelTimer timer(ctx, st);
#define RA_WEIGHTS_CASE(T_, D_, P_)                                                                              \
    if (!many && bf16 == std::is_same<T_, BF16>::value && wide == (D_ == 128) && paged == P_)                    \
        RA_LAUNCH_TIMED((token_weights_kernel<T_, D_, P_>), grid, dim3(256), SelectedRounds::bytes(layer->R_max), st, a);
    RA_WEIGHTS_CASE(BF16, 128, false) RA_WEIGHTS_CASE(BF16, 128, true) RA_WEIGHTS_CASE(BF16, 64, false) RA_WEIGHTS_CASE(BF16, 64, true)
    RA_WEIGHTS_CASE(F32, 128, false) RA_WEIGHTS_CASE(F32, 128, true) RA_WEIGHTS_CASE(F32, 64, false) RA_WEIGHTS_CASE(F32, 64, true)
#undef RA_WEIGHTS_CASE
#define RA_WEIGHTS_CASE(D_, P_) \
    if (many && wide == (D_ == 128) && paged == P_) RA_LAUNCH_TIMED((token_weights_rows_kernel<D_, P_>), grid, dim3(256), SelectedRounds::bytes(layer->R_max), st, a);
    RA_WEIGHTS_CASE(128, false) RA_WEIGHTS_CASE(128, true) RA_WEIGHTS_CASE(64, false) RA_WEIGHTS_CASE(64, true)
#undef RA_WEIGHTS_CASE
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
