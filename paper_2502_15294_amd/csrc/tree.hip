// Drafted tokens: attention of a tree of them over the selected rounds, the committed tokens of the current round and each
// other, and the accepted path's move behind the committed tokens.
//
// bf16 goes to the question kernels (attn_mfma.hip, attn_prefill_mfma.hip), which a tree is a question for whose rows see
// other parts of the current round.  This file holds the entry points, the kernel for fp32 caches and the move.
#include "attn_common.hpp"
#include "mfma_util.hpp"
#include "stream_kv.hpp"

namespace ra {

__device__ __forceinline__ floatx4_t mfma4(float a, float b, floatx4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// fp32 tree attention.  The query rows of a KV head are (node i, head h of the group), row = i * G + h, in blocks of 64: a
// workgroup owns a block, every wave 16 of its rows, and walks a piece of the sequence's key units (16 tokens) with all of
// them; a unit's keys and values pass through LDS once for the 64 rows.
//   S^T [16 tokens x 16 rows] = K [16 x D] . Q^T       D / 4 x mfma 16x16x4: lane % 16 = row, tokens 4 (lane / 16) + i
//   O^T [16 channels x 16 rows] += V^T [16 x 4] . P     4 per 16 channels, product i over tokens 4 q + i, q = 0 .. 3
// The contraction of S^T takes channels 16 j + 4 q + e in its product e of step j, so a lane's operands are 16 contiguous
// bytes of a key and of its query; in that of O^T a lane's P operand is the probability it holds and its V operand 16
// contiguous bytes of the transposed value tile.  All of it fp32: nothing is rounded to fewer bits.
template <int D, bool PAGED>
__global__ __launch_bounds__(256) void tree_f32_kernel(AttnArgs a, int n_rowblocks) {
    constexpr int kKeyPitch = D + 4, kValuePitch = 20, kQuads = D / 64;  // 16-byte pieces of keys (of values) a thread moves
    extern __shared__ __align__(16) char smem[];
    const DevView& vw = a.view;
    const int Hkv = vw.Hkv, G = a.G, b = blockIdx.z, s = blockIdx.x;
    const int rowblock = blockIdx.y / Hkv, g = blockIdx.y - rowblock * Hkv;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = lane & 15, q4 = lane >> 4;
    const int cap = vw.R_max + 1;
    SlotTable tab;
    tab.carve(smem, cap);
    float* keys = reinterpret_cast<float*>(smem + ((SlotTable::bytes(cap) + 15) & ~(size_t)15));
    float* values = keys + 16 * kKeyPitch;
    const PlanHeader hdr = load_plan(a.plan + (size_t)b * plan_stride(cap), cap, tab);
    if (s >= hdr.S_eff) return;
    __syncthreads();
    const int committed = committed_tokens(a, b), drafted = drafted_tokens(a, b, committed);
    const int u_lo = (int)(((long long)hdr.U * s) / hdr.S_eff), u_hi = (int)(((long long)hdr.U * (s + 1)) / hdr.S_eff);

    const int row = rowblock * 64 + wave * 16 + n;
    const bool row_ok = row < a.q_len * G;
    const int node = row_ok ? row / G : 0, head = row_ok ? row - node * G : 0;
    const size_t rowid = ((size_t)b * a.q_len + node) * a.Hq + (size_t)g * G + head;
    float4 q[D / 16];
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
        q[j] = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + rowid * D + 16 * j + 4 * q4);
    const uint32_t* mask = a.tree_mask + ((size_t)b * a.q_len + node) * a.tree_words;
    floatx4_t acc[D / 16];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[j] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    float m = kNegBig, l = 0.f;

    int slot = u_lo < u_hi ? find_slot(tab.cum, hdr.n_slots, u_lo) : 0;
    for (int u = u_lo; u < u_hi; ++u) {
        while (u >= tab.cum[slot + 1]) ++slot;
        const int len = tab.len[slot], tok0 = (u - tab.cum[slot]) * kUnitTokens, ntok = min(kUnitTokens, len - tok0);
        const bool is_cur = slot >= hdr.n_hist;
        // ---- the unit's 16 keys and its value tile into LDS (tokens past the segment's end: its last one again) --------
        const float *kp, *vp;
        size_t kstride = D;
        if (is_cur) {
            const size_t e0 = (((size_t)b * a.cur_cap + tok0) * Hkv + g) * D;
            kp = static_cast<const float*>(a.cur_k) + e0;
            vp = static_cast<const float*>(a.cur_v) + e0;
            kstride = (size_t)Hkv * D;
        } else if (PAGED) {
            const long long at = min(max(tab.off_k[slot] + tok0 / 16, 0ll), (long long)vw.max_blocks - 1);
            const size_t block = max(vw.block_table[(size_t)b * vw.max_blocks + at], 0);
            kp = static_cast<const float*>(vw.k) + (block * Hkv + g) * 16 * D;
            vp = static_cast<const float*>(vw.v) + (block * Hkv + g) * 16 * D;
        } else {
            kp = static_cast<const float*>(vw.k) + ((size_t)tab.off_k[slot] * Hkv + (size_t)g * len + tok0) * D;
            vp = static_cast<const float*>(vw.v) + ((size_t)tab.off_v[slot] * Hkv + (size_t)g * ((len + 15) & ~15) + tok0) * D;
        }
        float4 kx[kQuads], vx[kQuads];
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int x = tid + 256 * i, t = min(x / (D / 4), ntok - 1), c = x % (D / 4) * 4;
            kx[i] = *reinterpret_cast<const float4*>(kp + (size_t)t * kstride + c);
            if (is_cur) vx[i] = *reinterpret_cast<const float4*>(vp + (size_t)t * kstride + c);  // four channels of a token
            else vx[i] = *reinterpret_cast<const float4*>(vp + x * 4);                          // four tokens of a channel
        }
        __syncthreads();  // the unit before is read
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int x = tid + 256 * i, t = x / (D / 4), c = x % (D / 4) * 4;
            *reinterpret_cast<float4*>(keys + t * kKeyPitch + c) = kx[i];
            if (is_cur) {
                values[(c + 0) * kValuePitch + t] = vx[i].x;
                values[(c + 1) * kValuePitch + t] = vx[i].y;
                values[(c + 2) * kValuePitch + t] = vx[i].z;
                values[(c + 3) * kValuePitch + t] = vx[i].w;
            } else {
                *reinterpret_cast<float4*>(values + x / 4 * kValuePitch + x % 4 * 4) = vx[i];
            }
        }
        __syncthreads();
        // ---- logits ------------------------------------------------------------------------------------------------
        floatx4_t sc = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const float4 k = *reinterpret_cast<const float4*>(keys + n * kKeyPitch + 16 * j + 4 * q4);
            sc = mfma4(k.x, q[j].x, sc);
            sc = mfma4(k.y, q[j].y, sc);
            sc = mfma4(k.z, q[j].z, sc);
            sc = mfma4(k.w, q[j].w, sc);
        }
        uint32_t sees = 0xffffffffu;
        if (is_cur && tok0 + kUnitTokens > committed) sees = tree_sees(mask, a.tree_words, tok0, committed);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * q4 + i >= ntok || !(sees >> (4 * q4 + i) & 1)) sc[i] = -__builtin_inff();
        // ---- softmax and the output's products ---------------------------------------------------------------------
        const float m_new = vmax(m, xrow_max4(vmax(vmax(sc[0], sc[1]), vmax(sc[2], sc[3]))));
        const float alpha = fast_exp2((m - m_new) * a.c), mc = m_new * a.c;
        m = m_new;
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fast_exp2(__builtin_fmaf(sc[i], a.c, -mc));
        l = __builtin_fmaf(l, alpha, (p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const float4 v = *reinterpret_cast<const float4*>(values + (16 * j + n) * kValuePitch + 4 * q4);
            acc[j] *= alpha;
            acc[j] = mfma4(v.x, p[0], acc[j]);
            acc[j] = mfma4(v.y, p[1], acc[j]);
            acc[j] = mfma4(v.z, p[2], acc[j]);
            acc[j] = mfma4(v.w, p[3], acc[j]);
        }
    }
    l = xrow_sum4(l);
    if (node >= drafted) {  // no token of this sequence's tree: as a row that sees nothing
        m = kNegBig;
        l = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) acc[j] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }
    if (!row_ok) return;
    if (hdr.S_eff > 1) {
        const size_t pr = rowid * a.S + s;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) *reinterpret_cast<floatx4_t*>(a.part_acc + pr * D + 16 * j + 4 * q4) = acc[j];
        if (q4 == 0) {
            a.part_m[pr] = m;
            a.part_l[pr] = l;
        }
    } else {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            floatx4_t o = floatx4_t{0.f, 0.f, 0.f, 0.f};
            if (l > 0.f) o = floatx4_t{acc[j][0] / l, acc[j][1] / l, acc[j][2] / l, acc[j][3] / l};
            *reinterpret_cast<floatx4_t*>(a.out + rowid * D + 16 * j + 4 * q4) = o;
        }
        if (a.lse && q4 == 0) a.lse[rowid] = l > 0.f ? __builtin_fmaf(m, a.scale, __builtin_logf(l)) : -__builtin_inff();
    }
}

static int tree_attention_f32(ra_ctx* ctx, hipStream_t st, AttnArgs& a, int64_t max_tokens) {
    const int B = a.view.B, Hkv = a.view.Hkv, D = a.view.d, n_rowblocks = (a.q_len * a.G + 63) / 64;
    const long long inner = (long long)Hkv * n_rowblocks;
    RA_REQUIRE(inner <= 65535 && B <= kMaxBatch, RA_ERR_UNSUPPORTED, "tree: %lld blocks of rows or %d sequences are too many", inner, B);
    const size_t rows = (size_t)B * a.q_len * a.Hq;
    a.S = decode_splits(ctx->num_cu, B, (int)inner, max_tokens);
    const AttnWorkspace w = attn_workspace(rows, a.S, D, B, a.view.R_max);
    RA_REQUIRE(ctx->ws.base != nullptr && ctx->ws.bytes >= w.total, RA_ERR_WORKSPACE,
               "tree: workspace has %zu bytes, this call needs %zu", ctx->ws.bytes, w.total);
    a.min_units = attn_min_units();
    a.part_acc = reinterpret_cast<float*>(ctx->ws.base + w.acc_off);
    a.part_m = reinterpret_cast<float*>(ctx->ws.base + w.m_off);
    a.part_l = reinterpret_cast<float*>(ctx->ws.base + w.l_off);
    a.n_parts = reinterpret_cast<int*>(ctx->ws.base);
    a.plan = ctx->ws.base + w.plan_off;
    launch_plan(a, kUnitTokens, st);
    const dim3 grid((unsigned)a.S, (unsigned)inner, (unsigned)B);
    const size_t smem = align_up(SlotTable::bytes(a.view.R_max + 1), 16) + (16 * (D + 4) + D * 20) * sizeof(float);
    const bool paged = a.view.block_size != 0;
    KernelTimer timer(ctx, st);
    if (D == 128 && paged) RA_LAUNCH_TIMED((tree_f32_kernel<128, true>), grid, dim3(256), smem, st, a, n_rowblocks);
    else if (D == 128) RA_LAUNCH_TIMED((tree_f32_kernel<128, false>), grid, dim3(256), smem, st, a, n_rowblocks);
    else if (paged) RA_LAUNCH_TIMED((tree_f32_kernel<64, true>), grid, dim3(256), smem, st, a, n_rowblocks);
    else RA_LAUNCH_TIMED((tree_f32_kernel<64, false>), grid, dim3(256), smem, st, a, n_rowblocks);
    if (a.S > 1) launch_combine(a, D, rows, st);
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}

// ---- the accepted path ---------------------------------------------------------------------------------------------------
constexpr int kCommitLayers = 32;  // layers of one launch (their pointers are kernel arguments)
struct CommitLayers {
    uint4* p[2 * kCommitLayers];
};
constexpr int kCommitFlight = 8;  // rows that a thread has in flight

// grid (sequence, tensor of a layer, 16-byte columns of a row / 256).  A thread moves its 16 bytes of all rows of the path, in
// the path's order, a few rows at a time: row j is written when the rows before it and those read together with it have been
// read, and those behind it come from behind it, since path[j] >= j.
__global__ __launch_bounds__(256) void tree_commit_kernel(CommitLayers layers, int cur_cap, int row16, const int32_t* __restrict__ cur_len,
                                                          const int32_t* __restrict__ path, const int32_t* __restrict__ n_path,
                                                          int max_path, int32_t* __restrict__ new_len) {
    const int b = blockIdx.x, lane = threadIdx.x & 63, column = blockIdx.z * 256 + threadIdx.x;
    const int committed = min(max(cur_len[b], 0), cur_cap), room = cur_cap - committed;
    const int listed = min(max(n_path[b], 0), max_path);
    path += (size_t)b * max_path;
    int n = 0;  // entries before the first that is none
    for (int j0 = 0; j0 < listed && n == j0; j0 += 64) {
        const int j = j0 + lane, node = j < listed ? path[j] : -1;
        const unsigned long long bad = __ballot(node < j || node >= room);
        n = j0 + (bad ? __ffsll(bad) - 1 : 64);
    }
    if (new_len && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) new_len[b] = committed + n;
    if (column >= row16) return;
    uint4* rows = layers.p[blockIdx.y] + ((size_t)b * cur_cap + committed) * row16 + column;
    for (int j0 = 0; j0 < n; j0 += kCommitFlight) {
        uint4 v[kCommitFlight];
#pragma unroll
        for (int i = 0; i < kCommitFlight; ++i)
            if (j0 + i < n) v[i] = rows[(size_t)path[j0 + i] * row16];
#pragma unroll
        for (int i = 0; i < kCommitFlight; ++i)
            if (j0 + i < n) rows[(size_t)(j0 + i) * row16] = v[i];
    }
}

}  // namespace ra

using namespace ra;

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

extern "C" int ra_round_sparse_attn_tree(ra_ctx* ctx, void* stream, const void* q, int n_nodes, int Hq, const ra_kv_view* layer,
                                         const int32_t* sel_idx, const int32_t* n_sel, const void* cur_k, const void* cur_v,
                                         const int32_t* cur_len, int cur_cap, const uint32_t* tree_mask, const int32_t* tree_len,
                                         float scale, float* out, float* lse) {
    RA_REQUIRE(ctx != nullptr, RA_ERR_INVALID_ARG, "tree: ctx is NULL");
    RA_REQUIRE(n_nodes > 0, RA_ERR_INVALID_ARG, "tree: n_nodes must be positive");
    RA_REQUIRE(q != nullptr && out != nullptr, RA_ERR_INVALID_ARG, "tree: q or out is NULL");
    if (int rc = check_view(layer, true, "tree")) return rc;
    RA_REQUIRE(Hq > 0 && Hq % layer->Hkv == 0, RA_ERR_INVALID_ARG, "tree: Hq %d is not a multiple of Hkv %d", Hq, layer->Hkv);
    RA_REQUIRE((sel_idx == nullptr) == (n_sel == nullptr), RA_ERR_INVALID_ARG,
               "tree: sel_idx and n_sel must both be given or both be NULL");
    RA_REQUIRE(cur_k && cur_v && cur_len && tree_mask, RA_ERR_INVALID_ARG, "tree: cur_k, cur_v, cur_len or tree_mask is NULL");
    RA_REQUIRE(cur_cap >= n_nodes, RA_ERR_INVALID_ARG, "tree: cur_cap %d has no room for %d nodes", cur_cap, n_nodes);
    RA_REQUIRE(scale > 0.f && scale == scale, RA_ERR_INVALID_ARG, "tree: scale must be positive");
    RA_REQUIRE(layer->d == 64 || layer->d == 128, RA_ERR_UNSUPPORTED, "tree: head_dim %d not in {64, 128}", layer->d);
    const int G = Hq / layer->Hkv;
    RA_REQUIRE(G <= 16, RA_ERR_UNSUPPORTED, "tree: Hq / Hkv = %d exceeds 16", G);
    RA_REQUIRE(aligned16(q) && aligned16(layer->k) && aligned16(layer->v) && aligned16(cur_k) && aligned16(cur_v) && aligned16(out),
               RA_ERR_INVALID_ARG, "tree: q, keys, values and out must be 16-byte aligned");
    const TreeOperands tree = {cur_len, tree_mask, tree_len};
    if (layer->dtype == RA_BF16)
        return question_attention(ctx, "tree", stream, q, n_nodes, Hq, layer, sel_idx, n_sel, cur_k, cur_v, cur_cap, scale, out, lse,
                                  nullptr, nullptr, &tree);
    AttnArgs a = {};
    a.view = to_dev(layer);
    a.q = q;
    a.sel_idx = sel_idx;
    a.n_sel = n_sel;
    a.cur_k = cur_k;
    a.cur_v = cur_v;
    a.cur_len_dev = cur_len;
    a.cur_cap = cur_cap;
    a.max_tokens = layer->max_tokens;
    a.q_len = n_nodes;
    a.Hq = Hq;
    a.G = G;
    a.c = scale * kLog2e;
    a.scale = scale;
    a.out = out;
    a.lse = lse;
    a.tree_mask = tree_mask;
    a.tree_len = tree_len;
    a.tree_words = (n_nodes + 31) / 32;
    return tree_attention_f32(ctx, reinterpret_cast<hipStream_t>(stream), a, layer->max_tokens + cur_cap);
}

extern "C" int ra_tree_commit(ra_ctx* ctx, void* stream, void* const* cur_k_layers, void* const* cur_v_layers, int n_layers, int B,
                              int cur_cap, int Hkv, int d, int dtype, const int32_t* cur_len, const int32_t* path,
                              const int32_t* n_path, int max_path, int32_t* new_len) {
    RA_REQUIRE(ctx != nullptr, RA_ERR_INVALID_ARG, "tree_commit: ctx is NULL");
    RA_REQUIRE(n_layers > 0 && B > 0 && cur_cap > 0 && Hkv > 0 && d > 0 && max_path > 0, RA_ERR_INVALID_ARG,
               "tree_commit: non-positive dimension");
    RA_REQUIRE(cur_k_layers && cur_v_layers && cur_len && path && n_path && new_len, RA_ERR_INVALID_ARG, "tree_commit: NULL argument");
    RA_REQUIRE(dtype == RA_F32 || dtype == RA_BF16, RA_ERR_UNSUPPORTED, "tree_commit: unknown dtype %d", dtype);
    RA_REQUIRE(new_len != cur_len, RA_ERR_INVALID_ARG, "tree_commit: new_len must be another buffer than cur_len");
    const long long row_bytes = (long long)Hkv * d * (dtype == RA_BF16 ? 2 : 4);
    RA_REQUIRE(row_bytes % 16 == 0, RA_ERR_UNSUPPORTED, "tree_commit: a token's %lld bytes are no multiple of 16", row_bytes);
    const long long columns = (row_bytes / 16 + 255) / 256;
    RA_REQUIRE(columns <= 65535 && row_bytes / 16 < (1ll << 31), RA_ERR_UNSUPPORTED, "tree_commit: a token's %lld bytes are too many",
               row_bytes);
    for (int l = 0; l < n_layers; ++l)
        RA_REQUIRE(cur_k_layers[l] && cur_v_layers[l] && aligned16(cur_k_layers[l]) && aligned16(cur_v_layers[l]), RA_ERR_INVALID_ARG,
                   "tree_commit: layer %d is NULL or not 16-byte aligned", l);
    for (int l0 = 0; l0 < n_layers; l0 += kCommitLayers) {
        CommitLayers layers = {};
        const int n = n_layers - l0 < kCommitLayers ? n_layers - l0 : kCommitLayers;
        for (int l = 0; l < n; ++l) {
            layers.p[2 * l] = static_cast<uint4*>(cur_k_layers[l0 + l]);
            layers.p[2 * l + 1] = static_cast<uint4*>(cur_v_layers[l0 + l]);
        }
        hipLaunchKernelGGL(tree_commit_kernel, dim3((unsigned)B, (unsigned)(2 * n), (unsigned)columns), dim3(256), 0,
                           reinterpret_cast<hipStream_t>(stream), layers, cur_cap, (int)(row_bytes / 16), cur_len, path, n_path,
                           max_path, l0 == 0 ? new_len : nullptr);
    }
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
