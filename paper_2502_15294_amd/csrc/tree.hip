// Drafted tokens: attention of a tree of them over the selected rounds, the committed tokens of the current round and each
// other, and the accepted path's move behind the committed tokens.
//
// bf16 goes to the question kernels (attn_mfma.hip, attn_prefill_mfma.hip), which a tree is a question for whose rows see
// other parts of the current round, or to this file's kernel (tree_by_units).  This file also holds the kernel for fp32 caches
// and the move.
#include "attn_common.hpp"
#include "mfma_util.hpp"
#include "stream_kv.hpp"

#include <algorithm>

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

    // A thread's share of a unit's keys and values, on their way from memory while the unit before is worked on.
    struct Unit {
        floatx4_t k[kQuads], v[kQuads];
        int tok0, tokens;
        bool is_cur;
    };
    if (u_lo >= u_hi) {  // an empty key set (one piece)
        if (!row_ok) return;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) *reinterpret_cast<floatx4_t*>(a.out + rowid * D + 16 * j + 4 * q4) = acc[j];
        if (a.lse && q4 == 0) a.lse[rowid] = -__builtin_inff();
        return;
    }
    int slot = find_slot(tab.cum, hdr.n_slots, u_lo);
    auto load = [&](int u) {  // (tokens past the segment's end: its last one again)
        Unit x;
        while (u >= tab.cum[slot + 1]) ++slot;
        const int len = tab.len[slot], tok0 = (u - tab.cum[slot]) * kUnitTokens, ntok = min(kUnitTokens, len - tok0);
        const bool is_cur = slot >= hdr.n_hist;
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
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int e = tid + 256 * i, t = min(e / (D / 4), ntok - 1), c = e % (D / 4) * 4;
            x.k[i] = *reinterpret_cast<const floatx4_t*>(kp + (size_t)t * kstride + c);
            // four channels of a token of the current round, four tokens of a channel of any other
            x.v[i] = *reinterpret_cast<const floatx4_t*>(is_cur ? vp + (size_t)t * kstride + c : vp + e * 4);
        }
        x.tok0 = tok0;
        x.tokens = ntok;
        x.is_cur = is_cur;
        return x;
    };
    Unit x = load(u_lo);
    for (int u = u_lo; u < u_hi; ++u) {
        __syncthreads();  // the unit before is read
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int e = tid + 256 * i, t = e / (D / 4), c = e % (D / 4) * 4;
            *reinterpret_cast<floatx4_t*>(keys + t * kKeyPitch + c) = x.k[i];
            if (x.is_cur) {
                values[(c + 0) * kValuePitch + t] = x.v[i][0];
                values[(c + 1) * kValuePitch + t] = x.v[i][1];
                values[(c + 2) * kValuePitch + t] = x.v[i][2];
                values[(c + 3) * kValuePitch + t] = x.v[i][3];
            } else {
                *reinterpret_cast<floatx4_t*>(values + e / 4 * kValuePitch + e % 4 * 4) = x.v[i];
            }
        }
        __syncthreads();
        const int tok0 = x.tok0, ntok = x.tokens;
        const bool is_cur = x.is_cur;
        x = load(min(u + 1, u_hi - 1));  // (in any case: a load behind a condition would be waited for where the paths meet)
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

// ---- bf16, 128 channels, many query rows per KV head ---------------------------------------------------------------------------
// Arithmetic of the question kernel (S^T = K . Q^T, O^T += V^T . P, query row = lane % 16, the softmax reference of a row raised
// only when a logit exceeds it by more than 2^16 after scaling), but the keys come in steps of four UNITS of 16 tokens, a unit
// being what one value tile holds and never crossing a round, and the roles of the lanes are dealt out by unit:
//   * row r of the operand K of tile h (h = 0 .. 3) is token 4 h + r % 4 of unit r / 4, so that lane group q of the product holds
//     the logits of unit q, tokens 4 h .. 4 h + 3, and after tiles 2 m and 2 m + 1 the eight probabilities of tokens
//     8 m .. 8 m + 7 of unit q: the P operand of the products over those tokens of all four units;
//   * the V^T operand of lane group q is then 16 contiguous bytes of unit q's value tile.
// A unit needs one address for its keys and one for its values.  The workgroup looks up 256 units at a time (a thread each) and
// keeps the addresses in LDS; wave w brings the keys of a step's unit w, four instructions of four whole rows, and two channel
// groups of the values, all with one base address a lane and constant offsets.  So the loop has no segment walk, no block-table
// look-up and next to no address arithmetic, and one barrier per 64 tokens.  (The question kernel walks the segments in scalar
// registers, which it has too few of, once per 32 tokens; 60 drafted tokens of 64 heads over 32 paged dialogues of 4 900 tokens: 765
// -> 725 microseconds.)
// Units of the current round, whose values are token-major and whose keys lie Hkv rows apart, take a slower path: their values
// are gathered by 2-byte loads.
//
// P goes to the matrix cores as the sum of three bf16 numbers, which hold all of its 24 bits.  (With two, both rounded to the
// nearest, outputs were off by 2.5e-6 of themselves, twice what fp32 arithmetic is; the third costs 19 % at the size above.)
//
// Bound by the matrix cores and the vector ALUs in turn: at that size the matrix cores are busy for 41 % of the kernel's time (302 GFLOP
// of the formula, four halves of it as products: 830 TFLOP/s), the vector ALUs work for about as long, and a fifth is waiting
// for keys and values.  Tried: wave priorities, the products of the high parts first, both row tiles' softmax first: no change.
constexpr int kUnitsAhead = 256;                    // units that are looked up at a time
constexpr int kStepUnits = 4, kStepBytes = 32768;   // 16 KB of keys, 16 KB of values
constexpr int kTreeWaves = 2;                       // workgroups of a compute unit, waves of a SIMD

struct UnitTable {
    long long key[kUnitsAhead], value[kUnitsAhead];  // addresses of the unit's first key, and of its value tile (first value)
    int tokens[kUnitsAhead];                         // 1 .. 16; of the current round: + 32
    int first[kUnitsAhead];                          // first token inside its segment
};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // M0 is named as clobbered; the compiler sets it anew before each of its own uses
// As load_to_lds, OFFSET bytes behind `base`.  The instruction adds its offset to the LDS address too, and takes 16 bits of M0: the
// steps lie in the first 64 KB of LDS.
template <int OFFSET>
__device__ __forceinline__ void load_to_lds_at(long long base, unsigned lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off offset:%2" : : "v"(base), "s"(lds - OFFSET), "n"(OFFSET) : "memory", "m0");
}
#pragma clang diagnostic pop

// RT: 16-row tiles of a wave (one workgroup: four waves, 64 RT rows).  grid (pieces x row blocks x KV heads x sequences)
template <bool PAGED, int RT>
__global__ __launch_bounds__(256, kTreeWaves) void tree_rows_kernel(AttnArgs a, int n_rowblocks) {
    extern __shared__ __align__(16) char smem[];  // (all of the kernel's LDS: the steps come first)
    const DevView& vw = a.view;
    const int Hkv = vw.Hkv, G = a.G, cap = vw.R_max + 1;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char* tiles = smem;  // two steps
    UnitTable& units = *reinterpret_cast<UnitTable*>(smem + 2 * kStepBytes);
    int* cum = reinterpret_cast<int*>(smem + 2 * kStepBytes + sizeof(UnitTable));
    const unsigned tiles_lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(lptr_t)tiles);

    // Neighbours share keys (the row blocks of a piece, then the pieces): they go to the same die.
    const int dies = 8, die = blockIdx.x % dies, each = gridDim.x / dies, more = gridDim.x - each * dies;
    int item = die * each + min(die, more) + (int)blockIdx.x / dies;
    const int rowblock = item % n_rowblocks;
    item /= n_rowblocks;
    const int s = item % a.S;
    item /= a.S;
    const int g = item % Hkv, b = item / Hkv;

    const char* plan = a.plan + (size_t)b * plan_stride(cap);
    const PlanHeader hdr = *reinterpret_cast<const PlanHeader*>(plan);
    const long long* off_k = reinterpret_cast<const long long*>(plan + sizeof(PlanHeader));
    const long long* off_v = off_k + cap;
    const int* lens = reinterpret_cast<const int*>(off_v + cap);
    for (int i = tid; i <= cap; i += 256) cum[i] = lens[cap + i];
    const int committed = committed_tokens(a, b), drafted = drafted_tokens(a, b, committed);
    // ---- this wave's query rows: the block's 16-row tiles are dealt out to the waves in turn ---------------------------------
    const int rows = a.q_len * G;
    const RowsPerToken per_token(G);
    int node[RT];
    bool row_ok[RT];
    size_t rowid[RT];
    uint4 q[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = ((rowblock * RT + t) * 4 + wave) * 16 + n;
        row_ok[t] = row < rows;
        const int r = row_ok[t] ? row : 0;
        node[t] = per_token.token(r);
        rowid[t] = ((size_t)b * a.q_len + node[t]) * a.Hq + (size_t)g * G + (r - node[t] * G);
        const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const char*>(a.q) + rowid[t] * 256);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) q[t][kk] = qp[kk * 4 + q4];
    }
    const int n_slots = __builtin_amdgcn_readfirstlane(hdr.n_slots), n_hist = __builtin_amdgcn_readfirstlane(hdr.n_hist);
    const int S_eff = __builtin_amdgcn_readfirstlane(hdr.S_eff), U = __builtin_amdgcn_readfirstlane(hdr.U);
    if (s >= S_eff) return;
    const int u_lo = (int)(((long long)U * s) / S_eff), u_hi = (int)(((long long)U * (s + 1)) / S_eff);

    floatx4_t acc[RT][8];
    float m[RT], l[RT];
    const float slack = 16.f / a.c;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        m[t] = kNegBig;
        l[t] = 0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[t][dt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }
    // Keys: LDS row 16 h + r holds operand row r of tile h, its 16-byte chunk x at position (x + r) mod 16.  Wave w fills rows
    // 16 h + 4 w .. + 3 (unit w), 16 lanes a row: chunk of the lane, from the row's start.
    const unsigned key_chunk = (unsigned)((n - (4 * wave + q4)) & 15) * 16u;

    // What of a step does not come by direct loads: values of units of the current round, on their way through registers.
    struct Pending {
        uint4 v[4];
        bool some;
    };
    // Step `it` of the units looked up goes to `lds`.  Units past the last one repeat it (their tokens are masked).
    auto load_step = [&](int it, int n_units, unsigned lds) -> Pending {
        Pending p;
        p.some = false;
        p.v[0] = p.v[1] = p.v[2] = p.v[3] = make_uint4(0, 0, 0, 0);
        const int ku = min(it * kStepUnits + wave, n_units - 1), vu = min(it * kStepUnits + q4, n_units - 1);
        const int k_tokens = __builtin_amdgcn_readfirstlane(units.tokens[ku]), v_tokens = units.tokens[vu];
        const long long k0 = units.key[ku], v0 = units.value[vu];
        const unsigned kd = lds + 4 * wave * 256;
        if (k_tokens == 16 || (PAGED && k_tokens < 32)) {  // whole rows 256 bytes apart (a block has 16 of them in any case)
            const long long base = k0 + q4 * 256 + key_chunk;
            load_to_lds_at<0>(base, kd);
            load_to_lds_at<1 * 1024>(base, kd + 4096);
            load_to_lds_at<2 * 1024>(base, kd + 8192);
            load_to_lds_at<3 * 1024>(base, kd + 12288);
        } else {
            const long long stride = k_tokens >= 32 ? (long long)Hkv * 256 : 256;
            const int last = (k_tokens & 31) - 1;
#pragma unroll
            for (int h = 0; h < 4; ++h) load_to_lds_at<0>(k0 + min(4 * h + q4, last) * stride + key_chunk, kd + h * 4096);
        }
        // values: fragment (dt, m) holds lane L's 16 bytes at (2 dt + m) * 1024 + 16 L: tokens 8 m .. + 7 of unit L / 16, channel
        // 16 dt + L % 16; this wave: dt = 2 wave, 2 wave + 1
        const unsigned vd = lds + 16384 + 4 * wave * 1024;
        if (!__any(v_tokens >= 32)) {
            const long long base = v0 + wave * 1024 + n * 32;
            load_to_lds_at<0>(base, vd);
            load_to_lds_at<16>(base, vd + 1 * 1024);
            load_to_lds_at<512>(base, vd + 2 * 1024);
            load_to_lds_at<528>(base, vd + 3 * 1024);
        } else {
            p.some = true;
            const int last = (v_tokens & 31) - 1;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int channel = (2 * wave + f / 2) * 16 + n;
                if (v_tokens >= 32) {  // token-major: eight tokens of a channel
                    uint32_t e[8];
#pragma unroll
                    for (int t = 0; t < 8; ++t)
                        e[t] = *reinterpret_cast<const unsigned short*>(v0 + (long long)min(8 * (f & 1) + t, last) * Hkv * 256 + channel * 2);
                    p.v[f] = make_uint4(e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16), e[6] | (e[7] << 16));
                } else {
                    p.v[f] = *reinterpret_cast<const uint4*>(v0 + channel * 32 + (f & 1) * 16);
                }
            }
        }
        return p;
    };
    auto consume = [&](const char* buf, int it, int n_units) {
        const uint4* kb = reinterpret_cast<const uint4*>(buf);
        const uint4* vb = reinterpret_cast<const uint4*>(buf + 16384);
        const int unit = it * kStepUnits + q4, at = min(unit, n_units - 1);
        const int tokens = units.tokens[at], first = units.first[at];
        const int limit = unit < n_units ? tokens & 31 : 0;  // tokens of the lane's unit
        const bool drafts = tokens >= 32 && first + kUnitTokens > committed;
        const bool whole = __all(limit == 16 && !drafts);
        floatx4_t sc[RT][4];
#pragma unroll
        for (int h0 = 0; h0 < 4; h0 += 2) {
            uint4 kf[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) kf[h][kk] = kb[((h0 + h) * 16 + n) * 16 + ((kk * 4 + q4 + n) & 15)];
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)  // independent chains interleaved
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        sc[t][h0 + h] = mfma16(kf[h][kk], q[t][kk], kk ? sc[t][h0 + h] : floatx4_t{0.f, 0.f, 0.f, 0.f});
        }
        if (!whole) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                uint32_t sees = (1u << limit) - 1;
                if (drafts)
                    sees &= tree_sees(a.tree_mask + ((size_t)b * a.q_len + node[t]) * a.tree_words, a.tree_words, first, committed);
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(sees >> (4 * h + i) & 1)) sc[t][h][i] = -__builtin_inff();
            }
        }
        bool raise = false;
        float mx[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            mx[t] = vmax(max8(sc[t][0], sc[t][1]), max8(sc[t][2], sc[t][3]));
            raise |= mx[t] > m[t] + slack;
        }
        if (__any(raise)) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const float m_new = vmax(m[t], xrow_max4(mx[t])), alpha = fast_exp2((m[t] - m_new) * a.c);
                l[t] *= alpha;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) acc[t][dt] *= alpha;
                m[t] = m_new;
            }
        }
        // (tokens 8 m2 .. + 7 of every unit, row tile t), one after the other: its products on the matrix cores while the vector ALU
        // turns the next one's logits into probabilities
        constexpr int K = 2 * RT;
        uint4 part[2][3], vf[8];
        auto soften = [&](int k) {
            const int m2 = k / RT, t = k % RT;
            const float mc = m[t] * a.c;
            float p[8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) p[h * 4 + i] = fast_exp2(__builtin_fmaf(sc[t][2 * m2 + h][i], a.c, -mc));
            l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
            for (int i = 0; i < 3; ++i) part[k & 1][i] = take_part(p, i == 2);
        };
        soften(0);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int m2 = k / RT, t = k % RT;
            if (t == 0) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) vf[dt] = vb[(2 * dt + m2) * 64 + lane];
            }
            if (k + 1 < K) soften(k + 1);
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) acc[t][dt] = mfma16(vf[dt], part[k & 1][i], acc[t][dt]);
#pragma unroll
            for (int i = 0; i < 24; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);  // four vector instructions
            }
        }
    };

    for (int c0 = u_lo; c0 < u_hi; c0 += kUnitsAhead) {
        const int n_units = min(kUnitsAhead, u_hi - c0), n_steps = (n_units + kStepUnits - 1) / kStepUnits;
        __syncthreads();  // the prefix is there; the units and the steps before are read
        if (tid < n_units) {
            const int u = c0 + tid, slot = find_slot(cum, n_slots, u), first = (u - cum[slot]) * kUnitTokens, len = lens[slot];
            const int tokens = min(kUnitTokens, len - first);
            long long key, value;
            if (slot >= n_hist) {
                const size_t row = (((size_t)b * a.cur_cap + first) * Hkv + g) * 256;
                key = reinterpret_cast<long long>(a.cur_k) + row;
                value = reinterpret_cast<long long>(a.cur_v) + row;
            } else if (PAGED) {
                const long long entry = min(max(off_k[slot] + first / 16, 0ll), (long long)vw.max_blocks - 1);
                const size_t block = ((size_t)max(vw.block_table[(size_t)b * vw.max_blocks + entry], 0) * Hkv + g) * 4096;
                key = reinterpret_cast<long long>(vw.k) + block;
                value = reinterpret_cast<long long>(vw.v) + block;
            } else {
                key = reinterpret_cast<long long>(vw.k) + ((size_t)off_k[slot] * Hkv + (size_t)g * len + first) * 256;
                value = reinterpret_cast<long long>(vw.v) + ((size_t)off_v[slot] * Hkv + (size_t)g * ((len + 15) & ~15) + first) * 256;
            }
            units.key[tid] = key;
            units.value[tid] = value;
            units.tokens[tid] = tokens + (slot >= n_hist ? 32 : 0);
            units.first[tid] = first;
        }
        __syncthreads();
        Pending p = load_step(0, n_units, tiles_lds);
        for (int it = 0; it < n_steps; ++it) {
            char* buf = tiles + (it & 1) * kStepBytes;
            if (p.some) {
                uint4* vd = reinterpret_cast<uint4*>(buf + 16384) + 4 * wave * 64 + lane;
#pragma unroll
                for (int f = 0; f < 4; ++f) vd[f * 64] = p.v[f];
            }
            wait_for_direct_loads();  // this wave's part of the step has landed in LDS
            __syncthreads();
            if (it + 1 < n_steps) p = load_step(it + 1, n_units, tiles_lds + ((it + 1) & 1) * kStepBytes);
            consume(buf, it, n_units);
        }
    }

    // ---- the four lane groups hold partial sums of the same rows; each wave owns its rows --------------------------------------
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        l[t] = xrow_sum4(l[t]);
        if (node[t] >= drafted) {  // no token of this sequence's tree: as a row that sees nothing
            m[t] = kNegBig;
            l[t] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) acc[t][dt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
        }
        if (!row_ok[t]) continue;
        if (S_eff > 1) {
            const size_t pr = rowid[t] * a.S + s;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<floatx4_t*>(a.part_acc + pr * 128 + dt * 16 + q4 * 4) = acc[t][dt];
            if (q4 == 0) {
                a.part_m[pr] = m[t];
                a.part_l[pr] = l[t];
            }
        } else {
            const float inv = l[t] > 0.f ? 1.f / l[t] : 0.f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<floatx4_t*>(a.out + rowid[t] * 128 + dt * 16 + q4 * 4) = acc[t][dt] * inv;
            if (a.lse && q4 == 0) a.lse[rowid[t]] = l[t] > 0.f ? __builtin_fmaf(m[t], a.scale, __builtin_logf(l[t])) : -__builtin_inff();
        }
    }
}

// Pieces that every sequence is cut into at most, for `items` workgroups a piece of which `at_once` run at the same time: the
// number with which the turns of workgroups take the least time, a two-hundredth of a whole sequence reckoned for every piece's
// start and merge.
static int tree_pieces(long long items, long long at_once, int64_t max_units, int min_units) {
    int64_t most = max_units / min_units;
    most = most < 1 ? 1 : most > 64 ? 64 : most;
    int best = 1;
    double least = 1e30;
    for (int S = 1; S <= most; ++S) {
        const double cost = (double)((items * S + at_once - 1) / at_once) / S + 0.005 * S;
        if (cost < least) least = cost, best = S;
    }
    return best;
}

// Which kernel a bf16 tree with 128 channels gets (microseconds of whole calls, left the question kernels):
//   up to 16 query rows per KV head: the streaming kernel, which reads the keys once for 16 rows;
//   17 to 32: that kernel would read them twice (32 paged dialogues of 4 900 tokens, 24 rows: 200 and 171 here; 8 dialogues of
//     3 300, 20 rows: 51 and 45, 32 rows: 51 and 45);
//   more: the question kernel where it plans itself, with ranges that are equal over the whole batch (8 dialogues, 100 rows: 56
//     and 65; 32: 152 and 181; 12 paged ones, 480 rows: 292 and 312), this file's where it does not (32 paged dialogues of 50
//     rounds, 64 rows: 214 and 169, 128: 269 and 233, 480: 765 and 725; contiguous 699 and 710).
static bool tree_by_units(int B, int R_max, int rows) { return rows > 16 && (rows <= 32 || !attn_mfma_plans_inline(B, R_max)); }

static int tree_attention(ra_ctx* ctx, hipStream_t st, AttnArgs& a, bool bf16) {
    const int B = a.view.B, Hkv = a.view.Hkv, D = a.view.d, rows_total = a.q_len * a.G;
    const int row_tiles = bf16 && rows_total > 64 ? 2 : 1;  // of a wave
    const int n_rowblocks = (rows_total + 64 * row_tiles - 1) / (64 * row_tiles);
    const long long inner = (long long)Hkv * n_rowblocks;
    RA_REQUIRE(B <= kMaxBatch, RA_ERR_UNSUPPORTED, "tree: batch %d exceeds %d", B, kMaxBatch);
    RA_REQUIRE(inner <= 65535 && inner * B * 64 < (1ll << 31), RA_ERR_UNSUPPORTED, "tree: %lld blocks of rows are too many", inner);
    const int64_t max_tokens = a.max_tokens + a.cur_cap;
    RA_REQUIRE(max_tokens < (int64_t)1 << 30, RA_ERR_UNSUPPORTED, "tree: max_tokens too large");
    const size_t rows = (size_t)B * rows_total * Hkv;
    AttnWorkspace w = attn_workspace(rows, 1, D, B, a.view.R_max);
    RA_REQUIRE(ctx->ws.base != nullptr && ctx->ws.bytes >= w.total, RA_ERR_WORKSPACE,
               "tree: workspace has %zu bytes, this call needs %zu", ctx->ws.bytes, w.total);
    a.min_units = bf16 ? 8 : 2;  // (fp32 calls are small: one dialogue of 500 tokens)
    a.S = tree_pieces(inner * B, (long long)kTreeWaves * ctx->num_cu, max_tokens / kUnitTokens, a.min_units);
    w = attn_workspace(rows, a.S, D, B, a.view.R_max);
    while (a.S > 1 && w.total > ctx->ws.bytes) w = attn_workspace(rows, --a.S, D, B, a.view.R_max);
    a.part_acc = reinterpret_cast<float*>(ctx->ws.base + w.acc_off);
    a.part_m = reinterpret_cast<float*>(ctx->ws.base + w.m_off);
    a.part_l = reinterpret_cast<float*>(ctx->ws.base + w.l_off);
    a.n_parts = reinterpret_cast<int*>(ctx->ws.base);
    a.plan = ctx->ws.base + w.plan_off;
    launch_plan(a, kUnitTokens, st);
    const bool paged = a.view.block_size != 0;
    KernelTimer timer(ctx, st);
    if (bf16) {
        const dim3 grid((unsigned)(a.S * inner * B));
        const size_t smem = 2 * kStepBytes + sizeof(UnitTable) + (a.view.R_max + 2) * sizeof(int);
        if (paged && row_tiles == 2) RA_LAUNCH_TIMED((tree_rows_kernel<true, 2>), grid, dim3(256), smem, st, a, n_rowblocks);
        else if (paged) RA_LAUNCH_TIMED((tree_rows_kernel<true, 1>), grid, dim3(256), smem, st, a, n_rowblocks);
        else if (row_tiles == 2) RA_LAUNCH_TIMED((tree_rows_kernel<false, 2>), grid, dim3(256), smem, st, a, n_rowblocks);
        else RA_LAUNCH_TIMED((tree_rows_kernel<false, 1>), grid, dim3(256), smem, st, a, n_rowblocks);
    } else {
        const dim3 grid((unsigned)a.S, (unsigned)inner, (unsigned)B);
        const size_t smem = align_up(SlotTable::bytes(a.view.R_max + 1), 16) + (16 * (D + 4) + D * 20) * sizeof(float);
        if (D == 128 && paged) RA_LAUNCH_TIMED((tree_f32_kernel<128, true>), grid, dim3(256), smem, st, a, n_rowblocks);
        else if (D == 128) RA_LAUNCH_TIMED((tree_f32_kernel<128, false>), grid, dim3(256), smem, st, a, n_rowblocks);
        else if (paged) RA_LAUNCH_TIMED((tree_f32_kernel<64, true>), grid, dim3(256), smem, st, a, n_rowblocks);
        else RA_LAUNCH_TIMED((tree_f32_kernel<64, false>), grid, dim3(256), smem, st, a, n_rowblocks);
    }
    if (a.S > 1) launch_combine(a, D, rows, st);
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}

// ---- the accepted path ---------------------------------------------------------------------------------------------------
constexpr int kCommitLayers = 32;  // layers of one launch (their pointers are kernel arguments)
struct CommitLayers {
    u32x4_t* p[2 * kCommitLayers];
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
    u32x4_t* rows = layers.p[blockIdx.y] + ((size_t)b * cur_cap + committed) * row16 + column;
    for (int j0 = 0; j0 < n; j0 += kCommitFlight) {
        u32x4_t v[kCommitFlight];
#pragma unroll
        for (int i = 0; i < kCommitFlight; ++i)
            v[i] = rows[(size_t)path[min(j0 + i, n - 1)] * row16];  // (behind the last one: that one again, not written)
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
    const bool bf16 = layer->dtype == RA_BF16;
    if (bf16 && (layer->d != 128 || !tree_by_units(layer->B, layer->R_max, n_nodes * G)))  // (64 channels: the streaming kernel)
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
    return tree_attention(ctx, reinterpret_cast<hipStream_t>(stream), a, bf16);
}

extern "C" int ra_tree_commit(ra_ctx* ctx, void* stream, void* const* cur_k_layers, void* const* cur_v_layers, int n_layers, int B,
                              int cur_cap, int Hkv, int d, int dtype, const int32_t* cur_len, const int32_t* path,
                              const int32_t* n_path, int max_path, int32_t* new_len) {
    RA_REQUIRE(ctx != nullptr, RA_ERR_INVALID_ARG, "tree_commit: ctx is NULL");
    RA_REQUIRE(n_layers > 0 && B > 0 && cur_cap > 0 && Hkv > 0 && d > 0 && max_path > 0, RA_ERR_INVALID_ARG,
               "tree_commit: non-positive dimension");
    RA_REQUIRE(cur_k_layers && cur_v_layers && cur_len && path && n_path && new_len, RA_ERR_INVALID_ARG, "tree_commit: NULL argument");
    RA_REQUIRE(dtype == RA_F32 || dtype == RA_BF16, RA_ERR_UNSUPPORTED, "tree_commit: unknown dtype %d", dtype);
    RA_REQUIRE(new_len != cur_len && new_len != n_path && (new_len < path || new_len >= path + (size_t)B * max_path), RA_ERR_INVALID_ARG,
               "tree_commit: new_len must be another buffer than cur_len, path and n_path");
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
            layers.p[2 * l] = static_cast<u32x4_t*>(cur_k_layers[l0 + l]);
            layers.p[2 * l + 1] = static_cast<u32x4_t*>(cur_v_layers[l0 + l]);
        }
        hipLaunchKernelGGL(tree_commit_kernel, dim3((unsigned)B, (unsigned)(2 * n), (unsigned)columns), dim3(256), 0,
                           reinterpret_cast<hipStream_t>(stream), layers, cur_cap, (int)(row_bytes / 16), cur_len, path, n_path,
                           max_path, l0 == 0 ? new_len : nullptr);
    }
    RA_HIP_CHECK(hipGetLastError());
    return RA_OK;
}
