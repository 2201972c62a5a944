// Dense causal attention of packed prompts on v_mfma_f32_32x32x16_bf16.
#include "api_checks.h"
#include "kv_store.h"
#include <type_traits>

namespace ihip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPromptWaves = 4;
constexpr int kPromptRows = 64 * kPromptWaves;       // queries of a workgroup
constexpr int kTileKeys = 32;
constexpr int kTileEl = kTileKeys * kD;              // bf16 elements of a K or V tile in LDS
constexpr int kPromptStages = 4;
constexpr float kNegBigPrompt = -1.0e30f;            // finite stand-in for -inf in maxima
constexpr float kPromptMaxSum = 18446744073709551616.0f;      // 2^64: sum of exponentials beyond which a block is done again

int32_t check_packed(const char *who, const ihip_packed *p);

struct PromptArgs {
    int B, Hq, Hkv, G, rows_q, rows_k;
    const int32_t *cu_q, *cu_k;
    const uint16_t *q, *k, *v;
    int64_t q_sh, q_st, k_sh, k_st, v_sh, v_st;
    float scale_log2e;
    uint16_t *out;                   // [rows_q, Hq, d]
    float *lse;                      // [rows_q, Hq] or null
};

// 16 bytes a lane from a scalar base and the lane's byte offset to the LDS byte address dst + 16 l (counts on vmcnt).  M0 is left as it is:
// nothing else in this kernel reads it, and it is not the compiler's to keep values in.
__device__ inline void prompt_to_lds(uint32_t dst, const uint16_t *base, uint32_t byte_off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(dst), "v"(byte_off), "s"(base) : "memory");
}

__global__ __launch_bounds__(64 * kPromptWaves, 1) void prompt_attn_kernel(const PromptArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;

    // which head, which sequence, which of its blocks
    const int hs = blockIdx.x % a.Hq, g = hs % a.Hkv, h = g * a.G + hs / a.Hkv;
    int ti = blockIdx.x / a.Hq, b = -1, m = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int blocks = 0;
        if (b0 + lane < a.B) {
            const int c0 = min(max(a.cu_q[b0 + lane], 0), a.rows_q), c1 = min(max(a.cu_q[b0 + lane + 1], c0), a.rows_q);
            blocks = (c1 - c0 + kPromptRows - 1) / kPromptRows;
        }
        const int incl = (int)wave_scan_u32((uint32_t)blocks, lane);
        const unsigned long long past = __ballot(incl > ti);
        if (past != 0) {
            const int at = __builtin_ctzll(past);
            b = b0 + at;
            m = __builtin_amdgcn_readlane(incl, at) - 1 - ti;          // the longest blocks of a sequence come first
            break;
        }
        ti -= __builtin_amdgcn_readlane(incl, 63);
    }
    if (b < 0) return;
    const int q_first = min(max(a.cu_q[b], 0), a.rows_q), nq = min(max(a.cu_q[b + 1], q_first), a.rows_q) - q_first;
    const int k_first = min(max(a.cu_k[b], 0), a.rows_k), nk = min(max(a.cu_k[b + 1], k_first), a.rows_k) - k_first;
    const int row0 = m * kPromptRows + wave * 64;    // this wave's first query
    const int ahead = nk - nq;                       // query i sees keys 0 .. i + ahead
    const int n_keys = min(m * kPromptRows + kPromptRows, nq) + ahead;
    const int n_tiles = n_keys > 0 ? (n_keys + kTileKeys - 1) / kTileKeys : 0;

    bf16x8 qb[2][8];
    int last_key[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int row = min(row0 + s * 32 + n, nq - 1);
        last_key[s] = row + ahead;
        const uint16_t *qp = a.q + (int64_t)(q_first + row) * a.q_st + h * a.q_sh + half * 8;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qb[s][ks] = *reinterpret_cast<const bf16x8 *>(qp + ks * 16);
    }
    const uint16_t *kb = a.k + (int64_t)k_first * a.k_st + g * a.k_sh;
    const uint16_t *vb = a.v + (int64_t)k_first * a.v_st + g * a.v_sh;

    // Loads of a tile: 8 four-row instructions for K and 8 for V, two of each a wave: lane l brings 16 bytes of row 4 j + l / 16 to
    // base + 16 l.  The base of a tile is scalar; a lane's offset from it changes in a tile that reaches behind the last key only,
    // whose rows stand for the missing ones.  What would come after the last tile is the last tile again, so that every period
    // has as many loads on their way as any other.
    auto offset = [&](int i, int rows, int64_t st, bool is_v) {
        const int key = 4 * (wave + i * kPromptWaves) + (lane >> 4), at = min(key, rows - 1), slot = lane & 15;
        return (uint32_t)(at * (int)st + ((slot ^ (is_v ? (key & 3) << 2 : key & 15)) << 3)) * 2u;
    };
    const uint32_t k_off[2] = {offset(0, kTileKeys, a.k_st, false), offset(1, kTileKeys, a.k_st, false)};
    const uint32_t v_off[2] = {offset(0, kTileKeys, a.v_st, true), offset(1, kTileKeys, a.v_st, true)};
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem + wave * 4 * kD * 2;
    const bool cut = n_tiles * kTileKeys > nk;       // the last tile reaches behind the last key
    const uint16_t *k_next = kb, *v_next = vb;       // of the tiles to be requested next
    int k_tile = 0, v_tile = 0;
    auto request_k = [&](int st) {
        uint32_t off[2] = {k_off[0], k_off[1]};
        if (cut && k_tile == n_tiles - 1) {
            off[0] = offset(0, nk - k_tile * kTileKeys, a.k_st, false);
            off[1] = offset(1, nk - k_tile * kTileKeys, a.k_st, false);
        }
        prompt_to_lds(lds0 + st * kTileEl * 2, k_next, off[0]);
        prompt_to_lds(lds0 + st * kTileEl * 2 + 16 * kD * 2, k_next, off[1]);
        const bool more = k_tile < n_tiles - 1;
        k_next += more ? kTileKeys * a.k_st : 0;
        k_tile += more;
    };
    auto request_v = [&](int st) {
        uint32_t off[2] = {v_off[0], v_off[1]};
        if (cut && v_tile == n_tiles - 1) {
            off[0] = offset(0, nk - v_tile * kTileKeys, a.v_st, true);
            off[1] = offset(1, nk - v_tile * kTileKeys, a.v_st, true);
        }
        prompt_to_lds(lds0 + (kPromptStages + st) * kTileEl * 2, v_next, off[0]);
        prompt_to_lds(lds0 + (kPromptStages + st) * kTileEl * 2 + 16 * kD * 2, v_next, off[1]);
        const bool more = v_tile < n_tiles - 1;
        v_next += more ? kTileKeys * a.v_st : 0;
        v_tile += more;
    };
    const uint16_t *k_at[8], *v_at[4];               // this lane's addresses in stage 0
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) k_at[ks] = smem + n * kD + ((ks * 2 + half) ^ (n & 15)) * 8;
    {
        const int i = lane & 15, key = 4 * half + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
            const int chunk = dt * 4 + ((n >> 4) << 1) + ((i & 3) >> 1);
            v_at[dt] = smem + kPromptStages * kTileEl + key * kD + ((chunk ^ ((key & 3) << 2)) << 3) + ((i & 1) << 2);
        }
    }
    auto k_operand = [&](int st, int ks) { return *reinterpret_cast<const bf16x8 *>(k_at[ks] + st * kTileEl); };
    auto v_operand = [&](int st, int i) {            // i: 4 kk + dt
        const uint16_t *at = v_at[i & 3] + st * kTileEl + 16 * (i >> 2) * kD;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 8 * kD));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x16 o[2][4], sc[2];
    auto scores = [&](int st, int s) {
        sc[s] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(st, ks), qb[s][ks], sc[s], 0, 0, 0);
    };
    auto mask = [&](int tile, int s) {
        if (tile * kTileKeys + kTileKeys - 1 <= row0 + s * 32 + ahead) return;
        const int last = last_key[s] - 4 * half - tile * kTileKeys;
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[s][r] = 8 * (r >> 2) + (r & 3) > last ? -INFINITY : sc[s][r];
    };
    auto row_max = [&](const f32x16 &s) {            // scaled; of both halves
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        return fmaxf(mx, __shfl_xor(mx, 32, 64)) * a.scale_log2e;
    };

    uint32_t pw[2][8];                               // the probabilities of a set, in pairs of keys
    float m_ref[2] = {kNegBigPrompt, kNegBigPrompt}, l_run[2] = {0.f, 0.f};
    // two scores -> two probabilities (exp2(-inf) = 0).  The empty assembly keeps them where they are called: left to themselves all
    // exponentials of a phase would be computed in front of its matrix instructions instead of under them.
    auto exponentials = [&](int s, int i) {
        float x = fmaf(sc[s][2 * i], a.scale_log2e, -m_ref[s]), y = fmaf(sc[s][2 * i + 1], a.scale_log2e, -m_ref[s]);
        asm volatile("" : "+v"(x), "+v"(y));
        x = __builtin_amdgcn_exp2f(x);
        y = __builtin_amdgcn_exp2f(y);
        l_run[s] += x;
        l_run[s] += y;
        pw[s][i] = pack_bf16x2(x, y);
        asm volatile("" : "+v"(pw[s][i]), "+v"(l_run[s]));
    };
    auto probabilities = [&](int s, int kk) {
        return __builtin_bit_cast(bf16x8, make_uint4(pw[s][4 * kk], pw[s][4 * kk + 1], pw[s][4 * kk + 2], pw[s][4 * kk + 3]));
    };
    // Period t, for the two sets of 32 queries in turn: first product of tile t + 1 and second product of tile t, and under them the
    // exponentials of the other set, 16 matrix instructions and 16 scores a lane at a time.  K of tile t + 4 and V of tile t + 3 are
    // requested into the stages that period t - 1 has read, and have landed when period t + 1 ends; the first operands of period
    // t + 1 are read from LDS as this one ends.  Matrix instructions are written as assembly: of the 512 registers that the one wave of
    // a SIMD has, they can keep the accumulators in the upper half ("a") and everything else in the lower one, and they stay where
    // they are, each with its share of the vector instructions under it.  The compiler does not know the instructions' latency: a set's
    // scores are read by vector instructions eight matrix instructions after their last one.
    bf16x8 ka[8], va[8];
    auto first_operands = [&](int st, int st1) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            ka[i] = k_operand(st1, i);
            va[i] = v_operand(st, i);
        }
    };
    auto period = [&](int st, int st1, int st2, int st3, int t) {      // stages of tiles t, t + 1, t + 2, t + 3
        mask(t, 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == 1) mask(t + 1, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = r & 7;
                if (s == 0 && r < 6) ka[r + 2] = k_operand(st1, r + 2);
                if (s == 0 && r >= 6 && r < 12) va[r - 4] = v_operand(st, r - 4);
                if (s == 1 && r == 10) first_operands(st1, st2);
                if (r == 0) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=v"(sc[s]) : "v"(ka[0]), "v"(qb[s][0]));
                else if (r < 8) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(sc[s]) : "v"(ka[r]), "v"(qb[s][r]));
                else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o[s][i & 3]) : "v"(va[i]), "v"(probabilities(s, i >> 2)));
                if (r % 2 == 0) exponentials(1 - s, r / 2);
                if (s == 0 && r == 3) request_k(st);
                if (s == 0 && r == 9) request_v(st3);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        __syncthreads();
    };
    // Exponentials are taken against the row's maximum over the first tile (key 0 is in it, which every query with a key sees), not
    // against a running one: bf16 and fp32 have exponents to spare, nothing is lost while the scores stay within 2^64 of it.  Where a
    // row's sum says that they did not, the block is done again against the maxima over all tiles.
    for (int again = 0; n_tiles > 0 && again < 2; ++again) {
        if (again) {
            m_ref[0] = m_ref[1] = kNegBigPrompt;
            k_next = kb;
            k_tile = 0;
            for (int t = 0; t < n_tiles; ++t) {
                request_k(0);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    scores(0, s);
                    mask(t, s);
                    m_ref[s] = fmaxf(m_ref[s], row_max(sc[s]));
                }
                __syncthreads();
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            l_run[s] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[s][dt] = f32x16{};
        }
        k_next = kb; v_next = vb;
        k_tile = v_tile = 0;
#pragma unroll
        for (int st = 0; st < 4; ++st) request_k(st);
#pragma unroll
        for (int st = 0; st < 3; ++st) request_v(st);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            scores(0, s);
            mask(0, s);
            if (!again) m_ref[s] = fmaxf(kNegBigPrompt, row_max(sc[s]));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) exponentials(0, i);
        __syncthreads();                             // K(0) has been read
        first_operands(0, 1);
        int t = 0;
        for (; t + 4 < n_tiles; t += 4) {
            period(0, 1, 2, 3, t);
            period(1, 2, 3, 0, t + 1);
            period(2, 3, 0, 1, t + 2);
            period(3, 0, 1, 2, t + 3);
        }
        for (; t + 1 < n_tiles; ++t) period(t & 3, (t + 1) & 3, (t + 2) & 3, (t + 3) & 3, t);
        // the last tile, whose first products are done
        mask(t, 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) exponentials(1, i);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x8 vt = v_operand(t & 3, i);
#pragma unroll
            for (int s = 0; s < 2; ++s)
                asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o[s][i & 3]) : "v"(vt), "v"(probabilities(s, i >> 2)));
        }
        // (the compiler does not know that there are matrix instructions in the assembly, whose results take up to 19 wait states)
        asm volatile("s_nop 15\n\ts_nop 7" : "+a"(o[0][0]), "+a"(o[0][1]), "+a"(o[0][2]), "+a"(o[0][3]), "+a"(o[1][0]), "+a"(o[1][1]), "+a"(o[1][2]), "+a"(o[1][3]));
        l_run[0] += __shfl_xor(l_run[0], 32, 64);
        l_run[1] += __shfl_xor(l_run[1], 32, 64);
        if (again || __syncthreads_or(!(l_run[0] <= kPromptMaxSum && l_run[1] <= kPromptMaxSum)) == 0) break;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const float l = l_run[s];
        const int row = row0 + s * 32 + n;
        if (row >= nq) continue;
        const float inv = 1.0f / l;
        const int64_t at = (int64_t)(q_first + row) * a.Hq + h;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<uint2 *>(a.out + at * kD + dt * 32 + r4 * 8 + half * 4) =
                    l == 0.f ? make_uint2(0, 0)       // a query without keys
                             : make_uint2(pack_bf16x2(o[s][dt][r4 * 4] * inv, o[s][dt][r4 * 4 + 1] * inv), pack_bf16x2(o[s][dt][r4 * 4 + 2] * inv, o[s][dt][r4 * 4 + 3] * inv));
        if (a.lse != nullptr && half == 0) a.lse[at] = l == 0.f ? -INFINITY : (m_ref[s] + log2f(l)) * 0.69314718055994530942f;
    }
}

}  // namespace ihip

using namespace ihip;

extern "C" int32_t ihip_prompt_attn(const ihip_packed *packed, ihip_tensor q, ihip_tensor k, ihip_tensor v, const int32_t *cu_k,
                                    int32_t rows_k, float sm_scale, void *out, float *out_lse, void *stream)
{
    const char *who = "ihip_prompt_attn";
    int32_t rc;
    if ((rc = check_packed(who, packed)) != IHIP_OK) return rc;
    if (rows_k < 0 || (!cu_k && rows_k != packed->rows))
        return fail(IHIP_ERR_INVALID_ARG, "%s: rows_k = %d (without cu_k: the %d rows of q)", who, rows_k, packed->rows);
    if (packed->B == 0 || packed->rows == 0 || packed->max_q == 0) return IHIP_OK;
    if ((rc = check_tensor(q, who, "q")) != IHIP_OK) return rc;
    if (rows_k > 0 && ((rc = check_tensor(k, who, "k")) != IHIP_OK || (rc = check_tensor(v, who, "v")) != IHIP_OK)) return rc;
    if (!out || ((uintptr_t)out & 15)) return fail(IHIP_ERR_INVALID_ARG, "%s: out is NULL or not 16-byte aligned", who);
    PromptArgs a;
    a.B = packed->B; a.Hq = packed->Hq; a.Hkv = packed->Hkv; a.G = packed->Hq / packed->Hkv;
    a.rows_q = packed->rows; a.rows_k = rows_k;
    a.cu_q = packed->cu_q; a.cu_k = cu_k ? cu_k : packed->cu_q;
    a.q = (const uint16_t *)q.ptr; a.q_sh = q.stride_h; a.q_st = q.stride_t;
    a.k = (const uint16_t *)k.ptr; a.k_sh = k.stride_h; a.k_st = k.stride_t;
    a.v = (const uint16_t *)v.ptr; a.v_sh = v.stride_h; a.v_st = v.stride_t;
    // a tile's rows are addressed by 32-bit byte offsets from its first
    if (a.k_st < 0 || a.v_st < 0 || a.k_st >= (1 << 24) || a.v_st >= (1 << 24))
        return fail(IHIP_ERR_UNSUPPORTED, "%s: rows of k and v must be less than 2^24 elements apart", who);
    a.scale_log2e = sm_scale * 1.44269504088896340736f;
    a.out = (uint16_t *)out;
    a.lse = out_lse;
    // blocks of all sequences: at most a part of one in each beyond the whole ones, and no more than max_q gives each
    const int64_t by_rows = (int64_t)packed->rows / kPromptRows + packed->B, by_len = (int64_t)packed->B * ((packed->max_q - 1) / kPromptRows + 1);
    const int64_t groups = (by_rows < by_len ? by_rows : by_len) * packed->Hq;
    if (groups > INT32_MAX) return fail(IHIP_ERR_UNSUPPORTED, "%s: %lld workgroups are too many", who, (long long)groups);
    KernelTimer timer("prompt_attn", (hipStream_t)stream);
    hipLaunchKernelGGL(prompt_attn_kernel, dim3((uint32_t)groups), dim3(64 * kPromptWaves), kPromptStages * 2 * kTileEl * 2, (hipStream_t)stream, a);
    return check_launch(who);
}
