// Dense causal attention of packed prompts on v_mfma_f32_32x32x16_bf16.
#include "api_checks.h"
#include "kv_store.h"

namespace ihip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPromptWaves = 4;
constexpr int kPromptRows = 64 * kPromptWaves;       // queries of a workgroup
constexpr int kTileKeys = 32;
constexpr int kTileEl = kTileKeys * kD;              // bf16 elements of a K or V tile in LDS
constexpr int kPromptStages = 3;
constexpr float kNegBigPrompt = -1.0e30f;            // finite stand-in for -inf in running maxima
constexpr float kPromptMaxSum = 1024.0f;             // row sum of a tile above which the softmax reference moves

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

    f32x16 o[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[s][dt][r] = 0.f;
    float m_run[2] = {kNegBigPrompt, kNegBigPrompt}, l_run[2] = {0.f, 0.f};

    auto request = [&](int tile) {
        if (tile >= n_tiles) return;
        uint16_t *stage = smem + (tile % kPromptStages) * 2 * kTileEl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = wave + i * kPromptWaves;   // 0..7 K rows 4j.., 8..15 V rows 4(j-8)..
            const bool is_v = i >= 2;
            const int key = 4 * (j & 7) + (lane >> 4), slot = lane & 15;
            const int pos = min(tile * kTileKeys + key, nk - 1);
            const int chunk = is_v ? slot ^ ((key & 3) << 2) : slot ^ (key & 15);
            const uint16_t *src = (is_v ? vb + (int64_t)pos * a.v_st : kb + (int64_t)pos * a.k_st) + chunk * 8;
            const uint32_t dst = __builtin_amdgcn_readfirstlane(
                (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)(stage + j * 4 * kD));
            global_to_lds(dst, src);
        }
    };
    int voff[4];
    {
        const int i = lane & 15, key = 4 * half + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
            const int chunk = dt * 4 + ((n >> 4) << 1) + ((i & 3) >> 1);
            voff[dt] = key * kD + ((chunk ^ ((key & 3) << 2)) << 3) + ((i & 1) << 2);
        }
    }
    auto v_operand = [&](const uint16_t *cV, int dt, int kk) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)(cV + voff[dt] + (16 * kk) * kD));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)(cV + voff[dt] + (16 * kk + 8) * kD));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto exponentials = [&](const f32x16 &s, float ref, bf16x8 (&pb)[2]) {
        float ps = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float pw = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2e, -ref));   // exp2(-inf) = 0
            ps += pw;
            pb[r >> 3][r & 7] = (__bf16)pw;
        }
        return ps;
    };

    request(0);
    request(1);
    for (int tile = 0; tile < n_tiles; ++tile) {
        if (tile + 1 < n_tiles) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        request(tile + 2);
        const uint16_t *cK = smem + (tile % kPromptStages) * 2 * kTileEl + n * kD, *cV = smem + (tile % kPromptStages) * 2 * kTileEl + kTileEl;
        f32x16 sc[2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[s][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            const bf16x8 ka = *reinterpret_cast<const bf16x8 *>(&cK[((ks * 2 + half) ^ (n & 15)) * 8]);
#pragma unroll
            for (int s = 0; s < 2; ++s) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[s][ks], sc[s], 0, 0, 0);
        }
        if (tile * kTileKeys + kTileKeys - 1 > row0 + ahead) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (tile * kTileKeys + 8 * (r >> 2) + 4 * half + (r & 3) > last_key[s]) sc[s][r] = -INFINITY;
        }
        bf16x8 pb[2][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float ps = exponentials(sc[s], m_run[s], pb[s]);
            if (__any(!(ps <= kPromptMaxSum))) {
                float mx = sc[s][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[s][r]);
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float mn = fmaxf(m_run[s], mx * a.scale_log2e);
                const float corr = __builtin_amdgcn_exp2f(m_run[s] - mn);
                m_run[s] = mn;
                ps = exponentials(sc[s], mn, pb[s]);
                l_run[s] *= corr;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[s][dt] *= corr;
            }
            l_run[s] += ps;
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                const bf16x8 va = v_operand(cV, dt, kk);
#pragma unroll
                for (int s = 0; s < 2; ++s) o[s][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[s][kk], o[s][dt], 0, 0, 0);
            }
    }

#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const float l = l_run[s] + __shfl_xor(l_run[s], 32, 64);
        const int row = row0 + s * 32 + n;
        if (row >= nq) continue;
        const float inv = l > 0.f ? 1.0f / l : 0.f;  // a query without keys: 0
        const int64_t at = (int64_t)(q_first + row) * a.Hq + h;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<uint2 *>(a.out + at * kD + dt * 32 + r4 * 8 + half * 4) =
                    make_uint2(pack_bf16x2(o[s][dt][r4 * 4] * inv, o[s][dt][r4 * 4 + 1] * inv), pack_bf16x2(o[s][dt][r4 * 4 + 2] * inv, o[s][dt][r4 * 4 + 3] * inv));
        if (a.lse != nullptr && half == 0) a.lse[at] = l > 0.f ? (m_run[s] + log2f(l)) * 0.69314718055994530942f : -INFINITY;
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
