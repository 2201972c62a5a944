// Decode attention over all rows of a cache (bf16, E4M3 or MX FP4) that also says how much attention each row got:
//   s_hj = q_h k_j,   l_h = sum_j e^(c s_hj),   out_h = sum_j e^(c s_hj) v_j / l_h,   weight_j = decay before_j + sum_h e^(c s_hj) / l_h
// over the heads h of a KV head.  A weight needs the sum over all rows, so the scores wait for it in scratch.  Two launches: the first cuts a
// sequence's rows into parts, one workgroup each, and leaves scores and partial results; the second joins the parts, and turns scores into weights.
// (Where sequences are one part each, the first does it all.)
//
// A wave takes 32 rows at a time, the products on v_mfma_f32_16x16x32_bf16 (rows widened to bf16, exact); no value crosses lanes in between:
//   scores   16 K rows x twice 8 heads, or four times 4 (fewer repeat the last).  Lane (n, g) = (l % 16, l / 16) brings 16-byte pieces of row n, and gets
//            head n % 8's (n % 4's) scores of keys 4 g + r and 16 + 4 g + r.  A piece of bf16 is 8 of the dims 32 j + 8 g of step j, of E4M3 16 of 64 j + 16 g
//            (two steps), of 4 bits the 32 of 32 g, one scale's (four steps); the queries' pieces are the same.
//   output   16 rows x 32 keys x 16 dims, eight times: a lane's eight probabilities are its part of the left operand as they are, key
//            16 (i / 4) + 4 g + i % 4 for element i; for the right one it brings dims 8 n .. 8 n + 7 of the same keys, and column n of product j is dim 8 n + j.
// A probability goes into the products as three bf16 numbers, what one dropped in the next, which are its 24 bits.  Up to four heads have them in rows
// 0 .. 3, 8 .. 11 and 4 .. 7 (12 .. 15: 0); eight have two in rows 0 .. 7 and 8 .. 15, and the third in rows 0 .. 7 of eight products more.  The rows are
// added in LDS.  (Of 32 sequences in E4M3 0.02 % of the outputs are another bf16 number than float64's, with two parts 0.24 %.)
// Bound by memory: 4 sequences of 57,654 to 100,003 rows in bf16, 32 heads on 8, 1.39 GB, take 314 us (4.4 TB/s, a copy of 2 GB moves 5.0; the
// scores are 43 MB more) and 18 for the join; 32 of 7,383 to 16,384 in E4M3, 782 MB, 193 (4.1; scores 49 MB) and 18; 8 of 20,637 to 32,768 in
// MX FP4, 232 MB, 66 (3.5; scores 27 MB, and 20 requests for 32 rows) and 10.  One of 2,051 takes 7 and 4, chains of latencies.  (The two kernels
// by themselves, medians under the profiler.)
#include "api_checks.h"
#include "decode_softmax.h"
#include "kv_store.h"
#include <algorithm>
#include <type_traits>

namespace ihip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTrThreads = 256, kTrWaves = kTrThreads / kWave;
constexpr int kTrStep = 32;                          // rows of a wave at a time
constexpr int kTrMaxSplit = 768, kTrMinSplit = 128;  // rows of a part (multiples of 128: a step of every wave)
constexpr int kTrOnePart = 1024;                     // rows of sequences that are one part each, if there are few of them

struct TrackedArgs {
    Geometry ge;
    int max_len;
    const uint16_t *q; int64_t q_sb, q_sh;
    StoreView from;
    float scale_log2e, v_scale;
    int n_splits, per;               // parts of a problem, rows of one
    DecodeGrid grid;
    float *scores; int64_t score_stride;             // [P, G, score_stride], unscaled
    float *part_ml, *part_acc;       // [P, n_splits, G, 2] (reference, unscaled, and sum), [P, n_splits, G, 128]
    uint16_t *out;
    float *out_lse;
    const float *before;             // [P, weight_rows] or null
    float *weights;
    int weight_rows;
    float decay;
};

__device__ inline uint16_t to_bf16(float x) { return (uint16_t)pack_bf16x2(x, x); }        // (NaN stays it)
__device__ inline int tracked_len(const TrackedArgs &a, int b) { return min(max(a.ge.seq_lens[b], 0), a.max_len); }
// softmax_exp with the exponent rounded by itself: against the 26 of kSoftmaxShift its last five bits would go
__device__ inline float tracked_exp(float score, float ref, float scale_log2e) { return __builtin_amdgcn_exp2f((score - ref) * scale_log2e) * 0x1p-26f; }
// A row's probability is 2^(c (s - reference) - log2 of the sum of those); without a key that is there, 0.  sum: as it was added up, times 2^-kSoftmaxShift
__device__ inline float tracked_log2_sum(float sum) { return sum == 0.f ? INFINITY : log2f(sum) + kSoftmaxShift; }
// (a score of -inf, as of a row that is not there, is 0 beside any other scores, NaN among them)
__device__ inline float tracked_probability(float score, float2 all, float scale_log2e)
{
    const float p = __builtin_amdgcn_exp2f(fmaf(score - all.x, scale_log2e, -all.y));
    return score == -INFINITY ? 0.f : p;
}
__device__ inline void store_tracked_weight(const TrackedArgs &a, int64_t at, float w) { a.weights[at] = a.before ? fmaf(a.decay, a.before[at], w) : w; }

template <int FORMAT>
struct TrackedRows {
    typedef typename std::conditional<FORMAT == IHIP_KV_BF16, uint4, typename std::conditional<FORMAT == IHIP_KV_E4M3, uint2, uint32_t>::type>::type word;
    static constexpr int kPieces = FORMAT == IHIP_KV_BF16 ? 4 : FORMAT == IHIP_KV_E4M3 ? 2 : 1;
    uint4 k[2][kPieces];             // of rows n and 16 + n
    word v[8];                       // dims 8 n .. of keys 4 g + r and 16 + 4 g + r
    uint32_t k_scale[2], v_scale[8]; // 4-bit rows
};

template <int FORMAT, int HEADS>
__global__ __launch_bounds__(kTrThreads, FORMAT == IHIP_KV_BF16 ? 2 : 4) void attn_decode_tracked_kernel(const TrackedArgs a)
{
    typedef TrackedRows<FORMAT> Rows;
    const int p = a.grid.problem(), split = a.grid.part();
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int b = p / a.ge.Hkv, kv_head = p % a.ge.Hkv, G = a.ge.G;
    const int len = tracked_len(a, b);
    const int s0 = (int)min((int64_t)split * a.per, (int64_t)len), s1 = min(s0 + a.per, len), steps = (s1 - s0 + kTrStep - 1) / kTrStep;
    if (split > 0 && steps == 0) return;             // (part 0 of an idle place has its output to write)
    const int64_t pbase = ((int64_t)p * a.n_splits + split) * G;

    // where the part's rows are, in bytes from row 0; behind the last step: the waves' results, of four rows of the products at a time
    constexpr int kParts = HEADS == 4 ? 3 : 2;
    __shared__ __attribute__((aligned(16))) union {
        struct { int64_t k[kTrOnePart], v[kTrOnePart]; } row;
        float acc[kTrWaves][kParts][HEADS][kD];
    } sh;
    __shared__ uint32_t sh_there[kTrOnePart / kTrStep];     // which of a step's rows hold a key
    __shared__ float sh_m[kTrWaves][HEADS], sh_l[kTrWaves][HEADS];
    __shared__ float2 sh_all[HEADS];

    // The operand of step j: 16-byte pieces as above
    bf16x8 qb[4];
    {
        const uint16_t *qp = a.q + b * a.q_sb + (int64_t)(kv_head * G + min(n & (HEADS - 1), G - 1)) * a.q_sh;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            qb[j] = *reinterpret_cast<const bf16x8 *>(qp + (FORMAT == IHIP_KV_BF16 ? 32 * j + 8 * g : FORMAT == IHIP_KV_E4M3 ? 64 * (j >> 1) + 16 * g + 8 * (j & 1) : 32 * g + 8 * j));
    }
    // A row behind the part's last key stands for that one, a row on no page for one that can be read
    const int32_t *table = a.from.paged.block_table ? a.from.paged.block_table + (int64_t)b * a.from.paged.table_stride : nullptr;
    for (int i = tid; i < steps * kTrStep; i += kTrThreads) {
        const int row = min(s0 + i, s1 - 1);
        int first = b, in_page = row;
        if (table) {
            first = table[row >> a.from.paged.page_log2];
            in_page = row & ((1 << a.from.paged.page_log2) - 1);
        }
        const unsigned long long there = __ballot(s0 + i < s1 && first >= 0);
        if ((lane & 31) == 0) sh_there[i >> 5] = (uint32_t)(there >> (lane & 32));
        first = max(first, 0);
        sh.row.k[i] = first * a.from.k_sb + in_page * a.from.k_st;
        sh.row.v[i] = first * a.from.v_sb + in_page * a.from.v_st;
    }
    const uint8_t *kb = a.from.k + kv_head * a.from.k_sh + g * 16, *vb = a.from.v + kv_head * a.from.v_sh + n * (int)sizeof(typename Rows::word);
    const uint8_t *ksb = a.from.ks + kv_head * (a.from.k_sh / 16) + g, *vsb = a.from.vs + kv_head * (a.from.v_sh / 16) + (n >> 2);
    __syncthreads();

    auto load = [&](int step, Rows &r) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t off = sh.row.k[step * kTrStep + 16 * t + n];
#pragma unroll
            for (int j = 0; j < Rows::kPieces; ++j) r.k[t][j] = *reinterpret_cast<const uint4 *>(kb + off + 64 * j);
            if constexpr (FORMAT == IHIP_KV_MX4) r.k_scale[t] = ksb[off / 16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t v_off = sh.row.v[step * kTrStep + 16 * t + 4 * g + i];
                r.v[4 * t + i] = *reinterpret_cast<const typename Rows::word *>(vb + v_off);
                if constexpr (FORMAT == IHIP_KV_MX4) r.v_scale[4 * t + i] = vsb[v_off / 16];
            }
        }
    };
    // operand of step j of a lane's K row
    auto k_operand = [&](const Rows &r, int t, int j) {
        if constexpr (FORMAT == IHIP_KV_BF16) {
            return __builtin_bit_cast(bf16x8, r.k[t][j]);
        } else if constexpr (FORMAT == IHIP_KV_E4M3) {
            const uint4 w = r.k[t][j >> 1];
            return __builtin_bit_cast(bf16x8, fp8x8_to_bf16x8((j & 1) == 0 ? make_uint2(w.x, w.y) : make_uint2(w.z, w.w)));
        } else {
            const uint4 w = r.k[t][0];
            return __builtin_bit_cast(bf16x8, mx4_to_bf16x8(j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w, mx4_scale(r.k_scale[t])));
        }
    };
    // two dims of a V row, as bf16
    auto v_pair = [&](const Rows &r, int i, auto d) -> uint32_t {
        constexpr int D = decltype(d)::value;
        if constexpr (FORMAT == IHIP_KV_BF16) return D == 0 ? r.v[i].x : D == 1 ? r.v[i].y : D == 2 ? r.v[i].z : r.v[i].w;
        else if constexpr (FORMAT == IHIP_KV_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(D < 2 ? r.v[i].x : r.v[i].y, 1.0f, D % 2 == 1));
        else return mx4_pair<D>(r.v[i], mx4_scale(r.v_scale[i]));
    };

    // lanes whose first, and first and second parts of the probabilities other lanes bring; lanes that bring none
    const uint32_t not_first = (HEADS == 4 ? n < 4 : n < 8) ? 0u : ~0u, not_second = n >= 4 && n < 8 ? ~0u : 0u, none = n >= 12 ? 0u : ~0u;
    float *scores = a.scores + ((int64_t)p * G + min(n & (HEADS - 1), G - 1)) * a.score_stride + s0 + 4 * g;
    f32x4 acc[8];                                    // rows 4 g + r, dim 8 n + j
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kSoftmaxLowest, l = 0.f;               // of head n (m: the same in the four lanes of a head; l: of this lane's keys)
    Rows r, nx;
    // Wide rows are asked for a step ahead, two waves a SIMD; of narrow ones four waves have as many bytes on their way, and one step's registers
    // (three waves and a step ahead: as long in E4M3, 7 % longer in MX FP4)
    constexpr bool kAheadLoads = FORMAT == IHIP_KV_BF16;
    if (kAheadLoads && wv < steps) load(wv, r);
    for (int step = wv; step < steps; step += kTrWaves) {
        if (!kAheadLoads) load(step, r);
        else if (step + kTrWaves < steps) load(step + kTrWaves, nx);
        f32x4 c[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_operand(r, t, j), qb[j], c[t], 0, 0, 0);
        }
        const uint32_t there = __builtin_amdgcn_readfirstlane(sh_there[step]);
        if (there != ~0u) {                          // (what stands in the rows is not used, but has to be finite)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!((there >> (16 * (i >> 2) + 4 * g + (i & 3))) & 1)) {
                    c[i >> 2][i & 3] = -INFINITY;
                    r.v[i] = typename Rows::word{};
                    r.v_scale[i] = 127;
                }
        }
        // (lanes of the same head write the same: under a branch the compiler would not know how many requests are on their way, and wait for all)
#pragma unroll
        for (int t = 0; t < 2; ++t) *reinterpret_cast<f32x4 *>(scores + step * kTrStep + 16 * t) = c[t];
        float w[8], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = tracked_exp(c[i >> 2][i & 3], m, a.scale_log2e);    // of -inf: 0
            sum += w[i];
        }
        if (__any(!(sum <= kSoftmaxMaxSum))) {       // the reference follows where the scores outgrew it
            float top = c[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, c[i >> 2][i & 3]);
            const float mn = fmaxf(m, max_over_rows(top));
            const float corr = softmax_weight(m, mn, a.scale_log2e);
            m = mn;
            l *= corr;
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = tracked_exp(c[i >> 2][i & 3], m, a.scale_log2e);
                sum += w[i];
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const float x = __shfl(corr, 4 * g + h, 64);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j][h] *= x;
            }
        }
        l += sum;
        uint32_t part[4], third[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            auto dropped = [](float x, uint32_t p, int j) { return x - __uint_as_float(j == 0 ? p << 16 : p & 0xffff0000u); };
            const uint32_t first = pack_bf16x2(w[2 * i], w[2 * i + 1]), from_w = first & not_first;
            const float x = dropped(w[2 * i], HEADS == 4 ? from_w : first, 0), y = dropped(w[2 * i + 1], HEADS == 4 ? from_w : first, 1);
            const uint32_t next = pack_bf16x2(x, y);
            if constexpr (HEADS == 4) {              // (nothing is taken off in the lanes of the first parts, once in those of the second, twice of the third)
                const uint32_t from_x = next & not_second;
                part[i] = pack_bf16x2(dropped(x, from_x, 0), dropped(y, from_x, 1)) & none;
            } else {
                part[i] = not_first ? next : first;
                third[i] = pack_bf16x2(dropped(x, next, 0), dropped(y, next, 1)) & ~not_first;
            }
        }
        const bf16x8 pw = __builtin_bit_cast(bf16x8, make_uint4(part[0], part[1], part[2], part[3]));
        auto dims = [&](auto d) {                    // 8 n + 2 d and 8 n + 2 d + 1
            uint32_t x[8], lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = v_pair(r, i, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
                hi[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
            }
            f32x4 &even = acc[2 * decltype(d)::value], &odd = acc[2 * decltype(d)::value + 1];
            auto add = [&](const bf16x8 &p) {
                even = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), even, 0, 0, 0);
                odd = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), odd, 0, 0, 0);
            };
            add(pw);
            if constexpr (HEADS == 8) add(__builtin_bit_cast(bf16x8, make_uint4(third[0], third[1], third[2], third[3])));
        };
        dims(std::integral_constant<int, 0>{});
        dims(std::integral_constant<int, 1>{});
        dims(std::integral_constant<int, 2>{});
        dims(std::integral_constant<int, 3>{});
        if (kAheadLoads) r = nx;
    }

    // the waves and the parts are merged through LDS
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (lane < HEADS) { sh_m[wv][lane] = m; sh_l[wv][lane] = l; }
    __syncthreads();
    if (HEADS == 8 || g < kParts) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float *to = HEADS == 8 ? &sh.acc[wv][g >> 1][4 * (g & 1) + h][8 * n] : &sh.acc[wv][g][h][8 * n];
            *reinterpret_cast<float4 *>(to) = make_float4(acc[0][h], acc[1][h], acc[2][h], acc[3][h]);
            *reinterpret_cast<float4 *>(to + 4) = make_float4(acc[4][h], acc[5][h], acc[6][h], acc[7][h]);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < G * kD; idx += kTrThreads) {
        const int h = idx / kD, c = idx % kD;
        float M = kSoftmaxLowest;
#pragma unroll
        for (int w = 0; w < kTrWaves; ++w) M = fmaxf(M, sh_m[w][h]);
        float L = 0.f, A = 0.f;
#pragma unroll
        for (int w = 0; w < kTrWaves; ++w) {
            const float x = softmax_weight(sh_m[w][h], M, a.scale_log2e);
            L = fmaf(x, sh_l[w][h], L);
            A = fmaf(x, sh.acc[w][0][h][c] + (kParts == 3 ? sh.acc[w][1][h][c] + sh.acc[w][kParts - 1][h][c] : sh.acc[w][1][h][c]), A);
        }
        if (a.n_splits == 1) {                       // nothing to join
            const int64_t hq = (int64_t)b * a.ge.Hq + kv_head * G + h;
            a.out[hq * kD + c] = to_bf16(L == 0.f ? 0.f : A / L * a.v_scale);
            if (c == 0) {
                if (a.out_lse != nullptr) a.out_lse[hq] = softmax_lse(M, L, a.scale_log2e);
                sh_all[h] = make_float2(M, tracked_log2_sum(L));
            }
        } else {
            a.part_acc[(pbase + h) * kD + c] = A;
            if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + (pbase + h) * 2) = make_float2(M, L);
        }
    }
    if (a.n_splits > 1) return;
    __syncthreads();                                 // (the scores are this workgroup's own)
    const float *all = a.scores + (int64_t)p * G * a.score_stride;
    for (int row = tid; row < len; row += kTrThreads) {
        float w = 0.f;
        for (int h = 0; h < G; ++h) w += tracked_probability(all[h * a.score_stride + row], sh_all[h], a.scale_log2e);
        store_tracked_weight(a, (int64_t)p * a.weight_rows + row, w);
    }
}

// The parts joined, and weights: of the workgroups of a problem the first G take a head's output, the others kJoinRows rows each.
constexpr int kJoinRows = 1024, kJoinAhead = 8, kJoinGroups = kTrThreads / 32;
template <int G>
__global__ __launch_bounds__(kTrThreads) void attn_decode_tracked_join_kernel(const TrackedArgs a)
{
    const int p = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int b = p / a.ge.Hkv;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + (int64_t)p * a.n_splits * G;
    __shared__ float sh_m[kJoinGroups], sh_l[kJoinGroups];
    __shared__ float2 sh_all[G];
    __shared__ __attribute__((aligned(16))) float sh_a[kJoinGroups][kD];
    static_assert(G <= kJoinGroups, "");
    if ((int)blockIdx.y < G) {
        // a head's parts: 32 lanes a part, 4 dims each
        const int h = blockIdx.y, l32 = tid & 31, grp = tid >> 5, parts = (tracked_len(a, b) + a.per - 1) / a.per;
        const float4 *accs = reinterpret_cast<const float4 *>(a.part_acc + (int64_t)p * a.n_splits * G * kD) + l32;
        float M = kSoftmaxLowest, L = 0.f;
        float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = grp; s0 < parts; s0 += kJoinGroups * kJoinAhead) {
            float2 x[kJoinAhead];
            float4 v[kJoinAhead];
            float top = M;
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                const int64_t at = (int64_t)min(s0 + i * kJoinGroups, parts - 1) * G + h;
                x[i] = ml[at];
                v[i] = accs[at * (kD / 4)];
            }
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i)
                if (s0 + i * kJoinGroups < parts) top = fmaxf(top, x[i].x);
            const float corr = softmax_weight(M, top, a.scale_log2e);
            L *= corr;
            A = make_float4(A.x * corr, A.y * corr, A.z * corr, A.w * corr);
            M = top;
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                if (s0 + i * kJoinGroups >= parts) break;
                const float w = softmax_weight(x[i].x, M, a.scale_log2e);
                L = fmaf(w, x[i].y, L);
                A = make_float4(fmaf(w, v[i].x, A.x), fmaf(w, v[i].y, A.y), fmaf(w, v[i].z, A.z), fmaf(w, v[i].w, A.w));
            }
        }
        *reinterpret_cast<float4 *>(&sh_a[grp][4 * l32]) = A;
        if (l32 == 0) { sh_m[grp] = M; sh_l[grp] = L; }
        __syncthreads();
        if (tid >= kD) return;
        M = kSoftmaxLowest;
#pragma unroll
        for (int i = 0; i < kJoinGroups; ++i) M = fmaxf(M, sh_m[i]);
        float sum = 0.f, out = 0.f;
#pragma unroll
        for (int i = 0; i < kJoinGroups; ++i) {
            const float w = softmax_weight(sh_m[i], M, a.scale_log2e);
            sum = fmaf(w, sh_l[i], sum);
            out = fmaf(w, sh_a[i][tid], out);
        }
        const int64_t hq = (int64_t)b * a.ge.Hq + (p % a.ge.Hkv) * G + h;
        a.out[hq * kD + tid] = to_bf16(sum == 0.f ? 0.f : out / sum * a.v_scale);         // an idle place: 0
        if (a.out_lse != nullptr && tid == 0) a.out_lse[hq] = softmax_lse(M, sum, a.scale_log2e);
        return;
    }
    const int len = tracked_len(a, b), row0 = ((int)blockIdx.y - G) * kJoinRows;
    if (row0 >= len) return;
    // (what the weights are made of is on its way while the sums are joined)
    constexpr int kRows = kJoinRows / kTrThreads;
    const float *scores = a.scores + (int64_t)p * G * a.score_stride;
    float x[kRows][G], old[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int row = min(row0 + i * kTrThreads + tid, len - 1);
#pragma unroll
        for (int h = 0; h < G; ++h) x[i][h] = scores[h * a.score_stride + row];
        old[i] = a.before ? a.before[(int64_t)p * a.weight_rows + row] : 0.f;
    }
    const int parts = (len - 1) / a.per + 1;
    for (int h = wv; h < G; h += kTrWaves) {
        float M = kSoftmaxLowest, L = 0.f;
        for (int s = lane; s < parts; s += 64) {
            const float2 y = ml[(int64_t)s * G + h];
            const float top = fmaxf(M, y.x);
            L = fmaf(softmax_weight(y.x, top, a.scale_log2e), y.y, softmax_weight(M, top, a.scale_log2e) * L);
            M = top;
        }
        const float top = wave_max_f32(M);
        L *= softmax_weight(M, top, a.scale_log2e);
        M = top;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) L += __shfl_xor(L, d, 64);
        if (lane == 0) sh_all[h] = make_float2(M, tracked_log2_sum(L));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int row = row0 + i * kTrThreads + tid;
        if (row >= len) break;
        float w = 0.f;
#pragma unroll
        for (int h = 0; h < G; ++h) w += tracked_probability(x[i][h], sh_all[h], a.scale_log2e);
        a.weights[(int64_t)p * a.weight_rows + row] = a.before ? fmaf(a.decay, old[i], w) : w;
    }
}

// All parts have as many rows, so that workgroups take as long as each other where sequences do not: kTrMaxSplit, or fewer where that would leave
// compute units with less than two.  us a call, with probabilities of two bf16 numbers (three: 2 more in MX FP4, 1 in E4M3), for 768 / 512 / 1,024 / 2,048 rows: 8 sequences of 20,637 to 32,768 in MX FP4 74 / 77 / 78 / 83, 32 of
// 7,383 to 16,384 in E4M3 200 / 201 / 201 / 207, one of 200,001 in MX FP4 77 / 82 / 77 / 82; one of 30,001 in bf16, with 128 / 256 / 512 rows
// 39 / 32 / 29.  Short sequences in one part each need no join: 4 of 1,000 14.7 where parts take 17.8, 16 of 1,000 16.7 / 17.7, 32 of 1,024 to 1,055
// 20.3 / 19.6.
struct TrackedPlan { int splits, per; int64_t score_stride, ml; size_t bytes; };         // ml: floats of part_ml, in whole 16 bytes (part_acc is behind it)
static TrackedPlan tracked_plan(const ihip_shape &s)
{
    const int64_t total = s.max_seq_len, P = std::max<int64_t>(1, (int64_t)s.B * s.Hkv);
    TrackedPlan r;
    r.per = (int)std::min<int64_t>(kTrMaxSplit, (total * P / (2 * compute_units()) + kTrMinSplit) / kTrMinSplit * kTrMinSplit);
    if (total <= (P < compute_units() ? kTrOnePart : kTrOnePart / 2)) r.per = (int)((total + kTrMinSplit - 1) / kTrMinSplit * kTrMinSplit);
    r.splits = (int)((total - 1) / r.per + 1);
    r.score_stride = (total + kTrStep - 1) / kTrStep * kTrStep;
    const int64_t heads = (int64_t)s.B * s.Hq;
    r.ml = (heads * r.splits * 2 + 3) / 4 * 4;
    r.bytes = (size_t)(heads * (r.score_stride + (int64_t)r.splits * kD) + r.ml) * sizeof(float);
    return r;
}

}  // namespace ihip

using namespace ihip;

extern "C" size_t ihip_attn_decode_tracked_workspace_bytes(const ihip_shape *shape)
{
    if (check_shape(shape, "ihip_attn_decode_tracked_workspace_bytes") != IHIP_OK) return 0;
    return std::max<size_t>(tracked_plan(*shape).bytes, 256);
}

extern "C" int32_t ihip_attn_decode_tracked(const ihip_shape *shape, ihip_tensor q, const ihip_kv_store *store, float sm_scale,
                                            const float *before, float decay, const ihip_kv_track *track, void *out,
                                            float *out_lse, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ihip_attn_decode_tracked";
    int32_t rc;
    if ((rc = check_shape(shape, who)) != IHIP_OK) return rc;
    if (shape->B == 0) return IHIP_OK;
    if (shape->Tq != 1 || shape->b_q != 1) return fail(IHIP_ERR_INVALID_ARG, "%s: needs Tq == b_q == 1", who);
    if ((rc = check_tensor(q, who, "q")) != IHIP_OK) return rc;
    TrackedArgs a{};
    if ((rc = check_store(who, store, *shape, &a.from)) != IHIP_OK) return rc;
    if ((rc = check_track(who, track, shape->max_seq_len, false)) != IHIP_OK) return rc;
    if ((rc = check_before(who, before, decay, track, (int64_t)shape->B * shape->Hkv)) != IHIP_OK) return rc;
    if (!out) return fail(IHIP_ERR_INVALID_ARG, "%s: out is NULL", who);
    if ((rc = check_sm_scale(who, sm_scale, &a.scale_log2e)) != IHIP_OK) return rc;
    if ((rc = check_sm_scale(who, sm_scale * a.from.k_scale, &a.scale_log2e)) != IHIP_OK) return rc;
    const TrackedPlan plan = tracked_plan(*shape);
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < plan.bytes)
        return fail(IHIP_ERR_WORKSPACE, "%s: workspace of %zu bytes, 16-byte aligned, needed, %zu given", who, plan.bytes, ws_bytes);
    const int64_t P = (int64_t)shape->B * shape->Hkv;
    const int64_t join_groups = ((int64_t)shape->max_seq_len - 1) / kJoinRows + 1;
    if (join_groups > 65535 - 8) return fail(IHIP_ERR_UNSUPPORTED, "%s: max_seq_len = %d is too large", who, shape->max_seq_len);
    a.ge = make_geometry(*shape);
    a.max_len = shape->max_seq_len;
    a.q = (const uint16_t *)q.ptr; a.q_sb = q.stride_b; a.q_sh = q.stride_h;
    a.v_scale = a.from.v_scale;
    a.n_splits = plan.splits;
    a.per = plan.per;
    a.grid = decode_grid(a.ge, a.n_splits, false);
    if (P > (a.grid.problems_first ? (int64_t)UINT32_MAX / kTrThreads : 65535))
        return fail(IHIP_ERR_UNSUPPORTED, "%s: %lld sequences x KV heads are too many", who, (long long)P);
    a.scores = (float *)ws;
    a.score_stride = plan.score_stride;
    a.part_ml = a.scores + P * a.ge.G * plan.score_stride;
    a.part_acc = a.part_ml + plan.ml;
    a.out = (uint16_t *)out;
    a.out_lse = out_lse;
    a.before = before;
    a.weights = track->weights;
    a.weight_rows = track->rows;
    a.decay = decay;
    const hipStream_t st = (hipStream_t)stream;
    const dim3 grid = a.grid.dims((int)P, a.n_splits);
    {
        KernelTimer timer("attn_decode_tracked", st);
#define IHIP_AT(FMT)                                                                                                              \
        if (a.ge.G <= 4) hipLaunchKernelGGL((attn_decode_tracked_kernel<FMT, 4>), grid, dim3(kTrThreads), 0, st, a);              \
        else hipLaunchKernelGGL((attn_decode_tracked_kernel<FMT, 8>), grid, dim3(kTrThreads), 0, st, a)
        if (store->format == IHIP_KV_BF16) { IHIP_AT(IHIP_KV_BF16); }
        else if (store->format == IHIP_KV_E4M3) { IHIP_AT(IHIP_KV_E4M3); }
        else { IHIP_AT(IHIP_KV_MX4); }
#undef IHIP_AT
    }
    if ((rc = check_launch(who)) != IHIP_OK || a.n_splits == 1) return rc;
    KernelTimer timer("attn_decode_tracked_join", st);
    const dim3 join((uint32_t)P, (uint32_t)(a.ge.G + join_groups));
    if (a.ge.G == 1) hipLaunchKernelGGL(attn_decode_tracked_join_kernel<1>, join, dim3(kTrThreads), 0, st, a);
    else if (a.ge.G == 2) hipLaunchKernelGGL(attn_decode_tracked_join_kernel<2>, join, dim3(kTrThreads), 0, st, a);
    else if (a.ge.G == 4) hipLaunchKernelGGL(attn_decode_tracked_join_kernel<4>, join, dim3(kTrThreads), 0, st, a);
    else hipLaunchKernelGGL(attn_decode_tracked_join_kernel<8>, join, dim3(kTrThreads), 0, st, a);
    return check_launch(who);
}
