// squat_paged_attention: softmax(scale q k^T) v over a store of pages, straight from the packed codes.
//
// Rows are (new token, query head of a KV head) pairs of one sequence, in tiles of 16 or 32; a workgroup meets one tile and one KV
// head with a part of the sequence, its four wavefronts taking 32-token steps in turn.  Per step a wavefront computes
// S^T = K Q^T and O^T += V^T P^T with 16x16x32 fp16 matrix instructions: in both a lane's column is a query row, so that the
// softmax's maximum and sum stay in the lane, and the logits of a lane (tokens 4 h + i of the step's halves, h = lane / 16) are
// where the second product wants its operand: nothing is exchanged between lanes and nothing goes through LDS.
//
// Keys enter as raw integer codes (exact in fp16); scale and zero-point of a group come in behind, in fp32:
//     q . k_t = sum_g scale[t,g] (sum_{c in g} q_c code_c) + zero[t,g] (sum_{c in g} q_c).
// Codes are turned into fp16 by placing their bits in the mantissa of a power of two, bias + code, one or two operations per pair;
// the accumulator starts at -bias sum q.  Values are contracted over tokens, whose scales differ, so they are dequantized, one
// rounding (2^-11) each; a lane takes 8 channels of 8 tokens, which it needs as 8 operands of 8 tokens, one per channel, so
// that the order of channels and tokens in the products makes a transpose unnecessary.
//
// The running maximum m of a row is raised only when a logit passes it by more than 2^kSlack (the rows' sums are rescaled then, for
// all of them): p = 2^(x - m + kLift), at most 2^15, and small weights keep their bits down to 2^-(24 + kLift) of the largest.
#include <type_traits>

#include "squat_paged.h"

using namespace squat;

namespace {

constexpr int kStep = 32;                                 // tokens per step of a wavefront
constexpr int kWaves = 4;
constexpr float kLift = 11.0f, kSlack = 4.0f;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr int kPitch = kD + 4;                            // floats per row of a wavefront's sums in LDS

struct AttendParams {
    const unsigned char *kc, *km, *vc, *vm;
    const unsigned char* q;
    int64_t qst, qsh;                                     // elements
    unsigned char* out;
    int64_t ost, osh;
    float* lse;
    const int32_t *q_start, *kv_len, *pages;
    int64_t page_stride;
    int pages_per_seq, n_seqs, n_new, n_kv, qpk, n_pages, page_shift;
    float scale;                                          // out_scale * log2(e)
    int splits, least;                                    // parts of a sequence at most; steps per part at least
    int n_tiles;
    float* part_o;                                        // [splits, n_tiles, n_kv, rows, d]
    float2* part_ml;                                      // [splits, n_tiles, n_kv, rows]
};

// A tile of R rows of one sequence, and the part of the sequence it is met with.
struct Tile {
    int seq, start, rows;                                 // the sequence's first new token, and its rows in all
    int row0;                                             // first row of the tile
    int pos0;                                             // position of the first new token
    int end;                                              // tokens that the tile's last row sees
    int steps, parts;
};

// Tile w: sequence s has the tiles floor(q_start[s] qpk / R) + s onwards, one number at most unused.  Every lane probes one sequence a
// round (64 sequences: one round).  Device values are brought into range, so that whatever they hold, only rows of q and out are touched.
template <int R>
__device__ __forceinline__ bool find_tile(const AttendParams& p, int w, Tile& t) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    auto first = [&](int s) { return min(max(p.q_start[s], 0), p.n_new); };
    auto base = [&](int s) { return static_cast<int64_t>(first(s)) * p.qpk / R + s; };
    int lo = 0, hi = p.n_seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
        const bool at = s < hi && (lane == 0 || base(s) <= w);
        const uint64_t m = __ballot(at);
        lo += (63 - __builtin_clzll(m)) * step;
        hi = min(hi, lo + step);
    }
    t.seq = __builtin_amdgcn_readfirstlane(lo);
    t.start = first(t.seq);
    const int n = max(first(t.seq + 1) - t.start, 0);
    t.rows = n * p.qpk;
    const int64_t tile = w - base(t.seq);
    if (tile < 0 || tile * R >= t.rows) return false;
    t.row0 = static_cast<int>(tile) * R;
    const int64_t room = static_cast<int64_t>(p.pages_per_seq) << p.page_shift;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(p.kv_len[t.seq], 0)), room));
    t.pos0 = len - n;
    t.end = min(max(t.pos0 + (min(t.row0 + R, t.rows) - 1) / p.qpk + 1, 0), len);
    t.steps = (t.end + kStep - 1) / kStep;
    t.parts = min(max(t.steps / p.least, 1), p.splits);
    return true;
}

__device__ __forceinline__ half2v as_half2(uint32_t u) { return __builtin_bit_cast(half2v, u); }
__device__ __forceinline__ uint32_t byte_perm(uint32_t a, uint32_t b, uint32_t sel) { return __builtin_amdgcn_perm(a, b, sel); }   // bytes 0-3: b
__device__ __forceinline__ float half_lo(uint32_t u) { return static_cast<float>(as_half2(u)[0]); }
__device__ __forceinline__ float half_hi(uint32_t u) { return static_cast<float>(as_half2(u)[1]); }

// What is added to a code when its bits are put into an fp16 mantissa.
template <int BITS>
struct Bias {
    static constexpr float value = BITS == 2 ? 16.0f : BITS == 4 ? 64.0f : 1024.0f;
    static constexpr uint32_t bits = BITS == 2 ? 0x4C004C00u : BITS == 4 ? 0x54005400u : 0x64006400u;
};

__device__ __forceinline__ uint32_t shifted(uint32_t x, int left) { return left >= 0 ? x << left : x >> -left; }

// Two codes of `x` (halves), at bit b of each half (2 and 4 bits), as bias + code.
template <int BITS>
__device__ __forceinline__ uint32_t code_pair(uint32_t x, int b) {
    constexpr int at = BITS == 2 ? 6 : 4;
    constexpr uint32_t mask = ((1u << BITS) - 1u) << at;
    return (shifted(x, at - b) & (mask | (mask << 16))) | Bias<BITS>::bits;
}

// 8 channels of a key, in the order in which Queries holds the query's: 0 4 1 5 2 6 3 7 (8 bits: as they come).
template <int BITS>
struct KeyWord;
template <>
struct KeyWord<2> {
    uint32_t w;                                           // 16 channels, of which the lane's are the half h & 1
    __device__ __forceinline__ void load(const unsigned char* row, int s, int h) { w = *reinterpret_cast<const uint32_t*>(row + 8 * s + 4 * (h >> 1)); }
    __device__ __forceinline__ u32x4 pairs(int h) const {
        const uint32_t x = byte_perm(0u, w, (h & 1) ? 0x0C030C02u : 0x0C010C00u);
        return u32x4{code_pair<2>(x, 0), code_pair<2>(x, 2), code_pair<2>(x, 4), code_pair<2>(x, 6)};
    }
};
template <>
struct KeyWord<4> {
    uint32_t w;
    __device__ __forceinline__ void load(const unsigned char* row, int s, int h) { w = *reinterpret_cast<const uint32_t*>(row + 16 * s + 4 * h); }
    __device__ __forceinline__ u32x4 pairs(int) const { return u32x4{code_pair<4>(w, 0), code_pair<4>(w, 4), code_pair<4>(w, 8), code_pair<4>(w, 12)}; }
};
template <>
struct KeyWord<8> {
    u32x2 w;
    __device__ __forceinline__ void load(const unsigned char* row, int s, int h) { w = *reinterpret_cast<const u32x2*>(row + 32 * s + 8 * h); }
    __device__ __forceinline__ u32x4 pairs(int) const {
        return u32x4{byte_perm(0x64646464u, w[0], 0x04010400u), byte_perm(0x64646464u, w[0], 0x04030402u),
                     byte_perm(0x64646464u, w[1], 0x04010400u), byte_perm(0x64646464u, w[1], 0x04030402u)};
    }
};

// 8 channels of a value, lane m's: channels 8 m to 8 m + 7.
template <int BITS>
struct ValueWord {
    typename std::conditional<BITS == 8, u32x2, typename std::conditional<BITS == 4, uint32_t, uint16_t>::type>::type w;
    __device__ __forceinline__ void load(const unsigned char* row, int m) { w = *reinterpret_cast<const decltype(w)*>(row + m * BITS); }
};

// Channel j of two tokens, as bias + code.
template <int BITS>
__device__ __forceinline__ uint32_t value_pair(const ValueWord<BITS>& a, const ValueWord<BITS>& b, int j) {
    if constexpr (BITS == 2) {
        return code_pair<2>(static_cast<uint32_t>(a.w) | (static_cast<uint32_t>(b.w) << 16), 2 * j);
    } else if constexpr (BITS == 4) {
        return code_pair<4>(byte_perm(b.w, a.w, j < 4 ? 0x05040100u : 0x07060302u), 4 * (j & 3));
    } else {
        const uint32_t c = static_cast<uint32_t>(j & 3);
        return byte_perm(b.w[j >> 2], a.w[j >> 2], 0x0C000C00u | c | ((c + 4u) << 16)) | Bias<8>::bits;
    }
}

template <int BITS, int NG>
struct StepLoads {
    KeyWord<BITS> k[2][4];
    uint32_t km[2][4][NG];
    ValueWord<BITS> v[2][4];
    uint32_t vm[2][4];
};

template <int BITS, int NG, int NQ, int QDT>
__global__ void __launch_bounds__(256) attend_kernel(const AttendParams p) {
    constexpr int R = 16 * NQ;
    constexpr int ROW = kD * BITS / 8;                    // bytes of a token's codes
    constexpr bool SPLIT_P = QDT == SQUAT_F16;            // weights as high and low fp16 parts (the fp16 result has 3 bits more than bf16's)
    __shared__ float sums[kWaves][16][kPitch];
    __shared__ float2 stats[kWaves][R];
    const int bx = static_cast<int>(blockIdx.x), w_tile = bx / p.n_kv, kvh = bx - w_tile * p.n_kv;
    Tile t;
    if (!find_tile<R>(p, w_tile, t)) return;
    const int part = static_cast<int>(blockIdx.y);
    if (part >= t.parts) return;
    const int lane = static_cast<int>(threadIdx.x) & 63, m = lane & 15, h = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int first = static_cast<int>(static_cast<int64_t>(t.steps) * part / t.parts);
    const int last = static_cast<int>(static_cast<int64_t>(t.steps) * (part + 1) / t.parts);

    // The queries, as operands: step s is channels 32 s to 32 s + 31, a lane's are 8 of them from 32 s + 8 h on, in KeyWord's order.
    half8 qf[NQ][4];
    f32x4 start[NQ][NG];                                  // -bias * sum of a group's queries
    float qs[NQ][NG], scale[NQ];
    int seen[NQ];                                         // the last token that the lane's row sees
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = t.row0 + 16 * n + m;
        const bool live = row < t.rows;
        const int r = live ? row : t.rows - 1;
        const int i = r / p.qpk, hq = kvh * p.qpk + (r - i * p.qpk);
        seen[n] = live ? t.pos0 + i : -1;
        const unsigned char* src = p.q + ((t.start + i) * p.qst + hq * p.qsh + 8 * h) * 2;
        float sum[4], top = 0.0f;
        u32x4 raw[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) raw[s] = *reinterpret_cast<const u32x4*>(src + 64 * s);
        float factor = 1.0f;
        if constexpr (QDT == SQUAT_BF16) {                // by a power of two into [1/2, 1): exact, and whatever the row's size
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(as_f32(raw[s][e] << 16)), fabsf(as_f32(raw[s][e] & 0xFFFF0000u))));
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            int e = 0;
            if (top > 0.0f && top < INFINITY) (void)frexpf(top, &e);
            e = max(-100, min(100, e));
            factor = ldexpf(1.0f, -e);
            scale[n] = ldexpf(p.scale, e);
        } else {
            scale[n] = p.scale;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            _Float16 c[8];
            sum[s] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t u = raw[s][e >> 1];
                if constexpr (QDT == SQUAT_BF16) c[e] = static_cast<_Float16>(as_f32((e & 1) ? (u & 0xFFFF0000u) : (u << 16)) * factor);
                else c[e] = as_half2(u)[e & 1];
                if (!live) c[e] = static_cast<_Float16>(0.0f);
                sum[s] += static_cast<float>(c[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) qf[n][s][e] = BITS == 8 ? c[e] : c[(e >> 1) + 4 * (e & 1)];
            sum[s] += __shfl_xor(sum[s], 16, 64);
            sum[s] += __shfl_xor(sum[s], 32, 64);
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            qs[n][g] = 0.0f;
#pragma unroll
            for (int s = 0; s < 4 / NG; ++s) qs[n][g] += sum[g * (4 / NG) + s];
            const float b = -Bias<BITS>::value * qs[n][g];
            start[n][g] = f32x4{b, b, b, b};
        }
    }
    const int least_seen = t.pos0 + t.row0 / p.qpk;       // every live row sees this token and all before it

    f32x4 o[NQ][8];                                       // O^T: channels 8 (4 h + i) + j, column m
    float top[NQ], total[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        top[n] = -INFINITY;
        total[n] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[n][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const int32_t* list = p.pages + t.seq * p.page_stride;
    const int offset_mask = (1 << p.page_shift) - 1;
    // Rows of a half step of 16 tokens: the page's, or, past the end or in a page that does not exist, some that do; `limit` is the first
    // of its tokens that nobody sees.
    auto rows_of = [&](int token, int& limit) {
        const bool past = token >= t.end;
        const int page = list[(past ? token - 16 : token) >> p.page_shift];
        const bool ok = page >= 0 && page < p.n_pages && !past;
        limit = ok ? t.end : token;
        return ((static_cast<int64_t>(ok ? page : 0) * p.n_kv + kvh) << p.page_shift) + (token & offset_mask);
    };

    for (int step = first + wave; step < last; step += kWaves) {
        const int t0 = step * kStep;
        int limit[2];
        StepLoads<BITS, NG> in;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t rows = rows_of(t0 + 16 * u, limit[u]);
            const unsigned char* kc = p.kc + rows * ROW + m * ROW;
#pragma unroll
            for (int s = 0; s < 4; ++s) in.k[u][s].load(kc, s, h);
            const unsigned char* km = p.km + (rows + 4 * h) * (4 * NG);
            const unsigned char* vc = p.vc + (rows + 4 * h) * ROW;
            const unsigned char* vm = p.vm + (rows + 4 * h) * (4 * NG) + 4 * ((m * NG) >> 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (NG == 4) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(km + i * 16);
#pragma unroll
                    for (int g = 0; g < 4; ++g) in.km[u][i][g] = x[g];
                } else if constexpr (NG == 2) {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(km + i * 8);
                    in.km[u][i][0] = x[0];
                    in.km[u][i][1] = x[1];
                } else {
                    in.km[u][i][0] = *reinterpret_cast<const uint32_t*>(km + i * 4);
                }
                in.v[u][i].load(vc + i * ROW, m);
                in.vm[u][i] = *reinterpret_cast<const uint32_t*>(vm + i * (4 * NG));
            }
        }

        // logits: lane's column m, tokens t0 + 16 u + 4 h + i
        float x[NQ][2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            half8 kf[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) kf[s] = __builtin_bit_cast(half8, in.k[u][s].pairs(h));
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f32x4 a = start[n][g];
#pragma unroll
                    for (int s = 0; s < 4 / NG; ++s) a = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[g * (4 / NG) + s], qf[n][g * (4 / NG) + s], a, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float z = half_hi(in.km[u][i][g]) * qs[n][g];
                        x[n][u][i] = fmaf(half_lo(in.km[u][i][g]), a[i], g == 0 ? z : x[n][u][i] + z);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) x[n][u][i] = fmaf(x[n][u][i], 0.0f, x[n][u][i]) * scale[n];       // (infinite metadata: NaN)
            }
        }
        // the last tokens, the ones that not every row sees, and pages that do not exist
        const bool edge = t0 + kStep > least_seen + 1 || t0 + 16 > limit[0] || t0 + kStep > limit[1];       // uniform
        if (edge) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = t0 + 16 * u + 4 * h + i;
                    const bool there = token < limit[u];
                    if (!there) in.vm[u][i] = 0u;         // (whatever the page holds behind the last token)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
                        if (!there || token > seen[n]) x[n][u][i] = -INFINITY;
                }
            // A token that only some rows see spoils those alone: NaN and infinity would reach the others as 0 * NaN.
            bool odd = false;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    odd |= (in.vm[u][i] & 0x7C00u) == 0x7C00u || (in.vm[u][i] & 0x7C000000u) == 0x7C000000u;
            if (__ballot(odd)) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if ((in.vm[u][i] & 0x7C00u) == 0x7C00u || (in.vm[u][i] & 0x7C000000u) == 0x7C000000u) in.vm[u][i] = 0u;
                // this lane's sums are of the channels 32 h to 32 h + 31
                for (int k = 0; k < kStep; ++k) {
                    int lim;
                    const int64_t rows = rows_of(t0 + (k & 16), lim);
                    if (t0 + k >= lim) continue;
                    const uint32_t meta = *reinterpret_cast<const uint32_t*>(p.vm + (rows + (k & 15)) * (4 * NG) + 4 * ((h * NG) >> 2));
                    const bool spoilt = (meta & 0x7C00u) == 0x7C00u || (meta & 0x7C000000u) == 0x7C000000u;
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
                        if (spoilt && t0 + k <= seen[n])
#pragma unroll
                            for (int j = 0; j < 8; ++j) o[n][j] += NAN;
                }
            }
        }

        // weights
        half8 pf[NQ], pl[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float most = x[n][0][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) most = fmaxf(most, x[n][e >> 2][e & 3]);
            if (__ballot(most > top[n] + kSlack)) {
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const float now = fmaxf(top[n], most);
                const float by = now > -INFINITY ? __builtin_amdgcn_exp2f(top[n] - now) : 1.0f;
                top[n] = now;
                total[n] *= by;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[n][j] *= by;
            }
            const float from = top[n] > -INFINITY ? top[n] - kLift : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __builtin_amdgcn_exp2f(x[n][e >> 2][e & 3] - from);
                total[n] += w;
                pf[n][e] = static_cast<_Float16>(w);
                if constexpr (SPLIT_P) pl[n][e] = static_cast<_Float16>(w - static_cast<float>(pf[n][e]));
            }
        }

        // values: operand j is channel 8 m + j of the tokens t0 + 4 h + i, t0 + 16 + 4 h + i
        half2v vs[4], vz[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t a = in.vm[e >> 1][2 * (e & 1)], b = in.vm[e >> 1][2 * (e & 1) + 1];
            vs[e] = as_half2(byte_perm(b, a, 0x05040100u));
            vz[e] = as_half2(byte_perm(b, a, 0x07060302u));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4 raw;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const half2v c = as_half2(value_pair<BITS>(in.v[e >> 1][2 * (e & 1)], in.v[e >> 1][2 * (e & 1) + 1], j)) -
                                 half2v{static_cast<_Float16>(Bias<BITS>::value), static_cast<_Float16>(Bias<BITS>::value)};
                raw[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, vs[e], vz[e]));
            }
            const half8 vf = __builtin_bit_cast(half8, raw);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[n], o[n][j], 0, 0, 0);
                if constexpr (SPLIT_P) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pl[n], o[n][j], 0, 0, 0);
            }
        }
    }

    // the four wavefronts' sums, 16 rows at a time
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        total[n] += __shfl_xor(total[n], 16, 64);
        total[n] += __shfl_xor(total[n], 32, 64);
        if (h == 0) stats[wave][16 * n + m] = float2{top[n], total[n]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float* to = &sums[wave][m][8 * (4 * h + i)];
            *reinterpret_cast<f32x4*>(to) = f32x4{o[n][0][i], o[n][1][i], o[n][2][i], o[n][3][i]};
            *reinterpret_cast<f32x4*>(to + 4) = f32x4{o[n][4][i], o[n][5][i], o[n][6][i], o[n][7][i]};
        }
        __syncthreads();
        const int r = static_cast<int>(threadIdx.x) >> 4, c0 = (static_cast<int>(threadIdx.x) & 15) * 8;
        const int row = t.row0 + 16 * n + r;
        if (row < t.rows) {
            float all = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) all = fmaxf(all, stats[w][16 * n + r].x);
            float sum = 0.0f, acc[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float2 st = stats[w][16 * n + r];
                const float by = st.x > -INFINITY ? __builtin_amdgcn_exp2f(st.x - all) : 1.0f;
                sum += by * st.y;
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = fmaf(by, sums[w][r][c0 + c], acc[c]);
            }
            if (p.splits > 1) {
                const int64_t at = (static_cast<int64_t>(part) * p.n_tiles * p.n_kv + bx) * R + 16 * n + r;
                float* to = p.part_o + at * kD + c0;
                *reinterpret_cast<f32x4*>(to) = f32x4{acc[0], acc[1], acc[2], acc[3]};
                *reinterpret_cast<f32x4*>(to + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
                if (c0 == 0) p.part_ml[at] = float2{all, sum};
            } else {
                const int i = row / p.qpk, hq = kvh * p.qpk + (row - i * p.qpk);
                const float by = sum == 0.0f ? 1.0f : 1.0f / sum;
                unsigned char* to = p.out + ((t.start + i) * p.ost + hq * p.osh + c0) * 2;
                if constexpr (QDT == SQUAT_BF16) {
                    bf16x8 v;
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = static_cast<__bf16>(acc[c] * by);
                    *reinterpret_cast<bf16x8*>(to) = v;
                } else {
                    half8 v;
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = static_cast<_Float16>(acc[c] * by);
                    *reinterpret_cast<half8*>(to) = v;
                }
                if (p.lse && c0 == 0)
                    p.lse[static_cast<int64_t>(t.start + i) * p.n_kv * p.qpk + hq] =
                        sum == 0.0f ? -INFINITY : kLn2 * ((all - kLift) + __builtin_amdgcn_logf(sum));
            }
        }
        if (n + 1 < NQ) __syncthreads();
    }
}

// The parts of a row put together: one workgroup a row, a wavefront every fourth part, two channels a lane.
template <int R, int QDT>
__global__ void __launch_bounds__(256) attend_join_kernel(const AttendParams p) {
    __shared__ float2 sums[kWaves][64];
    __shared__ float totals[kWaves];
    const int bx = static_cast<int>(blockIdx.x), w_tile = bx / p.n_kv, kvh = bx - w_tile * p.n_kv;
    Tile t;
    if (!find_tile<R>(p, w_tile, t)) return;
    const int row = t.row0 + static_cast<int>(blockIdx.y);
    if (row >= t.rows) return;
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int64_t at = static_cast<int64_t>(bx) * R + blockIdx.y, stride = static_cast<int64_t>(p.n_tiles) * p.n_kv * R;
    float all = -INFINITY;
    for (int s = lane; s < t.parts; s += 64) all = fmaxf(all, p.part_ml[at + s * stride].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor(all, o, 64));
    float2 acc{0.0f, 0.0f};
    float sum = 0.0f;
#pragma unroll 4
    for (int s = wave; s < t.parts; s += kWaves) {
        const float2 ml = p.part_ml[at + s * stride];
        const float2 v = *reinterpret_cast<const float2*>(p.part_o + (at + s * stride) * kD + 2 * lane);
        const float by = ml.x > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - all) : 1.0f;
        sum += by * ml.y;
        acc.x = fmaf(by, v.x, acc.x);
        acc.y = fmaf(by, v.y, acc.y);
    }
    sums[wave][lane] = acc;
    if (lane == 0) totals[wave] = sum;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        acc.x += sums[w][lane].x;
        acc.y += sums[w][lane].y;
        sum += totals[w];
    }
    const int i = row / p.qpk, hq = kvh * p.qpk + (row - i * p.qpk);
    const float by = sum == 0.0f ? 1.0f : 1.0f / sum;
    unsigned char* to = p.out + ((t.start + i) * p.ost + hq * p.osh + 2 * lane) * 2;
    uint32_t both;
    if constexpr (QDT == SQUAT_BF16) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        both = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(acc.x * by), static_cast<__bf16>(acc.y * by)});
    } else {
        both = __builtin_bit_cast(uint32_t, half2v{static_cast<_Float16>(acc.x * by), static_cast<_Float16>(acc.y * by)});
    }
    *reinterpret_cast<uint32_t*>(to) = both;
    if (p.lse && lane == 0)
        p.lse[static_cast<int64_t>(t.start + i) * p.n_kv * p.qpk + hq] = sum == 0.0f ? -INFINITY : kLn2 * ((all - kLift) + __builtin_amdgcn_logf(sum));
}

struct Plan {
    int nq;                                               // row tiles of 16 nq rows
    int64_t tiles;
    int splits, least;
    size_t o_bytes, ml_bytes;
};

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

Plan plan_attend(const squat_paged_store* s, int n_seqs, int64_t n_new, int q_per_kv, int pages_per_seq, int64_t max_new, int64_t max_kv) {
    Plan a;
    const int64_t room = static_cast<int64_t>(pages_per_seq) * s->page_tokens;
    if (max_new < 1 || max_new > n_new) max_new = n_new;
    if (max_kv < 1 || max_kv > room) max_kv = room;
    a.nq = max_new * q_per_kv <= 16 ? 1 : 2;
    const int64_t rows = 16 * a.nq;
    a.tiles = n_new * q_per_kv / rows + n_seqs;
    // tiles with work: what the hints allow
    int64_t busy = n_seqs * ((max_new * q_per_kv + rows - 1) / rows);
    busy = (busy < a.tiles ? busy : a.tiles) * s->n_kv_heads;
    a.least = 4;
    const int64_t wanted = (4 * device_cu_count() + busy - 1) / busy;
    const int64_t most = (max_kv + kStep * a.least - 1) / (kStep * a.least);
    int64_t n = wanted < most ? wanted : most;
    n = n > 256 ? 256 : n;
    a.splits = n < 1 ? 1 : static_cast<int>(n);
    const size_t all = a.splits > 1 ? static_cast<size_t>(a.splits) * a.tiles * s->n_kv_heads * rows : 0;
    a.o_bytes = up256(all * kD * sizeof(float));
    a.ml_bytes = up256(all * sizeof(float2));
    return a;
}

// What the workspace query and the call itself ask of the sizes.
int check_sizes(const squat_paged_store* s, int n_seqs, int64_t n_new, int q_per_kv, int pages_per_seq) {
    if (q_per_kv < 1 || q_per_kv > 16 || n_seqs < 0 || n_new < 0 || pages_per_seq < 0) return SQUAT_E_BADSHAPE;
    if (n_new * q_per_kv > 0x3FFFFFFF) return SQUAT_E_BADSHAPE;
    if (static_cast<int64_t>(pages_per_seq) * s->page_tokens > 0x3FFFFFFF) return SQUAT_E_BADSHAPE;
    if ((n_new * q_per_kv / 16 + n_seqs) * s->n_kv_heads > 0x7FFFFFFF) return SQUAT_E_BADSHAPE;
    return SQUAT_OK;
}

template <int BITS, int NG, int NQ>
void launch_rows(squat_dtype dt, dim3 grid, hipStream_t s, const AttendParams& p) {
    if (dt == SQUAT_F16) hipLaunchKernelGGL((attend_kernel<BITS, NG, NQ, SQUAT_F16>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attend_kernel<BITS, NG, NQ, SQUAT_BF16>), grid, dim3(256), 0, s, p);
}
template <int BITS, int NG>
void launch_groups(int nq, squat_dtype dt, dim3 grid, hipStream_t s, const AttendParams& p) {
    if (nq == 1) launch_rows<BITS, NG, 1>(dt, grid, s, p);
    else launch_rows<BITS, NG, 2>(dt, grid, s, p);
}
template <int BITS>
void launch_bits(int group, int nq, squat_dtype dt, dim3 grid, hipStream_t s, const AttendParams& p) {
    switch (group) {
        case 32: launch_groups<BITS, 4>(nq, dt, grid, s, p); break;
        case 64: launch_groups<BITS, 2>(nq, dt, grid, s, p); break;
        default: launch_groups<BITS, 1>(nq, dt, grid, s, p); break;
    }
}
template <int R>
void launch_join(squat_dtype dt, dim3 grid, hipStream_t s, const AttendParams& p) {
    if (dt == SQUAT_F16) hipLaunchKernelGGL((attend_join_kernel<R, SQUAT_F16>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attend_join_kernel<R, SQUAT_BF16>), grid, dim3(256), 0, s, p);
}

}  // namespace

extern "C" size_t squat_paged_attention_workspace(const squat_paged_store* store, int n_seqs, int64_t n_new, int q_per_kv,
                                                  int pages_per_seq, int64_t max_new, int64_t max_kv) {
    if (check_store(store) || check_sizes(store, n_seqs, n_new, q_per_kv, pages_per_seq) || n_seqs == 0 || n_new == 0) return 0;
    const Plan a = plan_attend(store, n_seqs, n_new, q_per_kv, pages_per_seq, max_new, max_kv);
    return a.o_bytes + a.ml_bytes;
}

extern "C" int squat_paged_attention(const squat_paged_store* store, const void* q, squat_dtype q_dt, int64_t n_new, int q_per_kv,
                                     int64_t q_stride_token, int64_t q_stride_head, const int32_t* q_start, const int32_t* kv_len,
                                     const int32_t* pages, int64_t page_stride, int pages_per_seq, int n_seqs, int64_t max_new,
                                     int64_t max_kv, float out_scale, void* out, int64_t o_stride_token, int64_t o_stride_head,
                                     float* lse, void* ws, size_t ws_bytes, squat_stream stream) {
    int rc = check_store(store);
    if (rc) return rc;
    if (q_dt != SQUAT_F16 && q_dt != SQUAT_BF16) return SQUAT_E_BADDTYPE;
    rc = check_sizes(store, n_seqs, n_new, q_per_kv, pages_per_seq);
    if (rc) return rc;
    if (q_stride_token < kD || q_stride_head < kD || o_stride_token < kD || o_stride_head < kD || page_stride < pages_per_seq)
        return SQUAT_E_BADSHAPE;
    if ((q_stride_token % 8) || (q_stride_head % 8) || (o_stride_token % 8) || (o_stride_head % 8)) return SQUAT_E_ALIGN;
    if (out_scale != out_scale) return SQUAT_E_BADVALUE;
    if (n_new == 0 || n_seqs == 0) return SQUAT_OK;
    if (!q || !q_start || !kv_len || !out || (!pages && pages_per_seq > 0)) return SQUAT_E_NULLPTR;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(q_start, 4) || !aligned(kv_len, 4) || !aligned(pages, 4) || !aligned(lse, 4))
        return SQUAT_E_ALIGN;
    const Plan a = plan_attend(store, n_seqs, n_new, q_per_kv, pages_per_seq, max_new, max_kv);
    if (a.splits > 1) {
        if (!ws || ws_bytes < a.o_bytes + a.ml_bytes) return SQUAT_E_WORKSPACE;
        if (!aligned(ws, 256)) return SQUAT_E_ALIGN;
    }
    AttendParams p;
    p.kc = reinterpret_cast<const unsigned char*>(store->key_codes);
    p.km = reinterpret_cast<const unsigned char*>(store->key_meta);
    p.vc = reinterpret_cast<const unsigned char*>(store->value_codes);
    p.vm = reinterpret_cast<const unsigned char*>(store->value_meta);
    p.q = static_cast<const unsigned char*>(q);
    p.qst = q_stride_token;
    p.qsh = q_stride_head;
    p.out = static_cast<unsigned char*>(out);
    p.ost = o_stride_token;
    p.osh = o_stride_head;
    p.lse = lse;
    p.q_start = q_start;
    p.kv_len = kv_len;
    p.pages = pages;
    p.page_stride = page_stride;
    p.pages_per_seq = pages_per_seq;
    p.n_seqs = n_seqs;
    p.n_new = static_cast<int>(n_new);
    p.n_kv = store->n_kv_heads;
    p.qpk = q_per_kv;
    p.n_pages = static_cast<int>(store->n_pages);
    p.page_shift = 0;
    while ((1 << p.page_shift) < store->page_tokens) ++p.page_shift;
    p.scale = out_scale * kLog2e;
    p.splits = a.splits;
    p.least = a.least;
    p.n_tiles = static_cast<int>(a.tiles);
    p.part_o = static_cast<float*>(ws);
    p.part_ml = a.splits > 1 ? reinterpret_cast<float2*>(static_cast<unsigned char*>(ws) + a.o_bytes) : nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned gx = static_cast<unsigned>(a.tiles * store->n_kv_heads);
    const dim3 grid(gx, static_cast<unsigned>(a.splits));
    switch (store->bits) {
        case 2: launch_bits<2>(store->group, a.nq, q_dt, grid, s, p); break;
        case 4: launch_bits<4>(store->group, a.nq, q_dt, grid, s, p); break;
        default: launch_bits<8>(store->group, a.nq, q_dt, grid, s, p); break;
    }
    rc = check_launch();
    if (rc || a.splits == 1) return rc;
    if (a.nq == 1) launch_join<16>(q_dt, dim3(gx, 16), s, p);
    else launch_join<32>(q_dt, dim3(gx, 32), s, p);
    return check_launch();
}
