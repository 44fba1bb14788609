// squat_verify_drafts: which drafted tokens stand, and the token that follows them.
//
// Bound: HBM for a batch (two rows of the vocabulary per sequence: the target's and the draft's at the first refusal), the launches
// for one sequence.  The first kernel's workgroups each find the refusal on their own (a handful of numbers) and sum one piece of
// kPiece entries of the row that the next token comes from; the second kernel goes through a sequence's sums, finds the piece
// that holds the mark and searches it.  Sums are made in fp64 and in a fixed order: the same call gives the same token, and
// the order of a sum matters only where two tokens' borders are 1e-16 of the row apart.
#include "squat_internal.h"

using namespace squat;

namespace {

constexpr int kPiece = 4096;                              // entries per workgroup of the first kernel
constexpr int kThreads = 256;

struct VerifyParams {
    const int64_t* tokens;
    int n_seqs, n_drafts, vocab;
    const unsigned char *target, *draft;
    int64_t tss, tsp, dss, dsp;                           // elements
    const float *u, *u_next;
    const int32_t* n_draft;
    int32_t* accepted;
    int64_t* out;
    double2* sums;                                        // [n_seqs, pieces]: of the residual, of the target's row
    int pieces;
};

template <int DT>
__device__ __forceinline__ float entry(const unsigned char* p, int64_t i) {
    if constexpr (DT == SQUAT_F32) return *reinterpret_cast<const float*>(p + 4 * i);
    const uint16_t h = *reinterpret_cast<const uint16_t*>(p + 2 * i);
    return DT == SQUAT_BF16 ? as_f32(static_cast<uint32_t>(h) << 16) : static_cast<float>(__builtin_bit_cast(_Float16, h));
}

// A lane's neighbouring entries, 16 bytes of them wherever the row begins (an odd vocabulary's rows are off every boundary); 0 behind
// the row's end.
template <int DT>
constexpr int kPer = DT == SQUAT_F32 ? 4 : 8;

template <int DT>
__device__ __forceinline__ void entries(const unsigned char* row, int i, int n, float (&x)[kPer<DT>]) {
    if (i + kPer<DT> <= n) {
        if constexpr (DT == SQUAT_F32) {
            const u32x4 v = *reinterpret_cast<const u32x4_dwords*>(row + static_cast<int64_t>(i) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = as_f32(v[e]);
        } else {
            const u32x4 v = *reinterpret_cast<const u32x4_halves*>(row + static_cast<int64_t>(i) * 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t h = (e & 1) ? (v[e >> 1] >> 16) : (v[e >> 1] & 0xFFFFu);
                x[e] = DT == SQUAT_BF16 ? as_f32(h << 16) : static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(h)));
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < kPer<DT>; ++e) x[e] = i + e < n ? entry<DT>(row, i + e) : 0.0f;
    }
}

// How a sequence's drafts end: `accepted` of them, and the rows that the next token comes from (draft: NULL where p itself is meant).
struct Verdict {
    int accepted, limit;
    const unsigned char *p, *q;
    int64_t taken;                                        // the draft chosen outright that was refused, or -1
};

template <int DT>
__device__ __forceinline__ Verdict decide(const VerifyParams& p, int s) {
    constexpr int ES = DT == SQUAT_F32 ? 4 : 2;
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const int n = p.n_draft ? min(max(p.n_draft[s], 0), p.n_drafts) : p.n_drafts;
    bool refused = lane >= n;
    if (!refused) {
        const int64_t x = p.tokens[static_cast<int64_t>(s) * p.n_drafts + lane];
        const double u = p.u[static_cast<int64_t>(s) * p.n_drafts + lane];
        double px = 0.0, qx = 1.0;
        if (x >= 0 && x < p.vocab) {
            px = entry<DT>(p.target + (s * p.tss + lane * p.tsp) * ES, x);
            if (p.draft) qx = entry<DT>(p.draft + (s * p.dss + lane * p.dsp) * ES, x);
        }
        refused = !(u * qx < px);
    }
    const uint64_t m = __ballot(refused);
    Verdict v;
    v.limit = n;
    v.accepted = m ? min(__builtin_ctzll(m), n) : n;      // (64 drafts, all accepted: no lane is left to say so)
    v.p = p.target + (s * p.tss + v.accepted * p.tsp) * ES;
    v.q = v.accepted < n && p.draft ? p.draft + (s * p.dss + v.accepted * p.dsp) * ES : nullptr;
    v.taken = v.accepted < n && !p.draft ? p.tokens[static_cast<int64_t>(s) * p.n_drafts + v.accepted] : -1;
    return v;
}

// What a lane's entries of the row weigh in the draw of the next token.
template <int DT>
__device__ __forceinline__ void weights(const Verdict& v, int i, int n, double (&r)[kPer<DT>], double (&t)[kPer<DT>]) {
    float a[kPer<DT>], b[kPer<DT>];
    entries<DT>(v.p, i, n, a);
    if (v.q) entries<DT>(v.q, i, n, b);
#pragma unroll
    for (int e = 0; e < kPer<DT>; ++e) {
        t[e] = a[e];
        r[e] = v.q ? fmax(static_cast<double>(a[e]) - static_cast<double>(b[e]), 0.0) : (i + e == v.taken ? 0.0 : static_cast<double>(a[e]));
    }
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

template <int DT>
__global__ void __launch_bounds__(kThreads) verify_sums_kernel(const VerifyParams p) {
    __shared__ double2 part[kThreads / 64];
    const int s = static_cast<int>(blockIdx.y);
    const Verdict v = decide<DT>(p, s);
    double r = 0.0, t = 0.0;
#pragma unroll
    for (int k = 0; k < kPiece / (kThreads * kPer<DT>); ++k) {
        const int64_t i = static_cast<int64_t>(blockIdx.x) * kPiece + (k * kThreads + static_cast<int>(threadIdx.x)) * kPer<DT>;
        if (i >= p.vocab) break;
        double re[kPer<DT>], te[kPer<DT>];
        weights<DT>(v, static_cast<int>(i), p.vocab, re, te);
#pragma unroll
        for (int e = 0; e < kPer<DT>; ++e) {
            r += re[e];
            t += te[e];
        }
    }
    r = wave_sum(r);
    t = wave_sum(t);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = double2{r, t};
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w) {
            r += part[w].x;
            t += part[w].y;
        }
        p.sums[static_cast<int64_t>(s) * p.pieces + blockIdx.x] = double2{r, t};
    }
}

// The running sum up to and including the thread's x, over the workgroup's threads in order; `all`: over all of them.
__device__ __forceinline__ double block_scan(double x, double (&lds)[kThreads / 64], double& all) {
    const int lane = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();                                      // (the last round's readers are through)
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    double before = 0.0;
    all = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    return before + x;
}

template <int DT>
__global__ void __launch_bounds__(kThreads) verify_pick_kernel(const VerifyParams p) {
    __shared__ double lds[kThreads / 64];
    __shared__ int found, fallback;
    __shared__ double before_found;
    const int s = static_cast<int>(blockIdx.x), tid = static_cast<int>(threadIdx.x);
    Verdict v = decide<DT>(p, s);
    const double2* sums = p.sums + static_cast<int64_t>(s) * p.pieces;
    double total = 0.0, total_p = 0.0, all;
    for (int c = 0; c < p.pieces; c += kThreads) {        // uniform
        const double2 x = c + tid < p.pieces ? sums[c + tid] : double2{0.0, 0.0};
        (void)block_scan(x.x, lds, all);
        total += all;
        (void)block_scan(x.y, lds, all);
        total_p += all;
    }
    const bool plain = !(total > 0.0);                    // nothing is left of the residual: the target's own row
    if (plain) {
        total = total_p;
        v.q = nullptr;
        v.taken = -1;
    }
    const double mark = static_cast<double>(p.u_next[s]) * total;
    // the piece that holds the mark: the first whose running sum is over it
    if (tid == 0) {
        found = 0x7FFFFFFF;
        fallback = 0;
        before_found = 0.0;
    }
    double before = 0.0;
    for (int c = 0; c < p.pieces; c += kThreads) {        // uniform
        const double2 x = c + tid < p.pieces ? sums[c + tid] : double2{0.0, 0.0};
        const double mine = plain ? x.y : x.x, upto = before + block_scan(mine, lds, all);
        if (c + tid < p.pieces && upto > mark) atomicMin(&found, c + tid);
        if (mine > 0.0) atomicMax(&fallback, c + tid);
        __syncthreads();
        if (found < 0x7FFFFFFF) {                         // uniform: everybody is past the barrier
            if (found == c + tid) before_found = upto - mine;
            break;
        }
        before += all;
    }
    __syncthreads();
    const bool any = found < 0x7FFFFFFF;
    const int piece = any ? found : fallback;             // (a mark that rounding put on the very end: the last entry that counts)
    before = any ? before_found : -INFINITY;
    __syncthreads();
    if (tid == 0) {
        found = 0x7FFFFFFF;
        fallback = 0;
    }
    __syncthreads();
    int first = 0x7FFFFFFF, last = 0;                     // the thread's first entry over the mark, and its last that counts
    for (int k = 0; k < kPiece / (kThreads * kPer<DT>); ++k) {
        const int64_t i = static_cast<int64_t>(piece) * kPiece + (k * kThreads + tid) * kPer<DT>;
        double r[kPer<DT>], t[kPer<DT>], sum = 0.0;
        if (i < p.vocab) {
            weights<DT>(v, static_cast<int>(i), p.vocab, r, t);
        } else {
#pragma unroll
            for (int e = 0; e < kPer<DT>; ++e) r[e] = 0.0;
        }
#pragma unroll
        for (int e = 0; e < kPer<DT>; ++e) sum += r[e];
        double run = before + (block_scan(sum, lds, all) - sum);
#pragma unroll
        for (int e = 0; e < kPer<DT>; ++e) {
            run += r[e];
            if (r[e] > 0.0) {
                last = static_cast<int>(i) + e;
                if (run > mark) first = min(first, last);
            }
        }
        before += all;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        first = min(first, __shfl_xor(first, o, 64));
        last = max(last, __shfl_xor(last, o, 64));
    }
    if ((tid & 63) == 0) {
        atomicMin(&found, first);
        atomicMax(&fallback, last);
    }
    __syncthreads();
    const int picked = found < 0x7FFFFFFF ? found : fallback;
    if (tid <= p.n_drafts) {
        const int64_t x = tid < v.accepted ? p.tokens[static_cast<int64_t>(s) * p.n_drafts + tid] : (tid == v.accepted ? picked : -1);
        p.out[static_cast<int64_t>(s) * (p.n_drafts + 1) + tid] = x;
    }
    if (tid == 0) p.accepted[s] = v.accepted;
}

template <int DT>
int launch_verify(hipStream_t s, const VerifyParams& p) {
    hipLaunchKernelGGL((verify_sums_kernel<DT>), dim3(static_cast<unsigned>(p.pieces), static_cast<unsigned>(p.n_seqs)), dim3(kThreads), 0, s, p);
    const int rc = check_launch();
    if (rc) return rc;
    hipLaunchKernelGGL((verify_pick_kernel<DT>), dim3(static_cast<unsigned>(p.n_seqs)), dim3(kThreads), 0, s, p);
    return check_launch();
}

bool sizes_ok(int n_seqs, int64_t vocab) { return n_seqs >= 0 && n_seqs <= 65535 && vocab >= 1 && vocab <= 0x7FFFFFFF - kPiece; }

}  // namespace

extern "C" size_t squat_verify_drafts_workspace(int n_seqs, int64_t vocab) {
    if (!sizes_ok(n_seqs, vocab)) return 0;
    return static_cast<size_t>(n_seqs) * ((vocab + kPiece - 1) / kPiece) * sizeof(double2);
}

extern "C" int squat_verify_drafts(const int64_t* tokens, int n_seqs, int n_drafts, int64_t vocab, const void* target,
                                   int64_t t_stride_seq, int64_t t_stride_pos, const void* draft, int64_t d_stride_seq,
                                   int64_t d_stride_pos, squat_dtype dt, const float* u, const float* u_next,
                                   const int32_t* n_draft, int32_t* accepted, int64_t* out, void* ws, size_t ws_bytes,
                                   squat_stream stream) {
    if (!sizes_ok(n_seqs, vocab) || n_drafts < 0 || n_drafts > 64) return SQUAT_E_BADSHAPE;
    const int es = elem_size(dt);
    if (es == 0) return SQUAT_E_BADDTYPE;
    if (t_stride_seq < 0 || t_stride_pos < 0 || d_stride_seq < 0 || d_stride_pos < 0) return SQUAT_E_BADSHAPE;
    if (n_seqs == 0) return SQUAT_OK;
    if (!target || !u_next || !accepted || !out || (n_drafts > 0 && (!tokens || !u))) return SQUAT_E_NULLPTR;
    if (!aligned(target, es) || !aligned(draft, es) || !aligned(tokens, 8) || !aligned(out, 8) || !aligned(u, 4) || !aligned(u_next, 4) ||
        !aligned(n_draft, 4) || !aligned(accepted, 4))
        return SQUAT_E_ALIGN;
    if (!ws || ws_bytes < squat_verify_drafts_workspace(n_seqs, vocab)) return SQUAT_E_WORKSPACE;
    if (!aligned(ws, 256)) return SQUAT_E_ALIGN;
    VerifyParams p;
    p.tokens = tokens;
    p.n_seqs = n_seqs;
    p.n_drafts = n_drafts;
    p.vocab = static_cast<int>(vocab);
    p.target = static_cast<const unsigned char*>(target);
    p.draft = static_cast<const unsigned char*>(draft);
    p.tss = t_stride_seq;
    p.tsp = t_stride_pos;
    p.dss = d_stride_seq;
    p.dsp = d_stride_pos;
    p.u = u;
    p.u_next = u_next;
    p.n_draft = n_draft;
    p.accepted = accepted;
    p.out = out;
    p.sums = static_cast<double2*>(ws);
    p.pieces = static_cast<int>((vocab + kPiece - 1) / kPiece);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (dt) {
        case SQUAT_F32: return launch_verify<SQUAT_F32>(s, p);
        case SQUAT_F16: return launch_verify<SQUAT_F16>(s, p);
        case SQUAT_BF16: return launch_verify<SQUAT_BF16>(s, p);
    }
    return SQUAT_E_BADDTYPE;
}
