// squat_paged_write / squat_paged_read: tokens into and out of a store of pages (Section 2's quantizer, per token and group of
// channels; keys with an update matrix go through the kernel of squat_quantize_keys and are then dealt to their slots).
//
// Bound: HBM (a token-head in bf16 moves 512 bytes of keys and values and, 4 bits, groups of 32, 160 of store), for a few
// tokens the launch.  Eight lanes hold the 128 channels of a token-head, 16 each: a group's statistics are two or three lane
// exchanges, and a wavefront takes eight consecutive tokens of one head, whose rows lie next to each other in a page.
#include "squat_paged.h"
#include "squat_residual.h"

using namespace squat;

namespace {

constexpr int kTokens = 32;                               // tokens of one head per workgroup of 256 threads

struct PagedRows {
    uint32_t* codes[2];                                   // keys, values
    uint32_t* meta[2];                                    // (scale, zero-point) as one word
    int64_t n_slots;
    const int64_t* slots;
    int64_t n;
    int n_heads;
    int page_shift;
    int group;
    int first;                                            // blockIdx.z 0 is this one
};

// The row of (slot, head) in an array of pages, or -1.
__device__ __forceinline__ int64_t store_row(const PagedRows& p, int64_t t, int h) {
    const int64_t slot = p.slots[t];
    if (slot < 0 || slot >= p.n_slots) return -1;
    const int64_t page = slot >> p.page_shift;
    return (((page * p.n_heads + h) << p.page_shift)) + (slot & ((int64_t(1) << p.page_shift) - 1));
}

struct WriteParams {
    PagedRows rows;
    const unsigned char* x[2];
    int64_t st, sh;                                       // strides in BYTES
};

// A group's codes are decided as in 64 bits: u = (x - zero) / scale in fp32 is off by less than 2^-21 u, so only a value that lies
// closer than that to a rounding border (k + 1/2) needs the quotient itself; then the lane's channels are done again in fp64.
template <int BITS, int DT>
__global__ void __launch_bounds__(256) paged_write_kernel(const WriteParams p) {
    constexpr int ES = DT == SQUAT_F32 ? 4 : 2;
    constexpr int NW = BITS / 2;                          // words of a lane's 16 codes
    constexpr float TOP = static_cast<float>((1 << BITS) - 1);
    constexpr float NEAR = BITS == 8 ? 0.4998f : 0.49999f;
    const int part = static_cast<int>(threadIdx.x) & 7;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + (threadIdx.x >> 3);
    if (t >= p.rows.n) return;                            // the same for the eight lanes
    const int h = static_cast<int>(blockIdx.y);
    const int which = static_cast<int>(blockIdx.z) + p.rows.first;
    const unsigned char* src = p.x[which] + t * p.st + h * p.sh + part * (16 * ES);
    float x[16];
    load8<DT>(src, x);
    load8<DT>(src + 8 * ES, x + 8);
    const int64_t row = store_row(p.rows, t, h);
    float mn = x[0], mx = x[0], bad = 0.0f;               // bad: NaN if a channel is infinite or NaN
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        mn = fminf(mn, x[e]);
        mx = fmaxf(mx, x[e]);
        bad = fmaf(x[e], 0.0f, bad);
    }
    for (int o = 1; o < p.rows.group / 16; o <<= 1) {     // uniform
        mn = fminf(mn, __shfl_xor(mn, o, 64));
        mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        bad += __shfl_xor(bad, o, 64);
    }
    if (row < 0) return;
    const float step = static_cast<float>((static_cast<double>(mx) - static_cast<double>(mn)) / static_cast<double>(TOP));
    uint16_t sbits, zbits;
    const float s = round_f16(step + bad, sbits), z = round_f16(mn + bad, zbits);
    const bool live = s > 0.0f;
    const float inv = 1.0f / (live ? s : 1.0f);
    uint32_t words[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) words[w] = 0u;
    bool near = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float u = (x[e] - z) * inv, r = rintf(u);
        near |= fabsf(u - r) > NEAR;
        const uint32_t c = live ? static_cast<uint32_t>(fminf(fmaxf(r, 0.0f), TOP)) : 0u;
        words[e * BITS / 32] |= c << (e * BITS % 32);
    }
    if (near && live) {
#pragma unroll
        for (int w = 0; w < NW; ++w) words[w] = 0u;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const double r = rint((static_cast<double>(x[e]) - static_cast<double>(z)) / static_cast<double>(s));
            const uint32_t c = static_cast<uint32_t>(fmin(fmax(r, 0.0), static_cast<double>(TOP)));
            words[e * BITS / 32] |= c << (e * BITS % 32);
        }
    }
    uint32_t* out = p.rows.codes[which] + row * (kD * BITS / 32) + part * NW;
    if constexpr (NW == 1) out[0] = words[0];
    else if constexpr (NW == 2) *reinterpret_cast<u32x2*>(out) = u32x2{words[0], words[1]};
    else *reinterpret_cast<u32x4*>(out) = u32x4{words[0], words[1], words[2], words[3]};
    if ((part * 16) % p.rows.group == 0)
        p.rows.meta[which][row * (kD / p.rows.group) + part * 16 / p.rows.group] = sbits | (static_cast<uint32_t>(zbits) << 16);
}

// Rows that squat_quantize_keys' kernel wrote densely, [heads, n, ...], to their slots: eight lanes a row.
struct DealParams {
    PagedRows rows;
    const uint32_t* codes;
    const uint16_t *scale, *zero;
};

template <int BITS>
__global__ void __launch_bounds__(256) paged_deal_kernel(const DealParams p) {
    constexpr int NW = BITS / 2;
    const int part = static_cast<int>(threadIdx.x) & 7;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + (threadIdx.x >> 3);
    if (t >= p.rows.n) return;
    const int h = static_cast<int>(blockIdx.y);
    const int64_t row = store_row(p.rows, t, h);
    if (row < 0) return;
    const int64_t from = h * p.rows.n + t;
#pragma unroll
    for (int w = 0; w < NW; ++w)
        p.rows.codes[0][row * (kD * BITS / 32) + part * NW + w] = p.codes[from * (kD * BITS / 32) + part * NW + w];
    const int ng = kD / p.rows.group;
    if (part < ng) p.rows.meta[0][row * ng + part] = p.scale[from * ng + part] | (static_cast<uint32_t>(p.zero[from * ng + part]) << 16);
}

struct ReadParams {
    PagedRows rows;
    unsigned char* x[2];
    int64_t st, sh;                                       // strides in BYTES
};

// 16 values of one lane, rounded once
template <int DT>
__device__ __forceinline__ void store16(unsigned char* to, const float (&x)[16]) {
    if constexpr (DT == SQUAT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(to + 16 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    } else if constexpr (DT == SQUAT_F16) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            half8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = static_cast<_Float16>(x[8 * i + e]);
            *reinterpret_cast<half8*>(to + 16 * i) = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            bf16x8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(x[8 * i + e]);
            *reinterpret_cast<bf16x8*>(to + 16 * i) = v;
        }
    }
}

template <int BITS, int DT>
__global__ void __launch_bounds__(256) paged_read_kernel(const ReadParams p) {
    constexpr int ES = DT == SQUAT_F32 ? 4 : 2;
    constexpr int NW = BITS / 2;
    const int part = static_cast<int>(threadIdx.x) & 7;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + (threadIdx.x >> 3);
    if (t >= p.rows.n) return;
    const int h = static_cast<int>(blockIdx.y);
    const int which = static_cast<int>(blockIdx.z) + p.rows.first;
    const int64_t row = store_row(p.rows, t, h);
    float x[16];
    if (row < 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.0f;
    } else {
        const uint32_t* from = p.rows.codes[which] + row * (kD * BITS / 32) + part * NW;
        uint32_t words[4];
        if constexpr (NW == 1) {
            words[0] = from[0];
        } else if constexpr (NW == 2) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(from);
            words[0] = v[0];
            words[1] = v[1];
        } else {
            const u32x4 v = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) words[i] = v[i];
        }
        const uint32_t m = p.rows.meta[which][row * (kD / p.rows.group) + part * 16 / p.rows.group];
        const float s = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(m & 0xFFFFu)));
        const float z = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(m >> 16)));
#pragma unroll
        for (int e = 0; e < 16; ++e)
            x[e] = fmaf(static_cast<float>((words[e * BITS / 32] >> (e * BITS % 32)) & ((1u << BITS) - 1u)), s, z);
    }
    store16<DT>(p.x[which] + t * p.st + h * p.sh + part * (16 * ES), x);
}

int page_shift(int page_tokens) {
    int s = 0;
    while ((1 << s) < page_tokens) ++s;
    return s;
}

PagedRows rows_of(const squat_paged_store* s, const int64_t* slots, int64_t n) {
    PagedRows r;
    r.codes[0] = s->key_codes;
    r.codes[1] = s->value_codes;
    r.meta[0] = reinterpret_cast<uint32_t*>(s->key_meta);
    r.meta[1] = reinterpret_cast<uint32_t*>(s->value_meta);
    r.n_slots = s->n_pages * s->page_tokens;
    r.slots = slots;
    r.n = n;
    r.n_heads = s->n_kv_heads;
    r.page_shift = page_shift(s->page_tokens);
    r.group = s->group;
    r.first = 0;
    return r;
}

// What both directions ask of the tokens' tensors.
int check_tokens(const squat_paged_store* s, squat_dtype dt, int64_t n, int64_t st, int64_t sh) {
    if (elem_size(dt) == 0) return SQUAT_E_BADDTYPE;
    if (n < 0 || (n + kTokens - 1) / kTokens > 0x7FFFFFFF) return SQUAT_E_BADSHAPE;
    if (st < kD || (sh < kD && s->n_kv_heads > 1) || sh < 0) return SQUAT_E_BADSHAPE;
    if ((st % 8) || (sh % 8)) return SQUAT_E_ALIGN;
    return SQUAT_OK;
}

template <int BITS>
void launch_write(squat_dtype dt, dim3 grid, hipStream_t s, const WriteParams& p) {
    switch (dt) {
        case SQUAT_F32: hipLaunchKernelGGL((paged_write_kernel<BITS, SQUAT_F32>), grid, dim3(256), 0, s, p); break;
        case SQUAT_F16: hipLaunchKernelGGL((paged_write_kernel<BITS, SQUAT_F16>), grid, dim3(256), 0, s, p); break;
        case SQUAT_BF16: hipLaunchKernelGGL((paged_write_kernel<BITS, SQUAT_BF16>), grid, dim3(256), 0, s, p); break;
    }
}

template <int BITS>
void launch_read(squat_dtype dt, dim3 grid, hipStream_t s, const ReadParams& p) {
    switch (dt) {
        case SQUAT_F32: hipLaunchKernelGGL((paged_read_kernel<BITS, SQUAT_F32>), grid, dim3(256), 0, s, p); break;
        case SQUAT_F16: hipLaunchKernelGGL((paged_read_kernel<BITS, SQUAT_F16>), grid, dim3(256), 0, s, p); break;
        case SQUAT_BF16: hipLaunchKernelGGL((paged_read_kernel<BITS, SQUAT_BF16>), grid, dim3(256), 0, s, p); break;
    }
}

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

}  // namespace

extern "C" size_t squat_paged_write_workspace(const squat_paged_store* s, int64_t n_tokens, int has_update) {
    if (check_store(s) || n_tokens < 0 || !has_update || s->bits == 8) return 0;
    const size_t rows = static_cast<size_t>(n_tokens) * s->n_kv_heads;
    return up256(rows * (kD * s->bits / 8)) + 2 * up256(rows * (kD / s->group) * 2);
}

extern "C" int squat_paged_write(const squat_paged_store* store, const void* k, const void* v, squat_dtype dt, int64_t n_tokens,
                                 int64_t stride_token, int64_t stride_head, const int64_t* slots, const float* update, int g,
                                 void* ws, size_t ws_bytes, squat_stream stream) {
    int rc = check_store(store);
    if (rc) return rc;
    rc = check_tokens(store, dt, n_tokens, stride_token, stride_head);
    if (rc) return rc;
    if (update && store->bits == 8) return SQUAT_E_BADSHAPE;
    if (n_tokens == 0) return SQUAT_OK;
    if (!k || !v || !slots) return SQUAT_E_NULLPTR;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return SQUAT_E_ALIGN;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int es = elem_size(dt);
    WriteParams p;
    p.rows = rows_of(store, slots, n_tokens);
    p.x[0] = static_cast<const unsigned char*>(k);
    p.x[1] = static_cast<const unsigned char*>(v);
    p.st = stride_token * es;
    p.sh = stride_head * es;
    dim3 grid(static_cast<unsigned>((n_tokens + kTokens - 1) / kTokens), static_cast<unsigned>(store->n_kv_heads), 2);
    if (update) {
        // the keys: densely into the workspace, then to their slots
        const size_t need = squat_paged_write_workspace(store, n_tokens, 1);
        if (!ws || ws_bytes < need) return SQUAT_E_WORKSPACE;
        if (!aligned(ws, 256)) return SQUAT_E_ALIGN;
        const size_t rows = static_cast<size_t>(n_tokens) * store->n_kv_heads;
        unsigned char* at = static_cast<unsigned char*>(ws);
        DealParams d;
        d.rows = p.rows;
        uint32_t* codes = reinterpret_cast<uint32_t*>(at);
        at += up256(rows * (kD * store->bits / 8));
        uint16_t* scale = reinterpret_cast<uint16_t*>(at);
        uint16_t* zero = reinterpret_cast<uint16_t*>(at + up256(rows * (kD / store->group) * 2));
        d.codes = codes;
        d.scale = scale;
        d.zero = zero;
        rc = quantize_keys_into(k, dt, 1, store->n_kv_heads, n_tokens, kD, 0, stride_head, stride_token, update, 0, store->bits,
                                store->group, g, codes, scale, zero, n_tokens, 0, stream);
        if (rc) return rc;
        grid.z = 1;
        if (store->bits == 2) hipLaunchKernelGGL((paged_deal_kernel<2>), grid, dim3(256), 0, s, d);
        else hipLaunchKernelGGL((paged_deal_kernel<4>), grid, dim3(256), 0, s, d);
        rc = check_launch();
        if (rc) return rc;
        p.rows.first = 1;
    }
    switch (store->bits) {
        case 2: launch_write<2>(dt, grid, s, p); break;
        case 4: launch_write<4>(dt, grid, s, p); break;
        default: launch_write<8>(dt, grid, s, p); break;
    }
    return check_launch();
}

extern "C" int squat_paged_read(const squat_paged_store* store, const int64_t* slots, int64_t n_tokens, void* k_out, void* v_out,
                                squat_dtype out_dt, int64_t stride_token, int64_t stride_head, squat_stream stream) {
    int rc = check_store(store);
    if (rc) return rc;
    rc = check_tokens(store, out_dt, n_tokens, stride_token, stride_head);
    if (rc) return rc;
    if (n_tokens == 0 || (!k_out && !v_out)) return SQUAT_OK;
    if (!slots) return SQUAT_E_NULLPTR;
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(slots, 8)) return SQUAT_E_ALIGN;
    const int es = elem_size(out_dt);
    ReadParams p;
    p.rows = rows_of(store, slots, n_tokens);
    p.rows.first = k_out ? 0 : 1;
    p.x[0] = static_cast<unsigned char*>(k_out);
    p.x[1] = static_cast<unsigned char*>(v_out);
    p.st = stride_token * es;
    p.sh = stride_head * es;
    const dim3 grid(static_cast<unsigned>((n_tokens + kTokens - 1) / kTokens), static_cast<unsigned>(store->n_kv_heads),
                    k_out && v_out ? 2 : 1);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (store->bits) {
        case 2: launch_read<2>(out_dt, grid, s, p); break;
        case 4: launch_read<4>(out_dt, grid, s, p); break;
        default: launch_read<8>(out_dt, grid, s, p); break;
    }
    return check_launch();
}
