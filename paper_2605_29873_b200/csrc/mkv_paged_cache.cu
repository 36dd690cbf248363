// Writing the paged cache (with the rotation of keys and queries on the way) and reading its rows
// back as values.  Elementwise work: bound by memory for prompts, by the latency of a launch and
// three dependent loads (starts, lens, table) for single tokens.
#include "mkv_paged.cuh"

namespace mkv {
namespace {

constexpr int kAppendThreads = 256;

template <typename T> struct Vec8;   // eight channels
template <> struct Vec8<__nv_bfloat16> {
    static __device__ void load(const void* p, float (&x)[8]) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
    static __device__ void store(void* p, const float (&x)[8]) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <> struct Vec8<float> {
    static __device__ void load(const void* p, float (&x)[8]) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    static __device__ void store(void* p, const float (&x)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
};

struct TokenPlace {
    uint8_t* page;   // nullptr: the token is not stored
    int row;         // in its page
    int rot_pos;
    int skip;        // belongs to no sequence, or has no place: nothing is written for it
};

// Finds the sequence of token i and the place of the token in the cache.
__device__ TokenPlace token_place(const PagedAppendArgs& a, int i) {
    TokenPlace t;
    t.page = nullptr; t.row = 0; t.rot_pos = 0; t.skip = 1;
    int s = i;
    if (a.b.starts) {
        // last s with starts[s] <= i
        int lo = 0, hi = a.b.batch;
        if (a.b.starts[0] > i || a.b.starts[a.b.batch] <= i) return t;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.b.starts[mid] <= i) lo = mid; else hi = mid;
        }
        s = lo;
    }
    const PagedSpan sp = paged_span(a.c, a.b, s);
    const int j = i - sp.tok0;
    if (j < 0 || j >= sp.n) return t;
    // the length as given: a sequence that has outgrown its table keeps its other tokens' places
    const int pos = max(a.b.lens[s], 0) - sp.n + j;
    if (pos < 0) return t;
    t.skip = 0;
    t.rot_pos = a.positions ? a.positions[i] : pos;
    if ((pos >> a.c.page_shift) >= a.b.table_stride) return t;   // reported by paged_span
    const int page = a.b.table[(size_t)s * a.b.table_stride + (pos >> a.c.page_shift)];
    if ((unsigned)page >= (unsigned)a.c.n_pages) { paged_fail(a.c, MKV_ERR_INVALID_ARG); return t; }
    t.page = a.c.pages + (size_t)page * a.c.page_bytes;
    t.row = pos & ((1 << a.c.page_shift) - 1);
    return t;
}

// cos and sin of pos * inv_freq.  The product and its reduction to a fraction of a turn are in 64
// bits: at position 10^6 an fp32 angle would be off by 0.06.
__device__ inline double turn_fraction(int pos, float inv_freq) {
    const double turns = (double)pos * (double)inv_freq * 0.15915494309189533577;
    return 2.0 * (turns - rint(turns));
}

// One quantised piece: the four channels 4 * l .. 4 * l + 3 of a head, lanes of eight sharing a
// group.  In 64 bits up to the code, so that a value next to a border between two codes goes where
// the definition sends it.
struct Coded { uint32_t codes16; uint16_t scale, lowest; };
__device__ inline Coded quantise4(const double (&x)[4]) {
    double lo = fmin(fmin(x[0], x[1]), fmin(x[2], x[3])), hi = fmax(fmax(x[0], x[1]), fmax(x[2], x[3]));
    // fmin / fmax pass over a NaN, so finiteness is looked at apart
    int fine = isfinite(x[0]) && isfinite(x[1]) && isfinite(x[2]) && isfinite(x[3]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        lo = fmin(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmax(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        fine &= __shfl_xor_sync(0xffffffffu, fine, o);
    }
    Coded r;
    r.codes16 = 0;
    if (!fine) { r.scale = 0x7fc0; r.lowest = 0; return r; }
    const __nv_bfloat16 sb = __float2bfloat16_rn((float)(hi / 15.0 - lo / 15.0)), lb = __float2bfloat16_rn((float)lo);
    r.scale = __bfloat16_as_ushort(sb);
    r.lowest = __bfloat16_as_ushort(lb);
    const double s = (double)__bfloat162float(sb), l = (double)__bfloat162float(lb);
    if (s > 0.0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double n = fmin(15.0, fmax(0.0, rint((x[i] - l) / s)));
            r.codes16 |= (uint32_t)n << (4 * i);
        }
    }
    return r;
}

// TT tokens per CTA.  KIND: the cache's mkv_dtype.
template <typename T, int KIND, int D, int TT>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(const PagedAppendArgs a) {
    __shared__ TokenPlace place[TT];
    __shared__ float2 cs[TT][D / 2];
    __shared__ double2 csd[KIND == MKV_INT4 ? TT : 1][KIND == MKV_INT4 ? D / 2 : 1];
    const int tid = threadIdx.x, tok0 = blockIdx.x * TT;
    if (tid < TT && tok0 + tid < a.b.n_tokens) place[tid] = token_place(a, tok0 + tid);
    else if (tid < TT) place[tid].skip = 1;
    __syncthreads();
    const int half = a.rot_dim >> 1;
    for (int i = tid; i < TT * half; i += kAppendThreads) {
        const int t = i / half, f = i - t * half;
        if (place[t].skip) continue;
        const double x = turn_fraction(place[t].rot_pos, a.inv_freq[f]);
        if (KIND == MKV_INT4) {
            double sd, cd;
            sincospi(x, &sd, &cd);
            csd[t][f] = make_double2(cd, sd);
            cs[t][f] = make_float2((float)cd, (float)sd);
        } else {
            float sf, cf;
            sincospif((float)x, &sf, &cf);
            cs[t][f] = make_float2(cf, sf);
        }
    }
    __syncthreads();

    // q, and k and v of the 16- and 32-bit caches: items of two eight-channel chunks.  Halves
    // paired: chunk i with chunk i + half / 8.  Neighbours paired, or not rotated: two in a row.
    constexpr int kItems = D / 16;
    const int nq = a.q ? a.c.q_heads : 0, nkv = KIND == MKV_INT4 ? 0 : a.c.kv_heads;
    const int per_tok = (nq + 2 * nkv) * kItems;
    for (int i = tid; i < TT * per_tok; i += kAppendThreads) {
        const int t = i / per_tok, r = i - t * per_tok;
        if (place[t].skip) continue;
        const int h = r / kItems, it = r - h * kItems;
        const bool is_v = h >= nq + nkv, is_k = !is_v && h >= nq;
        if ((is_v || is_k) && !place[t].page) continue;
        const size_t tok = (size_t)(tok0 + t);
        const T* src = is_v   ? (const T*)a.v + tok * a.v_stride + (size_t)(h - nq - nkv) * D
                       : is_k ? (const T*)a.k + tok * a.k_stride + (size_t)(h - nq) * D
                              : (const T*)a.q + tok * a.q_stride + (size_t)h * D;
        uint8_t* dst8 = is_v   ? place[t].page + a.c.kv_bytes + (size_t)(h - nq - nkv) * a.c.head_bytes
                        : is_k ? place[t].page + (size_t)(h - nq) * a.c.head_bytes
                               : (uint8_t*)a.q_out + (tok * a.c.q_heads + h) * (size_t)D * sizeof(T);
        T* dst = (T*)dst8 + ((is_v || is_k) ? (size_t)place[t].row * D : 0);
        const bool turn = !is_v && it * 16 < a.rot_dim;
        int c0 = 16 * it, c1 = 16 * it + 8;
        if (turn && !a.interleaved) { c0 = 8 * it; c1 = 8 * it + half; }
        float x[8], y[8];
        Vec8<T>::load(src + c0, x);
        Vec8<T>::load(src + c1, y);
        if (turn) {
            const float2* w = cs[t] + 8 * it;
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 u = w[e], z = w[4 + e];
                    const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
                    x[2 * e] = x0 * u.x - x1 * u.y; x[2 * e + 1] = x1 * u.x + x0 * u.y;
                    y[2 * e] = y0 * z.x - y1 * z.y; y[2 * e + 1] = y1 * z.x + y0 * z.y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 u = w[e];
                    const float x0 = x[e], y0 = y[e];
                    x[e] = x0 * u.x - y0 * u.y; y[e] = y0 * u.x + x0 * u.y;
                }
            }
        }
        Vec8<T>::store(dst + c0, x);
        Vec8<T>::store(dst + c1, y);
    }

    if (KIND == MKV_INT4) {
        // a lane owns four channels of one head and token; D / 4 lanes make a head
        constexpr int kLanes = D / 4, NG = D / 32;
        const int per4 = 2 * a.c.kv_heads * kLanes;
        const int l = tid % kLanes;
        const int total = TT * per4;   // a multiple of 32: whole warps stay together in the shuffles
        for (int i = tid; i < (total + 31) / 32 * 32; i += kAppendThreads) {
            const int t = min(i / per4, TT - 1), r = i - t * per4;
            const int h = min(r / kLanes, 2 * a.c.kv_heads - 1);
            const bool is_v = h >= a.c.kv_heads, live = i < total && !place[t].skip && place[t].page;
            const int hk = is_v ? h - a.c.kv_heads : h;
            double x[4] = {0, 0, 0, 0};
            if (live) {
                const size_t tok = (size_t)(tok0 + t);
                const T* src = is_v ? (const T*)a.v + tok * a.v_stride + (size_t)hk * D
                                    : (const T*)a.k + tok * a.k_stride + (size_t)hk * D;
                const int c = 4 * l;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (double)(float)src[c + e];
                if (!is_v && c < a.rot_dim) {
                    if (a.interleaved) {
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const double2 w = csd[t][(c + e) >> 1];
                            const double x0 = x[e], x1 = x[e + 1];
                            x[e] = x0 * w.x - x1 * w.y; x[e + 1] = x1 * w.x + x0 * w.y;
                        }
                    } else {
                        const bool up = c >= half;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const double2 w = csd[t][up ? c + e - half : c + e];
                            const double o = (double)(float)src[up ? c + e - half : c + e + half];
                            x[e] = up ? x[e] * w.x + o * w.y : x[e] * w.x - o * w.y;
                        }
                    }
                }
            }
            const Coded z = quantise4(x);
            if (!live) continue;
            uint8_t* blk = place[t].page + (size_t)hk * a.c.head_bytes + (size_t)(place[t].row >> 4) * paged_block_bytes(D);
            const int row = place[t].row & 15, j = l >> 3, g = l & 7;
            uint8_t* codes = is_v ? blk + 8 * D + (row >> 1) * D + (g * NG + j) * 4 + (row & 1) * 2
                                  : blk + row * (D / 2) + ((g >> 1) * NG + j) * 4 + (g & 1) * 2;
            *reinterpret_cast<uint16_t*>(codes) = (uint16_t)z.codes16;
            if (g == 0) {
                uint8_t* par = blk + 16 * D + (is_v ? 64 * NG : 0);
                const int by_pair = ((row >> 1) * NG + j) * 4 + (row & 1) * 2;
                *reinterpret_cast<uint16_t*>(par + by_pair) = z.scale;
                *reinterpret_cast<uint16_t*>(par + 32 * NG + (is_v ? by_pair : (row * NG + j) * 2)) = z.lowest;
            }
        }
    }
}

// Rows [first, lens) of every sequence as values: out row i = the token at position first + i.
template <typename T, int KIND, int D>
__global__ void __launch_bounds__(kAppendThreads) paged_read_kernel(const PagedReadArgs a) {
    const int s = blockIdx.y, h = blockIdx.z;
    const PagedSpan sp = paged_span(a.c, a.b, s);
    int first = a.first ? a.first[s] : 0;
    if (first < 0) { paged_fail(a.c, MKV_ERR_INVALID_ARG); first = 0; }
    const int n = sp.len - first;
    if (n > a.rows) paged_fail(a.c, MKV_ERR_CAPACITY);
    const int rows = min(n, a.rows);
    constexpr int kPer = D / 8;   // threads of a row, eight channels each
    const int c = (threadIdx.x % kPer) * 8;
    for (int i = blockIdx.x * (kAppendThreads / kPer) + threadIdx.x / kPer; i < rows; i += gridDim.x * (kAppendThreads / kPer)) {
        const int pos = first + i;
        const uint8_t* head = a.c.pages + (size_t)paged_page(a.c, a.b, s, pos) * a.c.page_bytes + (size_t)h * a.c.head_bytes;
        const int row = pos & ((1 << a.c.page_shift) - 1);
        const size_t o = (((size_t)s * a.c.kv_heads + h) * a.rows + i) * D + c;
        if (KIND != MKV_INT4) {
            float x[8], y[8];
            Vec8<T>::load((const T*)head + (size_t)row * D + c, x);
            Vec8<T>::load((const T*)(head + a.c.kv_bytes) + (size_t)row * D + c, y);
            Vec8<T>::store((T*)a.K + o, x);
            Vec8<T>::store((T*)a.V + o, y);
        } else {
            constexpr int NG = D / 32;
            const uint8_t* blk = head + (size_t)(row >> 4) * paged_block_bytes(D);
            const int r = row & 15, j = c >> 5, t = (c & 31) >> 3;
            const uint32_t kw = *reinterpret_cast<const uint32_t*>(blk + r * (D / 2) + (t * NG + j) * 4);
            const uint8_t* vp = blk + 8 * D + (r >> 1) * D + (2 * t * NG + j) * 4 + (r & 1) * 2;
            const uint32_t vw = *reinterpret_cast<const uint16_t*>(vp) |
                                ((uint32_t)*reinterpret_cast<const uint16_t*>(vp + NG * 4) << 16);
            const uint8_t* par = blk + 16 * D;
            const int by_pair = ((r >> 1) * NG + j) * 4 + (r & 1) * 2;
            const float ks = paged_bf16(*reinterpret_cast<const uint16_t*>(par + by_pair));
            const float kl = paged_bf16(*reinterpret_cast<const uint16_t*>(par + 32 * NG + (r * NG + j) * 2));
            const float vs = paged_bf16(*reinterpret_cast<const uint16_t*>(par + 64 * NG + by_pair));
            const float vl = paged_bf16(*reinterpret_cast<const uint16_t*>(par + 96 * NG + by_pair));
            float x[8], y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = fmaf(ks, (float)((kw >> (4 * e)) & 15u), kl);
                y[e] = fmaf(vs, (float)((vw >> (4 * e)) & 15u), vl);
            }
            Vec8<T>::store((T*)a.K + o, x);
            Vec8<T>::store((T*)a.V + o, y);
        }
    }
}

template <typename T, int KIND, int D>
cudaError_t append_t(const PagedAppendArgs& a, cudaStream_t st) {
    constexpr int TT = 4;
    if (a.b.n_tokens <= 1024) paged_append_kernel<T, KIND, D, 1><<<a.b.n_tokens, kAppendThreads, 0, st>>>(a);
    else paged_append_kernel<T, KIND, D, TT><<<(a.b.n_tokens + TT - 1) / TT, kAppendThreads, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, int KIND, int D>
cudaError_t read_t(const PagedReadArgs& a, cudaStream_t st) {
    const int per = kAppendThreads / (D / 8);
    const dim3 grid((unsigned)min((a.rows + per - 1) / per, 64), (unsigned)a.b.batch, (unsigned)a.c.kv_heads);
    paged_read_kernel<T, KIND, D><<<grid, kAppendThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

#define MKV_PAGED_DISPATCH(FN, A)                                                                          \
    if (D == 128) {                                                                                        \
        if ((A).c.kv_dtype == MKV_BF16) return FN<__nv_bfloat16, MKV_BF16, 128>(A, st);                    \
        if ((A).c.kv_dtype == MKV_F32) return FN<float, MKV_F32, 128>(A, st);                              \
        return (A).c.io_f32 ? FN<float, MKV_INT4, 128>(A, st) : FN<__nv_bfloat16, MKV_INT4, 128>(A, st);   \
    }                                                                                                      \
    if ((A).c.kv_dtype == MKV_BF16) return FN<__nv_bfloat16, MKV_BF16, 64>(A, st);                         \
    if ((A).c.kv_dtype == MKV_F32) return FN<float, MKV_F32, 64>(A, st);                                   \
    return (A).c.io_f32 ? FN<float, MKV_INT4, 64>(A, st) : FN<__nv_bfloat16, MKV_INT4, 64>(A, st);

cudaError_t launch_paged_append(const PagedAppendArgs& a, int D, cudaStream_t st) { MKV_PAGED_DISPATCH(append_t, a) }
cudaError_t launch_paged_read(const PagedReadArgs& a, int D, cudaStream_t st) { MKV_PAGED_DISPATCH(read_t, a) }

}  // namespace mkv
