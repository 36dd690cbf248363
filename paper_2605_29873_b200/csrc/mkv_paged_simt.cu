// Attention of new tokens over the paged cache, scalar form: one warp per (new token, query head).
// For every cache type, head size and mask; the tensor-core kernels take over where they exist.
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s_j - m),  s_j = q . k_j * scale * log2(e)
// over the positions j that the token at position t sees: j <= t, j < lens, j > t - window.
#include "mkv_paged.cuh"

namespace mkv {
namespace {

constexpr int kSimpleWarps = 4;

__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int KIND, int D>
__device__ inline float cached(const PagedDev& c, const uint8_t* head, int row, int ch, bool v) {
    if (KIND == MKV_BF16) return __bfloat162float(((const __nv_bfloat16*)(head + (v ? c.kv_bytes : 0)))[(size_t)row * D + ch]);
    if (KIND == MKV_F32) return ((const float*)(head + (v ? c.kv_bytes : 0)))[(size_t)row * D + ch];
    constexpr int NG = D / 32;
    const uint8_t* blk = head + (size_t)(row >> 4) * paged_block_bytes(D);
    const int r = row & 15, j = ch >> 5, i = ch & 31;
    const uint8_t* par = blk + 16 * D + (v ? 64 * NG : 0);
    const int by_pair = ((r >> 1) * NG + j) * 4 + (r & 1) * 2;
    uint32_t code;
    if (v) code = *(const uint16_t*)(blk + 8 * D + (r >> 1) * D + ((i >> 2) * NG + j) * 4 + (r & 1) * 2) >> (4 * (i & 3));
    else code = *(const uint32_t*)(blk + r * (D / 2) + ((i >> 3) * NG + j) * 4) >> (4 * (i & 7));
    const float s = paged_bf16(*(const uint16_t*)(par + by_pair));
    const float l = paged_bf16(*(const uint16_t*)(par + 32 * NG + (v ? by_pair : (r * NG + j) * 2)));
    return fmaf(s, (float)(code & 15u), l);
}

template <int KIND, int D, bool IO32>
__global__ void __launch_bounds__(kSimpleWarps * 32) paged_simple_kernel(const PagedAttendArgs a) {
    __shared__ float qs[kSimpleWarps][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * kSimpleWarps + warp;
    if (w >= (long long)a.b.n_tokens * a.c.q_heads) return;
    const int tok = (int)(w / a.c.q_heads), h = (int)(w - (long long)tok * a.c.q_heads), hk = h / a.c.group;
    int s = tok;
    if (a.b.starts) {
        int lo = 0, hi = a.b.batch;
        if (a.b.starts[0] > tok || a.b.starts[a.b.batch] <= tok) return;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.b.starts[mid] <= tok) lo = mid; else hi = mid;
        }
        s = lo;
    }
    const PagedSpan sp = paged_span(a.c, a.b, s);
    const int j = tok - sp.tok0;
    if (j < 0 || j >= sp.n) return;
    if (sp.n > a.max_new) paged_fail(a.c, MKV_ERR_CAPACITY);
    const int pos = sp.len - sp.n + j;
    const int end = pos + 1;
    int begin = 0;
    if (a.window > 0 && end > a.window) begin = end - a.window;
    for (int c = lane; c < D; c += 32) {
        const size_t at = (size_t)tok * a.q_stride + (size_t)h * D + c;
        qs[warp][c] = IO32 ? ((const float*)a.q)[at] : __bfloat162float(((const __nv_bfloat16*)a.q)[at]);
    }
    __syncwarp();
    constexpr int EPL = D / 32;
    float o[EPL], m = kPagedNegInf, l = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] = 0.f;
    for (int j0 = begin; j0 < end; j0 += 32) {
        float x = kPagedNegInf;
        if (j0 + lane < end) {
            const int p = j0 + lane;
            const uint8_t* head = a.c.pages + (size_t)paged_page(a.c, a.b, s, p) * a.c.page_bytes + (size_t)hk * a.c.head_bytes;
            const int row = p & ((1 << a.c.page_shift) - 1);
            float acc = 0.f;
            for (int c = 0; c < D; ++c) acc = fmaf(qs[warp][c], cached<KIND, D>(a.c, head, row, c, false), acc);
            x = acc * a.scale_log2;
        }
        float mx = x;
#pragma unroll
        for (int k = 16; k; k >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
        mx = fmaxf(mx, m);
        const float ref = mx == kPagedNegInf ? 0.f : mx;
        const float p = ex2(x - ref), sc = ex2(m - ref);
        m = mx;
        float ps = p;
#pragma unroll
        for (int k = 16; k; k >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, k);
        l = fmaf(l, sc, ps);
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] *= sc;
        for (int k = 0; k < min(32, end - j0); ++k) {
            const float pk = __shfl_sync(0xffffffffu, p, k);
            const int pp = j0 + k;
            const uint8_t* head = a.c.pages + (size_t)paged_page(a.c, a.b, s, pp) * a.c.page_bytes + (size_t)hk * a.c.head_bytes;
            const int row = pp & ((1 << a.c.page_shift) - 1);
#pragma unroll
            for (int e = 0; e < EPL; ++e) o[e] = fmaf(pk, cached<KIND, D>(a.c, head, row, lane * EPL + e, true), o[e]);
        }
    }
    const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
    const size_t at = ((size_t)tok * a.c.q_heads + h) * D + lane * EPL;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        if (a.c.out_f32) ((float*)a.out)[at + e] = o[e] * inv;
        else ((__nv_bfloat16*)a.out)[at + e] = __float2bfloat16_rn(o[e] * inv);
    }
    if (a.lse && lane == 0)
        a.lse[(size_t)tok * a.c.q_heads + h] = l == 0.f ? kPagedNegInf : (m + log2f(l)) * 0.69314718055994531f;
}

template <int KIND, int D>
cudaError_t simple_t(const PagedAttendArgs& a, cudaStream_t st) {
    const long long blocks = ((long long)a.b.n_tokens * a.c.q_heads + kSimpleWarps - 1) / kSimpleWarps;
    if (a.c.io_f32) paged_simple_kernel<KIND, D, true><<<(unsigned)blocks, kSimpleWarps * 32, 0, st>>>(a);
    else paged_simple_kernel<KIND, D, false><<<(unsigned)blocks, kSimpleWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_simt(const PagedAttendArgs& a, int D, cudaStream_t st) {
    if (D == 128) {
        if (a.c.kv_dtype == MKV_BF16) return simple_t<MKV_BF16, 128>(a, st);
        if (a.c.kv_dtype == MKV_F32) return simple_t<MKV_F32, 128>(a, st);
        return simple_t<MKV_INT4, 128>(a, st);
    }
    if (a.c.kv_dtype == MKV_BF16) return simple_t<MKV_BF16, 64>(a, st);
    if (a.c.kv_dtype == MKV_F32) return simple_t<MKV_F32, 64>(a, st);
    return simple_t<MKV_INT4, 64>(a, st);
}

}  // namespace mkv
