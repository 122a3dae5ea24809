// Attention over the paged key/value cache, whole or over listed blocks.
#include "kv.cuh"

namespace ivfpq {
namespace kv {
namespace {

// One warp per (token, query head): a lane holds d / 32 consecutive elements, one key at a time, running maximum
// and sum of the softmax (online form: a larger maximum m' scales what was summed by exp(m - m')).
template <int E>
__global__ void __launch_bounds__(128) attend_kernel(AttendArgs a) {
    const Cache& c = a.c;
    const int lane = threadIdx.x % 32, e = lane * E, hq = a.group * c.nheads;
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    if (row >= (int64_t)a.b.ntok * hq) return;
    const int tok = (int)(row / hq), h = (int)(row % hq), head = h / a.group;
    int* status = reinterpret_cast<int*>(a.ws);
    const int r = request_of(a.b, tok);
    const int2 mine = tokens_of(a.b, r, status);
    const int len = length_of(a.b, c, r, status);
    const int pos = len - mine.y + (tok - mine.x);
    const int nb = pos < 0 || pos >= len ? 0 : (pos >> c.page_shift) + 1;
    float q[E], o[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        q[i] = to_float(reinterpret_cast<const uint16_t*>(a.q.p + 2 * (tok * a.q.ts + h * a.q.hs))[e + i], a.bf16) * a.scale;
        o[i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    const int32_t* list = a.blocks ? a.blocks + ((int64_t)tok * c.nheads + head) * a.nselect : nullptr;
    const int n = list ? a.nselect : nb;
    for (int j = 0; j < n; ++j) {
        const int blk = list ? list[j] : j;
        if (blk < 0 || blk >= nb) continue;
        const int page = page_of(a.b, c, r, blk, status);
        if (page < 0) continue;
        const int end = min(c.page, pos + 1 - (blk << c.page_shift));
        for (int t = 0; t < end; ++t) {
            float kx[E], vx[E];
            if (c.format != IVFPQ_KV_INT4) {
                const uint16_t* kp = reinterpret_cast<const uint16_t*>(c.k) + page * c.ks[0] + head * c.ks[1] + t * c.ks[2] + e;
                const uint16_t* vp = reinterpret_cast<const uint16_t*>(c.v) + page * c.vs[0] + head * c.vs[1] + t * c.vs[2] + e;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    kx[i] = to_float(kp[i], a.bf16);
                    vx[i] = to_float(vp[i], a.bf16);
                }
            } else {
                const uint8_t* rec = record_of(c, page, head, t / kTile);
                const int tt = t % kTile, g = e / 64, e8 = e / 8 * 8, sh = e % 8 * 4;
                const __half* kp = reinterpret_cast<const __half*>(rec + key_param(c.d, tt, g));
                const __half* vp = reinterpret_cast<const __half*>(rec + value_param(c.d, tt, g));
                const uint32_t kw = *reinterpret_cast<const uint32_t*>(rec + key_word(c.d, tt, e8)) >> sh;
                const uint32_t vw = *reinterpret_cast<const uint32_t*>(rec + value_word(c.d, tt, e8)) >> sh;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    kx[i] = fmaf(__half2float(kp[0]), (float)((kw >> (4 * i)) & 15u), __half2float(kp[1]));
                    vx[i] = fmaf(__half2float(vp[0]), (float)((vw >> (4 * i)) & 15u), __half2float(vp[2]));
                }
            }
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) x = fmaf(q[i], kx[i], x);
#pragma unroll
            for (int s = 16; s; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
            const float mn = fmaxf(m, x), f = __expf(m - mn), p = __expf(x - mn);
            m = mn;
            l = l * f + p;
#pragma unroll
            for (int i = 0; i < E; ++i) o[i] = fmaf(p, vx[i], o[i] * f);
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + row * c.d + e;
#pragma unroll
    for (int i = 0; i < E; ++i) out[i] = to_bits(o[i] * inv, a.bf16);
    if (a.lse && lane == 0) a.lse[row] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

size_t attend_workspace_bytes(int d) { return 256; }

cudaError_t launch_attend(const AttendArgs& a, cudaStream_t st) {
    const int64_t rows = (int64_t)a.b.ntok * a.c.nheads * a.group;
    const unsigned grid = (unsigned)((rows + 3) / 4);
    if (a.c.d == 64) attend_kernel<2><<<grid, 128, 0, st>>>(a);
    else if (a.c.d == 128) attend_kernel<4><<<grid, 128, 0, st>>>(a);
    else attend_kernel<8><<<grid, 128, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kv
}  // namespace ivfpq
