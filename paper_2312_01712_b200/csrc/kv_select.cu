// Filtering of the key/value cache: blocks chosen per token and kv head by the bounds of their keys.
#include "kv.cuh"

namespace ivfpq {
namespace kv {
namespace {

constexpr int kThreads = 256;

// Order-preserving key of a score; NaN below everything.
__device__ __forceinline__ uint32_t score_key(float s) {
    if (s != s) return 0u;
    const uint32_t u = __float_as_uint(s + 0.f);   // -0 and 0 are one score
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA per (token, kv head): keys of all visible blocks to shared memory, then the nselect largest by radix
// passes of 8 bits over a histogram, ties to the lowest block, written in ascending order.
__global__ void __launch_bounds__(kThreads) select_kernel(SelectArgs a) {
    extern __shared__ uint32_t s_key[];            // [blocks of the longest row]
    __shared__ int s_hist[256];
    __shared__ int s_pick[2];
    __shared__ int s_count[kThreads / 32][2];
    __shared__ float s_top[kThreads / 32];
    const Cache& c = a.c;
    const int tok = blockIdx.x, head = blockIdx.y, d = c.d, tid = threadIdx.x;
    int8_t* s_q = reinterpret_cast<int8_t*>(s_key + a.b.max_blocks);     // [group][d]
    int32_t* out = a.out + ((int64_t)tok * c.nheads + head) * a.nselect;
    const int r = request_of(a.b, tok);
    const int2 mine = tokens_of(a.b, r, a.status);
    const int len = length_of(a.b, c, r, a.status);
    const int pos = len - mine.y + (tok - mine.x);
    const int nb = pos < 0 || pos >= len ? 0 : (pos >> c.page_shift) + 1;
    if (nb <= a.nselect) {
        for (int i = tid; i < a.nselect; i += kThreads) out[i] = i < nb ? i : -1;
        return;
    }
    const char* q = a.q.p + 2 * (tok * a.q.ts + (int64_t)head * a.group * a.q.hs);
    float top = 0.f;
    for (int i = tid; i < a.group * d; i += kThreads)
        top = fmaxf(top, fabsf(to_float(reinterpret_cast<const uint16_t*>(q + 2 * (i / d) * a.q.hs)[i % d], a.bf16)));
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (tid % 32 == 0) s_top[tid / 32] = top;
    __syncthreads();
    top = s_top[0];
    for (int i = 1; i < kThreads / 32; ++i) top = fmaxf(top, s_top[i]);
    const float inv = code_factor(top);
    for (int i = tid; i < a.group * d; i += kThreads)
        s_q[i] = code8(to_float(reinterpret_cast<const uint16_t*>(q + 2 * (i / d) * a.q.hs)[i % d], a.bf16), inv);
    __syncthreads();
    for (int blk = tid; blk < nb; blk += kThreads) {
        uint32_t key = 0xffffffffu;
        if (blk >= a.nsink && blk < nb - a.nlocal) {
            const int page = page_of(a.b, c, r, blk, a.status);
            key = 0;
            if (page >= 0) {
                const int64_t at = (int64_t)page * c.nheads + head;
                const int8_t* bd = c.bounds + at * 2 * d;
                int best = INT_MIN;
                for (int h = 0; h < a.group; ++h) {
                    int sum = 0;
                    for (int i = 0; i < d; ++i) {
                        const int x = s_q[h * d + i];
                        sum += max(x * bd[i], x * bd[d + i]);
                    }
                    best = max(best, sum);
                }
                key = score_key(__fmul_rn((float)best, c.scale[at]));
            }
        }
        s_key[blk] = key;
    }
    __syncthreads();
    uint32_t prefix = 0;
    int need = a.nselect;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) s_hist[tid] = 0;
        __syncthreads();
        for (int blk = tid; blk < nb; blk += kThreads) {
            const uint32_t k = s_key[blk];
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int left = need, bin = 255;
            while (bin > 0 && s_hist[bin] < left) left -= s_hist[bin--];
            s_pick[0] = bin;
            s_pick[1] = left;
        }
        __syncthreads();
        prefix |= (uint32_t)s_pick[0] << shift;
        need = s_pick[1];
    }
    // keys above `prefix` are in, and the first `need` equal to it
    int base = 0, ties = 0;
    for (int b0 = 0; b0 < nb; b0 += kThreads) {
        const int blk = b0 + tid;
        const uint32_t k = blk < nb ? s_key[blk] : 0;
        const bool eq = blk < nb && k == prefix;
        const unsigned below = (1u << (tid % 32)) - 1, me = __ballot_sync(0xffffffffu, eq);
        __syncthreads();
        if (tid % 32 == 0) s_count[tid / 32][0] = __popc(me);
        __syncthreads();
        int rank = ties + __popc(me & below), all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < tid / 32) rank += s_count[w][0];
            all += s_count[w][0];
        }
        const bool in = blk < nb && (k > prefix || (eq && rank < need));
        const unsigned mi = __ballot_sync(0xffffffffu, in);
        if (tid % 32 == 0) s_count[tid / 32][1] = __popc(mi);
        __syncthreads();
        int at = base + __popc(mi & below), allin = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < tid / 32) at += s_count[w][1];
            allin += s_count[w][1];
        }
        if (in && at < a.nselect) out[at] = blk;
        base += allin;
        ties += all;
    }
}

}  // namespace

cudaError_t launch_select(const SelectArgs& a, cudaStream_t st) {
    const size_t smem = (size_t)a.b.max_blocks * 4 + (size_t)a.group * a.c.d;
    const cudaError_t e = cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    select_kernel<<<dim3(a.b.ntok, a.c.nheads), kThreads, smem, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kv
}  // namespace ivfpq
