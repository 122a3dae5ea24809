// Filtering of the key/value cache: blocks chosen per token and kv head by the bounds of their keys.
//
// The score of a block is a product of whole numbers: max(q u, q l) = q+ u + q- l with q+ = max(q, 0), q- = min(q, 0), so a
// row [q+, q-] of 2 d bytes times the block's [upper, lower] bytes, on the 8-bit matrix instruction (m16n8k32, 16 blocks by 8
// (token, query head) columns, 32-bit sums: exact in any order).  A lane reads 16 consecutive bytes of a block's bounds
// straight into the instruction's operand; the order in which the summed axis is dealt to lanes is free, as long as q has the
// same.  A CTA scores a tile of tokens of one request (one token in a decode step), so that a prompt reads the bounds once per
// tile, keeps the scores as order-preserving 32-bit keys in shared memory, and finds each token's nselect-th
// largest key two bits at a time: count the keys at or above the candidates, from the highest bit in which keys differ, until a count
// fits.
// With few rows and many blocks a cluster of CTAs shares a row's blocks and sends its keys to the first one's
// shared memory.
#include "kv.cuh"

namespace ivfpq {
namespace kv {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxTokens = 32;                     // of a tile

// Order-preserving key of a score; NaN below everything.
__device__ __forceinline__ uint32_t score_key(float s) {
    if (s != s) return 0u;
    const uint32_t u = __float_as_uint(s + 0.f);   // -0 and 0 are one score
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void mma_s8(int* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Address of this shared-memory location in the cluster's first CTA, and a store to it.
__device__ __forceinline__ uint32_t in_first_cta(const void* p) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)));
    return r;
}
__device__ __forceinline__ void store_cluster(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

struct SelectPlan {
    int32_t tokens;          // of a tile: 1, or 8 to 32
    int32_t split;           // CTAs (of a cluster) that share a tile's blocks
    int32_t cols;            // columns of a token: its query heads rounded up to 1, 2, 4 or a multiple of 8
    int32_t ntiles8;         // groups of 8 columns in all
};

// Writes the n largest of keys[0 .. nb), ties to the lowest index, in ascending order of index.  W warps work together
// (W = 1: a warp by itself); cnt: [32] zeroed counters, aux: [2 W] words; nb > n >= 1.  Two bits of the n-th largest key are found per
// pass, by counting the keys at or above three candidates.  NK > 0: a lane's keys, at most NK, stay in registers.
template <int W, int NK>
__device__ __forceinline__ void pick(const uint32_t* keys, int nb, int n, int32_t* out, int warp, int lane, unsigned long long* cnt, uint32_t* bits,
                                     int* aux) {
    auto sync = [] { if (W > 1) __syncthreads(); else __syncwarp(); };
    uint32_t kr[NK > 0 ? NK : 1];
    auto each = [&](auto f) {
        if (NK > 0) {
#pragma unroll
            for (int i = 0; i < NK; ++i)
                if (W * 32 * i < nb) f(kr[i]);     // past the end: key 0, below every candidate
        } else {
            for (int i = warp * 32 + lane; i < nb; i += W * 32) f(keys[i]);
        }
    };
    uint32_t all = 0xffffffffu, any = 0u;
    if (NK > 0) {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int at = (i * W + warp) * 32 + lane;
            kr[i] = at < nb ? keys[at] : 0u;
            if (at < nb) {
                all &= kr[i];
                any |= kr[i];
            }
        }
    } else {
        each([&](uint32_t k) {
            all &= k;
            any |= k;
        });
    }
    all = __reduce_and_sync(0xffffffffu, all);
    any = __reduce_or_sync(0xffffffffu, any);
    if (W > 1) {
        if (lane == 0) {
            atomicAnd(&bits[0], all);
            atomicOr(&bits[1], any);
        }
        sync();
        all = bits[0];
        any = bits[1];
    }
    const int high = 31 - __clz(all ^ any);        // -1: all keys are equal
    uint32_t t = high == 31 ? 0u : high < 0 ? all : all & ~((2u << high) - 1u);
    bool exact = false;
    for (int b = high; b >= 0 && !exact;) {
        const int lowbit = b > 0 ? b - 1 : 0;      // the pass finds bits b and lowbit (bit 0 alone at the end)
        const uint32_t c1 = t | (1u << lowbit), c2 = t | (1u << b), c3 = c2 | (1u << lowbit);
        int n1 = 0, n2 = 0, n3 = 0;
        each([&](uint32_t k) {
            n1 += k >= c1;
            n2 += k >= c2;
            n3 += k >= c3;
        });
        // counts of up to 2^15 + 2^5 keys in 21 bits each
        unsigned long long x;
        if (W == 1 && NK > 0) {                    // at most 1024 keys: 11 bits would do, two words of two
            const uint32_t y = __reduce_add_sync(0xffffffffu, (uint32_t)n1 | (uint32_t)n2 << 16);
            x = (y & 0xffffu) | (unsigned long long)(y >> 16) << 21 | (unsigned long long)__reduce_add_sync(0xffffffffu, n3) << 42;
        } else {
            x = (unsigned long long)__reduce_add_sync(0xffffffffu, n1) | (unsigned long long)__reduce_add_sync(0xffffffffu, n2) << 21 |
                (unsigned long long)__reduce_add_sync(0xffffffffu, n3) << 42;
        }
        if (W > 1) {
            if (lane == 0) atomicAdd(&cnt[b], x);
            sync();
            x = cnt[b];
        }
        const int m1 = (int)(x & 0x1fffff), m2 = (int)(x >> 21 & 0x1fffff), m3 = (int)(x >> 42);
        if (m3 >= n) {
            t = c3;
            exact = m3 == n;
        } else if (m2 >= n) {
            t = c2;
            exact = m2 == n;
        } else if (m1 >= n) {
            t = c1;
            exact = m1 == n;
        }
        b -= 2;
    }
    // each warp writes from a contiguous range of its own
    const int per = ((nb + W - 1) / W + 31) / 32 * 32, lo = min(warp * per, nb), hi = min(lo + per, nb);
    int gt = 0, eq = 0;
    for (int i = lo + lane; i < hi; i += 32) {
        gt += keys[i] > t;
        eq += keys[i] == t;
    }
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    int gt_before = 0, eq_before = 0, gt_all = gt;
    if (W > 1) {
        if (lane == 0) {
            aux[warp * 2] = gt;
            aux[warp * 2 + 1] = eq;
        }
        sync();
        gt_all = 0;
        for (int w = 0; w < W; ++w) {
            gt_all += aux[w * 2];
            if (w < warp) {
                gt_before += aux[w * 2];
                eq_before += aux[w * 2 + 1];
            }
        }
    }
    const int need = n - gt_all;                   // how many of the equal keys are in
    int at = gt_before + min(eq_before, need), ties = eq_before;
    const unsigned below = (1u << lane) - 1u;
    for (int i0 = lo; i0 < hi; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < hi ? keys[i] : 0u;
        const unsigned me = __ballot_sync(0xffffffffu, i < hi && k == t);
        const bool in = i < hi && (k > t || (k == t && ties + __popc(me & below) < need));
        const unsigned mi = __ballot_sync(0xffffffffu, in);
        if (in) out[at + __popc(mi & below)] = i;
        at += __popc(mi);
        ties += __popc(me);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) select_kernel(SelectArgs a, SelectPlan p) {
    constexpr int CH = 2 * D / 64;                 // 64-byte segments of a block's bounds
    constexpr int KS = 2 * CH;                     // matrix steps of 32 bytes
    extern __shared__ __align__(16) uint32_t s_key[];       // [tokens][blocks], then the queries' operands
    __shared__ unsigned long long s_cnt[32];
    __shared__ uint32_t s_bits[2];
    __shared__ int s_aux[2 * kWarps];
    const Cache& c = a.c;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, lr = lane / 4, lc = lane % 4;
    const int head = blockIdx.y, tile = blockIdx.x / p.split, rank = p.split > 1 ? (int)cluster_rank() : 0;
    const int stride = a.b.max_blocks;
    uint32_t* s_q = s_key + (((size_t)p.tokens * stride + 3) & ~(size_t)3);        // [columns / 8][KS][lane][2]
    if (p.split > 1) cluster_arrive();             // all CTAs of the cluster run before anybody stores to the first
    if (tid < 32) s_cnt[tid] = 0;
    if (tid == 0) {
        s_bits[0] = 0xffffffffu;
        s_bits[1] = 0u;
    }

    // ---- the tile's tokens: request r, rows tok0 .. tok0 + n, at positions pos0 ... ----
    int r = tile, j0 = 0;
    bool real = true;
    if (p.tokens == 1) {
        r = request_of(a.b, tile);
    } else {
        int lo = 0, hi = a.b.nreq - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.b.start[mid] / p.tokens + mid <= tile) lo = mid; else hi = mid - 1;
        }
        r = lo;
        j0 = (tile - (a.b.start[r] / p.tokens + r)) * p.tokens;
        real = j0 >= 0;
    }
    const int2 mine = tokens_of(a.b, r, a.status);
    if (p.tokens == 1) j0 = tile - mine.x;
    real = real && j0 >= 0 && j0 < mine.y;
    const int len = length_of(a.b, c, r, a.status);
    const int n = real ? min(p.tokens, mine.y - j0) : 0, tok0 = mine.x + j0, pos0 = len - mine.y + j0;
    auto blocks_of = [&](int j) { return pos0 + j < 0 ? 0 : ((pos0 + j) >> c.page_shift) + 1; };   // that token j of the tile sees
    const int nb_max = n > 0 ? blocks_of(n - 1) : 0;
    const bool score = nb_max > a.nselect;         // uniform over the cluster

    if (score) {
        // ---- queries: codes of the token's group, as matrix operands ----
        for (int j = warp; j < p.tokens; j += kWarps) {
            const char* q = a.q.p + 2 * ((int64_t)(tok0 + min(j, n - 1)) * a.q.ts + (int64_t)head * a.group * a.q.hs);
            float top = 0.f;
            for (int i = lane; i < a.group * (D / 8); i += 32) {
                float x[8];
                unpack8(*reinterpret_cast<const uint4*>(q + 2 * ((int64_t)(i / (D / 8)) * a.q.hs + i % (D / 8) * 8)), a.bf16, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(x[k]));
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float factor = code_factor(top);
            for (int i = lane; i < p.cols * (D / 8); i += 32) {
                const int g = i / (D / 8), e = i % (D / 8) * 8;
                float x[8];
                unpack8(*reinterpret_cast<const uint4*>(q + 2 * ((int64_t)(g < a.group ? g : 0) * a.q.hs + e)), a.bf16, x);
                uint32_t pos[2] = {0, 0}, neg[2] = {0, 0};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int v = code8(x[k], factor);
                    pos[k / 4] |= (uint32_t)(uint8_t)(int8_t)max(v, 0) << (8 * (k % 4));
                    neg[k / 4] |= (uint32_t)(uint8_t)(int8_t)min(v, 0) << (8 * (k % 4));
                }
                const int col = j * p.cols + g;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // bytes e .. e + 7 of the half: segment e / 64, lane part e % 64 / 16, words (e % 16) / 4 and the next
                    const int at = h * D + e;
                    const int word = ((col / 8 * KS + at / 64 * 2 + at % 16 / 8) * 32 + col % 8 * 4 + at % 64 / 16) * 2;
                    *reinterpret_cast<uint2*>(s_q + word) = h ? make_uint2(neg[0], neg[1]) : make_uint2(pos[0], pos[1]);
                }
            }
        }
    }
    __syncthreads();
    if (p.split > 1) cluster_wait();
    if (score) {
        // ---- scores of 16 blocks per warp and step ----
        const int groups = (nb_max + 15) / 16, share = (groups + p.split - 1) / p.split;
        const int g1 = min((rank + 1) * share, groups);
        const uint32_t key0 = p.split > 1 ? in_first_cta(s_key) : 0;
        const int per8 = p.cols < 8 ? 8 / p.cols : 1;                 // tokens of a group of 8 columns
        auto page_at = [&](int gr, int h) {
            const int blk = gr * 16 + lr + h * 8;
            return gr < g1 && blk < nb_max ? page_of(a.b, c, r, blk, a.status) : -1;
        };
        int next[2] = {page_at(rank * share + warp, 0), page_at(rank * share + warp, 1)};
        for (int gr = rank * share + warp; gr < g1; gr += kWarps) {
            uint32_t w[2][CH][4];
            float scale[2];
            bool ok[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int page = next[h];
                ok[h] = page >= 0;
                const int64_t at = (int64_t)max(page, 0) * c.nheads + head;
                scale[h] = c.scale[at];
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const uint4 x = __ldg(reinterpret_cast<const uint4*>(c.bounds + at * 2 * D + i * 64 + lc * 16));
                    w[h][i][0] = x.x; w[h][i][1] = x.y; w[h][i][2] = x.z; w[h][i][3] = x.w;
                }
            }
            next[0] = page_at(gr + kWarps, 0);     // while the bounds are on their way
            next[1] = page_at(gr + kWarps, 1);
            int best[4] = {INT_MIN, INT_MIN, INT_MIN, INT_MIN};
            for (int nt = 0; nt < p.ntiles8; ++nt) {
                int acc[4] = {0, 0, 0, 0};
                const uint32_t* q = s_q + (nt * KS * 32 + lane) * 2;
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const uint2 b = *reinterpret_cast<const uint2*>(q + (i * 2 + s) * 64);
                        const uint32_t f[4] = {w[0][i][2 * s], w[1][i][2 * s], w[0][i][2 * s + 1], w[1][i][2 * s + 1]};
                        mma_s8(acc, f, b.x, b.y);
                    }
                if (p.cols >= 2) {
                    acc[0] = max(acc[0], acc[1]);
                    acc[2] = max(acc[2], acc[3]);
                }
                if (p.cols >= 4) {
                    acc[0] = max(acc[0], __shfl_xor_sync(0xffffffffu, acc[0], 1));
                    acc[2] = max(acc[2], __shfl_xor_sync(0xffffffffu, acc[2], 1));
                }
                if (p.cols >= 8) {
                    acc[0] = max(acc[0], __shfl_xor_sync(0xffffffffu, acc[0], 2));
                    acc[2] = max(acc[2], __shfl_xor_sync(0xffffffffu, acc[2], 2));
                    best[0] = max(best[0], acc[0]);
                    best[2] = max(best[2], acc[2]);
                    if ((nt + 1) % (p.cols / 8)) continue;            // more of this token's heads follow
                    acc[0] = best[0];
                    acc[2] = best[2];
                    best[0] = best[2] = INT_MIN;
                }
                const int j = p.cols >= 8 ? nt / (p.cols / 8) : nt * per8 + (p.cols == 4 ? lc / 2 : p.cols == 2 ? lc : lc * 2);
                const bool writer = p.cols >= 8 ? lc == 0 : p.cols == 4 ? lc % 2 == 0 : true;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (x % 2 && p.cols > 1) continue;
                    const int jj = j + x % 2, h = x / 2, blk = gr * 16 + lr + h * 8;
                    if (!writer || jj >= n) continue;
                    const int nb = blocks_of(jj);
                    if (blk >= nb) continue;
                    uint32_t key = ok[h] ? score_key(__fmul_rn((float)acc[x], scale[h])) : 0u;
                    if (blk < a.nsink || blk >= nb - a.nlocal) key = 0xffffffffu;
                    if (p.split > 1) store_cluster(key0 + ((uint32_t)jj * stride + blk) * 4, key);
                    else s_key[(size_t)jj * stride + blk] = key;
                }
            }
        }
    }
    if (p.split > 1) {
        cluster_arrive();
        if (rank) return;
        cluster_wait();
    } else {
        __syncthreads();
    }

    // ---- the lists ----
    if (p.tokens == 1) {
        if (n == 0) return;
        int32_t* out = a.out + ((int64_t)tok0 * c.nheads + head) * a.nselect;
        if (score) {
            if (nb_max <= kThreads * 4) pick<kWarps, 4>(s_key, nb_max, a.nselect, out, warp, lane, s_cnt, s_bits, s_aux);
            else pick<kWarps, 0>(s_key, nb_max, a.nselect, out, warp, lane, s_cnt, s_bits, s_aux);
        } else {
            for (int i = tid; i < a.nselect; i += kThreads) out[i] = i < nb_max ? i : -1;
        }
    } else {
        for (int j = warp; j < n; j += kWarps) {
            int32_t* out = a.out + ((int64_t)(tok0 + j) * c.nheads + head) * a.nselect;
            const int nb = blocks_of(j);
            if (nb > a.nselect) {
                const uint32_t* keys = s_key + (size_t)j * stride;
                if (nb <= 32 * 8) pick<1, 8>(keys, nb, a.nselect, out, 0, lane, nullptr, nullptr, nullptr);
                else if (nb <= 32 * 24) pick<1, 24>(keys, nb, a.nselect, out, 0, lane, nullptr, nullptr, nullptr);
                else pick<1, 0>(keys, nb, a.nselect, out, 0, lane, nullptr, nullptr, nullptr);
            } else {
                for (int i = lane; i < a.nselect; i += 32) out[i] = i < nb ? i : -1;
            }
        }
    }
}

template <int D>
cudaError_t run(const SelectArgs& a, int sms, cudaStream_t st) {
    SelectPlan p{};
    p.cols = a.group <= 2 ? a.group : a.group <= 4 ? 4 : (a.group + 7) / 8 * 8;
    auto bytes = [&](int tokens) {
        return (((size_t)tokens * a.b.max_blocks + 3) & ~(size_t)3) * 4 + (size_t)((tokens * p.cols + 7) / 8) * 8 * 2 * D;
    };
    // a prompt: as many tokens per tile as two CTAs an SM have room for, and as leave every SM two CTAs
    p.tokens = 1;
    if (a.b.start && a.b.ntok >= 4 * (int64_t)a.b.nreq) {
        for (int t = kMaxTokens; t >= 8; t /= 2) {
            if (bytes(t) > 100 * 1024) continue;
            p.tokens = t;
            if (((int64_t)a.b.ntok / t + 1) * a.c.nheads >= 2 * sms) break;
        }
    }
    p.ntiles8 = (p.tokens * p.cols + 7) / 8;
    const int64_t tiles = p.tokens == 1 ? a.b.ntok : (int64_t)a.b.ntok / p.tokens + a.b.nreq;
    // few rows: a cluster shares a row's blocks, at least 128 of them each
    p.split = 1;
    while (p.split < 8 && p.tokens == 1 && tiles * a.c.nheads * p.split * 2 <= 2 * sms && a.b.max_blocks >= 256 * p.split) p.split *= 2;
    const size_t smem = bytes(p.tokens);
    auto kernel = select_kernel<D>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * p.split), a.c.nheads);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = p.split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a, p);
}

}  // namespace

cudaError_t launch_select(const SelectArgs& a, cudaStream_t st) {
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    if (a.c.d == 64) return run<64>(a, sms, st);
    if (a.c.d == 128) return run<128>(a, sms, st);
    return run<256>(a, sms, st);
}

}  // namespace kv
}  // namespace ivfpq
