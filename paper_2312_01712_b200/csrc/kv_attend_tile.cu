// Attention of a prompt's tokens over listed blocks.
//
// Every (token, kv head) has a list of its own, but neighbouring tokens' lists are much alike.  A CTA takes a tile of consecutive
// tokens of a request (up to 128 rows = token x query head) and one kv head, forms the union of their lists with one bit per token
// and block, and walks it in ascending order: a block comes from L2 once per tile instead of once per token, and a warp computes
// it only for those of its two groups of 8 rows that have a token that listed it.  Read once per token, 2048 tokens x 8
// heads x 1024 keys are 8.6 GB from L2 for 69 GFLOP, which bound the kernel of kv_attend.cu on this work.
#include <type_traits>

#include "kv_mma.cuh"

namespace ivfpq {
namespace kv {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 16 * kWarps;       // columns of S^T: two groups of 8 per warp
constexpr int kMaxTokens = 64;           // of a tile: bits of a block's mask
constexpr int kKeys = 32;                // of a stage

template <int D>
struct TileShape {
    static constexpr int kStages = D == 256 ? 3 : 4;
    static constexpr int kTileBytes = kKeys * D * 2;          // of keys, or of values
    static constexpr int kRing = kStages * 2 * kTileBytes;
};

struct TilePlan {
    int32_t tokens;          // of a tile
    int32_t cols;            // columns of a token: its query heads rounded up to 1, 2, 4 or a multiple of 8
    int32_t list_cap;        // entries of the union
};

template <bool BF, int D>
__global__ void __launch_bounds__(kThreads, 1) attend_tile_kernel(AttendArgs a, TilePlan p) {
    using S = TileShape<D>;
    constexpr int KSTEPS = D / 16, MT = D / 16, CH = D / 8, NT = 2;
    extern __shared__ __align__(128) char smem[];
    unsigned long long* s_mask = reinterpret_cast<unsigned long long*>(smem + S::kRing);      // [max_blocks], then by entry
    int2* s_list = reinterpret_cast<int2*>(s_mask + a.b.max_blocks);                           // [list_cap] (block, page)
    __shared__ int s_count[kWarps];
    __shared__ int s_total;
    const Cache& c = a.c;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, lr = lane / 4, lc = lane % 4, head = blockIdx.y;
    int* status = reinterpret_cast<int*>(a.ws);
    const uint32_t ring_u = smem_u32(smem);

    // ---- the tile's tokens: rows tok0 .. tok0 + n of request r, the first at position pos0 ----
    int lo = 0, hi = a.b.nreq - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.b.start[mid] / p.tokens + mid <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const int r = lo;
    const int j0 = ((int)blockIdx.x - (a.b.start[r] / p.tokens + r)) * p.tokens;
    const int2 mine = tokens_of(a.b, r, status);
    if (j0 < 0 || j0 >= mine.y) return;
    const int n = min(p.tokens, mine.y - j0), tok0 = mine.x + j0;
    const int pos0 = length_of(a.b, c, r, status) - mine.y + j0;
    const int lim_hi = max(pos0 + n, 0);
    const int nb = (lim_hi + c.page - 1) >> c.page_shift;

    // ---- union of the lists ----
    for (int i = tid; i < nb; i += kThreads) s_mask[i] = 0ull;
    __syncthreads();
    for (int i = tid; i < n * a.nselect; i += kThreads) {
        const int j = i / a.nselect;
        const int blk = a.blocks[((int64_t)(tok0 + j) * c.nheads + head) * a.nselect + (i - j * a.nselect)];
        if (blk >= 0 && (int64_t)blk << c.page_shift <= pos0 + j) atomicOr(&s_mask[blk], 1ull << j);
    }
    __syncthreads();
    int total = 0;
    for (int i0 = 0; i0 < nb; i0 += kThreads) {
        const int i = i0 + tid;
        const unsigned long long m = i < nb ? s_mask[i] : 0ull;
        const int page = m ? page_of(a.b, c, r, i, status) : -1;
        const unsigned in = __ballot_sync(0xffffffffu, page >= 0);
        if (lane == 0) s_count[warp] = __popc(in);
        __syncthreads();
        int at = total + __popc(in & ((1u << lane) - 1u));
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) at += s_count[w];
            total += s_count[w];
        }
        if (page >= 0) {
            s_list[at] = make_int2(i, page);
            s_mask[at] = m;                        // at <= i: entries before i0 are all read
        }
        __syncthreads();
    }

    // ---- queries and limits of the warp's columns ----
    const int col0 = warp * 16;
    uint32_t qf[NT][KSTEPS][2];
    int lim[NT][2], bit[NT][2];
    unsigned long long mine_mask[NT];
    const float fscale = fmaxf(fabsf(a.scale), 1e-30f) * kLog2e;
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int col = col0 + nt * 8 + lr, j = col / p.cols, g = col % p.cols;
        const bool real = j < n && g < a.group;
        const char* qp = a.q.p + 2 * ((int64_t)(tok0 + (real ? j : 0)) * a.q.ts + (int64_t)(head * a.group + (real ? g : 0)) * a.q.hs);
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            qf[nt][s][0] = real ? *reinterpret_cast<const uint32_t*>(qp + 2 * (16 * s + 2 * lc)) ^ flip : 0u;
            qf[nt][s][1] = real ? *reinterpret_cast<const uint32_t*>(qp + 2 * (16 * s + 8 + 2 * lc)) ^ flip : 0u;
        }
        mine_mask[nt] = 0ull;
        for (int x = 0; x < 8; ++x) {
            const int jj = (col0 + nt * 8 + x) / p.cols;
            if (jj < n) mine_mask[nt] |= 1ull << jj;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int jj = (col0 + nt * 8 + lc * 2 + x) / p.cols;
            bit[nt][x] = min(jj, 63);
            lim[nt][x] = jj < n ? max(pos0 + jj + 1, 0) : 0;
        }
    }
    const int lim_lo = max(pos0 + min(col0 / p.cols, n - 1) + 1, 0);      // of the warp's first column
    const bool packed = p.cols < 8;               // a group of 8 columns has several tokens

    float o[MT][NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[i][nt][x] = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -INFINITY;
        l[nt][0] = l[nt][1] = 0.f;
    }

    // ---- stages: 32 keys (a page of 16: its 16) of an entry ----
    const int per_shift = c.page_shift > 5 ? c.page_shift - 5 : 0;
    const int nstage = total << per_shift, keys = min(c.page, kKeys);
    auto issue = [&](int st) {
        if (st < nstage) {
            const int2 e = s_list[st >> per_shift];
            const int off = (st & ((1 << per_shift) - 1)) * kKeys, pos = (e.x << c.page_shift) + off;
            if (pos < lim_hi) {
                const uint32_t dst = ring_u + (st % S::kStages) * 2 * S::kTileBytes;
                const char* kp = c.k + 2 * (e.y * c.ks[0] + head * c.ks[1] + off * c.ks[2]);
                const char* vp = c.v + 2 * (e.y * c.vs[0] + head * c.vs[1] + off * c.vs[2]);
#pragma unroll
                for (int i = 0; i < kKeys * CH / kThreads; ++i) {
                    const int x = i * kThreads + tid, row = x / CH, ch = x % CH;
                    const uint32_t at = row * (2 * D) + ((ch ^ (row & 7)) * 16);
                    const bool real = row < keys && pos + row < lim_hi;
                    const int rr = real ? row : 0;
                    cp_async16(dst + at, kp + 2 * (rr * c.ks[2] + ch * 8), real);
                    cp_async16(dst + S::kTileBytes + at, vp + 2 * (rr * c.vs[2] + ch * 8), real);
                }
            }
        }
        cp_async_commit();
    };
    for (int i = 0; i < S::kStages - 1; ++i) issue(i);
    for (int st = 0; st < nstage; ++st) {
        cp_async_wait<S::kStages - 2>();
        __syncthreads();                          // the stage is here, and everybody is done with the one before
        issue(st + S::kStages - 1);
        const unsigned long long mask = s_mask[st >> per_shift];
        const bool need0 = (mask & mine_mask[0]) != 0, need1 = (mask & mine_mask[1]) != 0;
        const int pos = (s_list[st >> per_shift].x << c.page_shift) + (st & ((1 << per_shift) - 1)) * kKeys;
        if (pos >= lim_hi || !(need0 || need1)) continue;
        const uint32_t kt = ring_u + (st % S::kStages) * 2 * S::kTileBytes, vt = kt + S::kTileBytes;
        const bool masked = packed || pos + kKeys > lim_lo || keys < kKeys;
        auto work = [&](auto first, auto count) {
            constexpr int N0 = decltype(first)::value, N1 = N0 + decltype(count)::value;
            float s[2][NT][4];
            {
                const int row = (lane & 7) + ((lane >> 3) & 1) * 8, up = lane >> 4;
#pragma unroll
                for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t f[4];
                        ldmatrix4(f, kt + (i * 16 + row) * (2 * D) + (((2 * k + up) ^ (row & 7)) * 16));
#pragma unroll
                        for (int nt = N0; nt < N1; ++nt) {
                            if (k == 0) mma16816_first<BF>(s[i][nt], f[0], f[1], f[2], f[3], qf[nt][k][0], qf[nt][k][1]);
                            else mma16816<BF>(s[i][nt], f[0], f[1], f[2], f[3], qf[nt][k][0], qf[nt][k][1]);
                        }
                    }
            }
            if (masked) {
#pragma unroll
                for (int nt = N0; nt < N1; ++nt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const bool listed = (mask >> bit[nt][x & 1]) & 1ull;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int key = i * 16 + lr + (x >> 1) * 8;
                            if (!listed || key >= keys || pos + key >= lim[nt][x & 1]) s[i][nt][x] = -INFINITY;
                        }
                    }
            }
            bool need = false;
            float top[NT][2];
#pragma unroll
            for (int nt = N0; nt < N1; ++nt)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    top[nt][x] = fmaxf(fmaxf(s[0][nt][x], s[0][nt][x + 2]), fmaxf(s[1][nt][x], s[1][nt][x + 2]));
                    need |= fmaf(top[nt][x], fscale, -m[nt][x]) > kSlack;
                }
            if (__any_sync(0xffffffffu, need)) {
#pragma unroll
                for (int nt = N0; nt < N1; ++nt)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float y = top[nt][x];
#pragma unroll
                        for (int k = 4; k < 32; k <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, k));
                        const float mn = fmaxf(m[nt][x], y * fscale);
                        const float f = m[nt][x] == mn ? 1.f : ex2(m[nt][x] - mn);
                        m[nt][x] = mn;
                        l[nt][x] *= f;
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            o[i][nt][x] *= f;
                            o[i][nt][x + 2] *= f;
                        }
                    }
            }
            uint32_t pf[2][NT][2];
#pragma unroll
            for (int nt = N0; nt < N1; ++nt) {
                const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float e0 = ex2(fmaf(s[i][nt][0], fscale, -m0)), e1 = ex2(fmaf(s[i][nt][1], fscale, -m1));
                    const float e2 = ex2(fmaf(s[i][nt][2], fscale, -m0)), e3 = ex2(fmaf(s[i][nt][3], fscale, -m1));
                    l[nt][0] += e0 + e2;
                    l[nt][1] += e1 + e3;
                    pf[i][nt][0] = movmatrix(pack2<BF>(e0, e1));
                    pf[i][nt][1] = movmatrix(pack2<BF>(e2, e3));
                }
            }
            const int key = (lane & 7) + (lane >> 4) * 8, up = (lane >> 3) & 1;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t f[4];
                    ldmatrix4t(f, vt + (i * 16 + key) * (2 * D) + (((2 * mt + up) ^ (key & 7)) * 16));
#pragma unroll
                    for (int nt = N0; nt < N1; ++nt) mma16816<BF>(o[mt][nt], f[0], f[1], f[2], f[3], pf[i][nt][0], pf[i][nt][1]);
                }
        };
        using I0 = std::integral_constant<int, 0>;
        using I1 = std::integral_constant<int, 1>;
        if (need0 && need1) work(I0{}, std::integral_constant<int, 2>{});
        else if (need0) work(I0{}, I1{});
        else work(I1{}, I1{});
    }
    cp_async_wait<0>();
    __syncthreads();

    // ---- results through shared memory: [column][d] ----
    char* so = smem + warp * 16 * (D + 8) * 2;
    static_assert(kWarps * 16 * (D + 8) * 2 <= S::kRing, "the ring holds the rows");
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float y = l[nt][x];
#pragma unroll
            for (int k = 4; k < 32; k <<= 1) y += __shfl_xor_sync(0xffffffffu, y, k);
            const int cc = nt * 8 + lc * 2 + x, col = col0 + cc, j = col / p.cols, g = col % p.cols;
            const bool nan = y != y;
            const float inv = nan ? y : y > 0.f ? 1.f / y : 0.f;
            if (a.lse && lr == 0 && j < n && g < a.group)
                a.lse[(int64_t)(tok0 + j) * (c.nheads * a.group) + head * a.group + g] =
                    nan ? y : y > 0.f ? (m[nt][x] + log2f(y)) * 0.6931471805599453f : -INFINITY;
            uint16_t* at = reinterpret_cast<uint16_t*>(so) + cc * (D + 8) + lr;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                at[mt * 16] = to_bits(o[mt][nt][x] * inv, BF);
                at[mt * 16 + 8] = to_bits(o[mt][nt][x + 2] * inv, BF);
            }
        }
    __syncwarp();
    for (int i = lane; i < 16 * CH; i += 32) {
        const int cc = i / CH, ch = i % CH, col = col0 + cc, j = col / p.cols, g = col % p.cols;
        if (j < n && g < a.group)
            *reinterpret_cast<uint4*>(a.out + 2 * (((int64_t)(tok0 + j) * (c.nheads * a.group) + head * a.group + g) * D + ch * 8)) =
                *reinterpret_cast<const uint4*>(so + (cc * (D + 8) + ch * 8) * 2);
    }
}

template <int D>
size_t tile_smem(const AttendArgs& a, TilePlan* p) {
    p->cols = a.group <= 2 ? a.group : a.group <= 4 ? 4 : (a.group + 7) / 8 * 8;
    p->tokens = kRows / p->cols < kMaxTokens ? kRows / p->cols : kMaxTokens;
    const int64_t entries = (int64_t)p->tokens * a.nselect;
    p->list_cap = (int32_t)(entries < a.b.max_blocks ? entries : a.b.max_blocks);
    return (size_t)TileShape<D>::kRing + (size_t)a.b.max_blocks * 8 + (size_t)p->list_cap * 8;
}

template <bool BF, int D>
cudaError_t run(const AttendArgs& a, cudaStream_t st) {
    TilePlan p{};
    const size_t smem = tile_smem<D>(a, &p);
    auto kernel = attend_tile_kernel<BF, D>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kernel<<<dim3(a.b.ntok / p.tokens + a.b.nreq, a.c.nheads), kThreads, smem, st>>>(a, p);
    return cudaGetLastError();
}

}  // namespace

// Tiles pay where tokens of a request share lists: several tokens a request, and masks that fit beside the ring.
bool attend_tile_serves(const AttendArgs& a) {
    if (!a.blocks || !a.b.start || a.c.format == IVFPQ_KV_INT4 || a.b.ntok < 8 * (int64_t)a.b.nreq) return false;
    TilePlan p{};
    const size_t smem = a.c.d == 64 ? tile_smem<64>(a, &p) : a.c.d == 128 ? tile_smem<128>(a, &p) : tile_smem<256>(a, &p);
    return smem <= 220 * 1024;
}

cudaError_t launch_attend_tile(const AttendArgs& a, cudaStream_t st) {
    const bool bf = a.c.format == IVFPQ_KV_BF16;
    if (a.c.d == 64) return bf ? run<true, 64>(a, st) : run<false, 64>(a, st);
    if (a.c.d == 128) return bf ? run<true, 128>(a, st) : run<false, 128>(a, st);
    return bf ? run<true, 256>(a, st) : run<false, 256>(a, st);
}

}  // namespace kv
}  // namespace ivfpq
