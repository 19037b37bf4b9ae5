// head_tc.cu -- the matrix products of a head over a large vocabulary, on pairs of SMs (tcgen05 cta_group::2, TMEM, TMA):
//
//   HEAD_STATS    l = z w^T, of which a tile's rows leave their largest value, their sum of exponentials and the
//                 label's logit: the logits themselves are never written
//   HEAD_DLOGITS  the same product again, each logit turned into the loss' gradient by it, in bf16
//   HEAD_DZ       dz = dl w over a piece of the vocabulary, summed in fp32 over the pieces
//   HEAD_DW       dw = dl^T z over the tokens
//
// A tile is 256 x 256 outputs, 128 rows of it in each SM's TMEM, two tiles deep, so that the epilogue of one runs under
// the products of the next.  Roles and barriers are those of row_pair_kernel (gemm_tc2.cuh): warp 0 loads this SM's
// halves of A and B by TMA (operands that lie with the summed index outside as two boxes of 64 x 64), warp 1 of the
// leading SM issues the products, warps 2-9 are the epilogue, a thread a row and half of the columns.  What a tile leaves
// behind is read from TMEM in one go (128 values a thread), which frees it before any exponential is taken.
//
// Tokens that take part lie packed, and their number is known on the device alone: a role walks the tiles with a cursor
// over the heads.  Order: STATS and DLOGITS take all row tiles of a group of 32 under one column tile, so that the
// weights come from DRAM once and the tokens stay in L2; DZ all column tiles of a row tile, whose dl is the larger operand.
// DZ's tiles are few and long (a sum over the vocabulary): what does not fill all pairs is cut along the sum (DzShares).
//
// fp32 operands are three bf16 parts of 8 bits each (split3), and a product of theirs the six products of parts that are
// above 2^-24 of it, the smallest first.  Tensor cores cut a sum to fp32 at every step of 16, always towards zero, so the
// large products are taken a block at a time and the epilogue adds them up, rounding to nearest: dz over 5003 entries
// is then off by 2e-7 where one long sum is off by 1.6e-6.  4 heads of 500 tokens, 8000 entries, d 768: 539 us forward and
// backward; with two blocks 518, and twice the error of p - q where a teacher and the model are sure.
#include "gemm_tc2.cuh"
#include "head.cuh"

namespace vmoe {
namespace tc {

namespace {

constexpr int HB = HEAD_TILE;
static_assert(BK == HEAD_BLOCK, "HEAD_DW's last block of tokens");
constexpr int HG_ROWS = 32;  // row tiles that share a column tile

// Blocks of 64 of a tile's sum that the tensor cores add up by themselves: all, with SHORT two at a time, or in fp32 the five
// small products of parts and then one at a time of the large one.
template <int PARTS, bool SHORT>
__device__ __forceinline__ int sums_of(int kb) { return kb == 0 ? 0 : SHORT ? (kb + 1) / 2 : PARTS == 1 ? 1 : 1 + kb; }
template <int PARTS, bool SHORT>
__device__ __forceinline__ int sum_end(int kb, int i) {
    return SHORT ? min(kb, 2 * i + 2) : PARTS == 1 ? kb : 5 * kb + i;
}

struct HeadShape {
    static constexpr uint32_t A_BYTES = 128 * BK * 2, B_BYTES = 128 * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int STAGES = 6;
    static constexpr int EPI_BYTES = 8 * 4096;  // a warp's 32 rows x 64 bf16 columns
    static constexpr int NUM_BARS = 2 * STAGES + 5;
    static constexpr size_t SMEM_BYTES = 1024 + (size_t)STAGES * STAGE_BYTES + EPI_BYTES + NUM_BARS * 8 + 16;
    static_assert(SMEM_BYTES <= 232448, "over the 227 KB shared-memory limit");
};

// The parts of A and B in product i of np = 6: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0).
__device__ __forceinline__ int part_a(int np, int i) { return np == 1 ? 0 : i == 0 ? 2 : i == 2 || i == 3 ? 1 : 0; }
__device__ __forceinline__ int part_b(int np, int i) { return np == 1 ? 0 : i == 1 ? 2 : i == 2 || i == 4 ? 1 : 0; }

struct HTile {
    int t, m, n, rows, kb0, kb1;  // k-blocks of one product of parts
    int part;                     // HEAD_DZ: where a part of a tile goes, -1: a whole one
};

// A role's way through the tiles of all heads: every `step`-th one, then a part of HEAD_DZ's last ones.
template <int MODE>
struct Cursor {
    int t = -1, base = 0, cnt = 0, rows = 0, u, step;
    int full = 0x7fffffff, left = 0;
    __device__ Cursor(const HeadGemm &g, int first, int stride) : u(first), step(stride) {
        if (MODE != HEAD_DZ || !g.dz) return;
        int tiles = 0;
        for (int i = 0; i < g.T; ++i) tiles += (__ldcg(g.rows + i) + HB - 1) / HB * g.tiles_n;
        left = tiles % g.pairs;
        full = tiles - left;
    }
    __device__ bool seek(const HeadGemm &g, int at, HTile &x) {
        while (at - base >= cnt) {
            base += cnt;
            if (++t >= g.T) return false;
            rows = __ldcg(g.rows + t);  // not the read-only path: see `overlap`
            cnt = MODE == HEAD_DW ? g.tiles_m * g.tiles_n : (rows + HB - 1) / HB * g.tiles_n;
        }
        int local = at - base;
        x.t = t;
        x.rows = rows;
        x.part = -1;
        x.kb0 = 0;
        if (MODE == HEAD_STATS || MODE == HEAD_DLOGITS) {
            const int tm = (rows + HB - 1) / HB, g0 = local / (HG_ROWS * g.tiles_n);
            local -= g0 * HG_ROWS * g.tiles_n;
            const int gm = min(HG_ROWS, tm - g0 * HG_ROWS);
            x.n = local / gm;
            x.m = g0 * HG_ROWS + local - x.n * gm;
            x.kb1 = (g.d + BK - 1) / BK;
        } else {
            x.n = local % g.tiles_n;
            x.m = local / g.tiles_n;
            x.kb1 = MODE == HEAD_DZ ? (g.vn + BK - 1) / BK : (rows + BK - 1) / BK;
        }
        return true;
    }
    __device__ bool next(const HeadGemm &g, HTile &x) {
        if (MODE != HEAD_DZ || u < full) {
            const bool ok = seek(g, u, x);
            u += step;
            return ok;
        }
        // this pair's part of a tile that is left, once
        const int c = (int)(blockIdx.x >> 1);
        const DzShares s(left, g.pairs, (g.vn + BK - 1) / BK, dz_least(g.parts));
        if (u == 0x7fffffff || left == 0 || c >= left * s.cuts) return false;
        u = 0x7fffffff;
        if (!seek(g, full + c % left, x)) return false;
        x.kb0 = s.beg(c / left);
        x.kb1 = s.beg(c / left + 1);
        if (s.cuts > 1) x.part = c;
        return true;
    }
};

__device__ __forceinline__ void tma_store_plain(const CUtensorMap *map, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(src), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

// 64 columns of this warp's 32 rows as bf16, through its staging tile; rest: v becomes what bf16 leaves of it.
template <bool REST>
__device__ __forceinline__ void store64(const CUtensorMap *map, float *v, uint8_t *stg, int col, int row, int batch) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) bulk_wait_read0();  // the last store has read the tile
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float *p = v + 8 * j + 2 * i;
            w[i] = pack_bf16x2(p[0], p[1]);
            if (REST) {
                const float2 h = unpk2(bf16x2_to_f32x2(w[i]));
                p[0] -= h.x;
                p[1] -= h.y;
            }
        }
        *reinterpret_cast<uint4 *>(stg + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
        tma_store_plain(map, smem_u32(stg), col, row, batch);
        bulk_commit();
    }
}

__device__ __forceinline__ float ex2(float v) {
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
}

// STATS2: labels and a teacher at another temperature.  PARTS: 1 or 3.  SHORT: see sums_of.
template <int MODE, bool STATS2, int PARTS, bool SHORT = false>
__global__ void __launch_bounds__(THREADS, 1)
head_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                 const __grid_constant__ CUtensorMap tmD, HeadGemm args) {
    using S = HeadShape;
    constexpr int STAGES = S::STAGES;
    constexpr bool A_MN = MODE == HEAD_DW, B_MN = MODE == HEAD_DZ || MODE == HEAD_DW;
    constexpr uint32_t IDESC = idesc_bf16(HB, HB, A_MN, B_MN);

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    uint8_t *smem = smem_raw + ((1024u - (raw_addr & 1023u)) & 1023u);
    const uint32_t tiles_addr = smem_u32(smem);
    uint8_t *epi_base = smem + STAGES * S::STAGE_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(epi_base + S::EPI_BYTES);
    int *misc = reinterpret_cast<int *>(bars + S::NUM_BARS);  // [0] tmem base, [1] abort

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    auto bar_full = [&](int s) { return smem_u32(bars + s); };  // the leader's counts both CTAs
    auto bar_empty = [&](int s) { return smem_u32(bars + STAGES + s); };
    auto bar_tfull = [&](int a) { return smem_u32(bars + 2 * STAGES + a); };
    auto bar_tempty = [&](int a) { return smem_u32(bars + 2 * STAGES + 2 + a); };
    const uint32_t bar_drain = smem_u32(bars + 2 * STAGES + 4);
    volatile int *abort_flag = misc + 1;
    const uint32_t peer_abort = mapa_shared(smem_u32(misc + 1), rank ^ 1u);

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full(s), 1);
            mbar_init(bar_empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(bar_tfull(a), 1);
            mbar_init(bar_tempty(a), 16);
        }
        mbar_init(bar_drain, 1);
        misc[1] = 0;
        fence_barrier_init();
        fence_proxy_async();
        prefetch_map(&tmA);
        prefetch_map(&tmB);
        if (MODE == HEAD_DLOGITS || MODE == HEAD_DW) prefetch_map(&tmD);
    }
    if (warp == 0) {
        tmem_alloc_pair(smem_u32(misc), 2 * HB);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    cluster_sync_all();  // barriers initialised and TMEM allocated in both CTAs
    tc_fence_after();
    if (MODE == HEAD_DW && args.overlap) {
        // HEAD_DZ ahead may still run: it writes nothing that is read here and reads nothing that is written, and whatever
        // came before it had completed when it let this kernel start.  That is made visible as in wait_for_predecessor
        // (gemm_tc.cuh); its completion is waited for at the end, for whoever waits for this kernel.
        __threadfence();
        asm volatile("fence.proxy.async;" ::: "memory");
    } else {
        pdl_wait();
        if (MODE == HEAD_DZ && args.overlap) pdl_launch_dependents();
    }
    const uint32_t tmem_base = (uint32_t)misc[0];
    const int cid = blockIdx.x >> 1, ncl = gridDim.x >> 1;
    auto give_up = [&]() {
        if (*abort_flag && lane == 0) st_cluster_u32(peer_abort, 1u);
    };

    if (warp == 0) {
        // ------------------------------------------------------------ producer
        if (lane == 0) {
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true;
            Cursor<MODE> cur(args, cid, ncl);
            HTile x;
            while (ok && cur.next(args, x)) {
                const int a0 = x.m * HB + (int)rank * 128, b0 = x.n * HB + (int)rank * 128;
                for (int i = 0; i < args.np && ok; ++i) {
                    const int ta = x.t + args.T * part_a(args.np, i), tb = x.t + args.T * part_b(args.np, i);
                    for (int kb = x.kb0; kb < x.kb1; ++kb) {
                        if (!wait_phase(bar_empty(stage), phase ^ 1u, abort_flag, args.status)) {
                            ok = false;
                            break;
                        }
                        const uint32_t sa = tiles_addr + stage * S::STAGE_BYTES, sb = sa + S::A_BYTES;
                        const uint32_t fb = mapa_shared(bar_full(stage), 0);
                        if (leader) mbar_expect_tx(bar_full(stage), 2 * S::STAGE_BYTES);
                        const int k = kb * BK;
                        if (A_MN) {
                            tma_load_3d_pair(sa, &tmA, fb, a0, k, ta);
                            tma_load_3d_pair(sa + 8192, &tmA, fb, a0 + 64, k, ta);
                        } else {
                            tma_load_3d_pair(sa, &tmA, fb, k, a0, ta);
                        }
                        // HEAD_STATS, HEAD_DLOGITS: rows of w from the piece's first on; HEAD_DZ: its summed index
                        if (MODE == HEAD_DZ) {
                            tma_load_3d_pair(sb, &tmB, fb, b0, args.v0 + k, tb);
                            tma_load_3d_pair(sb + 8192, &tmB, fb, b0 + 64, args.v0 + k, tb);
                        } else if (MODE == HEAD_DW) {
                            tma_load_3d_pair(sb, &tmB, fb, b0, k, tb);
                            tma_load_3d_pair(sb + 8192, &tmB, fb, b0 + 64, k, tb);
                        } else {
                            tma_load_3d_pair(sb, &tmB, fb, k, args.v0 + b0, tb);
                        }
                        ++issued;
                        if (++stage == STAGES) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                }
            }
            if (MODE != HEAD_DZ || !args.overlap) pdl_launch_dependents();
            if (*abort_flag && leader) {  // copies in flight (both CTAs') land before the pair exits
                const unsigned long long t0 = global_ns();
                for (int s = 0; s < STAGES && s < issued; ++s)
                    while (!mbar_try_wait(bar_full(s), (uint32_t)(((issued - 1 - s) / STAGES) & 1)) &&
                           global_ns() - t0 < 200000000ull) {
                    }
            }
        }
        __syncwarp();
        give_up();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (leader)
        if (leader) {
            int stage = 0, it = 0;
            uint32_t phase = 0;
            bool ok = true;
            Cursor<MODE> cur(args, cid, ncl);
            HTile x;
            while (ok && cur.next(args, x)) {
                const int kb = x.kb1 - x.kb0, sums = sums_of<PARTS, SHORT>(kb);  // none without a token: the epilogue writes zeros
                for (int i = 0, k = 0; i < sums && ok; ++i, ++it) {
                    const int acc = it & 1, end = sum_end<PARTS, SHORT>(kb, i);
                    if (!wait_phase(bar_tempty(acc), (uint32_t)((it >> 1) & 1) ^ 1u, abort_flag, args.status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t dtmem = tmem_base + (uint32_t)(acc * HB);
                    for (const int beg = k; k < end; ++k) {
                        if (!wait_phase(bar_full(stage), phase, abort_flag, args.status)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t sa = tiles_addr + stage * S::STAGE_BYTES;
                            const uint64_t da = operand_desc(sa, 0, A_MN), db = operand_desc(sa + S::A_BYTES, 0, B_MN);
#pragma unroll
                            for (int kk = 0; kk < BK / 16; ++kk)
                                mma_pair_bf16(dtmem, desc_step(da, kk, A_MN), desc_step(db, kk, B_MN), IDESC,
                                              k != beg || kk != 0 ? 1u : 0u);
                            mma_pair_commit_both(bar_empty(stage));
                        }
                        __syncwarp();
                        if (++stage == STAGES) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                    if (!ok) break;
                    if (elect_one()) mma_pair_commit_both(bar_tfull(acc));
                    __syncwarp();
                }
            }
            if (elect_one()) {  // all MMAs of the pair complete before TMEM is freed
                mma_pair_commit_local(bar_drain);
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(bar_drain, 0) && global_ns() - t0 < 1000000000ull) {
                }
            }
            __syncwarp();
        }
        give_up();
    } else {
        // ------------------------------------------------------------ epilogue
        // warps w and w + 4 share TMEM lane quarter q = w & 3 and split the columns in halves; a thread owns a row
        const int q = warp & 3, half = (warp - 2) >> 2;
        uint8_t *stg = epi_base + (warp - 2) * 4096;
        int it = 0;
        Cursor<MODE> cur(args, cid, ncl);
        HTile x;
        while (cur.next(args, x)) {
            float v[128];
            const int row = x.m * HB + (int)rank * 128 + q * 32 + lane, col = x.n * HB + half * 128;
            const long long at = (long long)x.t * args.Np + row;
            const int sums = sums_of<PARTS, SHORT>(x.kb1 - x.kb0);
            if (PARTS > 1 || SHORT || sums == 0) {
#pragma unroll
                for (int i = 0; i < 128; ++i) v[i] = 0.0f;
            }
            // the teacher's entries in these 32 rows and 128 columns
            int ent = 0, ents = 0;
            const unsigned *list = nullptr;
            if (MODE == HEAD_STATS && args.off) {
                const long long block = (at - lane) >> 5;
                const int *o = args.off + block * (2 * args.tiles_n + 1) + 2 * x.n + half;
                ent = __ldg(o);
                ents = __ldg(o + 1);
                list = args.list + block * 32 * args.K;
            }
            bool ok = true;
            for (int i = 0; i < sums; ++i, ++it) {
                const int acc = it & 1;
                if (!(ok = wait_phase(bar_tfull(acc), (uint32_t)((it >> 1) & 1), abort_flag, args.status))) break;
                tc_fence_after();
                const uint32_t trow = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * HB + half * 128);
                if (PARTS == 1 && !SHORT) {
                    if (MODE == HEAD_STATS) {
                        for (; ent < ents; ent += 32) {  // their columns, by the column
                            const unsigned mine = ent + lane < ents ? __ldg(list + ent + lane) : 0u;
                            for (int e = 0; e < min(32, ents - ent); ++e) {
                                const unsigned what = __shfl_sync(0xffffffffu, mine, e);
                                uint32_t l;
                                asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(l) : "r"(trow + ((what >> 5) & 127u)));
                                tmem_ld_wait();
                                if (lane == (int)(what & 31u)) args.tl[at * args.K + (what >> 12)] = __uint_as_float(l);
                            }
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(trow + c * 32, *reinterpret_cast<uint32_t(*)[32]>(v + 32 * c));
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t r[32];
                        tmem_ld32(trow + c * 32, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[32 * c + j] += __uint_as_float(r[j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(mapa_shared(bar_tempty(acc), 0));
            }
            if (!ok) break;
            if (MODE == HEAD_DZ && PARTS == 1 && args.two) {  // a token's two rows
#pragma unroll
                for (int i = 0; i < 128; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], HEAD_HALF);
            }
            if (MODE == HEAD_STATS && (PARTS > 1 || SHORT)) {
                for (; ent < ents; ++ent) {
                    const unsigned what = __ldg(list + ent);
                    if (lane != (int)(what & 31u)) continue;
                    const int c = (int)((what >> 5) & 127u);
                    float l = 0.0f;
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (i == c) l = v[i];
                    args.tl[at * args.K + (what >> 12)] = l;
                }
            }
            if (MODE == HEAD_STATS) {
                if (col >= args.V) continue;  // the other half's columns are the last
                const int lab = args.label ? __ldg(args.label + at) - col : -1;
                if (lab >= 0 && lab < 128) {
                    float l = 0.0f;
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (i == lab) l = v[i];
                    args.picked[at] = l;
                }
                if (col + 128 > args.V) {
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (col + i >= args.V) v[i] = -INFINITY;
                }
                float m[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[j] = v[j];
#pragma unroll
                    for (int i = 1; i < 32; ++i) m[j] = fmaxf(m[j], v[4 * i + j]);
                }
                // finite where every logit here is -inf (their sum is then 0) or NaN
                const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), ref = fmaxf(top * args.c1, -3e38f);
                float s[4] = {};
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i & 3] += ex2(fmaf(v[i], args.c1, -ref));
                const long long o = ((long long)x.t * 2 * args.tiles_n + 2 * x.n + half) * args.Np + row;
                args.part[o] = make_float2(ref, (s[0] + s[1]) + (s[2] + s[3]));
                if (STATS2) {
                    const float ref2 = fmaxf(top * args.c2, -3e38f);
                    float s2[4] = {};
#pragma unroll
                    for (int i = 0; i < 128; ++i) s2[i & 3] += ex2(fmaf(v[i], args.c2, -ref2));
                    args.part2[o] = make_float2(ref2, (s2[0] + s2[1]) + (s2[2] + s2[3]));
                }
            } else if (MODE == HEAD_DLOGITS) {
                // a row of zeros among those of two a token is none: times an infinite weight it has a logit of NaN
                const bool live = PARTS == 1 && args.two ? two_token(row) < __ldcg(args.rows + args.T + x.t) : row < x.rows;
                const float4 cf = live ? __ldg(args.coef + at) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                const int lab = live && args.label ? __ldg(args.label + at) - args.v0 - col : -1;
                if (live) {
                    float there = 0.0f;  // the value at the label, whose first term cancels where it is formed as the others are
                    if (lab >= 0 && lab < 128) {
                        float l = 0.0f;
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (i == lab) l = v[i];
                        there = __ldg(args.at_label + at);
                        if (STATS2) there = fmaf(cf.z, ex2(fmaf(l, args.c2, -cf.w)), there);
                    }
#pragma unroll
                    for (int i = 0; i < 128; ++i) {
                        const float l = v[i];
                        v[i] = cf.x * ex2(fmaf(l, args.c1, -cf.y));
                        if (STATS2) v[i] = fmaf(cf.z, ex2(fmaf(l, args.c2, -cf.w)), v[i]);
                    }
                    if (lab >= 0 && lab < 128) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (i == lab) v[i] = there;
                    }
                    if (args.v0 + col + 128 > args.V) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (args.v0 + col + i >= args.V) v[i] = 0.0f;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 128; ++i) v[i] = 0.0f;
                }
                const int r0 = row - lane;
                if (PARTS == 1 && args.two && (lane & HEAD_HALF)) {  // the token's second row: what rounding leaves of the first
#pragma unroll
                    for (int i = 0; i < 128; ++i) v[i] -= __bfloat162float(__float2bfloat16_rn(v[i]));
                }
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    store64<(PARTS > 1)>(&tmD, v, stg, col, r0, x.t + args.T * part);
                    store64<(PARTS > 1)>(&tmD, v + 64, stg, col + 64, r0, x.t + args.T * part);
                }
            } else if (MODE == HEAD_DZ && args.dz && x.part < 0) {
                // straight into the tokens' rows
                const int to = row < x.rows ? __ldg(args.map + at) : -1;
                if (to >= 0) {
                    const long long o = ((long long)x.t * args.N + to) * args.d + col;
#pragma unroll
                    for (int i = 0; i < 128; i += 8) {
                        if (col + i >= args.d) break;
                        if (PARTS == 1) {
                            *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(args.dz) + o + i) = f32_to_bf16x8(v + i);
                        } else {
                            float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(args.dz) + o + i);
                            p[0] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                            p[1] = make_float4(v[i + 4], v[i + 5], v[i + 6], v[i + 7]);
                        }
                    }
                }
            } else if (MODE == HEAD_DZ || PARTS > 1) {
                // fp32: 32 bytes at a time, d and the columns being multiples of 8
                const bool live = MODE == HEAD_DZ ? row < x.rows : row < args.vn;
                float *o = MODE == HEAD_DW ? args.out + ((long long)x.t * args.V + args.v0 + row) * args.d + col
                           : x.part < 0    ? args.out + at * args.d + col
                                           : args.out + ((long long)x.part * HB + row - x.m * HB) * HB + half * 128;
                if (live) {
#pragma unroll
                    for (int i = 0; i < 128; i += 4) {
                        if (col + i >= args.d) break;
                        float4 r = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        float4 *p = reinterpret_cast<float4 *>(o + i);
                        if (MODE == HEAD_DZ && !args.dz && !args.first) {
                            const float4 b = *p;
                            r = make_float4(r.x + b.x, r.y + b.y, r.z + b.z, r.w + b.w);
                        }
                        *p = r;
                    }
                }
            } else {
                const int r0 = row - lane;
                if (r0 < args.vn) {  // rows past the vocabulary's end and columns past d are cut off by the map
                    if (col < args.d) store64<false>(&tmD, v, stg, col, args.v0 + r0, x.t);
                    if (col + 64 < args.d) store64<false>(&tmD, v + 64, stg, col + 64, args.v0 + r0, x.t);
                }
            }
        }
        if (lane == 0) bulk_wait_all();
        __syncwarp();
        give_up();
    }

    if (MODE == HEAD_DW && args.overlap) pdl_wait();
    tc_fence_before();
    cluster_sync_all();  // no MMA, copy or remote arrive of either CTA is still in flight
    tc_fence_after();
    if (warp == 0) tmem_dealloc_pair(tmem_base, 2 * HB);
}

// SM pairs that run the kernel at once on the current device, its shared memory granted first; 0: the query fails.
template <int MODE, bool STATS2, int PARTS, bool SHORT = false>
int pairs_of(cudaLaunchConfig_t *cfg, cudaLaunchAttribute (&attr)[2]) {
    auto kern = head_gemm_kernel<MODE, STATS2, PARTS, SHORT>;
    static std::atomic<int> smem_limit[64], fits[64];
    if (raise_smem_limit((const void *)kern, smem_limit, (int)HeadShape::SMEM_BYTES) != VMOE_OK) return 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    *cfg = {};
    cfg->gridDim = dim3(2 * (unsigned)num_sms());
    cfg->blockDim = dim3(THREADS);
    cfg->dynamicSmemBytes = HeadShape::SMEM_BYTES;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg->attrs = attr;
    cfg->numAttrs = 1;
    int n = fits[dev].load(std::memory_order_relaxed);
    if (!n) {
        if (cudaOccupancyMaxActiveClusters(&n, kern, cfg) != cudaSuccess || n <= 0) return 0;
        fits[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int MODE, bool STATS2, int PARTS, bool SHORT = false>
int launch(const CUtensorMap &ma, const CUtensorMap &mb, const CUtensorMap &md, const HeadGemm &g, long long tiles,
           cudaStream_t s, const char *name) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    const int fits = pairs_of<MODE, STATS2, PARTS, SHORT>(&cfg, attr);
    if (!fits) return VMOE_ERR_CUDA;
    const int pairs = g.pairs ? g.pairs : (int)(tiles < fits ? tiles : fits);
    cfg.stream = s;
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    trace_before(s, name);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, head_gemm_kernel<MODE, STATS2, PARTS, SHORT>, ma, mb, md, g);
    trace_after(s);
    return e == cudaSuccess ? VMOE_OK : VMOE_ERR_CUDA;
}

}  // namespace
}  // namespace tc

using namespace tc;

int head_dz_pairs(int parts) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    return parts > 1 ? pairs_of<HEAD_DZ, false, 3>(&cfg, attr) : pairs_of<HEAD_DZ, false, 1>(&cfg, attr);
}

int launch_head_gemm(int mode, const HeadPlan &h, HeadGemm g, const __nv_bfloat16 *z, const __nv_bfloat16 *w,
                     __nv_bfloat16 *dl, __nv_bfloat16 *dw, cudaStream_t s) {
    g.T = h.T;
    g.Np = h.Np;
    g.V = h.V;
    g.d = h.d;
    g.parts = h.parts;
    g.two = h.two;
    g.np = h.parts == 1 ? 1 : 6;
    g.c1 = h.c1;
    g.c2 = h.c2;
    if (!(g.status = device_status_word())) return VMOE_ERR_CUDA;
    const uint64_t batches = (uint64_t)h.T * h.parts;
    const int tn_v = (g.vn + HB - 1) / HB, tn_d = (h.d + HB - 1) / HB;
    const long long tm = (long long)h.T * (h.Np / HB);
    const bool f32 = h.parts > 1;
    CUtensorMap ma, mb, md;
    if (mode == HEAD_STATS || mode == HEAD_DLOGITS) {
        g.tiles_n = tn_v;
        if (!make_map(&ma, z, h.d, h.Np, batches, 128) || !make_map(&mb, w, h.d, h.V, batches, 128)) return VMOE_ERR_CUDA;
        // No more than a tile a pair: short sums cost half a microsecond, and what the tensor cores cut from a long one does not
        // reach the losses: kl of 46 tokens, 9055 entries, d 840, is off by 3e-7 instead of 1.75e-6.  With more tiles their reads
        // do not hide behind the next tile's products: 17 tasks of 1576 tokens, 6 and 4 blocks at a time, 809 and 876 us for 726.
        if (mode == HEAD_STATS && !f32 && tm * tn_v <= num_sms() / 2)
            return h.stats == 2 ? launch<HEAD_STATS, true, 1, true>(ma, mb, ma, g, tm * tn_v, s, "head_stats")
                                : launch<HEAD_STATS, false, 1, true>(ma, mb, ma, g, tm * tn_v, s, "head_stats");
        if (mode == HEAD_STATS)
            return h.stats == 2 ? (f32 ? launch<HEAD_STATS, true, 3>(ma, mb, ma, g, tm * tn_v, s, "head_stats")
                                       : launch<HEAD_STATS, true, 1>(ma, mb, ma, g, tm * tn_v, s, "head_stats"))
                                : (f32 ? launch<HEAD_STATS, false, 3>(ma, mb, ma, g, tm * tn_v, s, "head_stats")
                                       : launch<HEAD_STATS, false, 1>(ma, mb, ma, g, tm * tn_v, s, "head_stats"));
        if (!make_map(&md, dl, h.piece, h.Np, batches, 32)) return VMOE_ERR_CUDA;
        return h.stats == 2 ? (f32 ? launch<HEAD_DLOGITS, true, 3>(ma, mb, md, g, tm * tn_v, s, "head_dlogits")
                                   : launch<HEAD_DLOGITS, true, 1>(ma, mb, md, g, tm * tn_v, s, "head_dlogits"))
                            : (f32 ? launch<HEAD_DLOGITS, false, 3>(ma, mb, md, g, tm * tn_v, s, "head_dlogits")
                                   : launch<HEAD_DLOGITS, false, 1>(ma, mb, md, g, tm * tn_v, s, "head_dlogits"));
    }
    g.tiles_n = tn_d;
    if (mode == HEAD_DZ) {
        if (!make_map(&ma, dl, h.piece, h.Np, batches, 128) || !make_map(&mb, w, h.d, h.V, batches, 64)) return VMOE_ERR_CUDA;
        return f32 ? launch<HEAD_DZ, false, 3>(ma, mb, ma, g, tm * tn_d, s, "head_dz")
                   : launch<HEAD_DZ, false, 1>(ma, mb, ma, g, tm * tn_d, s, "head_dz");
    }
    g.tiles_m = tn_v;
    const long long tiles = (long long)h.T * tn_v * tn_d;
    if (!make_map(&ma, dl, h.piece, h.Np, batches, 64) || !make_map(&mb, z, h.d, h.Np, batches, 64)) return VMOE_ERR_CUDA;
    if (f32) return launch<HEAD_DW, false, 3>(ma, mb, ma, g, tiles, s, "head_dw");
    if (!make_map(&md, dw, h.d, h.V, h.T, 32)) return VMOE_ERR_CUDA;
    return launch<HEAD_DW, false, 1>(ma, mb, md, g, tiles, s, "head_dw");
}

}  // namespace vmoe
