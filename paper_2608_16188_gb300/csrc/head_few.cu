// head_few.cu -- the sums of a head's logits for a few tokens, as a served model scores or answers with them:
//
//   l = z w^T for at most 16 tokens, of which the largest value, the sum of exponentials and the label's logit stay
//
// What bounds it is the weights' way from DRAM, read once: V d 2 bytes.  A warp streams 32 rows of w at a time, whole rows
// that lie together, straight into the B fragments of mma.sync m16n8k16: a lane's 16 bytes are eight neighbouring
// k of one row, which the products take in an order of their own (two of four k each: any order of the sum will do, if A
// has the same); the tokens, 16 rows, are A, from shared memory.  A lane keeps the running maximum and sum of its two
// tokens, a CTA leaves one of each.
// 4 tokens, 128000 entries, d 1024 (262 MB, 38.6 us at the copy rate): 51 us, and 52 for the whole pass, whose packing runs
// under the first rows' way from DRAM; as 256 x 256 tiles of head_tc.cu, whose 128-byte pieces of 19000 rows at a time lose
// DRAM's pages, 57.
#include "head.cuh"

namespace vmoe {
namespace {

constexpr int FW_THREADS = 256, FW_WARPS = FW_THREADS / 32, FW_ROWS = 32;
constexpr int FW_AHEAD = 1536;  // bytes of a row of w that are fetched ahead
constexpr unsigned FULL = 0xffffffffu;

__device__ __forceinline__ float ex2(float v) {
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
}
// Running maximum (in units of log2) and sum of exponentials.
struct Sum {
    float m = -3e38f, s = 0.0f;
    __device__ __forceinline__ void join(float om, float os) {
        const float top = fmaxf(m, om);
        s = s * ex2(m - top) + os * ex2(om - top);
        m = top;
    }
};

// Pitch of a token's row in shared memory: 64 bytes past a multiple of 128, free of bank conflicts for 16-byte reads of
// two rows by eight lanes.
__host__ __device__ constexpr int fw_pitch(int d) { return (d + 63) / 64 * 64 + 32; }

template <bool STATS2>
__global__ void __launch_bounds__(FW_THREADS, 2)
head_few_kernel(HeadGemm args, const __nv_bfloat16 *__restrict__ z, const __nv_bfloat16 *__restrict__ w) {
    extern __shared__ __align__(16) __nv_bfloat16 fw_z[];  // [16][pitch]
    __shared__ float2 joined[2][FW_WARPS][HEAD_FEW];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
    const int d = args.d, V = args.V, pitch = fw_pitch(d);
    const __nv_bfloat16 *wt = w + (long long)t * V * d;
    // The warp's first rows, a lane each, on their way into L2 while head_pack runs: at most 120 MB of its 129 (2432 warps).
    // A pass of 4 tokens, 128000 entries, d 1024: 60.7 us without, 58.9 with 256 bytes a row, 57.4 with 512, 54.4 with 1024,
    // 52.2 with 1536 or 1792.  Fetched ahead all the way, a block's rows under the products of the last: 62.
    const int first = (blockIdx.x * FW_WARPS + warp) * FW_ROWS + lane;
    if (first < V)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(__cvta_generic_to_global(wt + (long long)first * d)),
                     "r"(min(d * 2, FW_AHEAD))
                     : "memory");
    pdl_wait();
    pdl_launch_dependents();
    for (int i = tid; i < HEAD_FEW * (pitch / 8); i += FW_THREADS) {
        const int r = i / (pitch / 8), c = (i - r * (pitch / 8)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c < d) v = __ldg(reinterpret_cast<const uint4 *>(z + ((long long)t * args.Np + r) * d + c));
        *reinterpret_cast<uint4 *>(fw_z + r * pitch + c) = v;
    }
    if (args.rows[t] == 0) return;  // nothing was packed, and nothing is read
    __syncthreads();
    const long long at = (long long)t * args.Np + g;
    const int lab[2] = {args.label ? __ldg(args.label + at) : -1, args.label ? __ldg(args.label + at + 8) : -1};
    const __nv_bfloat16 *za = fw_z + g * pitch + 8 * q, *zb = za + 8 * pitch;
    Sum one[2], two[2];
    const int blocks = (V + FW_ROWS - 1) / FW_ROWS;
    for (int b = blockIdx.x * FW_WARPS + warp; b < blocks; b += gridDim.x * FW_WARPS) {
        const int v0 = b * FW_ROWS;
        const __nv_bfloat16 *row[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) row[n] = wt + (long long)min(V - 1, v0 + 8 * n + g) * d + 8 * q;
        float sum[4][4] = {};
        constexpr int U = 4;  // steps of 32 k in flight: 8 KB a warp
        for (int k0 = 0; k0 < d; k0 += 32 * U) {
            uint4 x[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    x[u][n] = make_uint4(0, 0, 0, 0);
                    if (k0 + 32 * u + 8 * q < d) x[u][n] = __ldcs(reinterpret_cast<const uint4 *>(row[n] + k0 + 32 * u));
                }
            // 128 k at a time: the products cut every step of their sums towards zero (all 1024 in one: ce off by 1.1e-6; so 1e-7)
            float acc[4][4] = {};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k0 + 32 * u >= d) break;
                const uint4 a = *reinterpret_cast<const uint4 *>(za + k0 + 32 * u), c = *reinterpret_cast<const uint4 *>(zb + k0 + 32 * u);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    mma_bf16_16816(acc[n], a.x, c.x, a.y, c.y, x[u][n].x, x[u][n].y);
                    mma_bf16_16816(acc[n], a.z, c.z, a.w, c.w, x[u][n].z, x[u][n].w);
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[n][i] += acc[n][i];
        }
        // columns v0 + 8 n + 2 q, + 1 of tokens g (0, 1) and g + 8 (2, 3)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float l[8], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int col = v0 + 8 * (i >> 1) + 2 * q + (i & 1);
                l[i] = sum[i >> 1][2 * h + (i & 1)];
                if (col == lab[h]) args.picked[at + 8 * h] = l[i];
                if (col >= V) l[i] = -INFINITY;
                top = fmaxf(top, l[i]);
            }
            if (v0 + 2 * q >= V) continue;  // past the vocabulary's end; NaNs alone leave no top, but a sum
            auto add = [&](Sum &s, float c) {
                const float m = fmaxf(s.m, top * c);
                float v = s.s * ex2(s.m - m);
#pragma unroll
                for (int i = 0; i < 8; ++i) v += ex2(fmaf(l[i], c, -m));
                s.m = m;
                s.s = v;
            };
            add(one[h], args.c1);
            if (STATS2) add(two[h], args.c2);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            one[h].join(__shfl_xor_sync(FULL, one[h].m, o), __shfl_xor_sync(FULL, one[h].s, o));
            if (STATS2) two[h].join(__shfl_xor_sync(FULL, two[h].m, o), __shfl_xor_sync(FULL, two[h].s, o));
        }
        if (q == 0) {
            joined[0][warp][g + 8 * h] = make_float2(one[h].m, one[h].s);
            joined[1][warp][g + 8 * h] = make_float2(two[h].m, two[h].s);
        }
    }
    __syncthreads();
    if (tid >= HEAD_FEW) return;
    const long long o = ((long long)t * gridDim.x + blockIdx.x) * args.Np + tid;
    Sum s, s2;
    for (int i = 0; i < FW_WARPS; ++i) {
        s.join(joined[0][i][tid].x, joined[0][i][tid].y);
        if (STATS2) s2.join(joined[1][i][tid].x, joined[1][i][tid].y);
    }
    args.part[o] = make_float2(s.m, s.s);
    if (STATS2) args.part2[o] = make_float2(s2.m, s2.s);
}

}  // namespace

int launch_head_few(const HeadPlan &h, const HeadGemm &in, const __nv_bfloat16 *z, const __nv_bfloat16 *w, cudaStream_t s) {
    HeadGemm g = in;
    g.Np = h.Np;
    g.V = h.V;
    g.d = h.d;
    g.c1 = h.c1;
    g.c2 = h.c2;
    const size_t smem = (size_t)HEAD_FEW * fw_pitch(h.d) * 2;
    static std::atomic<int> limit[2][64];
    auto kern = h.stats == 2 ? head_few_kernel<true> : head_few_kernel<false>;
    if (smem > 40 * 1024)
        if (const int st = raise_smem_limit((const void *)kern, limit[h.stats == 2], (int)smem)) return st;
    trace_before(s, "head_few");
    const int st = launch_kernel(kern, dim3(h.few, h.T), dim3(FW_THREADS), smem, s, g, z, w);
    trace_after(s);
    return st;
}

}  // namespace vmoe
