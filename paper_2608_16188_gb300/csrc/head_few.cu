// head_few.cu -- the sums of a head's logits for a few tokens, as a served model scores or answers with them:
//
//   l = z w^T for at most 16 tokens, of which the largest value, the sum of exponentials and the label's logit stay
//
// What bounds it is the weights' way from DRAM, read once: V d 2 bytes.  A warp streams 32 rows of w at a time, whole rows
// that lie together, straight into the B fragments of mma.sync m16n8k16: a lane's 16 bytes are eight neighbouring
// k of one row, which the products take in an order of their own (two of four k each: any order of the sum will do, if A
// has the same); the tokens, 16 rows, are A, from shared memory.  A lane keeps the running maximum and sum of its two
// tokens, a CTA leaves one of each.
// 4 tokens, 128000 entries, d 1024 (262 MB, 38.6 us at the copy rate): 48 us, and 46 for the whole pass, whose packing runs
// under the first rows' way from DRAM; as 256 x 256 tiles of head_tc.cu, whose 128-byte pieces of 19000 rows at a time lose
// DRAM's pages, 57.
// fp32: a lane's eight values are split into three bf16 parts on their way, 16 rows at a time, for six products each; nothing
// but the weights themselves is read.  8 tokens, 50000 entries, d 1024 (205 MB, 30 us): 85 us the pass, bound by the splits'
// and products' issue; with the weights' parts written first and head_tc.cu 191.
#include "head.cuh"

namespace vmoe {
namespace {

constexpr int FW_THREADS = 256, FW_WARPS = FW_THREADS / 32;
constexpr int fw_tiles(int parts) { return parts == 1 ? 4 : 2; }              // of 8 rows of w, a warp at a time
constexpr int fw_ahead(int parts) { return 1536 * 4 / fw_tiles(parts); }      // bytes of a row of w that are fetched ahead
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

// Eight values of a row of w as the B fragments of their parts.
template <int PARTS>
struct Values;
template <>
struct Values<1> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool on) {
        v = make_uint4(0, 0, 0, 0);
        if (on) v = __ldcs(reinterpret_cast<const uint4 *>(p));
    }
    __device__ __forceinline__ void get(uint4 (&o)[1]) const { o[0] = v; }
};
template <>
struct Values<3> {
    float4 v[2];
    __device__ __forceinline__ void load(const float *p, bool on) {
        v[0] = v[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (on) v[0] = __ldcs(reinterpret_cast<const float4 *>(p)), v[1] = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void get(uint4 (&o)[3]) const {
        const float f[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
        split_weights(f, o);
    }
};

template <bool STATS2, int PARTS, typename W>
__global__ void __launch_bounds__(FW_THREADS, 2)
head_few_kernel(HeadGemm args, const __nv_bfloat16 *__restrict__ z, const W *__restrict__ w) {
    constexpr int NT = fw_tiles(PARTS), ROWS = 8 * NT;
    extern __shared__ __align__(16) __nv_bfloat16 fw_z[];  // [parts][16][pitch]
    __shared__ float2 joined[2][FW_WARPS][HEAD_FEW];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
    const int d = args.d, V = args.V, pitch = fw_pitch(d);
    const W *wt = w + (long long)t * V * d;
    // The warp's first rows, a lane each, on their way into L2 while head_pack runs: at most 120 MB of its 129 (2432 warps).
    // A pass of 4 tokens, 128000 entries, d 1024: 60.7 us without, 58.9 with 256 bytes a row, 57.4 with 512, 54.4 with 1024,
    // 52.2 with 1536 or 1792.  Fetched ahead all the way, a block's rows under the products of the last: 62.
    const int first = (blockIdx.x * FW_WARPS + warp) * ROWS + lane;
    if (lane < ROWS && first < V)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(__cvta_generic_to_global(wt + (long long)first * d)),
                     "r"(min(d * (int)sizeof(W), fw_ahead(PARTS)))
                     : "memory");
    pdl_wait();
    pdl_launch_dependents();
    const long long plane = (long long)args.T * args.Np * d;
    for (int i = tid; i < PARTS * HEAD_FEW * (pitch / 8); i += FW_THREADS) {
        const int r = i / (pitch / 8), c = (i - r * (pitch / 8)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c < d) v = __ldg(reinterpret_cast<const uint4 *>(z + r / HEAD_FEW * plane + ((long long)t * args.Np + r % HEAD_FEW) * d + c));
        *reinterpret_cast<uint4 *>(fw_z + r * pitch + c) = v;
    }
    if (args.rows[t] == 0) return;  // nothing was packed, and nothing is read
    __syncthreads();
    const long long at = (long long)t * args.Np + g;
    const int lab[2] = {args.label ? __ldg(args.label + at) : -1, args.label ? __ldg(args.label + at + 8) : -1};
    const __nv_bfloat16 *za = fw_z + g * pitch + 8 * q, *zb = za + 8 * pitch;
    Sum one[2], two[2];
    const int blocks = (V + ROWS - 1) / ROWS;
    for (int b = blockIdx.x * FW_WARPS + warp; b < blocks; b += gridDim.x * FW_WARPS) {
        const int v0 = b * ROWS;
        const W *row[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) row[n] = wt + (long long)min(V - 1, v0 + 8 * n + g) * d + 8 * q;
        float sum[NT][4] = {};
        constexpr int U = 4;  // steps of 32 k in flight: 8 KB a warp
        for (int k0 = 0; k0 < d; k0 += 32 * U) {
            Values<PARTS> x[U][NT];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n) x[u][n].load(row[n] + k0 + 32 * u, k0 + 32 * u + 8 * q < d);
            // 128 k at a time: the products cut every step of their sums towards zero (all 1024 in one: ce off by 1.1e-6; so 1e-7);
            // fp32: the large product 32 at a time (128: logits off by 3e-7 of themselves), the five small ones apart
            float acc[NT][4] = {}, low[NT][4] = {};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k0 + 32 * u >= d) break;
                uint4 a[PARTS], c[PARTS];
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    a[p] = *reinterpret_cast<const uint4 *>(za + p * HEAD_FEW * pitch + k0 + 32 * u);
                    c[p] = *reinterpret_cast<const uint4 *>(zb + p * HEAD_FEW * pitch + k0 + 32 * u);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 w8[PARTS];
                    x[u][n].get(w8);
                    auto product = [&](float(&o)[4], int i, int j) {
                        mma_bf16_16816(o, a[i].x, c[i].x, a[i].y, c[i].y, w8[j].x, w8[j].y);
                        mma_bf16_16816(o, a[i].z, c[i].z, a[i].w, c[i].w, w8[j].z, w8[j].w);
                    };
                    if constexpr (PARTS == 3) {
                        product(low[n], 2, 0), product(low[n], 0, 2), product(low[n], 1, 1);
                        product(low[n], 1, 0), product(low[n], 0, 1);
                    }
                    product(acc[n], 0, 0);
                    if constexpr (PARTS == 3) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            sum[n][i] += acc[n][i];
                            acc[n][i] = 0.0f;
                        }
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[n][i] += PARTS == 3 ? low[n][i] : acc[n][i];
        }
        // columns v0 + 8 n + 2 q, + 1 of tokens g (0, 1) and g + 8 (2, 3)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float l[2 * NT], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i) {
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
                for (int i = 0; i < 2 * NT; ++i) v += ex2(fmaf(l[i], c, -m));
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

template <bool STATS2, int PARTS, typename W>
int launch_few(const HeadPlan &h, const HeadGemm &g, const __nv_bfloat16 *z, const void *w, cudaStream_t s) {
    const size_t smem = (size_t)PARTS * HEAD_FEW * fw_pitch(h.d) * 2;
    static std::atomic<int> limit[64];
    auto kern = head_few_kernel<STATS2, PARTS, W>;
    if (smem > 40 * 1024)
        if (const int st = raise_smem_limit((const void *)kern, limit, (int)smem)) return st;
    return launch_kernel(kern, dim3(h.few, h.T), dim3(FW_THREADS), smem, s, g, z, (const W *)w);
}

}  // namespace

int launch_head_few(const HeadPlan &h, const HeadGemm &in, const __nv_bfloat16 *z, const void *w, cudaStream_t s) {
    HeadGemm g = in;
    g.T = h.T;
    g.Np = h.Np;
    g.V = h.V;
    g.d = h.d;
    g.c1 = h.c1;
    g.c2 = h.c2;
    trace_before(s, "head_few");
    const int st = h.parts == 1 ? (h.stats == 2 ? launch_few<true, 1, __nv_bfloat16>(h, g, z, w, s)
                                                : launch_few<false, 1, __nv_bfloat16>(h, g, z, w, s))
                                : (h.stats == 2 ? launch_few<true, 3, float>(h, g, z, w, s) : launch_few<false, 3, float>(h, g, z, w, s));
    trace_after(s);
    return st;
}

}  // namespace vmoe
