// norm.cu -- what surrounds an expert layer in its transformer block (Section 2.1:
// the experts stand in the place of a ViT block's MLP): the norm behind the branch,
// its gate and the residual, and the norm ahead of the next layer, in one pass.
//
//   w = norm(y; post_w, post_b)      (or w = y)
//   z = rho x + gate . w             (rounded to the tokens' dtype as it is stored)
//   u = norm(z; pre_w, pre_b)        (of z as stored, so that the backward, which has
//                                     only that, differentiates what was computed)
// norm(v) = (v - mean) rstd . weight + bias, rstd = 1 / sqrt(var + eps); the root-mean-
// square form has mean = 0.  With dzt = dz + (d u / d z)^T du:
//   dx = rho dzt,   dy = (d w / d y)^T (gate . dzt),
//   A = sum_n dzt . yhat,  B = sum_n dzt,
//   dpost_w = gate . A,  dpost_b = gate . B,  dgate = post_w . A + post_b . B,
//   dpre_w = sum_n du . zhat,  dpre_b = sum_n du.
// gate and weights do not depend on the token, so two sums a column carry the three
// gradients behind the branch.  Variances are sums of squared distances to the mean
// (two passes over registers), all sums fp32.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "around.cuh"

namespace cg = cooperative_groups;

namespace vmoe {

namespace {

// Eight consecutive elements as they lie in memory, and as four pairs of floats: the
// arithmetic runs on packed fp32 instructions, two elements each (60 instructions an
// element without them bound the forward at half the memory's rate, 30 do not).
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(f32x2 (&o)[4]) const {
        o[0] = bf16x2_to_f32x2(v.x);
        o[1] = bf16x2_to_f32x2(v.y);
        o[2] = bf16x2_to_f32x2(v.z);
        o[3] = bf16x2_to_f32x2(v.w);
    }
    __device__ __forceinline__ void set(const f32x2 (&in)[4]) {
        v = make_uint4(f32x2_to_bf16x2(in[0]), f32x2_to_bf16x2(in[1]), f32x2_to_bf16x2(in[2]), f32x2_to_bf16x2(in[3]));
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = v; }
};
template <>
struct Raw8<float> {
    ulonglong2 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const ulonglong2 *>(p)[0];
        b = reinterpret_cast<const ulonglong2 *>(p)[1];
    }
    __device__ __forceinline__ void zero() { a = b = make_ulonglong2(0, 0); }
    __device__ __forceinline__ void get(f32x2 (&o)[4]) const {
        o[0] = a.x;
        o[1] = a.y;
        o[2] = b.x;
        o[3] = b.y;
    }
    __device__ __forceinline__ void set(const f32x2 (&in)[4]) {
        a = make_ulonglong2(in[0], in[1]);
        b = make_ulonglong2(in[2], in[3]);
    }
    __device__ __forceinline__ void store(float *p) const {
        reinterpret_cast<ulonglong2 *>(p)[0] = a;
        reinterpret_cast<ulonglong2 *>(p)[1] = b;
    }
};

// Eight values of a [T, d] parameter, or a constant where there is none.
__device__ __forceinline__ void param8(const float *p, long long at, float none, f32x2 (&o)[4]) {
    Raw8<float> r;
    if (p) {
        r.load(p + at);
        r.get(o);
    } else {
        o[0] = o[1] = o[2] = o[3] = pk2(none);
    }
}

__device__ __forceinline__ float sum2(f32x2 v) {
    const float2 f = unpk2(v);
    return f.x + f.y;
}

template <int L>
__device__ __forceinline__ float lane_sum(float v) {  // over L neighbouring lanes
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// How rows lie on a CTA, forward and backward: W = ceil(d / 256) warps hold a row, or,
// up to 128 channels, 8 or 16 lanes; 8 columns a thread, so that a thread keeps its
// columns' parameters (and, in the backward, their gradients) in registers over all rows
// of the CTA's slice of a task.  A CTA has `groups` of such threads, each taking R rows
// at a time, with the next ones' loads in flight meanwhile.
int row_warps(int d) { return (d + 255) / 256; }
int row_threads(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32 * row_warps(d); }
int row_groups(int d) { return std::max(1, 128 / row_threads(d)); }
// Slices of a task's tokens: enough CTAs for `regs` registers a thread to fill 152 SMs
// once, and `least` steps for each.
int slices_of(const Dims &p, int R, int regs, int least) {
    const int groups = row_groups(p.d), threads = row_threads(p.d) * groups, rows = least * R * groups;
    const int resident = 152 * std::max(1, 65536 / (regs * threads));
    return std::max(1, std::min((p.N + rows - 1) / rows, resident / p.T));
}

// Rows at a time and CTAs of 128 threads an SM, for 1 to 4 warps a row.  Forward: two
// bf16 rows (one in fp32) and five CTAs; 33 us at 17 x 1576 tokens of 768 channels and 64
// at 8 x 6304 of 1024 without a post-norm, where four rows and four CTAs took 31 and 73, two
// rows and six CTAs 39 and 69.  Backward: two rows and three CTAs, 50 us at the former size
// (one row and three to five CTAs 56 to 60, before other steps that took 3 off both); fp32
// rows fill the registers of two CTAs: forward and backward of 3 x 1001 x 1000 26 us, 28 with
// one row and three CTAs, 8 x 4096 x 1024 205 and 209.
//
// Above 1024 channels the compiler does not know the number of warps: up to 16 of 128
// registers, with the next rows in flight, then 32 of 64 registers without (the backward
// spills 400 to 650 bytes a thread).  8 x 1576 x 1024, bf16, both norms: 20.0 us forward and
// 52.3 with the backward as above, 22.5 and 61.4 in the form for 16 warps; 4 x 1576 x 4096:
// 50.9 and 125 in that, 77.9 and 209 in the one for 32.  There bf16 rows still go in twos
// forward (29.0 us at 8 x 1576 x 1280, 42.7 one by one) and one by one backward (forward and
// backward 77.7 us, 86.0 in twos and 255 registers; 114 and 111 at 2048 channels).
constexpr int FR = 2, FB = 5, BR = 2, BB = 3, BB32 = 2;

struct FwdArgs {
    const void *x, *y;
    const float *post_w, *post_b, *gate, *pre_w, *pre_b;
    void *z, *u;
    float2 *post_stat, *pre_stat;
    float eps, rho;
    bool rms, post;
};

// Totals of R values over the W warps of a row, the same in every thread.  The first
// halvings of the butterfly sum two values at once; `buf` alternates between two
// halves, so one barrier a call is enough.
template <int WC, int L, int R>
struct Totals {
    float (*buf)[32][R];
    int first, flip;  // first warp of the group
    int W;            // WC, or where that is 0 the number of warps
    __device__ __forceinline__ void operator()(float (&v)[R]) {
        const int lane = threadIdx.x % L;
        int mine = 0;
#pragma unroll
        for (int h = R / 2, o = L / 2; h > 0; h >>= 1, o >>= 1) {
            const bool up = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < h; ++i) {
                const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
            mine += up ? h : 0;
        }
#pragma unroll
        for (int o = L / R / 2; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        float sum = v[0];
        if (WC != 1) {
            if (lane % (L / R) == 0) buf[flip][threadIdx.x >> 5][mine] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < (WC ? WC : W); ++w) sum += buf[flip][first + w][mine];
            flip ^= 1;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = __shfl_sync(0xffffffffu, sum, i * (L / R), L);
    }
};

// mean and rstd of R rows.
template <typename T, int WC, int L, int R>
__device__ __forceinline__ void stats(const Raw8<T> (&raw)[R], bool have, const FwdArgs &a, float share, Totals<WC, L, R> &totals,
                                      float2 (&s)[R]) {
    float m[R], q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) m[r] = 0.0f;
    if (!a.rms) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 v[4];
            raw[r].get(v);
            m[r] = have ? sum2(add2(add2(v[0], v[1]), add2(v[2], v[3]))) : 0.0f;
        }
        totals(m);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        f32x2 v[4], sq;
        raw[r].get(v);
        m[r] *= share;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = add2(v[i], pk2(-m[r]));
            sq = i ? fma2(v[i], v[i], sq) : mul2(v[i], v[i]);
        }
        q[r] = have ? sum2(sq) : 0.0f;
    }
    totals(q);
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = make_float2(m[r], rsqrtf(fmaf(q[r], share, a.eps)));
}

// The R rows' statistics, row by row of threads.
template <int R>
__device__ __forceinline__ void store_stats(float2 *out, const float2 (&s)[R], int th, int rows) {
    if (out == nullptr || th >= R || th >= rows) return;
    float2 o = s[0];
#pragma unroll
    for (int r = 1; r < R; ++r)
        if (th == r) o = s[r];
    out[th] = o;
}

template <typename T, int WC, int L, int MAXT, int MINB, int R, bool AHEAD>
__global__ void __launch_bounds__(MAXT, MINB)
norm_fwd_kernel(Dims p, FwdArgs a, int warps, int groups) {
    __shared__ float buf[2][32][R];
    const int W = WC ? WC : warps;
    const int group = threadIdx.x / (L * W), th = threadIdx.x - group * (L * W);
    const int t = blockIdx.y, N = p.N, d = p.d, c = 8 * th;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    const bool have = c < d;
    const float share = 1.0f / (float)d;
    Totals<WC, L, R> totals = {buf, group * W, 0, W};
    pdl_wait();
    const long long par = (long long)t * d + c, base = (long long)t * N;
    const T *x0 = (const T *)a.x + base * d, *y0 = (const T *)a.y + (a.y ? base * d : 0);
    T *z0 = (T *)a.z + (a.z ? base * d : 0), *u0 = (T *)a.u + (a.u ? base * d : 0);
    f32x2 post_w[4], post_b[4], pre_w[4], pre_b[4];
    {
        f32x2 gate[4];
        param8(have ? a.gate : nullptr, par, 1.0f, gate);
        param8(have ? a.post_w : nullptr, par, 1.0f, post_w);
        param8(have ? a.post_b : nullptr, par, 0.0f, post_b);
        param8(have ? a.pre_w : nullptr, par, 1.0f, pre_w);
        param8(have ? a.pre_b : nullptr, par, 0.0f, pre_b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            post_w[i] = mul2(post_w[i], gate[i]);
            post_b[i] = mul2(post_b[i], gate[i]);
        }
    }
    // Behind the last row and the last column others are read in their place, and what
    // comes of them is left out of the sums and not stored: predicated loads would cost
    // as many instructions again to zero their targets.  Offsets within a task fit 31 bits.
    const int cc = have ? c : 0;
    Raw8<T> nx[R], ny[R];
#pragma unroll
    for (int r = 0; r < R; ++r) ny[r].zero();
    auto fetch = [&](int n0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int at = min(n0 + group * R + r, end - 1) * d + cc;
            nx[r].load(x0 + at);
            if (a.y) ny[r].load(y0 + at);
        }
    };
    if (AHEAD && beg < end) fetch(beg);
    for (int n0 = beg; n0 < end; n0 += groups * R) {
        if (!AHEAD) fetch(n0);
        Raw8<T> x[R], y[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            x[r] = nx[r];
            y[r] = ny[r];
        }
        if (AHEAD && n0 + groups * R < end) fetch(n0 + groups * R);
        float2 s[R];
        const int n = n0 + group * R, rows = have ? end - n : 0, at = n * d + c;
        if (a.y) {
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] = make_float2(0.0f, 1.0f);
            if (a.post) {
                stats<T, WC, L, R>(y, have, a, share, totals, s);
                store_stats<R>(a.post_stat ? a.post_stat + base + n : nullptr, s, th, end - n);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f32x2 v[4], o[4];
                y[r].get(v);
                x[r].get(o);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o[i] = fma2(mul2(add2(v[i], pk2(-s[r].x)), pk2(s[r].y)), post_w[i], fma2(pk2(a.rho), o[i], post_b[i]));
                x[r].set(o);
                if (r < rows) x[r].store(z0 + at + r * d);
            }
        }
        if (!a.u) continue;
        stats<T, WC, L, R>(x, have, a, share, totals, s);
        store_stats<R>(a.pre_stat ? a.pre_stat + base + n : nullptr, s, th, end - n);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 v[4];
            x[r].get(v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fma2(mul2(add2(v[i], pk2(-s[r].x)), pk2(s[r].y)), pre_w[i], pre_b[i]);
            x[r].set(v);
            if (r < rows) x[r].store(u0 + at + r * d);
        }
    }
}

// ---------------------------------------------------------------------------
// Backward.  The four column sums stay in registers; a CTA's go to `parts`
// [T][slices][4][d]: A, B, dpre_w, dpre_b.
//
// With g = du . pre_w, e = dz + r_z g and aw = gate . post_w, the gradient behind the
// pre-norm is dzt = e - r_z (m1 + m2 zhat), m1 = sum g / d, m2 = sum g zhat / d, and what
// the post-norm needs of q = dzt . aw follows from sums over e, zhat and yhat:
//   sum q      = sum e aw - r_z (m1 sum aw + m2 sum zhat aw)
//   sum q yhat = sum e aw yhat - r_z (m1 sum aw yhat + m2 sum zhat aw yhat),
// so seven sums a row, taken together, replace two rounds of two that wait for one another.
// What the column sums of a task become.
struct JoinArgs {
    const float *parts, *post_w, *post_b, *gate;
    float *dpost_w, *dpost_b, *dgate, *dpre_w, *dpre_b;
    __device__ __forceinline__ void store(long long at, const float (&s)[4]) const {
        const float g = gate ? gate[at] : 1.0f, w = post_w ? post_w[at] : 1.0f, b = post_b ? post_b[at] : 0.0f;
        if (dpost_w) dpost_w[at] = g * s[0];
        if (dpost_b) dpost_b[at] = g * s[1];
        if (dgate) {  // a weight or a bias of 0, or none, adds nothing, also where the other sum is infinite
            const float bs = b == 0.0f && isinf(s[1]) ? 0.0f : b * s[1];
            dgate[at] = w == 0.0f && isinf(s[0]) ? bs : fmaf(w, s[0], bs);
        }
        if (dpre_w) dpre_w[at] = s[2];
        if (dpre_b) dpre_b[at] = s[3];
    }
};

struct BwdArgs {
    const void *y, *z;
    const float2 *post_stat, *pre_stat;
    const float *post_w, *post_b, *gate, *pre_w;
    const void *dz, *du;
    void *dx, *dy;
    float *parts;  // NULL: the slices are a cluster, which joins its sums itself
    JoinArgs join;
    float rho;
    bool rms, post;
};

int bwd_rows(const Dims &p) { return row_warps(p.d) <= 4 ? BR : 1; }
// Short tasks are a cluster of up to CLUSTER CTAs with at most JOIN_STEPS steps each, which
// joins its sums itself: one launch (the second costs the host 1.9 us).  On the GPU 4 to 8
// steps in all took 3.7 to 4.7 us so and 4.7 to 5.1 in two launches, 16 steps 4.8 to 6.0 and
// 4.6 to 5.0, 32 steps 6.1 to 8.1 and 4.8 to 6.1 (1 to 17 tasks, 128 to 1024 channels).
constexpr int CLUSTER = 8, JOIN_STEPS = 2;
bool bwd_cluster(const Dims &p) {
    return p.d <= 1024 && (p.N + bwd_rows(p) * row_groups(p.d) - 1) / (bwd_rows(p) * row_groups(p.d)) <= CLUSTER * JOIN_STEPS;
}
int bwd_slices(const Dims &p) {
    const int W = row_warps(p.d);
    if (bwd_cluster(p)) {
        const int steps = (p.N + bwd_rows(p) * row_groups(p.d) - 1) / (bwd_rows(p) * row_groups(p.d));
        int n = 1;  // no more than there are rows: a slice has one at least
        while (n < CLUSTER && 2 * n <= steps) n *= 2;
        return n;
    }
    return slices_of(p, bwd_rows(p), W <= 4 ? 512 / (p.bf16 ? BB : BB32) : W <= 16 ? 128 : 64, 2);
}

// Totals of 8 R values over L lanes: each halving step sums two lanes' values and keeps
// half of them, 16 shuffles for 16 totals.  Lane l ends with value l % 8 R; eight lanes
// with value l of each row.
template <int L, int R>
__device__ __forceinline__ void lane_totals(float (&v)[8 * R], float (&sum)[R]) {
    constexpr int M = L < 8 * R ? 8 : 8 * R;
    const int lane = threadIdx.x % L;
#pragma unroll
    for (int r = 0; r < 8 * R / M; ++r) {
        float *x = v + M * r;
#pragma unroll
        for (int h = M / 2; h > 0; h >>= 1) {
            const bool up = (lane & h) != 0;
#pragma unroll
            for (int i = 0; i < h; ++i) {
                const float give = up ? x[i] : x[i + h], keep = up ? x[i + h] : x[i];
                x[i] = keep + __shfl_xor_sync(0xffffffffu, give, h);
            }
        }
#pragma unroll
        for (int o = M; o < L; o <<= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
        sum[r] = x[0];
    }
}

template <typename T>
struct BwdRow {
    Raw8<T> y, z, dz, du;
    float2 py, pz;  // mean, rstd
    __device__ __forceinline__ void zero() {
        y.zero();
        z.zero();
        dz.zero();
        du.zero();
        py = pz = make_float2(0.0f, 0.0f);
    }
};

// POST: there is a branch and it has a norm.  ALL: and every input is there, known to the
// compiler (49 us at 17 x 1576 tokens of 768 channels, 55 without).
template <typename T, int WC, int L, int MAXT, int MINB, int R, bool AHEAD, bool POST, bool ALL>
__global__ void __launch_bounds__(MAXT, MINB)
norm_bwd_kernel(Dims p, BwdArgs a, int warps, int groups) {
    __shared__ float totals[2][32][16];
    extern __shared__ __align__(16) float join[];  // [max(1, groups - 1)][4][d]: the groups' sums, then the CTA's
    const int W = WC ? WC : warps;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x / (L * W), th = threadIdx.x - group * (L * W);
    const int t = blockIdx.y, N = p.N, d = p.d, c = 8 * th;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    const bool have = c < d;
    const float share = 1.0f / (float)d, centre = a.rms ? 0.0f : share;
    const bool has_u = ALL || a.du != nullptr, has_z = ALL || a.dz != nullptr, has_y = POST || a.y != nullptr;
    pdl_wait();
    f32x2 pw[4], aw[4];  // pre_w; gate . post_w
    float sum_aw;
    {
        const long long par = (long long)t * d + c;
        f32x2 g[4];
        param8(have ? a.pre_w : nullptr, par, 1.0f, pw);
        param8(have ? a.gate : nullptr, par, 1.0f, g);
        param8(have ? a.post_w : nullptr, par, 1.0f, aw);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // behind the last column 0, for the sums
            aw[i] = have ? mul2(aw[i], g[i]) : 0;
            pw[i] = have ? pw[i] : 0;
        }
        sum_aw = lane_sum<L>(sum2(add2(add2(aw[0], aw[1]), add2(aw[2], aw[3]))));
        if (WC != 1) {
            if (lane == 0) totals[0][warp][0] = sum_aw;
            __syncthreads();
            sum_aw = 0.0f;
            for (int w = 0; w < W; ++w) sum_aw += totals[0][group * W + w][0];
            __syncthreads();
        }
    }
    f32x2 A[4] = {}, B[4] = {}, Pw[4] = {}, Pb[4] = {};
    // as in the forward, others are read in the place of what lies behind the end; rows there
    // become zeros before they are used (a branch that the last step of a slice takes)
    const int cc = have ? c : 0;
    const long long base = (long long)t * N;
    auto task = [&](const void *p) { return (const T *)p + (p ? base * d : 0); };
    const T *y0 = task(a.y), *z0 = task(a.z), *dz0 = task(a.dz), *du0 = task(a.du);
    T *dx0 = (T *)task(a.dx), *dy0 = (T *)task(a.dy);
    const float2 *py0 = a.post_stat + (a.post_stat ? base : 0), *pz0 = a.pre_stat + (a.pre_stat ? base : 0);
    BwdRow<T> next[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        next[r].zero();
        next[r].py.y = next[r].pz.y = 1.0f;
    }
    auto fetch = [&](int n0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = min(n0 + group * R + r, end - 1), at = n * d + cc;
            if (has_u) {
                next[r].du.load(du0 + at);
                next[r].z.load(z0 + at);
                next[r].pz = pz0[n];
            }
            if (has_z) next[r].dz.load(dz0 + at);
            if (has_y) {
                next[r].y.load(y0 + at);
                if (POST) next[r].py = py0[n];
            }
        }
    };
    if (AHEAD && beg < end) fetch(beg);
    int flip = 0;
    for (int n0 = beg; n0 < end; n0 += groups * R, flip ^= 1) {
        if (!AHEAD) fetch(n0);
        f32x2 e[R][4], zh[R][4], yh[R][4];
        float rz[R], ry[R], v[8 * R];
        if (n0 + groups * R > end) {  // zeros add nothing to the columns' sums
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (n0 + group * R + r >= end) next[r].zero();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rz[r] = next[r].pz.y;
            ry[r] = next[r].py.y;
            const f32x2 mz = pk2(-next[r].pz.x), my = pk2(-next[r].py.x);
            f32x2 du[4], s[7];
            next[r].dz.get(e[r]);
            next[r].du.get(du);
            next[r].z.get(zh[r]);
            next[r].y.get(yh[r]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                zh[r][i] = mul2(add2(zh[r][i], mz), pk2(rz[r]));
                yh[r][i] = mul2(add2(yh[r][i], my), pk2(ry[r]));
                Pw[i] = fma2(du[i], zh[r][i], Pw[i]);
                Pb[i] = add2(Pb[i], du[i]);
                const f32x2 g = mul2(du[i], pw[i]);
                e[r][i] = fma2(pk2(rz[r]), g, e[r][i]);
                s[0] = i ? add2(s[0], g) : g;
                s[1] = i ? fma2(g, zh[r][i], s[1]) : mul2(g, zh[r][i]);
                if (!POST) continue;  // the others are for the norm on the branch
                const f32x2 ea = mul2(e[r][i], aw[i]), za = mul2(zh[r][i], aw[i]);
                s[2] = i ? add2(s[2], ea) : ea;
                s[3] = i ? fma2(ea, yh[r][i], s[3]) : mul2(ea, yh[r][i]);
                s[4] = i ? add2(s[4], za) : za;
                s[5] = i ? fma2(aw[i], yh[r][i], s[5]) : mul2(aw[i], yh[r][i]);
                s[6] = i ? fma2(za, yh[r][i], s[6]) : mul2(za, yh[r][i]);
            }
#pragma unroll
            for (int i = 0; i < 7; ++i) v[8 * r + i] = POST || i < 2 ? sum2(s[i]) : 0.0f;
            v[8 * r + 7] = 0.0f;
        }
        if (AHEAD && n0 + groups * R < end) fetch(n0 + groups * R);
        float sum[R];
        lane_totals<L, R>(v, sum);
        if (WC != 1) {
            if (lane < 8 * R) totals[flip][warp][lane] = sum[0];
            __syncthreads();  // the other half is written next: one barrier a step
            sum[0] = 0.0f;
#pragma unroll
            for (int w = 0; w < (WC ? WC : W); ++w) sum[0] += totals[flip][group * W + w][lane & (8 * R - 1)];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s[7];
#pragma unroll
            for (int i = 0; i < 7; ++i) s[i] = L < 8 * R ? __shfl_sync(0xffffffffu, sum[r], i, L) : __shfl_sync(0xffffffffu, sum[0], 8 * r + i, L);
            const int n = n0 + group * R + r;
            const float z1 = has_u ? rz[r] : 0.0f, m1 = z1 * centre * s[0], m2 = z1 * share * s[1];
            const float k1 = POST ? centre * (s[2] - m1 * sum_aw - m2 * s[4]) : 0.0f;
            const float k2 = POST ? share * (s[3] - m1 * s[5] - m2 * s[6]) : 0.0f;
            f32x2 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[r][i] = fma2(pk2(-m2), zh[r][i], add2(e[r][i], pk2(-m1)));
                A[i] = fma2(e[r][i], yh[r][i], A[i]);
                B[i] = add2(B[i], e[r][i]);
                const f32x2 ea = mul2(e[r][i], aw[i]);  // dy without a norm, whatever y holds
                q[i] = POST ? mul2(pk2(ry[r]), fma2(pk2(-k2), yh[r][i], fma2(e[r][i], aw[i], pk2(-k1)))) : ea;
                if (has_y) e[r][i] = mul2(e[r][i], pk2(a.rho));
            }
            if (have && n < end) {
                const int at = n * d + c;
                Raw8<T> o;
                o.set(e[r]);
                o.store(dx0 + at);
                if (has_y) {
                    o.set(q);
                    o.store(dy0 + at);
                }
            }
        }
    }
    // the groups' sums, in their order
    __syncthreads();
    Raw8<float> r;
    auto put = [&](float *o) {
        r.set(A);
        r.store(o);
        r.set(B);
        r.store(o + d);
        r.set(Pw);
        r.store(o + 2 * d);
        r.set(Pb);
        r.store(o + 3 * d);
    };
    if (group > 0 && have) put(join + (long long)(group - 1) * 4 * d + c);
    __syncthreads();
    const bool first = group == 0 && have;
    for (int g = 1; g < (first ? groups : 1); ++g) {
        const float *o = join + (long long)(g - 1) * 4 * d + c;
        auto add = [&](f32x2 (&to)[4], const float *from) {
            f32x2 f[4];
            r.load(from);
            r.get(f);
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = add2(to[i], f[i]);
        };
        add(A, o);
        add(B, o + d);
        add(Pw, o + 2 * d);
        add(Pb, o + 3 * d);
    }
    if (a.parts != nullptr) {
        if (first) put(a.parts + ((long long)t * gridDim.x + blockIdx.x) * 4 * d + c);
        return;
    }
    if (first) put(join + c);  // a thread overwrites what it alone has read
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int ranks = (int)cluster.num_blocks();
    for (int i = (int)cluster.block_rank() * blockDim.x + threadIdx.x; i < d; i += ranks * blockDim.x) {
        float s[4] = {};
        for (int q = 0; q < ranks; ++q) {
            const float *in = cluster.map_shared_rank(join, q);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += in[j * d + i];
        }
        a.join.store((long long)t * d + i, s);
    }
    cluster.sync();  // the sums stay until they are read
}

// The slices' column sums joined: 32 columns a CTA, JOIN threads a column, each a run
// of the slices.
constexpr int JOIN = 16;
__global__ void __launch_bounds__(32 * JOIN)
norm_join_kernel(Dims p, JoinArgs a, int slices) {
    __shared__ float part[JOIN][4][32];
    const int lane = threadIdx.x & 31, q = threadIdx.x >> 5, d = p.d, t = blockIdx.y, c = blockIdx.x * 32 + lane;
    const int beg = slices * q / JOIN, end = slices * (q + 1) / JOIN;
    pdl_wait();
    float s[4] = {};
    if (c < d)
#pragma unroll 4
        for (int i = beg; i < end; ++i) {
            const float *in = a.parts + ((long long)t * slices + i) * 4 * d + c;
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += in[(long long)j * d];
        }
#pragma unroll
    for (int j = 0; j < 4; ++j) part[q][j][lane] = s[j];
    __syncthreads();
    if (q > 0 || c >= d) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < JOIN; ++i) s[j] += part[i][j][lane];
    }
    a.store((long long)t * d + c, s);
}

template <typename T>
int run_fwd(const Dims &p, const FwdArgs &a, cudaStream_t s) {
    constexpr int R = sizeof(T) == 2 ? FR : FR / 2;
    const int W = row_warps(p.d), groups = row_groups(p.d), threads = row_threads(p.d) * groups;
    auto go = [&](auto kern, int rows, int regs) {
        return launch_kernel(kern, dim3(slices_of(p, rows, regs, 1), p.T), dim3(threads), 0, s, p, a, W, groups);
    };
    if (p.d <= 64) return go(norm_fwd_kernel<T, 1, 8, 128, FB, R, true>, R, 512 / FB);
    if (p.d <= 128) return go(norm_fwd_kernel<T, 1, 16, 128, FB, R, true>, R, 512 / FB);
    switch (W) {
        case 1: return go(norm_fwd_kernel<T, 1, 32, 128, FB, R, true>, R, 512 / FB);
        case 2: return go(norm_fwd_kernel<T, 2, 32, 128, FB, R, true>, R, 512 / FB);
        case 3: return go(norm_fwd_kernel<T, 3, 32, 96, FB * 4 / 3, R, true>, R, 512 / FB);
        case 4: return go(norm_fwd_kernel<T, 4, 32, 128, FB, R, true>, R, 512 / FB);
    }
    if (W <= 16) return go(norm_fwd_kernel<T, 0, 32, 512, 1, R, true>, R, 128);
    return go(norm_fwd_kernel<T, 0, 32, 1024, 1, 1, false>, 1, 64);
}

template <typename T, int WC, int L, int MAXT, int MINB, int R>
int launch_bwd(const Dims &p, const BwdArgs &a, cudaStream_t s) {
    const int W = row_warps(p.d), groups = row_groups(p.d), slices = bwd_slices(p);
    const dim3 grid(slices, p.T), block(row_threads(p.d) * groups);
    auto go = [&](auto kern) {
        if (a.parts) return launch_kernel(kern, grid, block, (size_t)(groups - 1) * 4 * p.d * sizeof(float), s, p, a, W, groups);
        return launch_cluster(kern, grid, block, (size_t)std::max(1, groups - 1) * 4 * p.d * sizeof(float), slices, s, p, a, W, groups);
    };
    if (!a.y || !a.post) return go(norm_bwd_kernel<T, WC, L, MAXT, MINB, R, MAXT <= 512, false, false>);
    if (WC && a.du && a.dz) return go(norm_bwd_kernel<T, WC, L, MAXT, MINB, R, MAXT <= 512, true, WC != 0>);
    return go(norm_bwd_kernel<T, WC, L, MAXT, MINB, R, MAXT <= 512, true, false>);
}
template <typename T>
int run_bwd(const Dims &p, const BwdArgs &a, cudaStream_t s) {
    constexpr int R = BR, B = sizeof(T) == 2 ? BB : BB32;
    if (p.d <= 64) return launch_bwd<T, 1, 8, 128, B, R>(p, a, s);
    if (p.d <= 128) return launch_bwd<T, 1, 16, 128, B, R>(p, a, s);
    const int W = row_warps(p.d);
    switch (W) {
        case 1: return launch_bwd<T, 1, 32, 128, B, R>(p, a, s);
        case 2: return launch_bwd<T, 2, 32, 128, B, R>(p, a, s);
        case 3: return launch_bwd<T, 3, 32, 96, B * 4 / 3, R>(p, a, s);
        case 4: return launch_bwd<T, 4, 32, 128, B, R>(p, a, s);
    }
    if (W <= 16) return launch_bwd<T, 0, 32, 512, 1, 1>(p, a, s);
    return launch_bwd<T, 0, 32, 1024, 1, 1>(p, a, s);
}

}  // namespace

size_t norm_bwd_workspace(const Dims &p) {
    return bwd_cluster(p) ? 16 : (size_t)p.T * bwd_slices(p) * 4 * p.d * sizeof(float);
}

int launch_block_norm(const Dims &p, const vmoe_norm *n, const void *x, const void *y, const float *post_w,
                      const float *post_b, const float *gate, const float *pre_w, const float *pre_b, void *z, void *u,
                      float *post_stat, float *pre_stat, cudaStream_t s) {
    const FwdArgs a = {x, y, post_w, post_b, gate, pre_w, pre_b, z, u, (float2 *)post_stat, (float2 *)pre_stat,
                       n->eps, n->residual_scale, (n->flags & VMOE_NORM_RMS) != 0, (n->flags & VMOE_NORM_POST) != 0};
    trace_before(s, "block_norm");
    const int st = p.bf16 ? run_fwd<__nv_bfloat16>(p, a, s) : run_fwd<float>(p, a, s);
    trace_after(s);
    return st;
}

int launch_block_norm_bwd(const Dims &p, const vmoe_norm *n, const void *y, const void *z, const float *post_stat,
                          const float *pre_stat, const float *post_w, const float *post_b, const float *gate,
                          const float *pre_w, const void *dz, const void *du, void *dx, void *dy, float *dpost_w,
                          float *dpost_b, float *dgate, float *dpre_w, float *dpre_b, float *parts, cudaStream_t s) {
    const bool cluster = bwd_cluster(p);
    const JoinArgs j = {parts, post_w, post_b, gate, dpost_w, dpost_b, dgate, dpre_w, dpre_b};
    const BwdArgs a = {y, z, (const float2 *)post_stat, (const float2 *)pre_stat, post_w, post_b, gate, pre_w, dz, du,
                       dx, dy, cluster ? nullptr : parts, j, n->residual_scale, (n->flags & VMOE_NORM_RMS) != 0,
                       (n->flags & VMOE_NORM_POST) != 0};
    trace_before(s, "block_norm_bwd");
    int st = p.bf16 ? run_bwd<__nv_bfloat16>(p, a, s) : run_bwd<float>(p, a, s);
    trace_after(s);
    if (st != VMOE_OK || cluster || !(dpost_w || dpost_b || dgate || dpre_w || dpre_b)) return st;
    trace_before(s, "block_norm_join");
    st = launch_kernel(norm_join_kernel, dim3((p.d + 31) / 32, p.T), dim3(32 * JOIN), 0, s, p, j, bwd_slices(p));
    trace_after(s);
    return st;
}

}  // namespace vmoe
