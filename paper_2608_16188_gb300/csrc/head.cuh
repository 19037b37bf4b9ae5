// head.cuh -- a head over a large vocabulary: shared declarations of its matrix products (head_tc.cu) and of what is
// around them (head.cu) (internal).
#pragma once

#include "common.cuh"

namespace vmoe {

constexpr int HEAD_K = 128;     // entries of a teacher's list at most
constexpr int HEAD_V = 1 << 20;  // entries of a vocabulary at most, with a teacher
constexpr int HEAD_FEW = 16;    // tokens of a head at most for head_few
// A few bf16 tokens a head (head_plan has the rule) have two rows each in the backward: token r (packed) row 32 (r / 16) + r % 16
// and the one 16 behind it, which a warp of an epilogue has both of.  z is the same in both, dl in the second what rounding
// takes from the first: it is then kept to 2^-16, and the sums need no other code.  map is -1 for the second.
constexpr int HEAD_HALF = 16;
__host__ __device__ constexpr int two_row(int r) { return 2 * HEAD_HALF * (r / HEAD_HALF) + r % HEAD_HALF; }
__host__ __device__ constexpr int two_token(int row) { return HEAD_HALF * (row / (2 * HEAD_HALF)) + row % HEAD_HALF; }
constexpr int HEAD_TILE = 256;  // rows and columns of a product's tile
constexpr int HEAD_BLOCK = 64;  // of its sum that are loaded at a time

// Eight fp32 weights as three bf16 parts each.  A part that would round to infinity is the largest finite value: of fp32's lowest
// value, and of -inf, the usual weights of entries that are switched off, plain rounding leaves -inf and then -inf - -inf, NaN.
__device__ __forceinline__ void split_weights(const float (&f)[8], uint4 (&o)[3]) {
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = f[2 * i], b = f[2 * i + 1];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(w[q][i]) : "f"(b), "f"(a));
            const float2 h = unpk2(bf16x2_to_f32x2(w[q][i]));
            a -= h.x;
            b -= h.y;
        }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) o[q] = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
}

// Sizes of a call, and where its scratch lies in the workspace (byte offsets).
struct HeadPlan {
    int T, N, d, V, K;   // heads, tokens of a head (all tasks' with a shared one), width, vocabulary, teacher's entries
    int Np;              // N in whole tiles: row pitch of what holds tokens
    int parts;           // bf16 parts of a value: 1, or 3 (fp32)
    int two;             // backward, 1: two rows a token, see HEAD_HALF
    int stats;           // sums of a row: 1, or 2 (labels and a teacher at another temperature)
    int piece;           // backward: columns of a piece of the vocabulary, whole tiles
    int pairs;           // backward: SM pairs, at most, that dz is shared out to; 0: in pieces of the vocabulary
    int few;             // forward: CTAs a head of head_few, 0: HEAD_STATS
    float tau;           // the temperature
    float c1, c2;        // log2(e), log2(e) / temperature
    size_t rows, mark, pos, map, label, z, w;  // both ways
    size_t part, part2, picked, off, list, tl; // forward
    size_t coef, at_label, dl, dzp;            // backward
    size_t bytes;
};

// One product of the head's, for launch_head_gemm.
enum { HEAD_STATS = 0, HEAD_DLOGITS = 1, HEAD_DZ = 2, HEAD_DW = 3 };
struct HeadGemm {
    int T, Np, V, d, parts, np;   // np: products of parts
    int two;
    const int *rows;              // [2][T] rows of tokens that take part, and those tokens
    int v0, vn;                   // the piece: first column, columns
    int tiles_n, tiles_m;         // tiles of columns; HEAD_DW: of rows
    int pairs, first;             // HEAD_DZ: SM pairs; whether this is the first piece
    int overlap;                  // HEAD_DZ: HEAD_DW follows and may run beside it; HEAD_DW: behind such a one
    float c1, c2;
    const int *label;             // [T][Np] of compact rows, -1: none
    float2 *part;                 // HEAD_STATS out: [T][2 tiles_n][Np] largest logit times c1, sum
    float2 *part2;                // the same at c2
    float *picked;                // [T][Np] the label's logit
    int K;                        // the teacher's entries: their logits go to tl [T][Np][K]
    const int *off;               // [T][Np / 32][2 tiles_n + 1] where each half tile's entries of 32 rows begin in list
    const unsigned *list;         // [T][Np / 32][32 K] row | column in the half tile << 5 | entry << 12
    float *tl;
    const float4 *coef;           // HEAD_DLOGITS: a, lse times log2(e), b, tlse times log2(e) of a row; infinite logarithms where a, b is 0
    const float *at_label;        // the first sum's share of the gradient there
    float *out;                   // HEAD_DZ: in pieces [T][Np][d], else [pairs][256][256] parts of tiles; HEAD_DW, fp32: [T][V][d]
    void *dz;                     // HEAD_DZ in one go: [T][N][d], row map[t][r] of it
    const int *map;
    int N;
    int *status;
};

// HEAD_DZ in one go has tiles for all SM pairs at once for a while, and then `left` more: their sums, of kb blocks each, are
// cut into `cuts` equal parts while there are pairs for them and a part keeps `least` blocks.  Pair c takes part c / left of
// tile c % left, so that neighbours go through the same weights and rows together, and leaves it in out[c].  (Equal shares
// of all the blocks left over, with cuts anywhere, fill the pairs better and lose that: a frozen head of 50304 entries, 64
// tiles over 76 pairs, 225 -> 342 us; 17 tasks of 32000, 53 tiles left, 815 -> 925.)
constexpr int dz_least(int parts) { return parts == 1 ? 16 : 8; }
struct DzShares {
    int full, left, kb, cuts;
    __host__ __device__ DzShares(int tiles, int pairs, int kb_, int least) {
        kb = kb_;
        left = tiles % pairs;
        full = tiles - left;
        cuts = left ? pairs / left : 1;
        if (cuts > kb / least) cuts = kb / least;
        if (cuts < 1) cuts = 1;
    }
    __host__ __device__ int beg(int cut) const { return (int)((long long)kb * cut / cuts); }
};

int head_dz_pairs(int parts);  // SM pairs that run HEAD_DZ at once, 0: the query fails
// a, b: the operands; dw: HEAD_DW's bf16 output; dl: HEAD_DLOGITS' output, [parts][T][Np][piece].
int launch_head_gemm(int mode, const HeadPlan &h, HeadGemm g, const __nv_bfloat16 *z, const __nv_bfloat16 *w,
                     __nv_bfloat16 *dl, __nv_bfloat16 *dw, cudaStream_t s);

// The sums of HEAD_STATS for at most HEAD_FEW tokens a head (head_few.cu): one entry of part a CTA, `few` CTAs a head.  z: the
// packed parts; w: the weights as they are given.
int launch_head_few(const HeadPlan &h, const HeadGemm &g, const __nv_bfloat16 *z, const void *w, cudaStream_t s);

struct HeadIn {
    const void *z, *w;
    const int32_t *label, *tidx;
    const float *tlogit;
};
// The plan for a workspace of `bytes` (0: the one that is recommended); false if they do not do.
bool head_plan(const Dims &p, const vmoe_head *head, bool label, size_t bytes, HeadPlan *out);
size_t head_min_workspace(const Dims &p, const vmoe_head *head);
int launch_head_loss(const Dims &p, const HeadPlan &h, const HeadIn &in, float *ce, float *lse, float *kl, float *tlse,
                     float *logp, void *workspace, cudaStream_t s);
int launch_head_loss_bwd(const Dims &p, const HeadPlan &h, const HeadIn &in, const float *ce, const float *lse,
                         const float *tlse, const float *logp, const float *dce, const float *dlse, const float *dkl,
                         void *dz, void *dw, void *workspace, cudaStream_t s);

}  // namespace vmoe
