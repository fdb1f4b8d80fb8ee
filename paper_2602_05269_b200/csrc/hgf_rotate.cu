// Norms of the heads of Q and K with the rotation by position, and their gradients, each in one pass.  For a head x of a token at position p,
//     u = x r,  r = (mean(x^2) + eps)^(-1/2),   y = R(p) (u (.) w)
// where R(p) turns pair i of the first `rot` dims by the angle p base^(-2 i / rot) and leaves the others.  Backward, with g = R(p)^T dy:
//     dw = sum over tokens and heads of g (.) u,   dx = r (g (.) w - u mean(g (.) w (.) u))
#include <cmath>

#include "hgf_common.cuh"
#include "hgf_warp.cuh"

namespace hgf {

struct RotateSide {
    const __nv_bfloat16 *x;   // [rows][heads * dh]
    const __nv_bfloat16 *dy;  // (backward)
    __nv_bfloat16 *out;       // y, or dx (may be null: the weights' gradient alone)
    const float *w;           // [dh], null: ones
    int heads;                // 0: this side is not asked for
};
struct RotateParams {
    RotateSide side[2];
    const int32_t *pos;
    float *part;              // (backward) [grid][2][dh] sums of the blocks, null: not asked for
    int rows, rot, pairs, per_warp;  // per_warp: groups of heads that a warp takes, one after the other
    float eps;
    double turns[64];         // base^(-2 i / rot) / (2 pi)
};

// DH / 16 lanes share a head, each with two eights of its dims, so that both dims of a pair are one lane's: pairs (i, i + rot / 2) lie in
// eights e and e + rot / 16, neighbours (2 i, 2 i + 1) in one.  In either case lane l has pairs 8 l .. 8 l + 7, if 8 l < rot / 2.
template <int DH>
struct RotateLane {
    static constexpr int LPH = DH / 16, HPW = 32 / LPH;  // lanes of a head, heads of a warp
    int l, head, e0, e1;
    bool turned, pairs;
    float cosine[8], sine[8];

    __device__ __forceinline__ RotateLane(const RotateParams &p, int lane) {
        l = lane % LPH;
        head = lane / LPH;
        turned = l < p.rot / 16;
        pairs = p.pairs != 0;
        e0 = turned && !pairs ? l : 2 * l;
        e1 = turned && !pairs ? l + p.rot / 16 : 2 * l + 1;
    }
    // The token's cosines and sines.  The angle is taken in turns and in 64 bits, its whole turns dropped: a far position loses no digits.
    // A lane forms those of its own number (and 32 on), the lanes exchange them.
    __device__ __forceinline__ void turn(const RotateParams &p, int pos, int lane) {
        float c[LPH / 4], s[LPH / 4];
#pragma unroll
        for (int n = 0; n < LPH / 4; ++n) {
            const int i = 32 * n + lane;
            c[n] = 1.0f;
            s[n] = 0.0f;
            if (2 * i < p.rot) {
                const double t = (double)pos * p.turns[i];
                sincospif(2.0f * (float)(t - rint(t)), &s[n], &c[n]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int from = (8 * l + e) & 31;
            cosine[e] = __shfl_sync(0xffffffffu, c[0], from);
            sine[e] = __shfl_sync(0xffffffffu, s[0], from);
            if constexpr (LPH == 8) {
                const float c1 = __shfl_sync(0xffffffffu, c[1], from), s1 = __shfl_sync(0xffffffffu, s[1], from);
                if (l >= 4) { cosine[e] = c1; sine[e] = s1; }
            }
        }
    }
    // v[0..7] the dims of e0, v[8..15] those of e1; BACK: by the angles' negatives
    template <bool BACK>
    __device__ __forceinline__ void rotate(float (&v)[16]) const {
        if (!turned) return;
        auto two = [&](float &a, float &b, int i) {
            const float s = BACK ? -sine[i] : sine[i], a0 = a;
            a = a0 * cosine[i] - b * s;
            b = a0 * s + b * cosine[i];
        };
        if (pairs) {
#pragma unroll
            for (int i = 0; i < 8; ++i) two(v[2 * i], v[2 * i + 1], i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) two(v[i], v[8 + i], i);
        }
    }
    __device__ __forceinline__ float head_sum(float v) const {
#pragma unroll
        for (int o = LPH / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    __device__ __forceinline__ void load(const __nv_bfloat16 *head_at, float (&v)[16]) const {
        const uint4 a = reinterpret_cast<const uint4 *>(head_at)[e0], b = reinterpret_cast<const uint4 *>(head_at)[e1];  // (the output may be the input)
        const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[2 * i] = bf16lo_to_float(x[i]);
            v[2 * i + 1] = bf16hi_to_float(x[i]);
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *head_at, const float (&v)[16]) const {
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            x[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        reinterpret_cast<uint4 *>(head_at)[e0] = make_uint4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<uint4 *>(head_at)[e1] = make_uint4(x[4], x[5], x[6], x[7]);
    }
    __device__ __forceinline__ void weights(const float *w, float (&v)[16]) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = w ? __ldg(w + 8 * (i < 8 ? e0 : e1) + (i & 7)) : 1.0f;
    }
};

constexpr int kRotateThreads = 256;

// A warp takes `per_warp` neighbouring groups of HPW heads of one token; Q's groups come before K's.
template <int DH>
__global__ void __launch_bounds__(kRotateThreads)
qk_norm_rotate_kernel(const __grid_constant__ RotateParams p) {
    using R = RotateLane<DH>;
    const int lane = threadIdx.x & 31;
    R r(p, lane);
    const int gq = (p.side[0].heads + R::HPW - 1) / R::HPW, groups = gq + (p.side[1].heads + R::HPW - 1) / R::HPW;
    const int parts = (groups + p.per_warp - 1) / p.per_warp;
    const long long unit = (long long)blockIdx.x * (kRotateThreads / 32) + (threadIdx.x >> 5);
    const long long row = unit / parts;
    if (row >= p.rows) return;
    const int first = (int)(unit % parts) * p.per_warp, last = min(first + p.per_warp, groups);
    r.turn(p, __ldg(p.pos + row), lane);
    float w[16];
    int side = -1;
    for (int grp = first; grp < last; ++grp) {
        const int s = grp >= gq;
        const RotateSide &a = p.side[s];
        if (s != side) {
            r.weights(a.w, w);
            side = s;
        }
        const int head = (grp - (s ? gq : 0)) * R::HPW + r.head;
        const bool there = head < a.heads;
        const size_t at = ((size_t)row * a.heads + (there ? head : 0)) * DH;
        float v[16], sum = 0.0f;
        r.load(a.x + at, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(v[i], v[i], sum);
        const float n = rsqrtf(r.head_sum(sum) * (1.0f / DH) + p.eps);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = v[i] * n * w[i];
        r.template rotate<false>(v);
        if (there) r.store(a.out + at, v);
    }
}

template <int DH>
__global__ void __launch_bounds__(kRotateThreads)
qk_norm_rotate_backward_kernel(const __grid_constant__ RotateParams p) {
    using R = RotateLane<DH>;
    __shared__ float s_dw[kRotateThreads / 32][DH];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    R r(p, lane);
    const long long warps = (long long)gridDim.x * (kRotateThreads / 32), me = (long long)blockIdx.x * (kRotateThreads / 32) + warp;
#pragma unroll 1
    for (int s = 0; s < 2; ++s) {
        const RotateSide &a = p.side[s];
        const int groups = (a.heads + R::HPW - 1) / R::HPW, parts = (groups + p.per_warp - 1) / p.per_warp;
        float dw[16] = {}, w[16];
        r.weights(a.w, w);
        for (long long unit = me; unit < (long long)p.rows * parts; unit += warps) {
            const long long row = unit / parts;
            const int first = (int)(unit % parts) * p.per_warp, last = min(first + p.per_warp, groups);
            r.turn(p, __ldg(p.pos + row), lane);
            for (int grp = first; grp < last; ++grp) {
                const int head = grp * R::HPW + r.head;
                const bool there = head < a.heads;
                const size_t at = ((size_t)row * a.heads + (there ? head : 0)) * DH;
                float x[16], g[16], sum = 0.0f, mean = 0.0f;
                r.load(a.x + at, x);
                r.load(a.dy + at, g);
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
                const float n = rsqrtf(r.head_sum(sum) * (1.0f / DH) + p.eps);
                r.template rotate<true>(g);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[i] *= n;
                    if (there) dw[i] = fmaf(g[i], x[i], dw[i]);
                    g[i] *= w[i];
                    mean = fmaf(g[i], x[i], mean);
                }
                mean = r.head_sum(mean) * (1.0f / DH);
#pragma unroll
                for (int i = 0; i < 16; ++i) g[i] = n * fmaf(-x[i], mean, g[i]);
                if (there && a.out) r.store(a.out + at, g);
            }
        }
        if (!p.part) continue;
        // the block's sum for each dim, in one order: over the heads of a warp, then over the warps
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int o = 16; o >= R::LPH; o >>= 1) dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
        if (lane < R::LPH)
#pragma unroll
            for (int i = 0; i < 16; ++i) s_dw[warp][8 * (i < 8 ? r.e0 : r.e1) + (i & 7)] = dw[i];
        __syncthreads();
        if (threadIdx.x < DH) {
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < kRotateThreads / 32; ++q) v += s_dw[q][threadIdx.x];
            p.part[((size_t)blockIdx.x * 2 + s) * DH + threadIdx.x] = v;
        }
        __syncthreads();
    }
}

// The blocks' sums added up, in 64 bits: a block takes 32 dims of a side, its warps every eighth block's sums.
__global__ void __launch_bounds__(256) rotate_weight_sums_kernel(const float *part, int n, int dh, float *dwq, float *dwk) {
    __shared__ double s_sum[8][32];
    const int per_side = dh / 32, s = blockIdx.x / per_side, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, dim = (blockIdx.x % per_side) * 32 + lane;
    float *out = s ? dwk : dwq;
    if (!out) return;
    double v = 0.0;
    for (int i = warp; i < n; i += 8) v += part[((size_t)i * 2 + s) * dh + dim];
    s_sum[warp][lane] = v;
    __syncthreads();
    if (warp == 0) {
        for (int q = 1; q < 8; ++q) v += s_sum[q][lane];
        out[dim] = (float)v;
    }
}

constexpr int kRotateMaxGrid = 1024;

static void rotate_plan(RotateParams &p, int dh, double base, int sms) {
    for (int i = 0; i < p.rot / 2; ++i) p.turns[i] = pow(base, -2.0 * i / p.rot) / 6.283185307179586476925286766559;
    // few tokens: a warp a group of heads; many: up to eight, so that a token's angles are formed rarely
    const int hpw = 32 / (dh / 16), groups = (p.side[0].heads + hpw - 1) / hpw + (p.side[1].heads + hpw - 1) / hpw;
    const long long all = (long long)p.rows * groups, want = (long long)sms * 32;
    p.per_warp = 1;
    while (p.per_warp < 8 && p.per_warp < groups && all / (2 * p.per_warp) >= want) p.per_warp *= 2;
}

static hgf_status rotate_arguments(RotateParams &p, const void *q, const void *k, int64_t n_rows, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                                   const int32_t *positions, const float *q_weight, const float *k_weight, float eps, double base, int32_t rotary_dim,
                                   uint32_t flags) {
    if ((!q && !k) || !positions || n_rows <= 0 || (q && q_heads <= 0) || (k && k_heads <= 0) || (flags & ~HGF_FLAG_ROTATE_PAIRS) || !(eps >= 0.0f) || !(base > 0.0) ||
        std::isinf(base) || std::isinf(eps))
        return HGF_ERR_INVALID_ARG;
    if ((head_dim != 64 && head_dim != 128) || n_rows > 0x7fffffff || rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 16 || q_heads > (1 << 20) || k_heads > (1 << 20))
        return HGF_ERR_UNSUPPORTED_SHAPE;
    if ((((uintptr_t)q) | ((uintptr_t)k) | ((uintptr_t)q_weight) | ((uintptr_t)k_weight) | ((uintptr_t)positions)) & 15u) return HGF_ERR_MISALIGNED;
    p.side[0].x = (const __nv_bfloat16 *)q;
    p.side[0].w = q_weight;
    p.side[0].heads = q ? q_heads : 0;
    p.side[1].x = (const __nv_bfloat16 *)k;
    p.side[1].w = k_weight;
    p.side[1].heads = k ? k_heads : 0;
    p.pos = positions;
    p.rows = (int)n_rows;
    p.rot = rotary_dim;
    p.pairs = (flags & HGF_FLAG_ROTATE_PAIRS) != 0;
    p.eps = eps;
    return HGF_OK;
}

}  // namespace hgf

using namespace hgf;

extern "C" hgf_status hgf_qk_norm_rotate(const void *q, const void *k, int64_t n_rows, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                                         const int32_t *positions, const float *q_weight, const float *k_weight, float eps, double base, int32_t rotary_dim,
                                         void *q_out, void *k_out, uint32_t flags, void *stream) {
    RotateParams p = {};
    const hgf_status st = rotate_arguments(p, q, k, n_rows, q_heads, k_heads, head_dim, positions, q_weight, k_weight, eps, base, rotary_dim, flags);
    if (st != HGF_OK) return st;
    if ((q && !q_out) || (k && !k_out)) return HGF_ERR_INVALID_ARG;
    if ((((uintptr_t)q_out) | ((uintptr_t)k_out)) & 15u) return HGF_ERR_MISALIGNED;
    p.side[0].out = (__nv_bfloat16 *)q_out;
    p.side[1].out = (__nv_bfloat16 *)k_out;
    const int sms = device_sm_count();
    if (!sms) return HGF_ERR_CUDA;
    rotate_plan(p, head_dim, base, sms);
    const int hpw = 32 / (head_dim / 16), groups = (p.side[0].heads + hpw - 1) / hpw + (p.side[1].heads + hpw - 1) / hpw;
    const long long units = (long long)p.rows * ((groups + p.per_warp - 1) / p.per_warp), blocks = (units + kRotateThreads / 32 - 1) / (kRotateThreads / 32);
    if (blocks > 0x7fffffffll) return HGF_ERR_UNSUPPORTED_SHAPE;
    if (head_dim == 64) qk_norm_rotate_kernel<64><<<(unsigned)blocks, kRotateThreads, 0, (cudaStream_t)stream>>>(p);
    else qk_norm_rotate_kernel<128><<<(unsigned)blocks, kRotateThreads, 0, (cudaStream_t)stream>>>(p);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? HGF_OK : HGF_ERR_CUDA;
}

extern "C" size_t hgf_qk_norm_rotate_workspace_bytes(int32_t head_dim) {
    return head_dim == 64 || head_dim == 128 ? (size_t)kRotateMaxGrid * 2 * head_dim * sizeof(float) : 0;
}

extern "C" hgf_status hgf_qk_norm_rotate_backward(const void *q, const void *k, int64_t n_rows, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                                                  const int32_t *positions, const float *q_weight, const float *k_weight, float eps, double base,
                                                  int32_t rotary_dim, const void *dq_out, const void *dk_out, const hgf_rotate_grads *grads, void *workspace,
                                                  size_t workspace_bytes, uint32_t flags, void *stream) {
    RotateParams p = {};
    const hgf_status st = rotate_arguments(p, q, k, n_rows, q_heads, k_heads, head_dim, positions, q_weight, k_weight, eps, base, rotary_dim, flags);
    if (st != HGF_OK) return st;
    if (!grads || (q && !dq_out) || (k && !dk_out)) return HGF_ERR_INVALID_ARG;
    if ((!q && (grads->dq || grads->dwq)) || (!k && (grads->dk || grads->dwk))) return HGF_ERR_INVALID_ARG;
    if ((((uintptr_t)dq_out) | ((uintptr_t)dk_out) | ((uintptr_t)grads->dq) | ((uintptr_t)grads->dk) | ((uintptr_t)grads->dwq) | ((uintptr_t)grads->dwk)) & 15u)
        return HGF_ERR_MISALIGNED;
    if (grads->dwq || grads->dwk) {
        if (!workspace || workspace_bytes < hgf_qk_norm_rotate_workspace_bytes(head_dim)) return HGF_ERR_WORKSPACE;
        if ((uintptr_t)workspace & 255u) return HGF_ERR_MISALIGNED;
        p.part = (float *)workspace;
    }
    if (!grads->dq && !grads->dwq) p.side[0].heads = 0;
    if (!grads->dk && !grads->dwk) p.side[1].heads = 0;
    if (!p.side[0].heads && !p.side[1].heads) return HGF_OK;
    p.side[0].dy = (const __nv_bfloat16 *)dq_out;
    p.side[1].dy = (const __nv_bfloat16 *)dk_out;
    p.side[0].out = (__nv_bfloat16 *)grads->dq;
    p.side[1].out = (__nv_bfloat16 *)grads->dk;
    const int sms = device_sm_count();
    if (!sms) return HGF_ERR_CUDA;
    rotate_plan(p, head_dim, base, sms);
    const int hpw = 32 / (head_dim / 16), most = p.side[0].heads > p.side[1].heads ? p.side[0].heads : p.side[1].heads, groups = (most + hpw - 1) / hpw;
    const long long units = (long long)p.rows * ((groups + p.per_warp - 1) / p.per_warp), blocks = (units + kRotateThreads / 32 - 1) / (kRotateThreads / 32);
    const int cap = 2 * sms < kRotateMaxGrid ? 2 * sms : kRotateMaxGrid, grid = blocks < cap ? (int)blocks : cap;
    if (head_dim == 64) qk_norm_rotate_backward_kernel<64><<<grid, kRotateThreads, 0, (cudaStream_t)stream>>>(p);
    else qk_norm_rotate_backward_kernel<128><<<grid, kRotateThreads, 0, (cudaStream_t)stream>>>(p);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) return HGF_ERR_CUDA;
    if (p.part) {
        rotate_weight_sums_kernel<<<2 * head_dim / 32, 256, 0, (cudaStream_t)stream>>>(p.part, grid, head_dim, grads->dwq, grads->dwk);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return HGF_ERR_CUDA;
    }
    return HGF_OK;
}
