// Causal differential attention of new tokens over the 8-bit paged K/V cache (include/hgf.h, hgf_diff_attention_cached).
//
// What a page's head costs to read is 3 * 64 * DH bytes, and every byte is used for few products: the kernel is a stream from memory.  The work is
// cut into units of that size - a page of a sequence and K/V head, or 32 open tokens - and the units of all (sequence, group of query rows, head)
// items are laid in one sequence, which is dealt in equal shares to the warps of one CTA an SM.  Each warp has a ring of units in shared memory that
// one bulk copy each fills, and works alone: no barrier between warps.  An item that lies within one warp's share is finished there; of an item
// that several share each leaves its softmax statistics and sums in the workspace, and a second kernel joins them, in the order of the tokens.
//
// Products are int8 tensor-core products on the codes as they lie in the page (m16n8k32, the codes as left operand), exact:
//   scores   q as a 23-bit fixed-point number of the row's power of two, cut into three signed digits in base 256: three columns of the right operand
//   values   probabilities as 24-bit fixed-point numbers of the running maximum (bits of 1 + p), three unsigned digits
// so nothing is rounded to fewer than 22 bits on the way, at any output type.  The open tokens' bf16 go through bf16 products, with the probabilities
// as sums of three bf16.
//
// Two forms: ROWS = 1 for single tokens with heads of their own (both streams' digits fit the eight columns of one product), ROWS = 8 otherwise (a
// product for each digit, eight query rows as its columns).
#include "hgf_cache.cuh"
#include "hgf_warp.cuh"

namespace hgf {

constexpr int kCaMaxSms = 160;   // CTAs at most (the workspace has room for them)
constexpr int kCaStages = 2;     // units in a warp's ring

template <int DH>
struct CaCfg {
    static constexpr int WARPS = DH == 64 ? 8 : 4, THREADS = WARPS * 32;
    static constexpr int UNIT = 3 * kCacheBlock * DH;            // bytes of a unit
    static constexpr int STAGE = (UNIT + 16 + 127) / 128 * 128;  // with the page's scales
    static constexpr int KT = DH / 32, MT = DH / 16;
};
constexpr int kCaScoreStride = 68;  // floats between rows of scores: eight rows' writes hit all banks
template <int ROWS>
constexpr int kCaScoreBytes = ROWS == 1 ? 2 * kCacheBlock * 4 : 8 * kCaScoreStride * 4;

struct CaParams {
    CacheView c;
    const __nv_bfloat16 *q;
    const int32_t *slots, *starts;
    void *out;
    int4 *items;          // [workers][2]: what the joining kernel does for a worker
    float *parts;         // [workers][2][ROWS][4 + 2 DH]: maximum and sum of stream 1, of stream 2, sums of values
    unsigned int *status;
    int n_seqs, n_rows, group, bf16;
    float lambda, out_scale, scale_log2;
};

__device__ __forceinline__ void mma_s8s8(int (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_s8u8(int (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ldmatrix4(uint32_t addr) {
    uint4 v;
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ldmatrix4_trans(uint32_t addr) {
    uint4 v;
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

// A sequence of the call and an item's place in it.
struct CaSeq {
    int slot, row0, m, length, pages, units;
    int tiles;
};
template <int ROWS>
__device__ __forceinline__ CaSeq ca_sequence(const CaParams &p, int i) {
    CaSeq s = {};
    s.slot = p.slots[i];
    s.row0 = p.starts[i];
    s.m = p.starts[i + 1] - s.row0;
    if (s.slot < 0 || s.slot >= p.c.n_slots || s.row0 < 0 || s.m <= 0 || s.m > p.n_rows - s.row0) {
        s.slot = s.slot == -1 || s.m == 0 ? -1 : -2;
        s.m = 0;
        return s;
    }
    s.length = p.c.length[s.slot];
    if (!cache_slot_ok(p.c, p.c.held[s.slot], s.length)) {
        s.slot = -2;
        s.m = 0;
        s.length = 0;
        return s;
    }
    s.pages = s.length >> 6;
    const int open = s.length & 63;
    s.units = s.pages + (open > 0) + (open > 32);
    s.tiles = (s.m * p.group + ROWS - 1) / ROWS;
    return s;
}

struct CaCursor {
    CaSeq s;
    int seq, tile, head, unit;
};

template <int DH, int ROWS>
__global__ void __launch_bounds__(CaCfg<DH>::THREADS, 1) cached_attention_kernel(CaParams p) {
    using C = CaCfg<DH>;
    constexpr int PART = 4 + 2 * DH;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, H = p.c.H;
    uint8_t *ring = smem + warp * (kCaStages * C::STAGE);
    float *scores = reinterpret_cast<float *>(smem + C::WARPS * kCaStages * C::STAGE + warp * kCaScoreBytes<ROWS>);
    long long *prefix = reinterpret_cast<long long *>(smem + C::WARPS * (kCaStages * C::STAGE + kCaScoreBytes<ROWS>));
    __shared__ long long wide[C::WARPS + 1];
    __shared__ __align__(8) uint64_t bars[C::WARPS][kCaStages];
    const uint32_t ring_a = dsmem_u32(ring);
    if (lane < kCaStages) dmbar_init(dsmem_u32(&bars[warp][lane]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    pdl_launch_dependents();

    // ---- plan: the running sum of units over the sequences, by every CTA for itself
    long long total = 0;
    for (int i0 = 0; i0 < p.n_seqs; i0 += C::THREADS) {
        const int i = i0 + tid;
        long long mine = 0;
        if (i < p.n_seqs) {
            const CaSeq s = ca_sequence<ROWS>(p, i);
            mine = (long long)s.tiles * H * s.units;
            if (blockIdx.x == 0 && s.slot == -2) atomicOr(p.status, kStatusCache);
        }
        long long sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) wide[warp] = sum;
        __syncthreads();
        long long before = total, all = 0;
#pragma unroll
        for (int w = 0; w < C::WARPS; ++w) {
            if (w < warp) before += wide[w];
            all += wide[w];
        }
        if (i < p.n_seqs) prefix[i] = before + sum - mine;
        total += all;
        __syncthreads();
    }
    if (tid == 0) prefix[p.n_seqs] = total;
    __syncthreads();

    // rows that see nothing because the sequence is empty
    const int width = H * p.group * DH;
    for (int i = blockIdx.x; i < p.n_seqs; i += gridDim.x)
        if (prefix[i + 1] == prefix[i]) {
            const CaSeq s = ca_sequence<ROWS>(p, i);
            const size_t at = (size_t)s.row0 * width, n = (size_t)s.m * width;
            for (size_t e = tid; e < n; e += C::THREADS) {
                if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[at + e] = __float2bfloat16(0.0f);
                else reinterpret_cast<float *>(p.out)[at + e] = 0.0f;
            }
        }

    // (no more workers than units, so that none is empty between two of an item; their numbers go round the CTAs)
    const int workers = (int)min((long long)gridDim.x * C::WARPS, total), worker = warp * gridDim.x + blockIdx.x;
    if (worker >= workers) {
        if (lane == 0) p.items[2 * worker] = make_int4(0, 0, 0, 0);
        return;
    }
    const long long u0 = total * worker / workers, u1 = total * (worker + 1) / workers;
    auto place = [&](long long u, CaCursor &k) {
        int lo = 0, hi = p.n_seqs - 1;
        while (lo < hi) {  // the last sequence that begins at or before u (of empty ones at the same place the last, which is not empty)
            const int mid = (lo + hi + 1) >> 1;
            if (prefix[mid] <= u) lo = mid; else hi = mid - 1;
        }
        k.seq = lo;
        k.s = ca_sequence<ROWS>(p, lo);
        const long long in = u - prefix[lo], item = in / k.s.units;
        k.unit = (int)(in - item * k.s.units);
        k.tile = (int)(item / H);
        k.head = (int)(item - (long long)k.tile * H);
    };
    auto advance = [&](CaCursor &k) {  // to the next unit; true: of another item
        if (++k.unit < k.s.units) return false;
        k.unit = 0;
        if (++k.head < H) return true;
        k.head = 0;
        if (++k.tile < k.s.tiles) return true;
        k.tile = 0;
        do ++k.seq; while (k.seq < p.n_seqs - 1 && prefix[k.seq + 1] == prefix[k.seq]);
        if (k.seq < p.n_seqs) k.s = ca_sequence<ROWS>(p, k.seq);
        return true;
    };
    // Tokens that query row r of a tile sees: those before row_sees().
    auto row_sees = [&](const CaCursor &k, int r) {
        const int at = k.tile * ROWS + r;
        return at < k.s.m * p.group ? k.s.length - k.s.m + at / p.group + 1 : 0;
    };
    auto unit_token = [&](const CaCursor &k) { return k.unit < k.s.pages ? k.unit << 6 : (k.s.pages << 6) + ((k.unit - k.s.pages) << 5); };
    auto tile_sees = [&](const CaCursor &k) {  // of the tile's last row
        return k.s.length - k.s.m + min(k.tile * ROWS + ROWS - 1, k.s.m * p.group - 1) / p.group + 1;
    };

    // ---- the ring: page numbers 32 at a time, one bulk copy a unit
    uint32_t loaded = 0;  // per stage: its unit was fetched
    int pages32 = 0, pages_at = -32, pages_seq = -1;
    auto fetch = [&](const CaCursor &k, int stage) {
        const uint32_t bar = dsmem_u32(&bars[warp][stage]), dst = ring_a + stage * C::STAGE;
        bool ok = unit_token(k) < tile_sees(k);
        if (k.unit < k.s.pages) {
            if (pages_seq != k.seq || (k.unit & ~31) != pages_at) {
                pages_seq = k.seq;
                pages_at = k.unit & ~31;
                pages32 = pages_at + lane < k.s.pages ? p.c.table[(size_t)k.s.slot * p.c.max_pages + pages_at + lane] : 0;
            }
            const int page = __shfl_sync(0xffffffffu, pages32, k.unit & 31);
            if (ok && (page < 0 || page >= p.c.n_pages)) {
                ok = false;
                if (lane == 0) atomicOr(p.status, kStatusCache);
            }
            if (ok && lane == 0) {
                const size_t at = (size_t)page * H + k.head;
                announce(bar, C::UNIT + 16);
                bulk_load_announced(dst, p.c.codes + at * C::UNIT, C::UNIT, bar);
                bulk_load_announced(dst + C::UNIT, p.c.scales + at, 16, bar);
            }
        } else if (ok && lane == 0) {
            const int half = k.unit - k.s.pages, rows = min(32, (k.s.length & 63) - 32 * half);
            const __nv_bfloat16 *src = p.c.open + (((size_t)k.s.slot * H + k.head) * 3 * kCacheBlock + 32 * half) * DH;
            announce(bar, 3 * rows * DH * 2);
#pragma unroll
            for (int n = 0; n < 3; ++n) bulk_load_announced(dst + n * 32 * DH * 2, src + (size_t)n * kCacheBlock * DH, rows * DH * 2, bar);
        }
        loaded = ok ? loaded | 1u << stage : loaded & ~(1u << stage);
    };
    uint32_t phases = 0;
    auto arrived = [&](int stage) {  // waits, bounded, for the stage's copies
        const uint32_t bar = dsmem_u32(&bars[warp][stage]), parity = phases >> stage & 1u;
        bool got = dmbar_try_wait(bar, parity);
        if (__all_sync(0xffffffffu, got)) return true;
        const unsigned long long since = dec_timer_ns();
        for (uint32_t polls = 1; !got && !(got = dmbar_try_wait(bar, parity)); ++polls)
            if ((polls & 255u) == 0 && dec_timer_ns() - since > kDecWaitLimitNs) break;
        if (!got) atomicExch(p.status, 0xb00u);
        return (bool)__all_sync(0xffffffffu, got);
    };

    CaCursor ahead, k;
    place(u0, ahead);
    k = ahead;
    long long ahead_u = u0;
    __syncwarp();
#pragma unroll
    for (int s = 0; s < kCaStages; ++s)
        if (ahead_u < u1) {
            fetch(ahead, s);
            advance(ahead);
            ++ahead_u;
        }

    // ---- state of the item
    // ROWS = 1: m, l of the lane's stream (lanes 0-15 stream 1, 16-31 stream 2); acc[mt][e]: dims 16 mt + g + 8 e, in lanes t of stream t / 2.
    // ROWS = 8: m[st], l[st] of row g; acc[st][mt][e]: dim 16 mt + g + 8 (e / 2), row 2 t + e % 2.
    constexpr int NS = ROWS == 1 ? 1 : 2, NE = ROWS == 1 ? 2 : 4;
    float m[NS], l[NS], acc[NS][C::MT][NE];
    uint32_t qd[2][ROWS == 1 ? 1 : 3][C::KT][2];  // right operand of the scores: digits of q
    float qs[NS];                                 // what a digit sum is worth, with 1 / sqrt(d) and log2 e
    const int my_stream = lane >> 4, limb = g & 3;
    const uint32_t limb_sel = 0x0040u + (uint32_t)((2 - limb) & 3) * 0x0011u;  // byte 2 - limb of two words
    const uint32_t limb_xor = limb == 0 ? 0x80808080u : 0u, limb_keep = limb == 3 ? 0u : 0xffffffffu;

    auto begin_item = [&] {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            m[s] = -INFINITY;
            l[s] = 0.0f;
#pragma unroll
            for (int a = 0; a < C::MT; ++a)
#pragma unroll
                for (int e = 0; e < NE; ++e) acc[s][a][e] = 0.0f;
        }
        // q's digits: q = f * 2^(E - 21) with E the exponent of the row's largest magnitude, so |f| < 2^22; f + 0x808080 has in each byte the
        // balanced digit plus 128.
        const int heads = H * p.group;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int r = ROWS == 1 ? 0 : g, at = k.tile * ROWS + r;
            const bool there = at < k.s.m * p.group && (ROWS == 8 || (g >> 2) == n);
            const __nv_bfloat16 *src = p.q + ((size_t)(k.s.row0 + (there ? at / p.group : 0)) * 2 + n) * heads * DH + (size_t)(k.head * p.group + (there ? at % p.group : 0)) * DH;
            uint2 w[C::KT][2];
            uint32_t top = 0;
#pragma unroll
            for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    w[kt][h] = there ? *reinterpret_cast<const uint2 *>(src + kt * 32 + h * 16 + 4 * t) : make_uint2(0, 0);
                    top = __vmaxu2(top, __vmaxu2(w[kt][h].x & 0x7fff7fffu, w[kt][h].y & 0x7fff7fffu));
                }
            top = max(top >> 16, top & 0xffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int E = max((int)(top >> 7) - 127, -100);  // (below 2^-100 the scores are zero for any purpose, above that 2^(21 - E) is a float)
            const float f = __uint_as_float((uint32_t)(127 + 21 - E) << 23);
            const float back = top >= 0x7f80u ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(127 - 21 + E) << 23);
            if (ROWS == 8 || n == my_stream) qs[ROWS == 1 ? 0 : n] = back * p.scale_log2;
#pragma unroll
            for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t d[4];
                    d[0] = (uint32_t)__float2int_rn(bf16lo_to_float(w[kt][h].x) * f) + 0x808080u;
                    d[1] = (uint32_t)__float2int_rn(bf16hi_to_float(w[kt][h].x) * f) + 0x808080u;
                    d[2] = (uint32_t)__float2int_rn(bf16lo_to_float(w[kt][h].y) * f) + 0x808080u;
                    d[3] = (uint32_t)__float2int_rn(bf16hi_to_float(w[kt][h].y) * f) + 0x808080u;
                    if (ROWS == 1) {
                        const uint32_t v = __byte_perm(__byte_perm(d[0], d[1], limb_sel), __byte_perm(d[2], d[3], limb_sel), 0x5410) ^ 0x80808080u;
                        qd[n][0][kt][h] = there ? v & limb_keep : 0u;
                    } else {
#pragma unroll
                        for (int j = 0; j < 3; ++j) {
                            const uint32_t sel = 0x0040u + (uint32_t)(2 - j) * 0x0011u;
                            qd[n][ROWS == 1 ? 0 : j][kt][h] = __byte_perm(__byte_perm(d[0], d[1], sel), __byte_perm(d[2], d[3], sel), 0x5410) ^ 0x80808080u;
                        }
                    }
                }
        }
    };

    // Softmax step of a row on `x` (16 or 8 tokens of this lane, the row's others in the lanes with the same g): new maximum, the probabilities in
    // place of the scores, and what the sums so far are to be multiplied with.
    auto softmax_step = [&](auto &x, float &mx, float &sum) {
        constexpr int N = sizeof(x) / sizeof(float);
        float top = x[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = fmaxf(top, x[j]);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float now = fmaxf(mx, top), base = now == -INFINITY ? 0.0f : now, alpha = exp2_approx(mx - base);
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            x[j] = exp2_approx(x[j] - base);
            s += x[j];
        }
        mx = now;
        sum = fmaf(sum, alpha, s);
        return alpha;
    };

    bool fresh = true;                       // the unit begins an item, or the share
    const bool begins_inside = k.unit != 0;  // the share's first item began in another share
    bool first_item = true;
    int4 join = make_int4(0, 0, 0, 0), join_at = join;

    for (long long u = u0; u < u1; ++u) {
        const int stage = (int)(u - u0) & (kCaStages - 1);
        if (fresh) begin_item();
        const uint8_t *unit = ring + stage * C::STAGE;
        if (loaded >> stage & 1u) {
            if (!arrived(stage)) {
                if (loaded >> (stage ^ 1) & 1u) arrived(stage ^ 1);  // (no copy outlives the CTA)
                break;
            }
            phases ^= 1u << stage;
            const int token0 = unit_token(k);
            if (k.unit < k.s.pages) {
                const float4 sc = *reinterpret_cast<const float4 *>(unit + C::UNIT);
                if constexpr (ROWS == 1) {
                    const float wa = t & 1 ? 1.0f : 65536.0f, wb = t & 1 ? 0.0f : 256.0f;
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) {
                        int d[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int kt = 0; kt < C::KT; ++kt) {
                                const uint4 a = *reinterpret_cast<const uint4 *>(unit + n * kCacheBlock * DH + ((mt * C::KT + kt) * 32 + lane) * 16);
                                mma_s8s8(d, a, qd[n][0][kt][0], qd[n][0][kt][1]);
                            }
                        float lo = fmaf((float)d[0], wa, (float)d[1] * wb), hi = fmaf((float)d[2], wa, (float)d[3] * wb);
                        lo += __shfl_xor_sync(0xffffffffu, lo, 1);
                        hi += __shfl_xor_sync(0xffffffffu, hi, 1);
                        scores[(t >> 1) * kCacheBlock + mt * 16 + g + (t & 1) * 8] = t & 1 ? hi : lo;
                    }
                    __syncwarp();
                    const float f = qs[0] * (my_stream ? sc.y : sc.x);
                    float x[16];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 v = *reinterpret_cast<const float4 *>(scores + my_stream * kCacheBlock + j * 16 + 4 * t);
                        x[4 * j] = v.x * f;
                        x[4 * j + 1] = v.y * f;
                        x[4 * j + 2] = v.z * f;
                        x[4 * j + 3] = v.w * f;
                    }
                    const int sees = row_sees(k, 0) - token0;
                    if (sees < kCacheBlock) {
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if ((j >> 2) * 16 + 4 * t + (j & 3) >= sees) x[j] = -INFINITY;
                    }
                    const float alpha = softmax_step(x, m[0], l[0]);
                    uint32_t b[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(1.0f + x[4 * j + e]);
                        b[j] = (__byte_perm(__byte_perm(w[0], w[1], limb_sel), __byte_perm(w[2], w[3], limb_sel), 0x5410) ^ limb_xor) & limb_keep;
                    }
                    const float scale = __shfl_sync(0xffffffffu, alpha, (t >> 1) * 16);
                    // digits of 2^23 p: weights 2^-7, 2^-15, 2^-23
                    const float va = sc.z * (t & 1 ? 1.1920928955078125e-7f : 0.0078125f), vb = t & 1 ? 0.0f : sc.z * 3.0517578125e-5f;
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        int d[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            const uint4 a = *reinterpret_cast<const uint4 *>(unit + 2 * kCacheBlock * DH + ((mt * 2 + kt) * 32 + lane) * 16);
                            mma_s8u8(d, a, b[2 * kt], b[2 * kt + 1]);
                        }
                        acc[0][mt][0] = fmaf((float)d[0], va, fmaf((float)d[1], vb, acc[0][mt][0] * scale));
                        acc[0][mt][1] = fmaf((float)d[2], va, fmaf((float)d[3], vb, acc[0][mt][1] * scale));
                    }
                } else {
                    const int sees = row_sees(k, g) - token0;
                    const bool partly = row_sees(k, 0) - token0 < kCacheBlock || row_sees(k, 7) - token0 < kCacheBlock;
                    uint32_t b[2][3][4];
                    float alpha[2];
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
#pragma unroll
                        for (int mt = 0; mt < 4; ++mt) {
                            int d[3][4] = {};
#pragma unroll
                            for (int kt = 0; kt < C::KT; ++kt) {
                                const uint4 a = *reinterpret_cast<const uint4 *>(unit + n * kCacheBlock * DH + ((mt * C::KT + kt) * 32 + lane) * 16);
#pragma unroll
                                for (int j = 0; j < 3; ++j) mma_s8s8(d[j], a, qd[n][j][kt][0], qd[n][j][kt][1]);
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                scores[(2 * t + (e & 1)) * kCaScoreStride + mt * 16 + g + (e >> 1) * 8] = fmaf((float)(d[0][e] * 256 + d[1][e]), 256.0f, (float)d[2][e]);
                        }
                        __syncwarp();
                        const float f = qs[n] * (n ? sc.y : sc.x);
                        float x[16];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float4 v = *reinterpret_cast<const float4 *>(scores + g * kCaScoreStride + j * 16 + 4 * t);
                            x[4 * j] = v.x * f;
                            x[4 * j + 1] = v.y * f;
                            x[4 * j + 2] = v.z * f;
                            x[4 * j + 3] = v.w * f;
                        }
                        __syncwarp();  // (the other stream's scores follow in the same place)
                        if (partly) {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                if ((j >> 2) * 16 + 4 * t + (j & 3) >= sees) x[j] = -INFINITY;
                        }
                        alpha[n] = softmax_step(x, m[n], l[n]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(1.0f + x[4 * j + e]);
#pragma unroll
                            for (int z = 0; z < 3; ++z) {
                                const uint32_t sel = 0x0040u + (uint32_t)(2 - z) * 0x0011u;
                                b[n][z][j] = __byte_perm(__byte_perm(w[0], w[1], sel), __byte_perm(w[2], w[3], sel), 0x5410) ^ (z ? 0u : 0x80808080u);
                            }
                        }
                    }
                    float scale[2][2], worth[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        scale[0][e] = __shfl_sync(0xffffffffu, alpha[0], (2 * t + e) * 4);
                        scale[1][e] = __shfl_sync(0xffffffffu, alpha[1], (2 * t + e) * 4);
                        // (a row that sees none of the page takes nothing of it, not even a scale that is NaN)
                        worth[e] = row_sees(k, 2 * t + e) > token0 ? sc.z * 1.1920928955078125e-7f : 0.0f;
                    }
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        uint4 a[2];
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) a[kt] = *reinterpret_cast<const uint4 *>(unit + 2 * kCacheBlock * DH + ((mt * 2 + kt) * 32 + lane) * 16);
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            int d[3][4] = {};
#pragma unroll
                            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                                for (int z = 0; z < 3; ++z) mma_s8u8(d[z], a[kt], b[n][z][2 * kt], b[n][z][2 * kt + 1]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float v = fmaf((float)(d[0][e] * 256 + d[1][e]), 256.0f, (float)d[2][e]);
                                acc[n][mt][e] = fmaf(v, worth[e & 1], acc[n][mt][e] * scale[n][e & 1]);
                            }
                        }
                    }
                }
            } else {
                // ---- 32 open tokens
                const int half = k.unit - k.s.pages, rows = min(32, (k.s.length & 63) - 32 * half);
                uint8_t *mine = ring + stage * C::STAGE;
                const uint32_t at = ring_a + stage * C::STAGE;
                // what lies behind the last row is no value: V's rows there become zero (K's only give scores that are not looked at)
                for (int e = lane; e < (32 - rows) * (DH / 8); e += 32) *reinterpret_cast<uint4 *>(mine + 2 * 32 * DH * 2 + rows * DH * 2 + e * 16) = make_uint4(0, 0, 0, 0);
                __syncwarp();
                const int heads = H * p.group;
                float alpha[NS], f[NS];
                uint32_t b[NS][ROWS == 1 ? 1 : 3][2][2];
                // (a query that is not finite: digits mean nothing, but the products of its bf16 values do; qs is NaN then)
#pragma unroll
                for (int n = 0; n < NS; ++n) f[n] = qs[n] == qs[n] ? p.scale_log2 : qs[n];
                auto q_pair = [&](int n, int col) -> uint32_t {  // q's values col, col + 1 of this lane's column
                    const int r = ROWS == 1 ? 0 : g, rr = k.tile * ROWS + r;
                    const bool there = rr < k.s.m * p.group && (ROWS == 8 || g == 4 * n);
                    if (!there) return 0;
                    return *reinterpret_cast<const uint32_t *>(p.q + ((size_t)(k.s.row0 + rr / p.group) * 2 + n) * heads * DH + (size_t)(k.head * p.group + rr % p.group) * DH + col);
                };
                auto k_eight = [&](int n, int mt, int kt) {
                    const int r = mt * 16 + (lane & 15);
                    return ldmatrix4(at + n * 32 * DH * 2 + r * DH * 2 + cache_open_eight(r, kt * 2 + (lane >> 4)) * 16);
                };
                if constexpr (ROWS == 1) {
                    float d[2][4] = {};
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int kt = 0; kt < DH / 16; ++kt) {
                            const uint32_t b0 = q_pair(n, kt * 16 + 2 * t), b1 = q_pair(n, kt * 16 + 8 + 2 * t);
#pragma unroll
                            for (int mt = 0; mt < 2; ++mt) mma_bf16(d[mt], k_eight(n, mt, kt), b0, b1);
                        }
                    if (!(t & 1)) {
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt) {
                            scores[(t >> 1) * kCacheBlock + mt * 16 + g] = d[mt][0];
                            scores[(t >> 1) * kCacheBlock + mt * 16 + g + 8] = d[mt][2];
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    if constexpr (ROWS == 8) {
                        float d[2][4] = {};
#pragma unroll
                        for (int kt = 0; kt < DH / 16; ++kt) {
                            const uint32_t b0 = q_pair(n, kt * 16 + 2 * t), b1 = q_pair(n, kt * 16 + 8 + 2 * t);
#pragma unroll
                            for (int mt = 0; mt < 2; ++mt) mma_bf16(d[mt], k_eight(n, mt, kt), b0, b1);
                        }
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) scores[(2 * t + (e & 1)) * kCaScoreStride + mt * 16 + g + (e >> 1) * 8] = d[mt][e];
                    }
                    __syncwarp();
                    const float *row = scores + (ROWS == 1 ? my_stream * kCacheBlock : g * kCaScoreStride);
                    const int sees = min(rows, row_sees(k, ROWS == 1 ? 0 : g) - token0);
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {  // tokens 8 j + 2 t, 8 j + 2 t + 1
                        const float2 v = *reinterpret_cast<const float2 *>(row + 8 * j + 2 * t);
                        x[2 * j] = 8 * j + 2 * t < sees ? v.x * f[n] : -INFINITY;
                        x[2 * j + 1] = 8 * j + 2 * t + 1 < sees ? v.y * f[n] : -INFINITY;
                    }
                    __syncwarp();
                    alpha[n] = softmax_step(x, m[n], l[n]);
                    // p as a sum of three bf16, each the rounding of what the ones before leave
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float a0 = x[2 * j], a1 = x[2 * j + 1];
#pragma unroll
                        for (int z = 0; z < 3; ++z) {
                            const __nv_bfloat162 v = __floats2bfloat162_rn(a0, a1);
                            const uint32_t w = *reinterpret_cast<const uint32_t *>(&v);
                            if (ROWS == 8) b[n][ROWS == 8 ? z : 0][j >> 1][j & 1] = w;
                            else if (limb == z) b[n][0][j >> 1][j & 1] = w;
                            a0 -= bf16lo_to_float(w);
                            a1 -= bf16hi_to_float(w);
                        }
                        if (ROWS == 1 && limb == 3) b[n][0][j >> 1][j & 1] = 0;
                    }
                }
                auto v_eight = [&](int mt, int kt) {
                    const int r = kt * 16 + (lane & 7) + (lane >> 4) * 8;
                    return ldmatrix4_trans(at + 2 * 32 * DH * 2 + r * DH * 2 + cache_open_eight(r, mt * 2 + (lane >> 3 & 1)) * 16);
                };
                if constexpr (ROWS == 1) {
                    const float scale = __shfl_sync(0xffffffffu, alpha[0], (t >> 1) * 16), wb = t & 1 ? 0.0f : 1.0f;
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) mma_bf16(d, v_eight(mt, kt), b[0][0][kt][0], b[0][0][kt][1]);
                        acc[0][mt][0] = fmaf(d[1], wb, fmaf(acc[0][mt][0], scale, d[0]));
                        acc[0][mt][1] = fmaf(d[3], wb, fmaf(acc[0][mt][1], scale, d[2]));
                    }
                } else {
                    float scale[2][2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        scale[0][e] = __shfl_sync(0xffffffffu, alpha[0], (2 * t + e) * 4);
                        scale[1][e] = __shfl_sync(0xffffffffu, alpha[NS - 1], (2 * t + e) * 4);
                    }
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        const uint4 a[2] = {v_eight(mt, 0), v_eight(mt, 1)};
#pragma unroll
                        for (int n = 0; n < NS; ++n) {
                            float d[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) d[e] = acc[n][mt][e % NE] * scale[n][e & 1];
#pragma unroll
                            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                                for (int z = 0; z < 3; ++z) mma_bf16(d, a[kt], b[n][ROWS == 8 ? z : 0][kt][0], b[n][ROWS == 8 ? z : 0][kt][1]);
                            // (a row that sees none of these tokens takes nothing of them, not even a value that is NaN)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (row_sees(k, 2 * t + (e & 1)) > token0) acc[n][mt][e % NE] = d[e];
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");  // (the next copy into the stage comes after the zeros)
            }
        }
        __syncwarp();
        if (ahead_u < u1) {
            fetch(ahead, stage);
            advance(ahead);
            ++ahead_u;
        } else {
            loaded &= ~(1u << stage);
        }

        // ---- the item's end, or the share's
        const bool item_ends = k.unit == k.s.units - 1;
        if (item_ends || u + 1 == u1) {
            const bool whole = item_ends && !(first_item && begins_inside);
            float *part = p.parts + ((size_t)worker * 2 + (first_item ? 0 : 1)) * (ROWS * PART);
            if (!item_ends && !(first_item && begins_inside)) {
                // the item begins here and goes on elsewhere: this worker's entry names what is to be joined, to the last worker of the item
                const long long end = u - k.unit + k.s.units;  // (its end in the sequence of units)
                const int last = (int)((end * workers - 1) / total);
                join = make_int4(first_item ? 1 : 2, last, k.head, k.tile);
                join_at = make_int4(k.s.row0, k.s.m, 0, 0);
            }
            if constexpr (ROWS == 1) {
                l[0] += __shfl_xor_sync(0xffffffffu, l[0], 1);
                l[0] += __shfl_xor_sync(0xffffffffu, l[0], 2);
                const float l1 = __shfl_sync(0xffffffffu, l[0], 0), l2 = __shfl_sync(0xffffffffu, l[0], 16);
                const float m1 = __shfl_sync(0xffffffffu, m[0], 0), m2 = __shfl_sync(0xffffffffu, m[0], 16);
                const float i1 = l1 != 0.0f ? p.out_scale / l1 : 0.0f, i2 = l2 != 0.0f ? p.lambda * p.out_scale / l2 : 0.0f;
                const size_t at = ((size_t)(k.s.row0 + k.tile / p.group) * H * p.group + k.head * p.group + k.tile % p.group) * DH;
#pragma unroll
                for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float v = acc[0][mt][e];
                        v += __shfl_xor_sync(0xffffffffu, v, 1);
                        const float other = __shfl_xor_sync(0xffffffffu, v, 2);  // in lanes t = 0: stream 2's
                        const int dim = mt * 16 + g + 8 * e;
                        if (whole) {
                            const float y = v * i1 - other * i2;
                            if (t == 0) {
                                if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[at + dim] = __float2bfloat16(y);
                                else reinterpret_cast<float *>(p.out)[at + dim] = y;
                            }
                        } else if (!(t & 1)) {
                            part[4 + (t >> 1) * DH + dim] = v;
                        }
                    }
                if (!whole && lane == 0) *reinterpret_cast<float4 *>(part) = make_float4(m1, l1, m2, l2);
            } else {
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    l[n] += __shfl_xor_sync(0xffffffffu, l[n], 1);
                    l[n] += __shfl_xor_sync(0xffffffffu, l[n], 2);
                }
                if (!whole && t == 0) *reinterpret_cast<float4 *>(part + g * PART) = make_float4(m[0], l[0], m[NS - 1], l[NS - 1]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 2 * t + e, rr = k.tile * ROWS + r;
                    const float l1 = __shfl_sync(0xffffffffu, l[0], r * 4), l2 = __shfl_sync(0xffffffffu, l[NS - 1], r * 4);
                    const float i1 = l1 != 0.0f ? p.out_scale / l1 : 0.0f, i2 = l2 != 0.0f ? p.lambda * p.out_scale / l2 : 0.0f;
                    const bool there = rr < k.s.m * p.group;
                    const size_t at = ((size_t)(k.s.row0 + rr / p.group) * H * p.group + k.head * p.group + rr % p.group) * DH;
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float v1 = acc[0][mt][(2 * h + e) % NE], v2 = acc[NS - 1][mt][(2 * h + e) % NE];
                            const int dim = mt * 16 + g + 8 * h;
                            if (!whole) {
                                part[r * PART + 4 + dim] = v1;
                                part[r * PART + 4 + DH + dim] = v2;
                            } else if (there) {
                                const float y = v1 * i1 - v2 * i2;
                                if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[at + dim] = __float2bfloat16(y);
                                else reinterpret_cast<float *>(p.out)[at + dim] = y;
                            }
                        }
                }
            }
            first_item = false;
        }
        fresh = advance(k);
    }
    if (lane == 0) {
        p.items[2 * worker] = join;
        p.items[2 * worker + 1] = join_at;
    }
}

// Joins the parts of the items that several workers shared: block w the one that begins in worker w's share and does not end there, if there is one.
template <int DH, int ROWS>
__global__ void __launch_bounds__(512) cached_attention_join_kernel(CaParams p) {
    constexpr int PART = 4 + 2 * DH, WAYS = 512 / DH;  // threads: a dim each, the parts dealt to WAYS of them
    __shared__ float sums[WAYS][2][DH], stat[WAYS][4];
    const int dim = threadIdx.x % DH, way = threadIdx.x / DH, w0 = blockIdx.x;
    pdl_wait();
    const int4 item = p.items[2 * w0];
    if (!item.x) return;
    const int4 at = p.items[2 * w0 + 1];
    const int H = p.c.H, n = item.y - w0 + 1;
    for (int r = 0; r < ROWS; ++r) {
        const int rr = item.w * ROWS + r;
        if (rr >= at.y * p.group) break;
        float m1 = -INFINITY, l1 = 0.0f, m2 = -INFINITY, l2 = 0.0f, o1 = 0.0f, o2 = 0.0f;
#pragma unroll 4
        for (int j = way; j < n; j += WAYS) {
            const float *part = p.parts + ((size_t)(w0 + j) * 2 + (j == 0 && item.x == 2 ? 1 : 0)) * (ROWS * PART) + r * PART;
            const float4 s = *reinterpret_cast<const float4 *>(part);
            const float v1 = part[4 + dim], v2 = part[4 + DH + dim];
            const float n1 = fmaxf(m1, s.x), n2 = fmaxf(m2, s.z), b1 = n1 == -INFINITY ? 0.0f : n1, b2 = n2 == -INFINITY ? 0.0f : n2;
            const float a1 = exp2_approx(m1 - b1), c1 = exp2_approx(s.x - b1), a2 = exp2_approx(m2 - b2), c2 = exp2_approx(s.z - b2);
            l1 = l1 * a1 + s.y * c1;
            o1 = o1 * a1 + v1 * c1;
            l2 = l2 * a2 + s.w * c2;
            o2 = o2 * a2 + v2 * c2;
            m1 = n1;
            m2 = n2;
        }
        sums[way][0][dim] = o1;
        sums[way][1][dim] = o2;
        if (dim == 0) {
            stat[way][0] = m1;
            stat[way][1] = l1;
            stat[way][2] = m2;
            stat[way][3] = l2;
        }
        __syncthreads();
        if (way == 0) {
            float y[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float top = -INFINITY, l = 0.0f, o = 0.0f;
#pragma unroll
                for (int j = 0; j < WAYS; ++j) top = fmaxf(top, stat[j][2 * s]);
                const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
                for (int j = 0; j < WAYS; ++j) {
                    const float a = exp2_approx(stat[j][2 * s] - base);
                    l += stat[j][2 * s + 1] * a;
                    o += sums[j][s][dim] * a;
                }
                y[s] = l != 0.0f ? o / l : 0.0f;
            }
            const float v = (y[0] - p.lambda * y[1]) * p.out_scale;
            const size_t o = ((size_t)(at.x + rr / p.group) * H * p.group + item.z * p.group + rr % p.group) * DH + dim;
            if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[o] = __float2bfloat16(v);
            else reinterpret_cast<float *>(p.out)[o] = v;
        }
        __syncthreads();
    }
}

// One row an item where the call's rows are single tokens with heads of their own (on average: any call is right in either form).
static int ca_rows(int64_t n_seqs, int64_t n_rows, int group) { return n_rows * group <= n_seqs ? 1 : 8; }

template <int DH, int ROWS>
static cudaError_t launch_cached_attention(const CaParams &p, cudaStream_t stream) {
    using C = CaCfg<DH>;
    constexpr int SMEM = C::WARPS * (kCaStages * C::STAGE + kCaScoreBytes<ROWS>) + (kCacheMaxSeqs + 1) * 8;
    static_assert(SMEM <= 226 * 1024, "shared memory of a CTA");
    static std::atomic<unsigned long long> attr_done{0};
    cudaError_t e = ensure_dynamic_smem(cached_attention_kernel<DH, ROWS>, SMEM, attr_done);
    if (e != cudaSuccess) return e;
    const int sms = device_sm_count();
    if (!sms) return cudaErrorInvalidDevice;
    const int grid = sms < kCaMaxSms ? sms : kCaMaxSms;
    cached_attention_kernel<DH, ROWS><<<grid, C::THREADS, SMEM, stream>>>(p);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(grid * C::WARPS));
    cfg.blockDim = dim3(512);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, cached_attention_join_kernel<DH, ROWS>, p);
    if (e != cudaSuccess) return e;
    count_launch(2);
    return cudaSuccess;
}

static size_t ca_items_bytes(int head_dim) { return align_up((size_t)kCaMaxSms * (head_dim == 64 ? CaCfg<64>::WARPS : CaCfg<128>::WARPS) * 2 * sizeof(int4), 256); }
static size_t ca_workspace(int head_dim, int rows) {
    return ca_items_bytes(head_dim) + align_up((size_t)kCaMaxSms * (head_dim == 64 ? CaCfg<64>::WARPS : CaCfg<128>::WARPS) * 2 * rows * (4 + 2 * head_dim) * 4, 256);
}

}  // namespace hgf

using namespace hgf;

extern "C" size_t hgf_cached_workspace_bytes(const hgf_cache *cache, int64_t n_seqs, int64_t n_rows, int32_t n_heads) {
    if (!cache || (cache->head_dim != 64 && cache->head_dim != 128) || cache->n_heads <= 0 || n_heads <= 0 || n_rows <= 0 || n_seqs <= 0) return 256;
    return ca_workspace(cache->head_dim, ca_rows(n_seqs, n_rows, n_heads / cache->n_heads));
}

extern "C" hgf_status hgf_diff_attention_cached(const hgf_cache *cache, const void *q, int64_t n_rows, int32_t n_heads, const int32_t *slots,
                                                const int32_t *starts, int64_t n_seqs, float lambda, float out_scale, void *out, void *workspace,
                                                size_t workspace_bytes, uint32_t flags, void *stream) {
    if (!q || !slots || !starts || !out || n_rows <= 0 || n_heads <= 0 || (flags & ~HGF_FLAG_OUT_BF16)) return HGF_ERR_INVALID_ARG;
    CaParams p = {};
    if (const hgf_status st = parse_cache(cache, n_seqs, &p.c)) return st;
    if (n_heads % cache->n_heads || n_heads > 65535 || n_rows > (1 << 24) || n_rows * (n_heads / cache->n_heads) > 0x3fffffffll) return HGF_ERR_UNSUPPORTED_SHAPE;
    if (((uintptr_t)q | (uintptr_t)out) & 15u) return HGF_ERR_MISALIGNED;
    const int group = n_heads / cache->n_heads, rows = ca_rows(n_seqs, n_rows, group), dh = cache->head_dim;
    if (!workspace || workspace_bytes < ca_workspace(dh, rows)) return HGF_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255u) return HGF_ERR_MISALIGNED;
    p.q = (const __nv_bfloat16 *)q;
    p.slots = slots;
    p.starts = starts;
    p.out = out;
    p.items = (int4 *)workspace;
    p.parts = (float *)((char *)workspace + ca_items_bytes(dh));
    p.status = device_status_word();
    if (!p.status) return HGF_ERR_CUDA;
    p.n_seqs = (int)n_seqs;
    p.n_rows = (int)n_rows;
    p.group = group;
    p.bf16 = (flags & HGF_FLAG_OUT_BF16) != 0;
    p.lambda = lambda;
    p.out_scale = out_scale;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)dh));
    cudaError_t e;
    if (dh == 64) e = rows == 1 ? launch_cached_attention<64, 1>(p, (cudaStream_t)stream) : launch_cached_attention<64, 8>(p, (cudaStream_t)stream);
    else e = rows == 1 ? launch_cached_attention<128, 1>(p, (cudaStream_t)stream) : launch_cached_attention<128, 8>(p, (cudaStream_t)stream);
    return e == cudaSuccess ? HGF_OK : HGF_ERR_CUDA;
}
