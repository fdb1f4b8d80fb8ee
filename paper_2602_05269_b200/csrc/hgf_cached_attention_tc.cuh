// Cached differential attention of many rows a sequence, on tcgen05 (included by hgf_cached_attention.cu).
//
// An item is 128 rows (row: token times heads of the group) of a sequence and K/V head, a step one page of 64 tokens (the open tokens are one step more).
// All items' steps are one sequence, dealt in equal shares to one CTA an SM: a CTA walks segments, each the steps of one item that lie in its share; a
// segment that is not its whole item leaves maximum, sum and sums of values in the workspace, and the joining kernel adds such parts in the order of the
// tokens.  Within a CTA:
//   warp 14      brings pages into a ring of shared memory, a bulk copy each
//   warps 0-3    write query tiles, and the pages' codes as bf16 (exact: a code has seven bits and a sign) into rings of K and of V, as the operands' layouts
//                have them; V lies transposed in a page, so both operands have their contraction index contiguous
//   warps 12, 13 issue the products of a stream each: S = Q K^T of the codes, and O += P V of the codes
//   warps 4-7    softmax of stream 1, warps 8-11 of stream 2: a thread owns a row; scores times the page's scale of K, the page's scale of V in the exponent
// A probability enters the second product as a sum of three bf16, off by 2^-24 of itself at most, whatever the output's type.  All sums are fp32.  The products' are cut
// off, not rounded, and lose 2^-26 of themselves with each addition (4.4e-6 after 41 steps), so every eight steps they are added up elsewhere and begin anew: in
// shared memory 64 wide, else in the room that the CTA has in the workspace for parts, whose place is free until the part is.
// Tensor memory (512 columns) holds scores and probabilities of two steps a stream beside O 64 wide.  128 wide O takes 256 of them, and a step's
// scores and probabilities 96 (the third parts behind the 64 that scores and the others share): one step a stream, whose scores follow P V of the step before.
//
// What bounds it 64 wide is the instructions: 2300 a step and scheduler with waits and segments' ends, and their fetching, as the roles' loops together are longer than
// what a scheduler keeps (49 % of the issue slots used; tensor pipe 22 %, exponentials 22 %, memory 5 %).  128 wide (2340, 37 % of the slots, tensor pipe 27 %) it is the
// chain scores, softmax, P V of a stream, of which one step is under way at a time.
// Measured, calls back to back, either type of output: 16 heads of 64, 2 sequences of 6000 tokens, 256 rows each: 102 us; 8 K/V heads with four query heads each, 30000
// tokens, 128 rows: 219; 8 heads of 128, 4 sequences of 8192 tokens, 128 rows: 121; one of 30000, 512 rows: 359 (the last two with the int8 form 208 and 705).
// With probabilities in two parts, 16 bits, and sums that run on 64 steps (off by 7.5e-6 after 30000 tokens, growing with the length; plain fp32 3.9e-6, here 1.4e-6) 85, 171, 98 and
// 275.  Steps (the first case in fp32): codes from global memory into registers, segments kept in registers (spills went to the L2 cache) 99;
// segments in shared memory 91; the parts' sixteen bytes of neighbouring rows side by side 104 -> 100 (sequences of one length; the third case 155 -> 117);
// two converting warps of a larger share of registers 99 for 82.
#pragma once
#include "hgf_tc.cuh"

namespace hgf {

constexpr int kCtRows = 128, kCtThreads = 480;
constexpr int kCtFlush = 8;  // a power of two
constexpr float kCtSlack = 8.0f, kCtNone = -3e38f;  // (a maximum of nothing: finite, so that differences of two are zero)

template <int DH>
struct CtCfg {
    static constexpr int NBLK = DH / 64, KST = DH == 128 ? 2 : 3, GST = KST, NS = DH == 128 ? 1 : 2;  // stages of the operands, of the pages (as many as shared memory takes); scores a stream
    static constexpr int Q_BYTES = NBLK * kCtRows * 128, K_BYTES = NBLK * kCacheBlock * 128, V_BYTES = DH * 128;
    static constexpr int OFF_K = 2 * Q_BYTES, OFF_V = OFF_K + KST * 2 * K_BYTES, OFF_G = OFF_V + KST * V_BYTES,
                         UNIT = 3 * kCacheBlock * DH, G_BYTES = (UNIT + 16 + 127) / 128 * 128, OFF_BAR = OFF_G + GST * G_BYTES;
    static constexpr int BAR_QFULL = 0, BAR_QEMPTY = 1, BAR_OEMPTY = 2, BAR_L = 3, BAR_END = 5, BAR_KFULL = 7, BAR_KEMPTY = BAR_KFULL + KST, BAR_VFULL = BAR_KEMPTY + KST,
                         BAR_VEMPTY = BAR_VFULL + KST, BAR_SFULL = BAR_VEMPTY + KST /* [stream][buffer] */, BAR_PFULL = BAR_SFULL + 4, BAR_GFULL = BAR_PFULL + 4, BAR_GEMPTY = BAR_GFULL + GST,
                         BAR_COUNT = BAR_GEMPTY + GST;
    static constexpr int OFF_SCALES = OFF_BAR + 384;             // [8] float4: K1, K2, V of step g % 8, and 0 where its page is none
    static constexpr int OFF_ODD = OFF_SCALES + 128;             // [8][4] ints: of segment % 8, a warp found open values that are not finite
    static constexpr int OFF_L = OFF_ODD + 128;                  // [2][2][128] floats
    static constexpr int OFF_F = OFF_L + 2 * 2 * kCtRows * 4;    // [2][2][128] floats
    static constexpr int OFF_ACC = OFF_F + 2 * 2 * kCtRows * 4;  // (64 wide) [2][128][64] floats, sixteen bytes c of row r at place c ^ (r & 7)
    static constexpr int OFF_PREFIX = OFF_ACC + (DH == 64 ? 2 * kCtRows * DH * 4 : 0);
    static constexpr int SMEM = OFF_PREFIX + (kCacheMaxSeqs + 2) * 8 + 1024;
    static constexpr int COL_O = 256;  // O: + stream DH
    static __host__ __device__ constexpr int col_s(int stream, int buf) { return NS == 2 ? (2 * stream + buf) * 64 : stream * 96; }                      // scores, and the probabilities' first and second parts
    static __host__ __device__ constexpr int col_p3(int stream, int buf) { return NS == 2 ? COL_O + 2 * DH + (2 * stream + buf) * 32 : stream * 96 + 64; }  // their third parts
    static constexpr int PART = 4 + 2 * DH;
    static constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kCacheBlock >> 3) << 17) | ((uint32_t)(kCtRows >> 4) << 24);
    static constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(DH >> 3) << 17) | ((uint32_t)(kCtRows >> 4) << 24);
    static_assert(BAR_COUNT * 8 + 16 <= 384 && COL_O + 2 * DH + (NS == 2 ? 128 : 0) <= 512 && SMEM <= 226 * 1024, "barriers, tensor and shared memory");
};

__device__ __forceinline__ CaSeq ct_sequence(const CaParams &p, int i) {
    CaSeq s = ca_sequence(p, kCtRows, i);
    s.units = s.pages + ((s.length & 63) != 0);
    return s;
}
// The steps unit .. end - 1 of an item: those of the share's next segment.
struct CtSegment {
    CaSeq s;
    int seq, tile, head, unit, end, visible;  // visible: steps that a row of the tile sees something of
    long long u;                              // of `unit`
    __device__ __forceinline__ int stop() const { return min(end, visible); }
    __device__ __forceinline__ bool whole() const { return unit == 0 && end == s.units; }
    __device__ __forceinline__ void bound(const CaParams &p, long long u1) {
        end = (int)min((long long)s.units, unit + (u1 - u));
        const int at = (tile + 1) * kCtRows - 1, last = s.length - s.m + 1 + min(s.m - 1, p.group == 1 ? at : at / p.group);
        visible = (last + 63) >> 6;
    }
    __device__ __forceinline__ void first(const CaParams &p, const long long *prefix, long long u0, long long u1) {
        int lo = 0, hi = p.n_seqs - 1;
        while (lo < hi) {  // the last sequence that begins at or before u0 (of empty ones at the same place the last, which is not empty)
            const int mid = (lo + hi + 1) >> 1;
            if (prefix[mid] <= u0) lo = mid; else hi = mid - 1;
        }
        u = u0;
        seq = lo;
        s = ct_sequence(p, lo);
        const long long in = u0 - prefix[lo], item = in / s.units;
        unit = (int)(in - item * s.units);
        tile = (int)(item / p.c.H);
        head = (int)(item - (long long)tile * p.c.H);
        tile += s.tile0;
        bound(p, u1);
    }
    __device__ __forceinline__ bool next(const CaParams &p, const long long *prefix, long long u1) {
        u += end - unit;
        if (u >= u1) return false;
        unit = 0;
        if (++head == p.c.H) {
            head = 0;
            if (++tile == s.tiles) {
                do ++seq; while (seq < p.n_seqs - 1 && prefix[seq + 1] == prefix[seq]);
                s = ct_sequence(p, seq);
                tile = s.tile0;
            }
        }
        bound(p, u1);
        return true;
    }
};

// Four codes as bf16: of a byte c, 128 + its low seven bits less 128 or, for a negative one, 256.
__device__ __forceinline__ uint2 ct_bf16(uint32_t codes) {
    const uint32_t w[2] = {__byte_perm(codes, 0x43434343u, 0x4140), __byte_perm(codes, 0x43434343u, 0x4342)};
    uint32_t r[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t x = w[i] & 0xff7fff7fu, y = w[i] & 0xff80ff80u;
        const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
        r[i] = *reinterpret_cast<const uint32_t *>(&d);
    }
    return make_uint2(r[0], r[1]);
}

template <int DH>
__global__ void __launch_bounds__(kCtThreads, 1) cached_attention_tc_kernel(CaParams p) {
    using C = CtCfg<DH>;
    constexpr int KV = kCacheBlock, NS = C::NS;
    extern __shared__ uint8_t ct_smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)ct_smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem), bar0 = sbase + C::OFF_BAR;
    auto bar = [&](int i) { return bar0 + 8u * i; };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::OFF_BAR + C::BAR_COUNT * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::OFF_BAR + C::BAR_COUNT * 8 + 4);
    __shared__ volatile int page_ok[C::GST];
    // [segment % 4][stream][32 rows] of a segment's queries, those with a value that is not finite, a bit a row.  (Queries are written when the scores of the segment before
    // are complete, so its softmax may be behind by the NS steps that scores run ahead, which can be NS segments.)
    __shared__ volatile uint32_t odd_q[4][2][4];
    // A warp's segment lies in shared memory, where its first lane moves it on: in registers it costs every role sixteen of them, and what they spilled went
    // through the L2 cache, since the L1 has no room beside so much shared memory.
    __shared__ CtSegment segments[kCtThreads / 32 + 2];
    int *unseen = reinterpret_cast<int *>(smem + C::OFF_BAR + C::BAR_COUNT * 8 + 8);
    float4 *scales = reinterpret_cast<float4 *>(smem + C::OFF_SCALES);
    volatile int *odd = reinterpret_cast<volatile int *>(smem + C::OFF_ODD);
    float *s_l = reinterpret_cast<float *>(smem + C::OFF_L), *s_f = reinterpret_cast<float *>(smem + C::OFF_F);
    long long *prefix = reinterpret_cast<long long *>(smem + C::OFF_PREFIX);
    __shared__ long long wide[kCtThreads / 32];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, H = p.c.H;

    if (tid == 0) {
        mbar_init(bar(C::BAR_QFULL), 4);
        mbar_init(bar(C::BAR_QEMPTY), 2);  // a commit from each issuer
        mbar_init(bar(C::BAR_OEMPTY), 8);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(C::BAR_L + i), 8);
            mbar_init(bar(C::BAR_END + i), 1);
        }
        for (int s = 0; s < C::KST; ++s) {
            mbar_init(bar(C::BAR_KFULL + s), 4);
            mbar_init(bar(C::BAR_KEMPTY + s), 2);
            mbar_init(bar(C::BAR_VFULL + s), 4);
            mbar_init(bar(C::BAR_VEMPTY + s), 2);
        }
        for (int s = 0; s < C::GST; ++s) {
            mbar_init(bar(C::BAR_GFULL + s), 1);
            mbar_init(bar(C::BAR_GEMPTY + s), 4);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(bar(C::BAR_SFULL + i), 1);
            mbar_init(bar(C::BAR_PFULL + i), 4);
        }
        *abort_flag = 0;
        *unseen = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_proxy_async();
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    pdl_wait();
    pdl_launch_dependents();

    // ---- plan, by every CTA for itself
    if (tid == 0) p.items[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    long long total = 0;
    for (int i0 = 0; i0 < p.n_seqs; i0 += kCtThreads) {
        const int i = i0 + tid;
        long long mine = 0;
        if (i < p.n_seqs) {
            const CaSeq s = ct_sequence(p, i);
            if (blockIdx.x == 0 && s.slot == -2) atomicOr(p.status, kStatusCache);
            if (s.m > s.length) *unseen = 1;
            mine = (long long)(s.tiles - s.tile0) * H * s.units;
        }
        long long sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) wide[warp] = sum;
        __syncthreads();
        long long before = total;
        for (int w = 0; w < kCtThreads / 32; ++w) {
            if (w < warp) before += wide[w];
            total += wide[w];
        }
        if (i < p.n_seqs) prefix[i] = before + sum - mine;
        __syncthreads();
    }
    if (tid == 0) prefix[p.n_seqs] = total;
    __syncthreads();
    if (*unseen) {  // rows that see no token
        const int width = H * p.group * DH;
        for (int i = blockIdx.x; i < p.n_seqs; i += gridDim.x) {
            const CaSeq s = ct_sequence(p, i);
            const size_t at = (size_t)s.row0 * width, n = (size_t)max(s.m - s.length, 0) * width;
            if (p.bf16) for (size_t e = 8 * tid; e < n; e += 8 * kCtThreads) *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(p.out) + at + e) = make_uint4(0, 0, 0, 0);
            else for (size_t e = 4 * tid; e < n; e += 4 * kCtThreads) *reinterpret_cast<uint4 *>(reinterpret_cast<float *>(p.out) + at + e) = make_uint4(0, 0, 0, 0);
        }
    }
    const int ctas = (int)min((long long)gridDim.x, total);
    const bool works = (int)blockIdx.x < ctas;
    const long long c0 = works ? ca_share(total, blockIdx.x, ctas) : 0, c1 = works ? ca_share(total, blockIdx.x + 1, ctas) : 0;

    auto first_segment = [&](CtSegment &s) {
        if (lane == 0) s.first(p, prefix, c0, c1);
        __syncwarp();
    };
    auto next_segment = [&](CtSegment &s) {
        int more = 0;
        __syncwarp();
        if (lane == 0) more = s.next(p, prefix, c1);
        more = __shfl_sync(0xffffffffu, more, 0);
        __syncwarp();
        return more != 0;
    };
    if (works && warp < 4) {
        // ------------------------------------------------------------------ queries, keys and values into shared memory
        const int g4 = lane >> 2, t = lane & 3;
        auto wait = [&](int i, uint32_t par, unsigned int code) { return __all_sync(0xffffffffu, mbar_wait(bar(i), par, abort_flag, p.status, code)) != 0; };
        auto there = [&](int i) {  // what this warp wrote is there for the products
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(i));
        };
        constexpr int KN = DH / 16, VN = DH / 32;  // tiles of 16 x 32 codes of a warp: of K, of V
        bool ok = true;
        int ks = 0, vs = 0, gs = 0, g = 0, segment = 0;
        uint32_t kph = 1, vph = 1, gph = 0, qph = 1;
        CtSegment &seg = segments[warp];
        first_segment(seg);
        bool more = true;
        for (; ok && more; more = next_segment(seg)) {
            const int stop = seg.stop(), first = seg.unit, pages = seg.s.pages;
            if (first >= stop) continue;
            // sixteen codes of a tile: four neighbouring ones of two rows and two places
            auto store = [&](uint8_t *rows, int row0, int chunk0, const uint4 &x) {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = row0 + g4 + 8 * (i & 1), chunk = chunk0 + 2 * (i >> 1) + (t >> 1);
                    *reinterpret_cast<uint2 *>(rows + row * 128 + ((chunk ^ g4) << 4) + (t & 1) * 8) = ct_bf16(w[i]);
                }
            };
            if (!(ok = wait(C::BAR_QEMPTY, qph, 0xc10u))) break;
            {
                const int at = seg.tile * kCtRows + tid, token = p.group == 1 ? at : at / p.group;
                const bool in = token < seg.s.m;
                const size_t row = (size_t)(seg.s.row0 + (in ? token : 0)) * 2 * H * p.group + seg.head * p.group + (in ? at - token * p.group : 0);
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (row + (size_t)st * H * p.group) * DH);
                    uint8_t *dst = smem + st * C::Q_BYTES + tid * 128;
                    uint4 v[DH / 8];
#pragma unroll
                    for (int c = 0; c < DH / 8; ++c) v[c] = in ? src[c] : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < DH / 8; ++c) *reinterpret_cast<uint4 *>(dst + (c >> 3) * kCtRows * 128 + (((c & 7) ^ (tid & 7)) << 4)) = v[c];
                    uint32_t top = 0;
#pragma unroll
                    for (int c = 0; c < DH / 8; ++c) top = absmax8_bits(top, v[c]);
                    const uint32_t which = __ballot_sync(0xffffffffu, max(top >> 16, top & 0xffffu) >= 0x7f80u);
                    if (lane == 0) odd_q[segment & 3][st][warp] = which;
                }
                there(C::BAR_QFULL);
                qph ^= 1u;
            }
            for (int j = first; j < stop; ++j, ++g) {
                const bool page = j < pages;
                const int rows = page ? KV : seg.s.length & 63;
                const uint4 *open = reinterpret_cast<const uint4 *>(p.c.open + ((size_t)seg.s.slot * H + seg.head) * 3 * KV * DH);
                if (page && !(ok = wait(C::BAR_GFULL + gs, gph, 0xc18u + gs))) break;
                const uint4 *codes = reinterpret_cast<const uint4 *>(smem + C::OFF_G + gs * C::G_BYTES) + lane;
                const bool good = page && page_ok[gs];
                if (!(ok = wait(C::BAR_KEMPTY + ks, kph, 0xc20u + ks))) break;
                uint8_t *k = smem + C::OFF_K + ks * 2 * C::K_BYTES;
                if (page) {
                    // (Not unrolled: instructions are fetched from afar - a third of all waits - and the less code the loops have the better.  2 x 256 rows of 6000
                    // tokens 96 us unrolled, 89 not; 4 x 128 rows of 8192 tokens 128 wide 107 and 99.)
#pragma unroll 1
                    for (int i = 0; i < KN; ++i) {  // tile n of stream n / (4 KT): sixteen tokens, 32 dims
                        const int n = 4 * i + warp, stream = n / (DH / 8), mt = n % (DH / 8) / (DH / 32), kt = n % (DH / 32);
                        store(k + stream * C::K_BYTES + (kt >> 1) * KV * 128, mt * 16, (kt & 1) * 4, good ? codes[n * 32] : make_uint4(0, 0, 0, 0));
                    }
                } else {  // (the rows' eights lie in the places that the operand's layout gives them)
#pragma unroll 4
                    for (int e = tid; e < 2 * KV * DH / 8; e += 128) {
                        const int stream = e / (KV * DH / 8), r = e / (DH / 8) % KV, c = e % (DH / 8);
                        *reinterpret_cast<uint4 *>(k + stream * C::K_BYTES + (c >> 3) * KV * 128 + r * 128 + ((c & 7) << 4)) = r < rows ? open[e] : make_uint4(0, 0, 0, 0);
                    }
                }
                if (tid == 0) {
                    float4 sc = page && good ? *reinterpret_cast<const float4 *>(smem + C::OFF_G + gs * C::G_BYTES + C::UNIT) : make_float4(1.0f, 1.0f, 1.0f, 0.0f);
                    sc.w = page && !good ? 0.0f : 1.0f;
                    scales[g & 7] = sc;
                }
                there(C::BAR_KFULL + ks);
                if (++ks == C::KST) { ks = 0; kph ^= 1u; }
                if (!(ok = wait(C::BAR_VEMPTY + vs, vph, 0xc30u + vs))) break;
                uint8_t *v = smem + C::OFF_V + vs * C::V_BYTES;
                if (page) {
#pragma unroll 1
                    for (int i = 0; i < VN; ++i) {  // sixteen dims, 32 tokens
                        const int n = 4 * i + warp;
                        store(v, (n >> 1) * 16, (n & 1) * 4, good ? codes[(4 * KN + n) * 32] : make_uint4(0, 0, 0, 0));
                    }
                } else {  // values that are not finite become zero here, and the rows that see them are told at the end: zero times such a value is no zero
                    bool some = false;
                    const int r = tid & 63;
#pragma unroll 4
                    for (int c = tid >> 6; c < DH / 8; c += 2) {
                        const uint4 x = r < rows ? open[2 * KV * DH / 8 + r * (DH / 8) + cache_open_eight(r, c)] : make_uint4(0, 0, 0, 0);
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            uint32_t bits = w[q >> 1] >> (16 * (q & 1)) & 0xffffu;
                            if ((bits & 0x7f80u) == 0x7f80u) {
                                bits = 0;
                                some = true;
                            }
                            *reinterpret_cast<uint16_t *>(v + (8 * c + q) * 128 + (((r >> 3) ^ q) << 4) + (r & 7) * 2) = (uint16_t)bits;
                        }
                    }
                    some = __any_sync(0xffffffffu, some);
                    if (lane == 0) odd[4 * (segment & 7) + warp] = some;
                }
                if (page) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::BAR_GEMPTY + gs));
                    if (++gs == C::GST) { gs = 0; gph ^= 1u; }
                }
                there(C::BAR_VFULL + vs);
                if (++vs == C::KST) { vs = 0; vph ^= 1u; }
            }
            ++segment;
        }
    } else if (works && warp == 14) {
        // ------------------------------------------------------------------ pages into shared memory
        uint32_t issued[C::GST] = {};
        bool ok = true, more = true;
        int gs = 0, pages32 = 0;
        uint32_t gph = 1;
        CtSegment &seg = segments[warp];
        first_segment(seg);
        for (; ok && more; more = next_segment(seg)) {
            const int first = seg.unit, pages = seg.s.pages, head = seg.head, stop = min(seg.stop(), pages);
            const int32_t *table = p.c.table + (size_t)seg.s.slot * p.c.max_pages;
            for (int j = first; j < stop; ++j) {
                if (j == first || (j & 31) == 0) pages32 = (j & ~31) + lane < pages ? table[(j & ~31) + lane] : 0;
                const int page = __shfl_sync(0xffffffffu, pages32, j & 31);
                const bool good = page >= 0 && page < p.c.n_pages;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(C::BAR_GEMPTY + gs), gph, abort_flag, p.status, 0xc90u + gs)) != 0;
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t full = bar(C::BAR_GFULL + gs), dst = sbase + C::OFF_G + gs * C::G_BYTES;
                    const size_t at = (size_t)(good ? page : 0) * H + head;
                    page_ok[gs] = good;
                    if (good) {
                        mbar_arrive_expect_tx(full, C::UNIT + 16);
                        bulk_load_1d(dst, p.c.codes + at * C::UNIT, C::UNIT, full);
                        bulk_load_1d(dst + C::UNIT, p.c.scales + at, 16, full);
                    } else {
                        atomicOr(p.status, kStatusCache);
                        mbar_arrive(full);
                    }
                }
                ++issued[gs];
                if (++gs == C::GST) { gs = 0; gph ^= 1u; }
            }
        }
        // never leave with a copy in flight
        for (int q = 0; q < C::GST; ++q)
            if (issued[q])
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(bar(C::BAR_GFULL + q), (issued[q] - 1u) & 1u); ++i) {}
    } else if (works && (warp == 12 || warp == 13)) {
        // ------------------------------------------------------------------ the products of a stream
        const int st = warp - 12;
        auto wait = [&](int i, uint32_t par, unsigned int code) { return __all_sync(0xffffffffu, mbar_wait_poll(bar(i), par, abort_flag, p.status, code)) != 0; };
        const uint64_t q_desc = make_sw128_desc(sbase + st * C::Q_BYTES), k_desc = make_sw128_desc(sbase + C::OFF_K + st * C::K_BYTES), v_desc = make_sw128_desc(sbase + C::OFF_V);
        // The scores run NS steps ahead of P V: the products execute in order, so P of a step has been read when the scores of NS steps on replace it.
        bool ok = true, s_more = true, p_more = true;
        int ks = 0, vs = 0, g = 0, sj = 0;
        uint32_t kph = 0, vph = 0, sqph = 0, poph = 1;
        CtSegment &sseg = segments[warp], &pseg = segments[warp - 12 + kCtThreads / 32];
        int s_first = 0, s_stop = 0, p_first = 0, p_stop = 0;
        auto full = [&](CtSegment &s, bool &more, int &first, int &stop) {  // on to a segment with steps
            while (more && s.unit >= s.stop()) more = next_segment(s);
            first = s.unit;
            stop = s.stop();
        };
        first_segment(sseg);
        first_segment(pseg);
        full(sseg, s_more, s_first, s_stop);
        full(pseg, p_more, p_first, p_stop);
        sj = s_first;
        auto next_scores = [&](int buf) {
            if (sj == s_first && !wait(C::BAR_QFULL, sqph, 0xc40u)) return false;
            if (!wait(C::BAR_KFULL + ks, kph, 0xc48u + ks)) return false;
            tc_fence_after();
            const uint64_t kd = k_desc + (uint64_t)(ks * (2 * C::K_BYTES >> 4));
#pragma unroll
            for (int blk = 0; blk < C::NBLK; ++blk)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    warp_mma_f16(tmem_base + C::col_s(st, buf), q_desc + (uint64_t)(blk * (kCtRows * 128 >> 4) + 2 * kk), kd + (uint64_t)(blk * (KV * 128 >> 4) + 2 * kk), C::IDESC_S, (blk | kk) ? 1u : 0u);
            warp_commit(bar(C::BAR_SFULL + 2 * st + buf));  // also: P V of NS steps before is complete
            warp_commit(bar(C::BAR_KEMPTY + ks));
            if (++ks == C::KST) { ks = 0; kph ^= 1u; }
            if (++sj == s_stop) {
                warp_commit(bar(C::BAR_QEMPTY));
                sqph ^= 1u;
                s_more = next_segment(sseg);
                full(sseg, s_more, s_first, s_stop);
                sj = s_first;
            }
            return true;
        };
        for (int i = 0; ok && i < NS && s_more; ++i) ok = next_scores(i);
        while (ok && p_more) {
            if (!(ok = wait(C::BAR_OEMPTY, poph, 0xc50u))) break;
            poph ^= 1u;
            const uint32_t o_col = tmem_base + C::COL_O + st * DH;
            for (int j = p_first; j < p_stop; ++j, ++g) {
                const int buf = NS == 2 ? g & 1 : 0;
                if (!(ok = wait(C::BAR_VFULL + vs, vph, 0xc58u + vs))) break;
                if (!(ok = wait(C::BAR_PFULL + 2 * st + buf, (uint32_t)(g >> (NS - 1)) & 1u, 0xc60u + st))) break;
                tc_fence_after();
                const uint64_t vd = v_desc + (uint64_t)(vs * (C::V_BYTES >> 4));
#pragma unroll
                for (int part = 0; part < 3; ++part)
#pragma unroll
                    for (int kk = 0; kk < KV / 16; ++kk)
                        warp_mma_f16_ts(o_col, tmem_base + (part < 2 ? C::col_s(st, buf) + 32 * part : C::col_p3(st, buf)) + 8 * kk, vd + (uint64_t)(2 * kk), C::IDESC_PV,
                                        (((j - p_first) & (kCtFlush - 1)) != 0 || part || kk) ? 1u : 0u);
                warp_commit(bar(C::BAR_VEMPTY + vs));
                if (j + 1 == p_stop) warp_commit(bar(C::BAR_END + st));
                if (++vs == C::KST) { vs = 0; vph ^= 1u; }
                if (s_more) { if (!(ok = next_scores(buf))) break; }
                else warp_commit(bar(C::BAR_SFULL + 2 * st + buf));
            }
            p_more = next_segment(pseg);
            full(pseg, p_more, p_first, p_stop);
        }
    } else if (works && warp < 12) {
        // ------------------------------------------------------------------ softmax of one stream, one row per thread
        const int st = warp >= 8 ? 1 : 0, quarter = warp & 3, row = 32 * quarter + lane;
        const uint32_t lane_base = tmem_base + ((uint32_t)(32 * quarter) << 16);
        auto wait = [&](int i, uint32_t par, unsigned int code) { return __all_sync(0xffffffffu, mbar_wait_poll(bar(i), par, abort_flag, p.status, code)) != 0; };
        bool ok = true, more = true;
        int g = 0, segment = 0;
        CtSegment &seg = segments[warp];
        first_segment(seg);
        for (; ok && more; more = next_segment(seg)) {
            const int first = seg.unit, stop = seg.stop(), at = seg.tile * kCtRows + row, token = p.group == 1 ? at : at / p.group;
            const int sees = token < seg.s.m ? seg.s.length - seg.s.m + 1 + token : 0;
            const bool whole = seg.whole();
            // The row's place for the segment as a part: the CTA's first if the item begins in front of the share or with it (then it is the first segment), else the
            // second, which the last segment alone can need as a part.
            // Sixteen bytes of a row lie kCtRows * 16 bytes apart, those of neighbouring rows side by side, as neighbouring threads have them.
            float4 *const part = reinterpret_cast<float4 *>(p.cta_parts + ((size_t)blockIdx.x * 2 + (seg.u - seg.unit > c0)) * kCtRows * C::PART) + row;
            auto sums_at = [&](int stream, int c) { return part + (1 + stream * (DH / 4) + c) * kCtRows; };
            auto put_ml = [&](float m, float l) { reinterpret_cast<float2 *>(part)[st] = make_float2(m, l); };
            auto acc_at = [&](int stream, int c) {  // sixteen bytes of the row's sums from before the products' last new beginning
                return DH == 64 ? reinterpret_cast<float4 *>(smem + C::OFF_ACC + ((size_t)stream * kCtRows + row) * DH * 4 + ((c ^ (row & 7)) << 4)) : sums_at(stream, c);
            };
            if (const long long from = seg.u - seg.unit, to = from + seg.s.units; !whole && to > c1 && from >= c0 && warp == 4 && lane == 0) {
                p.items[2 * blockIdx.x] = make_int4(from > c0 ? 2 : 1, ca_share_of(total, to - 1, ctas), seg.head, seg.tile);
                p.items[2 * blockIdx.x + 1] = make_int4(seg.s.row0, seg.s.m, 0, 0);
            }
            if (first >= stop) {  // (never a whole item: its first step is visible)
                put_ml(kCtNone, 0.0f);
                for (int c = 0; c < DH / 4; ++c) *sums_at(st, c) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                continue;
            }
            const uint32_t o_addr = lane_base + C::COL_O + st * DH;
            float m = kCtNone;
            uint64_t l2 = 0;  // the row's sum, two partial sums
            float m_acc = kCtNone;
            bool flushed = false;
            for (int j = first; j < stop; ++j, ++g) {
                const int buf = NS == 2 ? g & 1 : 0;
                const uint32_t s_addr = lane_base + C::col_s(st, buf), p3_addr = lane_base + C::col_p3(st, buf);
                if (!(ok = wait(C::BAR_SFULL + 2 * st + buf, (uint32_t)(g >> (NS - 1)) & 1u, 0xc70u + st))) break;
                tc_fence_after();
                // (A query that is infinite may have no score but -inf, which would be no weight: its maximum is NaN from the beginning, and with it all that follows.)
                if (j == first && sees > 0 && (odd_q[segment & 3][st][quarter] >> lane & 1u)) m = __uint_as_float(0x7fc00000u);
                const float4 sc = scales[g & 7];
                const int n = sc.w != 0.0f ? sees - KV * j : 0;  // of the step's tokens, those that the row sees: none of a page whose number is out of range
                // O is at rest once P V of the step before is complete: the barrier of scores that were issued behind it says so, the step's own where a stream has
                // one step of scores, else the next step's.
                auto at_rest = [&](unsigned int code) {
                    if (NS == 1) return true;
                    if (!wait(C::BAR_SFULL + 2 * st + (buf ^ 1), (uint32_t)((g + 1) >> 1) & 1u, code)) return false;
                    tc_fence_after();
                    return true;
                };
                if (j > first && ((j - first) & (kCtFlush - 1)) == 0) {
                    // (2 x 256 rows of 6000 tokens, error against 64 bits: 1.3e-6, without it 4.4e-6, and 92 us for 99)
                    if (!(ok = at_rest(0xc7cu + st))) break;
                    const float beta = flushed ? exp2_approx(m_acc - m) : 0.0f;
#pragma unroll
                    for (int cc = 0; cc < DH; cc += 16) {
                        uint32_t o[16];
                        float4 a[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) a[u] = flushed ? *acc_at(st, (cc >> 2) + u) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        tmem_ld16(o_addr + cc, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            *acc_at(st, (cc >> 2) + u) = make_float4(fmaf(a[u].x, beta, __uint_as_float(o[4 * u])), fmaf(a[u].y, beta, __uint_as_float(o[4 * u + 1])),
                                                                     fmaf(a[u].z, beta, __uint_as_float(o[4 * u + 2])), fmaf(a[u].w, beta, __uint_as_float(o[4 * u + 3])));
                    }
                    m_acc = m;
                    flushed = true;
                }
                if (__all_sync(0xffffffffu, n <= 0)) {
                    uint32_t zero[32];
#pragma unroll
                    for (int u = 0; u < 32; ++u) zero[u] = 0u;
                    tmem_st32(s_addr, zero);
                    tmem_st32(s_addr + 32, zero);
                    tmem_st32(p3_addr, zero);
                } else {
                    // (a page of zeros has the factor 0, and what is masked has to stay at -inf; of a page that the row sees nothing of not even a NaN counts.)
                    const float f = n > 0 ? p.scale_log2 * (st ? sc.y : sc.x) + 1.17549435e-38f : 1.0f;
                    // (a page of zeros has the scale 0 and codes 0)
                    const float sv = n > 0 && sc.z != 0.0f ? sc.z : 1.0f;
                    uint32_t v0[32], v1[32];
                    tmem_ld32(s_addr, v0);
                    tmem_ld32(s_addr + 32, v1);
                    tmem_ld_wait();
                    if (__any_sync(0xffffffffu, n < KV)) {
#pragma unroll
                        for (int u = 0; u < 32; ++u) {
                            if (u >= n) v0[u] = 0xff800000u;
                            if (32 + u >= n) v1[u] = 0xff800000u;
                        }
                    }
                    float m0 = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
                    for (int u = 0; u < 32; u += 4) {
                        m0 = fmaxf(m0, fmaxf(__uint_as_float(v0[u]), __uint_as_float(v0[u + 1])));
                        m1 = fmaxf(m1, fmaxf(__uint_as_float(v0[u + 2]), __uint_as_float(v0[u + 3])));
                        m2 = fmaxf(m2, fmaxf(__uint_as_float(v1[u]), __uint_as_float(v1[u + 1])));
                        m3 = fmaxf(m3, fmaxf(__uint_as_float(v1[u + 2]), __uint_as_float(v1[u + 3])));
                    }
                    const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)), here = top * f;
                    // The reference of the exponentials follows the maximum only where that has moved by more than kCtSlack, so O and l are rescaled rarely.
                    const float now = here - m > kCtSlack ? here : m;
                    if (j > first && __any_sync(0xffffffffu, now != m)) {
                        if (!(ok = at_rest(0xc78u + st))) break;
                        const float alpha = exp2_approx(m - now);
                        const uint64_t a2 = pack_f32x2(alpha, alpha);
                        l2 = mul_f32x2(l2, a2);
#pragma unroll
                        for (int cc = 0; cc < DH; cc += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_addr + cc, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int u = 0; u < 16; ++u) o[u] = __float_as_uint(__uint_as_float(o[u]) * alpha);
                            tmem_st16(o_addr + cc, o);
                        }
                    }
                    m = now;
                    const uint64_t f2 = pack_f32x2(f, f), minus = top == -INFINITY ? 0 : pack_f32x2(-top, -top), rest2 = pack_f32x2(here - m, here - m), minus1 = pack_f32x2(-1.0f, -1.0f), sv2 = pack_f32x2(sv, sv);
                    uint64_t sum_a = 0, sum_b = 0;
                    // (relative to the step's largest first, which is then exact however large the scores)
                    // 32 scores -> their probabilities, times the scale of V, in three parts, sixteen columns each
                    auto part_of = [&](const uint32_t (&v)[32], uint64_t &sum, int at) {
                        uint32_t hi[16], lo[16], third[16];
#pragma unroll
                        for (int u = 0; u < 16; ++u) {
                            float x0, x1;
                            unpack_f32x2(fma_f32x2(add_f32x2(pack_f32x2(__uint_as_float(v[2 * u]), __uint_as_float(v[2 * u + 1])), minus), f2, rest2), x0, x1);
                            uint64_t e = pack_f32x2(exp2_approx(x0), exp2_approx(x1));
                            sum = add_f32x2(sum, e);
                            e = mul_f32x2(e, sv2);
                            unpack_f32x2(e, x0, x1);
                            const __nv_bfloat162 first = __floats2bfloat162_rn(x0, x1);
                            hi[u] = *reinterpret_cast<const uint32_t *>(&first);
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(hi[u] << 16), __uint_as_float(hi[u] & 0xffff0000u)), minus1, e), x0, x1);
                            const __nv_bfloat162 second = __floats2bfloat162_rn(x0, x1);
                            lo[u] = *reinterpret_cast<const uint32_t *>(&second);
                            const __nv_bfloat162 rest = __floats2bfloat162_rn(x0 - __uint_as_float(lo[u] << 16), x1 - __uint_as_float(lo[u] & 0xffff0000u));
                            third[u] = *reinterpret_cast<const uint32_t *>(&rest);
                        }
                        tmem_st16(s_addr + at, hi);
                        tmem_st16(s_addr + 32 + at, lo);
                        tmem_st16(p3_addr + at, third);
                    };
                    part_of(v0, sum_a, 0);
                    part_of(v1, sum_b, 16);
                    l2 = add_f32x2(l2, add_f32x2(sum_a, sum_b));
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::BAR_PFULL + 2 * st + buf));
            }
            if (!ok) break;
            // ---- the segment's end
            if (!(ok = wait(C::BAR_END + st, (uint32_t)segment & 1u, 0xc80u + st))) break;
            float la, lb;
            unpack_f32x2(l2, la, lb);
            const float l = la + lb;
            // open values that are not finite were left out: NaN where a row sees them
            const int open0 = 64 * seg.s.pages, open_seen = stop > seg.s.pages ? min(sees - open0, seg.s.length - open0) : 0;
            const volatile int *o4 = odd + 4 * (segment & 7);
            const bool checked = stop > seg.s.pages && (o4[0] | o4[1] | o4[2] | o4[3]);
            const __nv_bfloat16 *values = p.c.open + (((size_t)seg.s.slot * H + seg.head) * 3 + 2) * KV * DH;
            auto not_finite = [&](int dim) {
                for (int r = 0; r < open_seen; ++r)
                    if ((__bfloat16_as_ushort(values[(size_t)r * DH + cache_open_eight(r, dim >> 3) * 8 + (dim & 7)]) & 0x7f80) == 0x7f80) return true;
                return false;
            };
            const float flush_scale = flushed ? exp2_approx(m_acc - m) : 0.0f;
            if (whole) {
                s_l[((segment & 1) * 2 + st) * kCtRows + row] = l;
                s_f[((segment & 1) * 2 + st) * kCtRows + row] = flush_scale;  // (`flushed` is alike for all rows and both streams)
            }
            auto add_flushed = [&](uint32_t (&v)[32], int stream, int cc, float scale) {
                if (flushed) {  // (with a scale of zero as well: what is not finite stays so)
#pragma unroll
                    for (int u = 0; u < 32; u += 4) {
                        const float4 a = *acc_at(stream, (cc + u) >> 2);
                        v[u] = __float_as_uint(fmaf(a.x, scale, __uint_as_float(v[u])));
                        v[u + 1] = __float_as_uint(fmaf(a.y, scale, __uint_as_float(v[u + 1])));
                        v[u + 2] = __float_as_uint(fmaf(a.z, scale, __uint_as_float(v[u + 2])));
                        v[u + 3] = __float_as_uint(fmaf(a.w, scale, __uint_as_float(v[u + 3])));
                    }
                }
            };
            // (both streams have got so far: their O are complete, their sums there)
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::BAR_L + (segment & 1)));
            if (!(ok = wait(C::BAR_L + (segment & 1), (uint32_t)(segment >> 1) & 1u, 0xc88u))) break;
            tc_fence_after();
            if (whole) {
                const float *sl = s_l + (segment & 1) * 2 * kCtRows;
                const float l1 = sl[row], l2 = sl[kCtRows + row];
                const float w1 = l1 != 0.0f ? p.out_scale / l1 : 0.0f, w2 = l2 != 0.0f ? p.out_scale * p.lambda / l2 : 0.0f;
                const uint32_t o_base = lane_base + C::COL_O;
                const size_t out = ((size_t)(seg.s.row0 + token) * H * p.group + seg.head * p.group + at - token * p.group) * DH;
#pragma unroll
                for (int cc = st * (DH / 2); cc < (st + 1) * (DH / 2); cc += 32) {
                    uint32_t v1[32], v2[32];
                    tmem_ld32(o_base + cc, v1);
                    tmem_ld32(o_base + DH + cc, v2);
                    tmem_ld_wait();
                    add_flushed(v1, 0, cc, s_f[(segment & 1) * 2 * kCtRows + row]);
                    add_flushed(v2, 1, cc, s_f[((segment & 1) * 2 + 1) * kCtRows + row]);
                    if (token < seg.s.m) {
#pragma unroll
                        for (int u = 0; u < 32; ++u) v1[u] = __float_as_uint(__uint_as_float(v1[u]) * w1 - __uint_as_float(v2[u]) * w2);
                        if (p.bf16) {
#pragma unroll
                            for (int u = 0; u < 32; u += 8) {
                                uint32_t o[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const __nv_bfloat162 y = __floats2bfloat162_rn(__uint_as_float(v1[u + 2 * e]), __uint_as_float(v1[u + 2 * e + 1]));
                                    o[e] = *reinterpret_cast<const uint32_t *>(&y);
                                }
                                *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(p.out) + out + cc + u) = make_uint4(o[0], o[1], o[2], o[3]);
                            }
                        } else {
#pragma unroll
                            for (int u = 0; u < 32; u += 4) *reinterpret_cast<uint4 *>(reinterpret_cast<float *>(p.out) + out + cc + u) = make_uint4(v1[u], v1[u + 1], v1[u + 2], v1[u + 3]);
                        }
                    }
                    __syncwarp();  // (tcgen05.ld takes the whole warp, in the next round again)
                }
                if (checked && token < seg.s.m)
                    for (int dim = st * (DH / 2); dim < (st + 1) * (DH / 2); ++dim)
                        if (not_finite(dim)) {
                            if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[out + dim] = __ushort_as_bfloat16(0x7fc0);
                            else reinterpret_cast<float *>(p.out)[out + dim] = __uint_as_float(0x7fc00000u);
                        }
            } else {
                put_ml(m, l);
#pragma unroll
                for (int cc = 0; cc < DH; cc += 32) {
                    uint32_t v[32];
                    tmem_ld32(o_addr + cc, v);
                    tmem_ld_wait();
                    add_flushed(v, st, cc, flush_scale);
#pragma unroll
                    for (int u = 0; u < 32; u += 4) *reinterpret_cast<uint4 *>(sums_at(st, (cc + u) >> 2)) = make_uint4(v[u], v[u + 1], v[u + 2], v[u + 3]);
                }
                if (checked)
                    for (int dim = 0; dim < DH; ++dim)
                        if (not_finite(dim)) reinterpret_cast<float *>(sums_at(st, dim >> 2))[dim & 3] = __uint_as_float(0x7fc00000u);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::BAR_OEMPTY));
            ++segment;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(512) : "memory");
    }
}

}  // namespace hgf
